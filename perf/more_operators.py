"""The operators of speculative decoding and beam search over a paged K/V cache, as they are measured.

Kinds of case (``kind``):

- ``attend``: the tokens of drafted trees attend to their sequences in the cache: every earlier token
  (``sink`` leading ones and the last ``local`` before a node's position; ``local`` -1: all of them) and
  the node's own ancestors and itself, with the logarithm of the softmax sum of every row;
- ``commit``: what a step does around the model: the trees' positions and ancestor masks from the nodes'
  parents; then, with the model's choice after each node, the walk down each tree and the accepted nodes'
  rows moved to the places that they keep, in the caches of ``layers`` layers. A node without a place in
  its tree (one of ``absent`` per cent, padding) is on no path;
- ``beam``: the best ``best`` of all continuations of a group's ``beams`` beams: the beam's score plus the
  logarithm of the token's softmax over the vocabulary (``vocab`` logits, ``type``);
- ``reorder``: the beams' page tables take the order of the beams they go on from, complete pages are
  shared, and the rows of the page that is still being filled are copied where two beams go on from one,
  in the caches of ``layers`` layers.

``hq`` / ``hkv`` query and KV heads (head size 128, bf16), ``cache`` the cache's type (``bf16``, or
``e4m3`` with a power-of-two scale per token and head), ``page`` tokens of a page, ``seqs`` sequences (of
``beam`` and ``reorder``: groups of beams) whose trees have ``new_lo`` to ``new_hi`` nodes and whose lengths
(new tokens included) spread from ``len_lo`` to ``len_hi``, geometrically.
"""

from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DH = 128
E4M3_MAX = 448.0
LOW_EXP = -100  # the smallest scale is 2^LOW_EXP


def listed():
    llama = dict(hq=32, hkv=8)
    return [
        # The smallest verification: one short tree at 2K on 4 query heads.
        dict(name="attend-1x8-2k", kind="attend", cache="bf16", page=64, seqs=1, new_lo=8, new_hi=8, len_lo=2048,
             len_hi=2048, sink=0, local=-1, hq=4, hkv=1),
        # One user's tree of 25 nodes at the end of 128K, 8-bit: the split of one long sequence.
        dict(name="attend-1x25-128k", kind="attend", cache="e4m3", page=64, seqs=1, new_lo=25, new_hi=25,
             len_lo=131071, len_hi=131071, sink=0, local=-1, **llama),
        # A batch of sequences of very different lengths with trees of 1 to 40 nodes, bf16 pages of 16 tokens.
        dict(name="attend-33-ragged", kind="attend", cache="bf16", page=16, seqs=33, new_lo=1, new_hi=40, len_lo=130,
             len_hi=20000, sink=0, local=-1, hq=28, hkv=4),
        # Trees of 60 nodes beside sinks and a window, 8-bit.
        dict(name="attend-9-window", kind="attend", cache="e4m3", page=64, seqs=9, new_lo=60, new_hi=60, len_lo=1000,
             len_hi=12000, sink=64, local=4000, **llama),
        # Sixteen long sequences with trees of 64 nodes: the largest.
        dict(name="attend-16x64-32k", kind="attend", cache="bf16", page=64, seqs=16, new_lo=64, new_hi=64,
             len_lo=20000, len_hi=32768, sink=0, local=-1, **llama),
        # One tree accepted, in one layer's cache: latency.
        dict(name="commit-1x16", kind="commit", cache="bf16", page=64, seqs=1, new_lo=16, new_hi=16, len_lo=300,
             len_hi=300, layers=1, absent=0, hkv=8),
        # A batch's trees, padded, in the 8-bit caches of 32 layers.
        dict(name="commit-48x61", kind="commit", cache="e4m3", page=16, seqs=48, new_lo=61, new_hi=61, len_lo=100,
             len_hi=400, layers=32, absent=20, hkv=8),
        # One group of four beams over a small vocabulary: latency.
        dict(name="beam-1x4-32k", kind="beam", type="bf16", seqs=1, beams=4, vocab=32000, best=8),
        # Eleven groups of five beams over a vocabulary of odd size, fp32 logits.
        dict(name="beam-11x5-100k", kind="beam", type="fp32", seqs=11, beams=5, vocab=100003, best=10),
        # A large batch: 64 groups of eight beams, twice as many continuations kept.
        dict(name="beam-64x8-128k", kind="beam", type="bf16", seqs=64, beams=8, vocab=128000, best=16),
        # One group's caches reordered in one layer: latency.
        dict(name="reorder-1x4", kind="reorder", cache="bf16", page=64, seqs=1, beams=4, len_lo=1000, len_hi=1000,
             layers=1, hkv=8),
        # Sixteen groups of eight beams, 8-bit, in all layers.
        dict(name="reorder-16x8", kind="reorder", cache="e4m3", page=64, seqs=16, beams=8, len_lo=200, len_hi=700,
             layers=32, hkv=8),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["attend", "attend", "attend", "commit", "beam", "beam", "reorder"])
    if kind == "beam":
        beams, vocab = size(1, 32), size(100, 160000)
        return dict(kind=kind, type=rng.choice(["bf16", "fp32"]), seqs=max(1, min(size(1, 64), 60000000 // (beams * vocab))),
                    beams=beams, vocab=vocab, best=min(64, size(1, 2 * beams), vocab))
    hq, hkv = rng.choice([(32, 8), (32, 8), (28, 4), (16, 8), (8, 1), (6, 2), (4, 4)])
    c = dict(kind=kind, cache=rng.choice(["bf16", "e4m3"]), page=rng.choice([16, 64, 128, 48]), hkv=hkv)
    if kind == "reorder":
        c.update(seqs=size(1, 24), beams=size(2, 16), layers=size(1, 32))
        hi = size(40, 900)
        while c["layers"] * c["seqs"] * (c["beams"] * 2 * c["page"] + hi) * hkv > 8000000:
            c["layers"] = (c["layers"] + 1) // 2
            c["seqs"] = (c["seqs"] + 1) // 2
        c.update(len_lo=hi if c["seqs"] == 1 else max(1, hi // 4), len_hi=hi)
        return c
    if kind == "commit":
        seqs, new_hi = size(1, 64), size(1, 200)
        hi = new_hi + size(1, 600)
        c.update(seqs=seqs, layers=size(1, 32), absent=rng.choice([0, 0, 20]))
        while c["layers"] * seqs * (hi + c["page"]) * hkv > 8000000:
            c["layers"] = (c["layers"] + 1) // 2
            seqs = c["seqs"] = (seqs + 1) // 2
        c.update(new_lo=new_hi if seqs == 1 else size(1, new_hi), new_hi=new_hi,
                 len_lo=hi if seqs == 1 else max(1, hi // 3), len_hi=hi)
        return c
    c.update(hq=hq)
    c.update(dict(sink=rng.choice([0, 4, 64, 128]), local=rng.choice([256, 1000, 4096])) if rng.random() < 0.3 else
             dict(sink=0, local=-1))
    seqs, new_hi = size(1, 48), size(1, 200)
    hi = max(2 * new_hi, size(200, 120000 if seqs == 1 else min(32000, 500000 // seqs)))
    seqs = max(1, min(seqs, 34000000 // (new_hi * hi)))
    c.update(seqs=seqs, new_lo=new_hi if seqs == 1 else size(1, new_hi), new_hi=new_hi,
             len_lo=hi if seqs == 1 else max(1, hi // rng.choice([1, 8, 60])), len_hi=hi)
    return c


def _spread(lo, hi, n, turn):
    """n sizes from lo to hi, evenly on a logarithmic scale, in an order of their own."""
    if n == 1:
        return [hi]
    up = [int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]
    return [up[i * turn % n] for i in range(n)] if math.gcd(turn, n) == 1 else up[::-1]


def _lens(c):
    """(new tokens, length with them) of every sequence; for beams (0, length) of every group."""
    lens = _spread(c["len_lo"], c["len_hi"], c["seqs"], 7)
    if c["kind"] == "reorder":
        return [(0, n) for n in lens]
    new = _spread(c["new_lo"], c["new_hi"], c["seqs"], 5)
    return [(min(a, n), n) for a, n in zip(new, lens)]


# ---------------------------------------------------------------- inputs


def _tree(rng, n, absent):
    """Parents of n nodes, level by level from one root (-1); -2: no node."""
    parent = [-1] + sorted(int(0.7 * (i - 1) * rng.random() ** 0.8) for i in range(1, n))
    leaf = set(range(n)) - set(parent)
    for i in range(1, n):
        if i in leaf and rng.random() * 100 < absent:
            parent[i] = -2
    return parent


def _path(rng, parent):
    """Nodes that the model accepts: a way down from the root, where no accepted row lies in a place
    that another one is moved to (so that a pass can be repeated on the rows it has moved)."""
    for _ in range(50):
        path, most = [0], rng.randint(1, 8)
        while len(path) < most:
            down = [i for i, p in enumerate(parent) if p == path[-1]]
            if not down:
                break
            path.append(rng.choice(down))
        if all(x == i or x >= len(path) for i, x in enumerate(path)):
            return path
    return [0]


def _trees(st, c, seed):
    """Parents of all rows, and for every row its position; the tokens and the model's choices of a commit."""
    rng = random.Random(seed)
    parents, tokens, choices = [], [], []
    for new, _ in st["lens"]:
        parent = _tree(rng, new, c.get("absent", 0))
        token = [rng.randrange(30000) for _ in parent]
        choice = [30000 + rng.randrange(1000) for _ in parent]
        path = _path(rng, parent)
        for x, y in zip(path, path[1:]):
            choice[x] = token[y]
        parents += parent
        tokens += token
        choices += choice
    as_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    st["parents"], st["tokens"], st["choices"] = as_int(parents), as_int(tokens), as_int(choices)
    st["first"] = st["tokens"][st["row_start"][:-1].long()].clone()  # the root is the token chosen before


def _mixture(gen, n, heads, groups):
    """[n][heads][128] fp32: a component of norm 3 of the head's group plus N(0, 1)."""
    kvh = torch.arange(heads, device="cuda") // (heads // groups.shape[0])
    ids = torch.randint(0, groups.shape[1], (n, heads), generator=gen, device="cuda")
    return groups[kvh, ids] + torch.randn(n, heads, DH, generator=gen, device="cuda")


def _groups(gen, hkv):
    x = torch.randn(hkv, 256, DH, generator=gen, device="cuda")
    return 3.0 * x / x.norm(dim=-1, keepdim=True)


def _power(e):
    """2^e of whole numbers e in -126..127, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """e4m3 rows of fp32 rows [..., 128] and the exponents + 127 of their scales (uint8)."""
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=LOW_EXP)  # amax <= 448 * 2^e
    e = torch.where(amax > 0, e, LOW_EXP)
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _pool(c, gen, pages, layers=None):
    """An empty cache (or one for each of `layers` layers) of so many pages."""
    st = {}
    lead = (pages,) if layers is None else (layers, pages)
    for x in "kv":
        kind = torch.float8_e4m3fn if c["cache"] == "e4m3" else torch.bfloat16
        st[x + "_pages"] = torch.zeros(*lead, c["page"], c["hkv"], DH, dtype=kind, device="cuda")
        if c["cache"] == "e4m3":
            st[x + "_scales"] = torch.full((*lead, c["hkv"], c["page"]), 127, dtype=torch.uint8, device="cuda")
    return st


def _table(gen, counts, spare=0):
    """Page table of sequences of so many pages each, in a shuffled pool with `spare` more."""
    used = sum(counts)
    order = torch.randperm(used + spare, generator=gen, device="cuda").int()
    table = torch.full((len(counts), max(counts)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, p in enumerate(counts):
        table[b, :p] = order[at: at + p]
        at += p
    return table, used + spare


def _fill(st, c, gen, groups):
    """Keys and values of every token of the sequences."""
    page = c["page"]
    for b, (_, n) in enumerate(st["lens"]):
        for a in range(0, n, 32768 // page * page):
            m = min(n - a, 32768 // page * page)
            pages = st["table"][b, a // page: -(-(a + m) // page)].long()
            for x in "kv":
                rows = torch.zeros(pages.numel() * page, c["hkv"], DH, device="cuda")
                rows[:m] = _mixture(gen, m, c["hkv"], groups) if x == "k" else torch.randn(
                    m, c["hkv"], DH, generator=gen, device="cuda")
                rows = rows.view(pages.numel(), page, c["hkv"], DH)
                if c["cache"] == "e4m3":
                    codes, e = _quantise(rows)
                    st[x + "_pages"].view(torch.uint8)[pages] = codes.view(torch.uint8)
                    st[x + "_scales"][pages] = e.transpose(1, 2).contiguous()
                else:
                    st[x + "_pages"][pages] = rows.bfloat16()


def _fill_all(st, c, gen):
    """Every row of every layer: what is moved is not looked at."""
    for x in "kv":
        pages = st[x + "_pages"]
        for layer in pages:
            layer.view(torch.uint8 if c["cache"] == "e4m3" else torch.bfloat16).copy_(
                torch.randn(layer.shape, generator=gen, device="cuda").to(layer.dtype).view(
                    torch.uint8 if c["cache"] == "e4m3" else torch.bfloat16))
        if c["cache"] == "e4m3":
            st[x + "_scales"].copy_(torch.randint(110, 130, st[x + "_scales"].shape, generator=gen, device="cuda"))


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = {"c": c}
    if c["kind"] == "beam":
        rows = c["seqs"] * c["beams"]
        z = torch.randn(rows, c["vocab"], generator=gen, device="cuda") * 2.5
        liked = torch.randint(0, c["vocab"], (rows, 12), generator=gen, device="cuda")
        z.scatter_add_(1, liked, torch.rand(rows, 12, generator=gen, device="cuda") * 14.0)
        st["logits"] = z.bfloat16() if c["type"] == "bf16" else z
        st["scores"] = -30.0 * torch.rand(c["seqs"], c["beams"], generator=gen, device="cuda")
    else:
        st["lens"] = _lens(c)
        page = c["page"]
        if c["kind"] == "reorder":
            _beams(st, c, gen, seed)
        else:
            starts = [0]
            for a, _ in st["lens"]:
                starts.append(starts[-1] + a)
            st["rows"] = starts[-1]
            st["most"] = max(a for a, _ in st["lens"])
            st["words"] = -(-st["most"] // 32)
            st["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
            st["kv_len"] = torch.tensor([n for _, n in st["lens"]], dtype=torch.int32, device="cuda")
            st["table"], pages = _table(gen, [-(-n // page) for _, n in st["lens"]], 3)
            st.update(_pool(c, gen, pages, c.get("layers")))
            _trees(st, c, seed)
            # every row's sequence and its place among its new tokens
            st["seq"] = torch.repeat_interleave(torch.arange(len(st["lens"]), device="cuda"),
                                                torch.tensor([a for a, _ in st["lens"]], device="cuda"))
            st["local"] = torch.arange(st["rows"], device="cuda") - st["row_start"].long()[st["seq"]]
            st["base"] = st["kv_len"].long() - (st["row_start"][1:] - st["row_start"][:-1]).long()
            if c["kind"] == "attend":
                groups = _groups(gen, c["hkv"])
                _fill(st, c, gen, groups)
                st["q"] = _mixture(gen, st["rows"], c["hq"], groups).bfloat16()
                st["positions"], st["masks"] = _plan_plain(st)
            else:
                _fill_all(st, c, gen)
    if own:
        _handles(st)
    return st


def _beams(st, c, gen, seed):
    """Beams whose prompt's pages are shared, each with a page of its own that is being filled and the next."""
    page, n = c["page"], c["beams"]
    counts = []
    for _, length in st["lens"]:
        counts.append(length // page)
    shared = sum(counts)
    pages = shared + 2 * n * c["seqs"] + 3
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((c["seqs"] * n, max(counts) + 2), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, k in enumerate(counts):
        mine = table[s * n: (s + 1) * n]
        mine[:, :k] = order[at: at + k]
        at += k
        mine[:, k: k + 2] = order[at: at + 2 * n].view(n, 2)
        at += 2 * n
    st["table"], st["pages"] = table, pages
    st["kv_len"] = torch.tensor([x for _, x in st["lens"]], dtype=torch.int32, device="cuda").repeat_interleave(n)
    rng = random.Random(seed)
    # the beams that go on: the better ones more often
    st["parents"] = torch.tensor([[int(n * rng.random() ** 1.5) for _ in range(n)] for _ in range(c["seqs"])],
                                 dtype=torch.int32, device="cuda")
    st.update(_pool(c, gen, pages, c["layers"]))
    _fill_all(st, c, gen)


# ---------------------------------------------------------------- the framework's calls


def _handles(st):
    """Descriptors, workspace and outputs, as a program keeps them between calls."""
    from paper_2609_31568_gb300 import scale as S

    c = st["c"]
    ints = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
    if c["kind"] == "beam":
        st["beam"] = S.beam_params(n_groups=c["seqs"], n_beams=c["beams"], vocab=c["vocab"], n_best=c["best"])
        st["best"] = torch.empty(c["seqs"], c["best"], device="cuda")
        st["best_beams"], st["best_tokens"] = ints(c["seqs"], c["best"]), ints(c["seqs"], c["best"])
        st["ws"] = torch.empty(S.scale_beam_workspace_size(st["beam"]), dtype=torch.uint8, device="cuda")
        return
    scales = lambda i: [st[x][i] if x in st else None for x in ("k_scales", "v_scales")]  # noqa: E731
    if "layers" in c:
        st["caches"] = S.cache_layers([S.kv_cache(st["k_pages"][i], st["v_pages"][i], *scales(i))
                                       for i in range(c["layers"])])
    if c["kind"] == "reorder":
        n = c["seqs"] * c["beams"]
        st["moves"] = S.cache_moves(ints(n * c["page"]), ints(n * c["page"]), n_groups=n)
        st["table_out"] = torch.empty_like(st["table"])
        return
    st["batch"] = S.kv_batch(st["row_start"], st["kv_len"], st["table"], st["rows"], st["most"])
    if c["kind"] == "commit":
        st["positions"], st["masks"] = ints(st["rows"]), ints(st["rows"], st["words"])
        st["tree"] = S.draft_tree(st["parents"], st["positions"], st["masks"])
        st["moves"] = S.cache_moves(ints(st["rows"]), ints(st["rows"]), st["row_start"])
        st["path"], st["next"] = ints(st["rows"]), ints(c["seqs"])
        st["n_accepted"], st["new_len"] = ints(c["seqs"]), ints(c["seqs"])
        return
    st["tree"] = S.draft_tree(st["parents"], st["positions"], st["masks"])
    st["cache"] = S.kv_cache(st["k_pages"], st["v_pages"], st.get("k_scales"), st.get("v_scales"))
    st["attend"] = S.attend_params(num_q_heads=c["hq"], n_sink=c["sink"], n_local=c["local"])
    st["out"] = torch.empty(st["rows"], c["hq"], DH, dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.empty(st["rows"], c["hq"], device="cuda")
    size = S.scale_cache_attend_workspace_size(st["attend"], st["cache"], st["batch"])
    st["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(st["ws"])


def _run_own(st):
    from paper_2609_31568_gb300 import scale as S

    kind = st["c"]["kind"]
    if kind == "attend":
        S.scale_cache_attend_tree(st["attend"], st["tree"], st["cache"], st["batch"], st["q"], st["out"], st["lse"],
                                  st["ws"])
        return {"out": st["out"], "lse": st["lse"]}
    if kind == "beam":
        S.scale_beam_select(st["beam"], st["logits"], st["scores"], st["best"], st["best_beams"], st["best_tokens"],
                            st["ws"])
        return {"score": st["best"], "beam": st["best_beams"], "token": st["best_tokens"]}
    if kind == "reorder":
        S.scale_beam_reorder(st["caches"], st["table"], st["kv_len"], st["parents"], st["table_out"], st["moves"])
        S.scale_cache_move(st["caches"], st["moves"])
        return {"table": st["table_out"], **_held(st)}
    S.scale_tree_plan(st["tree"], st["batch"])
    S.scale_tree_accept(st["tree"], st["caches"], st["batch"], st["tokens"], st["choices"], st["first"],
                        st["n_accepted"], st["path"], st["next"], st["new_len"], st["moves"])
    S.scale_cache_move(st["caches"], st["moves"])
    return {"positions": st["positions"], "masks": st["masks"], "n_accepted": st["n_accepted"], "path": st["path"],
            "next": st["next"], "new_len": st["new_len"], **_held(st)}


def _held(st):
    """The caches: their rows, 8-bit ones as the values of their codes beside their scales."""
    return {x: st[x] for x in ("k_pages", "v_pages", "k_scales", "v_scales") if x in st}


# ---------------------------------------------------------------- the plain forms


def _plan_plain(st):
    """Position of every row (-1: no node) and its ancestors and itself as bits, int32 [rows][words]."""
    rows, local, parent = st["rows"], st["local"], st["parents"].long()
    start = st["row_start"].long()[st["seq"]]
    every = torch.arange(rows, device="cuda")
    bad = (parent < -1) | (parent >= local)
    seen = torch.zeros(rows, 32 * st["words"], dtype=torch.bool, device="cuda")
    at, depth = local.clone(), torch.zeros_like(local)
    gone = torch.zeros(rows, dtype=torch.bool, device="cuda")
    while bool((at >= 0).any()):
        on = at >= 0
        seen[every[on], at[on]] = True
        row = start + at.clamp(min=0)
        gone |= on & bad[row]
        at = torch.where(on & ~bad[row], parent[row], -1)
        depth += at >= 0
    seen &= ~gone[:, None]
    weight = torch.tensor([1 << i for i in range(32)], device="cuda")
    words = (seen.view(rows, -1, 32) * weight).sum(-1)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
    return torch.where(gone, -1, st["base"][st["seq"]] + depth).int(), words


def _commit_plain(st):
    c, page = st["c"], st["c"]["page"]
    positions, masks = _plan_plain(st)
    seqs, n = c["seqs"], st["most"]
    here = (st["seq"], st["local"])
    parent = torch.full((seqs, n), -3, device="cuda")
    parent[here] = torch.where(positions >= 0, st["parents"].long(), -3)
    token = torch.full((seqs, n), -1, device="cuda")
    token[here] = st["tokens"].long()
    choice = torch.zeros(seqs, n, dtype=torch.long, device="cuda")
    choice[here] = st["choices"].long()
    at, want = torch.full((seqs,), -1, device="cuda"), st["first"].long()
    count = torch.zeros(seqs, dtype=torch.long, device="cuda")
    path = torch.full((seqs, n), -1, device="cuda")
    on = torch.ones(seqs, dtype=torch.bool, device="cuda")
    index = torch.arange(n, device="cuda")
    every = torch.arange(seqs, device="cuda")
    while bool(on.any()):
        fits = (parent == at[:, None]) & (token == want[:, None])
        down = torch.where(fits, index, n).amin(-1)
        on &= down < n
        path[every[on], count[on]] = down[on]
        count += on
        at = torch.where(on, down, at)
        want = torch.where(on, choice[every, at.clamp(min=0)], want)
    step, node = (path >= 0).nonzero()[:, 1], path[path >= 0]
    b = (path >= 0).nonzero()[:, 0]
    moved = node != step
    b, src, dst = b[moved], (st["base"][b] + node)[moved], (st["base"][b] + step)[moved]
    table = st["table"].long()
    _move(st, table[b, src // page], src % page, table[b, dst // page], dst % page)
    return {"positions": positions, "masks": masks, "n_accepted": count.int(), "path": path[here].int(),
            "next": want.int(), "new_len": (st["base"] + count).int(), **_held(st)}


def _move(st, src_page, src_slot, dst_page, dst_slot):
    """Rows of all layers' caches from places to places, all read before any is written."""
    for x in ("k_pages", "v_pages"):
        if x in st:
            rows = st[x].view(torch.uint8 if st[x].dtype == torch.float8_e4m3fn else st[x].dtype)
            rows[:, dst_page, dst_slot] = rows[:, src_page, src_slot]
    for x in ("k_scales", "v_scales"):
        if x in st:
            scales = st[x].transpose(2, 3)
            scales[:, dst_page, dst_slot] = scales[:, src_page, src_slot]


def _reorder_plain(st):
    c, page, n = st["c"], st["c"]["page"], st["c"]["beams"]
    parent = st["parents"].long()
    index = torch.arange(n, device="cuda")
    child = parent[:, None, :] == index[:, None]               # [group][parent][child]
    keeper = torch.where(child, index, n).amin(-1)             # the first beam that goes on from it
    keeper = torch.where(parent == index, index, keeper)       # or itself
    keeps = keeper.gather(1, parent) == index
    dead = keeper == n
    # the k-th beam that keeps nothing takes the pages of the k-th that nobody goes on from
    order = torch.argsort(dead.int(), dim=1, descending=True, stable=True)
    rank = ((~keeps).cumsum(1) - 1).clamp(min=0)
    donor = torch.where(keeps, parent, order.gather(1, rank))
    first = torch.arange(c["seqs"], device="cuda")[:, None] * n
    parent, donor = (first + parent).flatten(), (first + donor).flatten()
    full = st["kv_len"].long() // page                         # complete pages
    column = torch.arange(st["table"].shape[1], device="cuda")
    table = torch.where(column < full[:, None], st["table"][parent], st["table"][donor])
    slot = torch.arange(page, device="cuda")
    copied = (donor != parent)[:, None] & (slot < (st["kv_len"].long() % page)[:, None])
    b, slots = copied.nonzero()[:, 0], copied.nonzero()[:, 1]
    old = st["table"].long()
    _move(st, old[parent[b], full[b]], slots, old[donor[b], full[b]], slots)
    return {"table": table, **_held(st)}


def _beam_plain(st):
    """Scores in 64 bits: that of two beams' continuations may differ by less than 32 bits hold."""
    c = st["c"]
    z = st["logits"].double()
    top = z.amax(-1, keepdim=True)
    z = z - (top + (z - top).exp().sum(-1, keepdim=True).log())
    z = (z.view(c["seqs"], c["beams"], -1) + st["scores"].double()[..., None]).flatten(1)
    # stable among equals: the lowest beam and token
    limit = z.topk(c["best"], dim=-1).values[:, -1:]
    most = int((z >= limit).sum(-1).max())
    index = torch.arange(z.shape[1], device="cuda")
    kept = torch.where(z >= limit, index, z.shape[1]).topk(most, dim=-1, largest=False).values
    value = torch.where(kept < z.shape[1], z.gather(1, kept.clamp(max=z.shape[1] - 1)), -math.inf)
    value, at = value.sort(dim=-1, descending=True, stable=True)
    value, kept = value[:, : c["best"]], kept.gather(1, at)[:, : c["best"]]
    return {"score": value.float(), "beam": (kept // c["vocab"]).int(), "token": (kept % c["vocab"]).int()}


def _values(pages, scales):
    """fp32 values of pages [..., page, hkv, 128] (scales [..., hkv, page])."""
    if scales is None:
        return pages.float()
    return pages.float() * _power(scales.transpose(-1, -2)[..., None].int() - 127)


def _seen_new(st):
    """Which of its sequence's new tokens a row sees, [rows][most], from the masks' bits."""
    bits = (st["masks"][..., None] >> torch.arange(32, device="cuda")) & 1
    return bits.flatten(1)[:, : st["most"]] != 0


def _attend_plain(st):
    """Sequences side by side, padded to the longest; every KV head's query heads share its keys."""
    c = st["c"]
    hkv, g, seqs = c["hkv"], c["hq"] // c["hkv"], len(st["lens"])
    new, top = st["most"], max(n for _, n in st["lens"])
    table = st["table"].clamp(min=0).long()
    kv = [_values(st[x + "_pages"].view(torch.uint8 if c["cache"] == "e4m3" else torch.bfloat16)[table].view(
        st[x + "_pages"].dtype), None if x + "_scales" not in st else st[x + "_scales"][table])
        .flatten(1, 2)[:, :top].transpose(1, 2).reshape(seqs * hkv, top, DH) for x in "kv"]
    here = (st["seq"], st["local"])
    q = torch.zeros(seqs, new, c["hq"], DH, device="cuda")
    q[here] = st["q"].float()
    q = q.view(seqs, new, hkv, g, DH).permute(0, 2, 3, 1, 4).reshape(seqs * hkv, g * new, DH)
    z = torch.bmm(q, kv[0].transpose(1, 2)).mul_(1.0 / math.sqrt(DH)).view(seqs, hkv * g, new, top)
    pos = torch.full((seqs, new), -1, device="cuda")
    pos[here] = st["positions"].long()
    t = torch.arange(top, device="cuda")
    hidden = (t >= st["base"][:, None, None]).expand(seqs, new, top) | (pos[..., None] < 0)
    if c["local"] >= 0:
        hidden |= (t < pos[..., None] - c["local"]) & (t >= c["sink"])
    row, node = _seen_new(st).nonzero().unbind(1)
    hidden[st["seq"][row], st["local"][row], st["base"][st["seq"][row]] + node] = False
    z.masked_fill_(hidden[:, None], -math.inf)
    top_z = z.amax(-1, keepdim=True)
    z.sub_(top_z.clamp(min=-1e30)).exp_()
    total = z.sum(-1, keepdim=True)
    out = torch.bmm(z.view(seqs * hkv, g * new, top), kv[1]).view(seqs, hkv * g, new, DH)
    out /= total.clamp(min=1e-30)
    lse = (total.log() + top_z)[..., 0]
    return {"out": out.transpose(1, 2)[here].bfloat16(), "lse": lse.transpose(1, 2)[here]}


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _attend_plain, "beam": _beam_plain, "reorder": _reorder_plain,
            "commit": _commit_plain}[state["c"]["kind"]](state)


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    c = dict(case)
    if c["kind"] == "beam":
        rows = c["seqs"] * c["beams"]
        size = 2 if c["type"] == "bf16" else 4
        return {"bytes": rows * (c["vocab"] * size + 4) + c["seqs"] * c["best"] * 12, "flops": 4 * rows * c["vocab"]}
    lens = _lens(c)
    row = DH * 2
    held = DH + 1 if c["cache"] == "e4m3" else row  # a row of the cache
    if c["kind"] == "reorder":
        # tables read and written; about half of the beams' unfinished pages read and written
        tables = sum(2 * 4 * c["beams"] * (n // c["page"] + 2) for _, n in lens)
        rows = sum(c["beams"] // 2 * (n % c["page"]) for _, n in lens)
        return {"bytes": tables + c["layers"] * rows * c["hkv"] * 2 * held * 2, "flops": 0}
    new = sum(a for a, _ in lens)
    words = -(-max(a for a, _ in lens) // 32)
    if c["kind"] == "commit":
        # parents, tokens and choices read, positions, masks and paths written, three rows of a tree moved
        moved = sum(min(3, a - 1) for a, _ in lens)
        return {"bytes": new * (5 * 4 + 4 * words) + c["layers"] * moved * c["hkv"] * 2 * held * 2, "flops": 0}
    pairs = keys = 0
    for a, n in lens:
        old = n - a
        seen = min(old, c["local"]) + min(c["sink"], max(0, old - c["local"])) if c["local"] >= 0 else old
        pairs += a * (seen + 1 + min(a - 1, 4))
        keys += seen + a
    return {"bytes": new * (c["hq"] * (2 * row + 4) + 4 + 4 * words) + keys * c["hkv"] * 2 * held,
            "flops": 4 * DH * c["hq"] * pairs}


# ---------------------------------------------------------------- in 64 bits


def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_rows(st, x, b, n):
    """Keys or values [n][hkv][128] of sequence b, from the pages."""
    page = st["c"]["page"]
    pages = st["table"][b, : -(-n // page)].long()
    if st["c"]["cache"] == "bf16":
        return st[x + "_pages"][pages].double().flatten(0, 1)[:n]
    code = st[x + "_pages"].view(torch.uint8)[pages].long()
    e = st[x + "_scales"][pages].long().transpose(1, 2)[..., None] - 127
    power, low = (code >> 3) & 15, (code & 7).double()
    size = torch.where(power > 0, (8 + low) * _exact_power(power - 10), low * 2.0 ** -9)
    return (torch.where(code > 127, -size, size) * _exact_power(e)).flatten(0, 1)[:n]


def _exact_tree(parent):
    """Nodes from the root to every node, itself last; none for what has no place."""
    ways = []
    for i, p in enumerate(parent):
        if p == -1:
            ways.append([i])
        else:
            ways.append(ways[p] + [i] if 0 <= p < i and ways[p] else [])
    return ways


def _exact_attend(st):
    c, out, lse, at = st["c"], [], [], 0
    for b, (a, n) in enumerate(st["lens"]):
        k, v = (_exact_rows(st, x, b, n) for x in "kv")
        ways = _exact_tree(st["parents"][at: at + a].tolist())
        seen = torch.zeros(a, n, dtype=torch.bool)
        for i, way in enumerate(ways):
            if not way:
                continue
            p = n - a + len(way) - 1
            seen[i, : n - a] = True
            if c["local"] >= 0:
                seen[i, c["sink"]: max(c["sink"], min(n - a, p - c["local"]))] = False
            seen[i, [n - a + x for x in way]] = True
        seen = seen.cuda()
        o = torch.empty(a, c["hq"], DH, dtype=torch.float64, device="cuda")
        s = torch.empty(a, c["hq"], dtype=torch.float64, device="cuda")
        for h in range(c["hq"]):
            kvh = h // (c["hq"] // c["hkv"])
            z = st["q"][at: at + a, h].double() @ k[:, kvh].t() / math.sqrt(DH)
            z = torch.where(seen, z, -math.inf)
            s[:, h] = torch.logsumexp(z, -1)
            o[:, h] = torch.softmax(z, -1).nan_to_num(0.0) @ v[:, kvh]
        out.append(o)
        lse.append(s)
        at += a
    return {"out": torch.cat(out), "lse": torch.cat(lse)}


def _exact_move(st, moves):
    """Rows (page, slot) of all layers to (page, slot), one after another."""
    held = {x: st[x].view(torch.uint8) if st[x].element_size() == 1 else st[x] for x in _held(st)}
    old = {x: {} for x in held}
    for (p, s), _ in moves:
        for x, t in held.items():
            old[x][p, s] = (t[:, p, :, s] if x.endswith("scales") else t[:, p, s]).clone()
    for src, (p, s) in moves:
        for x, t in held.items():
            if x.endswith("scales"):
                t[:, p, :, s] = old[x][src]
            else:
                t[:, p, s] = old[x][src]
    return {x: st[x].double() if x.endswith("pages") else st[x] for x in held}


def _exact_commit(st):
    page, at, moves = st["c"]["page"], 0, []
    got = {x: [] for x in ("positions", "masks", "n_accepted", "path", "next", "new_len")}
    table = st["table"].tolist()
    tokens, choices, first = st["tokens"].tolist(), st["choices"].tolist(), st["first"].tolist()
    for b, (a, n) in enumerate(st["lens"]):
        base = n - a
        parent = st["parents"][at: at + a].tolist()
        ways = _exact_tree(parent)
        got["positions"] += [base + len(w) - 1 if w else -1 for w in ways]
        for w in ways:
            words = np.zeros(st["words"], np.uint32)
            for x in w:
                words[x // 32] |= np.uint32(1 << (x % 32))
            got["masks"].append(words.view(np.int32))
        path, want, p = [], first[b], -1
        while True:
            down = [i for i in range(a) if ways[i] and parent[i] == p and tokens[at + i] == want]
            if not down:
                break
            p = down[0]
            path.append(p)
            want = choices[at + p]
        place = lambda t: (table[b][t // page], t % page)  # noqa: E731
        moves += [(place(base + x), place(base + i)) for i, x in enumerate(path) if x != i]
        got["n_accepted"].append(len(path))
        got["path"] += path + [-1] * (a - len(path))
        got["next"].append(want)
        got["new_len"].append(base + len(path))
        at += a
    ints = {x: torch.from_numpy(np.array(y, dtype=np.int32)) for x, y in got.items()}
    return {**ints, **_exact_move(st, moves)}


def _exact_reorder(st):
    c, page, n, moves = st["c"], st["c"]["page"], st["c"]["beams"], []
    old, new = st["table"].tolist(), []
    for s, (_, length) in enumerate(st["lens"]):
        full, parents = length // page, st["parents"][s].tolist()
        keeper = {}
        for i, p in enumerate(parents):
            keeper.setdefault(p, i)
        keeper.update({i: i for i, p in enumerate(parents) if p == i})
        free = [p for p in range(n) if p not in keeper]
        for i, p in enumerate(parents):
            donor = p if keeper[p] == i else free.pop(0)
            new.append(old[s * n + p][:full] + old[s * n + donor][full:])
            if donor != p:
                moves += [((old[s * n + p][full], t), (old[s * n + donor][full], t)) for t in range(length % page)]
    return {"table": torch.tensor(new, dtype=torch.int32), **_exact_move(st, moves)}


def _exact_beam(st):
    c, got = st["c"], {"score": [], "beam": [], "token": []}
    for s in range(c["seqs"]):
        z = st["logits"][s * c["beams"]: (s + 1) * c["beams"]].double()
        z = (st["scores"][s].double()[:, None] + z - torch.logsumexp(z, -1, keepdim=True)).flatten()
        picks = []
        for _ in range(c["best"]):
            top = z.max()
            picks.append((top, (z == top).nonzero()[0, 0]))
            z[picks[-1][1]] = -math.inf
        flat = torch.stack([x for _, x in picks])
        got["score"].append(torch.stack([x for x, _ in picks]))
        got["beam"].append((flat // c["vocab"]).int())
        got["token"].append((flat % c["vocab"]).int())
    return {x: torch.stack(y) for x, y in got.items()}


def exact(case, seed):
    st = prepare(case, seed)
    return {"attend": _exact_attend, "beam": _exact_beam, "reorder": _exact_reorder,
            "commit": _exact_commit}[case["kind"]](st)

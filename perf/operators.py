"""The operators of a serving step over a paged K/V cache, as they are measured.

Kinds of case (``kind``):

- ``rope``: rotary positions with one axis (text) or three (time, height, width) on the queries and
  keys of ``n`` tokens; ``fused``: they are slices of the rows a joint QKV projection wrote; ``order``
  is how the pairs are taken (``half``: dimension i with i + 64; ``adjacent``: 2 i with 2 i + 1);
- ``append``: new tokens go into the cache, their keys (and queries) turned to their positions on the
  way (``axes`` > 0), and are read back as bf16, as the selection of later layers reads them;
- ``read``: whole sequences read from the cache as contiguous bf16 rows;
- ``attend``: new tokens attend causally to their sequences in the cache (``sink`` leading tokens and
  the last ``local`` tokens before a token; ``local`` -1: all of them), with the logarithm of the
  softmax sum of every row.

``hq`` / ``hkv`` query and KV heads (head size 128, bf16), ``cache`` the cache's type (``bf16``, or
``e4m3`` with a power-of-two scale per token and head), ``page`` tokens of a page, ``seqs`` sequences
whose new tokens spread from ``new_lo`` to ``new_hi`` and whose lengths (new tokens included) from
``len_lo`` to ``len_hi``, geometrically.
"""

from __future__ import annotations

import math

import torch

own = False

DH = 128
ROPE_BASE = 500000.0
E4M3_MAX = 448.0
LOW_EXP = -100  # the smallest scale is 2^LOW_EXP


def listed():
    llama = dict(hq=32, hkv=8)
    return [
        # One decode step's 16 tokens, a million tokens into their sequences: latency.
        dict(name="rope-16", kind="rope", n=16, axes=1, order="half", fused=False, far=1048576, **llama),
        # A 32K prompt with images, on the slices of a joint projection (28 query heads on 4 KV heads).
        dict(name="rope-32k-3axes", kind="rope", n=32709, axes=3, order="half", fused=True, far=0, hq=28, hkv=4),
        # One decode step of 64 sequences into an 8-bit cache.
        dict(name="append-64x1", kind="append", cache="e4m3", page=64, seqs=64, new_lo=1, new_hi=1, len_lo=500,
             len_hi=30000, axes=1, **llama),
        # A chunk of prompt pieces of odd lengths, bf16 pages of 16 tokens.
        dict(name="append-ragged-bf16", kind="append", cache="bf16", page=16, seqs=7, new_lo=33, new_hi=2500,
             len_lo=333, len_hi=9000, axes=3, hq=28, hkv=4),
        # An outer chunk of 8192 tokens into an 8-bit cache.
        dict(name="append-8k", kind="append", cache="e4m3", page=64, seqs=1, new_lo=8192, new_hi=8192, len_lo=65536,
             len_hi=65536, axes=1, **llama),
        # A short sequence read back; and a 128K one, 8-bit.
        dict(name="read-4k-bf16", kind="read", cache="bf16", page=16, seqs=1, len_lo=4096, len_hi=4096, **llama),
        dict(name="read-128k", kind="read", cache="e4m3", page=64, seqs=1, len_lo=131071, len_hi=131071, **llama),
        # The smallest decode step: one token at 4K on 4 query heads.
        dict(name="attend-1x4k", kind="attend", cache="bf16", page=64, seqs=1, new_lo=1, new_hi=1, len_lo=4096,
             len_hi=4096, sink=0, local=-1, hq=4, hkv=1),
        # One token at the end of 128K, 8-bit: the split of one long sequence.
        dict(name="attend-1x128k", kind="attend", cache="e4m3", page=64, seqs=1, new_lo=1, new_hi=1, len_lo=131071,
             len_hi=131071, sink=0, local=-1, **llama),
        # A decode step of 48 sequences of very different lengths, bf16 pages of 16 tokens.
        dict(name="attend-48-ragged", kind="attend", cache="bf16", page=16, seqs=48, new_lo=1, new_hi=1, len_lo=130,
             len_hi=30000, sink=0, local=-1, hq=28, hkv=4),
        # Prompt pieces beside decoding sequences (1 to 700 new tokens), sinks and a window, 8-bit.
        dict(name="attend-mixed-window", kind="attend", cache="e4m3", page=64, seqs=9, new_lo=1, new_hi=700,
             len_lo=1000, len_hi=12000, sink=64, local=4000, **llama),
        # An outer chunk's half, 4096 tokens, over a 64K sequence: the largest.
        dict(name="attend-4k-over-64k", kind="attend", cache="bf16", page=64, seqs=1, new_lo=4096, new_hi=4096,
             len_lo=65536, len_hi=65536, sink=0, local=-1, **llama),
    ]


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["rope", "append", "append", "read", "attend", "attend", "attend", "attend"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (28, 4), (16, 8), (8, 1), (6, 2), (4, 4)])
    c = dict(kind=kind, hq=hq, hkv=hkv)
    if kind == "rope":
        c.update(n=size(1, 32768), axes=rng.choice([1, 3]), order=rng.choice(["half", "adjacent"]),
                 fused=rng.random() < 0.5, far=rng.choice([0, 100000, 1048576]))
        return c
    c.update(cache=rng.choice(["bf16", "e4m3"]), page=rng.choice([16, 64, 128, 48]))
    if kind == "read":
        hi = size(300, 100000)
        seqs = min(size(1, 40), max(1, 130000 // hi))
        c.update(seqs=seqs, len_lo=max(1, int(hi * rng.random())) if seqs > 1 else hi, len_hi=hi)
        return c
    if kind == "append":
        seqs = size(1, 64)
        new_hi = size(1, max(1, 8192 // seqs))
        len_hi = max(new_hi, size(100, 20000))
        c.update(seqs=seqs, new_lo=size(1, new_hi) if seqs > 1 else new_hi, new_hi=new_hi,
                 len_lo=max(1, len_hi // 8) if seqs > 1 else len_hi, len_hi=len_hi, axes=rng.choice([0, 1, 3]))
        return c
    window = dict(sink=rng.choice([0, 4, 64, 128]), local=rng.choice([256, 1000, 4096])) if rng.random() < 0.3 else \
        dict(sink=0, local=-1)
    c.update(window)
    if rng.random() < 0.5:  # a decode step
        seqs = size(1, 64)
        len_hi = size(100, 120000 if seqs == 1 else min(30000, 1600000 // seqs))
        c.update(seqs=seqs, new_lo=1, new_hi=rng.choice([1, 1, 1, 3]), len_lo=max(1, len_hi // rng.choice([1, 8, 60])),
                 len_hi=len_hi)
    else:
        new_hi = size(2, 4096)
        len_hi = max(new_hi, size(500, 60000))
        seqs = min(size(1, 8), max(1, 100000000 // (new_hi * len_hi)))
        c.update(seqs=seqs, new_lo=size(1, new_hi), new_hi=new_hi, len_lo=max(1, len_hi // rng.choice([1, 8])),
                 len_hi=len_hi)
    if c["seqs"] == 1:
        c.update(new_lo=c["new_hi"], len_lo=c["len_hi"])
    return c


def _spread(lo, hi, n, turn):
    """n sizes from lo to hi, evenly on a logarithmic scale, in an order of their own."""
    if n == 1:
        return [hi]
    up = [int(round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]
    return [up[i * turn % n] for i in range(n)] if math.gcd(turn, n) == 1 else up[::-1]


def _lens(c):
    """(new tokens, length with them) of every sequence."""
    lens = _spread(c["len_lo"], c["len_hi"], c["seqs"], 7)
    if c["kind"] == "read":
        return [(n, n) for n in lens]
    new = _spread(c["new_lo"], c["new_hi"], c["seqs"], 5)
    return [(min(a, n), n) for a, n in zip(new, lens)]


# ---------------------------------------------------------------- inputs


def _mixture(gen, n, heads, groups):
    """[n][heads][128] fp32: a component of norm 3 of the head's group plus N(0, 1)."""
    kvh = torch.arange(heads, device="cuda") // (heads // groups.shape[0])
    ids = torch.randint(0, groups.shape[1], (n, heads), generator=gen, device="cuda")
    return groups[kvh, ids] + torch.randn(n, heads, DH, generator=gen, device="cuda")


def _groups(gen, hkv):
    x = torch.randn(hkv, 256, DH, generator=gen, device="cuda")
    return 3.0 * x / x.norm(dim=-1, keepdim=True)


def _positions(gen, n, axes, first):
    """int32 [axes][n]: text counts up; with three axes, images of 24 x 32 patches lie between texts."""
    t = torch.arange(n, device="cuda")
    if axes == 1:
        return (first + t).int()[None].contiguous()
    in_image = (t // 1000) % 2 == 1
    at = t % 1000
    pos = torch.stack([first + t - torch.where(in_image, at, 0), first + t - at + torch.where(in_image, at // 32, at),
                       first + t - at + torch.where(in_image, at % 32, at)])
    return pos.int().contiguous()


def _axis_of_pair(axes):
    """The axis whose position turns pair i: three axes take 16, 24 and 24 pairs."""
    return [0] * 64 if axes == 1 else [0] * 16 + [1] * 24 + [2] * 24


def _power(e):
    """2^e of whole numbers e in -126..127, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """e4m3 codes (uint8) of fp32 rows [..., 128] and the exponents + 127 of their scales (uint8)."""
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=LOW_EXP)  # amax <= 448 * 2^e
    e = torch.where(amax > 0, e, LOW_EXP)
    codes = (x * _power(-e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, (e + 127).to(torch.uint8)


def _pool(c, gen, lens):
    """An empty cache with a few spare pages, and the sequences' page table."""
    page, hkv = c["page"], c["hkv"]
    width = max(-(-n // page) for _, n in lens)
    used = sum(-(-n // page) for _, n in lens)
    order = torch.randperm(used + 3, generator=gen, device="cuda").int()
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, (_, n) in enumerate(lens):
        p = -(-n // page)
        table[b, :p] = order[at: at + p]
        at += p
    st = {"table": table}
    for x in "kv":
        kind = torch.uint8 if c["cache"] == "e4m3" else torch.bfloat16
        st[x + "_pages"] = torch.zeros(used + 3, page, hkv, DH, dtype=kind, device="cuda")
        if c["cache"] == "e4m3":
            st[x + "_scales"] = torch.full((used + 3, hkv, page), 127, dtype=torch.uint8, device="cuda")
    return st


def _fill(st, c, gen, lens, groups):
    """Keys and values of every token of the sequences."""
    page = c["page"]
    for b, (_, n) in enumerate(lens):
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
                    st[x + "_pages"][pages] = codes
                    st[x + "_scales"][pages] = e.transpose(1, 2).contiguous()
                else:
                    st[x + "_pages"][pages] = rows.bfloat16()


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv = c["hq"], c["hkv"]
    groups = _groups(gen, hkv)
    st = {"c": c}
    axes = c.get("axes", 0)
    if axes:
        st["inv_freq"] = ROPE_BASE ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
        st["axis"] = torch.tensor(_axis_of_pair(axes), device="cuda")
    if c["kind"] == "rope":
        n = c["n"]
        rows = [_mixture(gen, n, hq, groups).bfloat16(), _mixture(gen, n, hkv, groups).bfloat16()]
        if c["fused"]:
            joint = torch.empty(n, (hq + 2 * hkv) * DH, dtype=torch.bfloat16, device="cuda")
            views = [joint[:, : hq * DH].view(n, hq, DH), joint[:, hq * DH: (hq + hkv) * DH].view(n, hkv, DH)]
            for v, r in zip(views, rows):
                v.copy_(r)
            rows = views
        st["q"], st["k"] = rows
        st["positions"] = _positions(gen, n, axes, c["far"])
    else:
        lens = _lens(c)
        st["lens"] = lens
        st.update(_pool(c, gen, lens))
        starts = [0]
        for a, _ in lens:
            starts.append(starts[-1] + a)
        st["rows"] = starts[-1]
        st["row_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        st["kv_len"] = torch.tensor([n for _, n in lens], dtype=torch.int32, device="cuda")
        if c["kind"] != "append":
            _fill(st, c, gen, lens, groups)
        if c["kind"] != "read":
            st["q"] = _mixture(gen, st["rows"], hq, groups).bfloat16()
        if c["kind"] == "append":
            st["k"] = _mixture(gen, st["rows"], hkv, groups).bfloat16()
            st["v"] = torch.randn(st["rows"], hkv, DH, generator=gen, device="cuda").bfloat16()
            if axes:
                first = torch.cat([_positions(gen, a, axes, n - a) for a, n in lens], dim=1)
                st["positions"] = first.contiguous()
        # where every row lies: its sequence, its position there, its row of the pool
        st["seq"] = torch.repeat_interleave(torch.arange(len(lens), device="cuda"),
                                            torch.tensor([a for a, _ in lens], device="cuda"))
        back = st["row_start"].long()[st["seq"] + 1] - torch.arange(st["rows"], device="cuda")
        st["pos"] = st["kv_len"].long()[st["seq"]] - back
        st["page_of"] = st["table"][st["seq"], st["pos"] // c["page"]].long()
        st["slot_of"] = st["pos"] % c["page"]
    if own:
        _handles(st)
    return st


# ---------------------------------------------------------------- the framework's calls


def _handles(st):
    """Descriptors, workspace and output rows, as a program keeps them between calls."""
    from paper_2609_31568_gb300 import scale as S

    c = st["c"]
    empty = lambda n, h: torch.empty(n, h, DH, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    if c.get("axes"):
        st["rope"] = S.rope_axes(st["inv_freq"], st["positions"], _axis_of_pair(c["axes"]),
                                 c.get("order") == "adjacent")
    if c["kind"] == "rope":
        st["q_out"], st["k_out"] = empty(c["n"], c["hq"]), empty(c["n"], c["hkv"])
        return
    st["cache"] = S.kv_cache(st["k_pages"], st["v_pages"], st.get("k_scales"), st.get("v_scales"))
    st["batch"] = S.kv_batch(st["row_start"], st["kv_len"], st["table"], st["rows"], max(a for a, _ in st["lens"]))
    if c["kind"] == "append" and c["axes"]:
        st["q_out"] = empty(st["rows"], c["hq"])
    if c["kind"] != "attend":
        st["k_out"], st["v_out"] = empty(st["rows"], c["hkv"]), empty(st["rows"], c["hkv"])
        return
    st["attend"] = S.attend_params(num_q_heads=c["hq"], n_sink=c["sink"], n_local=c["local"])
    st["out"] = empty(st["rows"], c["hq"])
    st["lse"] = torch.empty(st["rows"], c["hq"], device="cuda")
    size = S.scale_cache_attend_workspace_size(st["attend"], st["cache"], st["batch"])
    st["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(st["ws"])


def _run_own(st):
    from paper_2609_31568_gb300 import scale as S

    kind = st["c"]["kind"]
    if kind == "rope":
        S.scale_rope(st["rope"], st["q"], st["k"], st["q_out"], st["k_out"])
        return {"q": st["q_out"], "k": st["k_out"]}
    if kind == "append":
        if "rope" in st:
            S.scale_cache_append(st["cache"], st["batch"], st["k"], st["v"], st["rope"], st["q"], st["q_out"])
        else:
            S.scale_cache_append(st["cache"], st["batch"], st["k"], st["v"])
        S.scale_cache_read(st["cache"], st["batch"], st["k_out"], st["v_out"])
        return {"q": st.get("q_out"), "k": st["k_out"], "v": st["v_out"]}
    if kind == "read":
        S.scale_cache_read(st["cache"], st["batch"], st["k_out"], st["v_out"])
        return {"k": st["k_out"], "v": st["v_out"]}
    S.scale_cache_attend(st["attend"], st["cache"], st["batch"], st["q"], st["out"], st["lse"], st["ws"])
    return {"out": st["out"], "lse": st["lse"]}


# ---------------------------------------------------------------- the plain forms


def _turned(st, x, order):
    """x [n][heads][128] turned to its positions, fp32; the angles in 64 bits."""
    angle = st["positions"][st["axis"]].double().t() * st["inv_freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float()
    if order == "adjacent":
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    a, b = x[..., :64], x[..., 64:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _values(pages, scales):
    """fp32 values of pages [..., page, hkv, 128] (scales [..., hkv, page])."""
    if scales is None:
        return pages.float()
    return pages.view(torch.float8_e4m3fn).float() * _power(scales.transpose(-1, -2)[..., None].int() - 127)


def _rows_back(st, x):
    pages, scales = st[x + "_pages"], st.get(x + "_scales")
    rows = pages[st["page_of"], st["slot_of"]]
    if scales is None:
        return rows
    e = scales[st["page_of"], :, st["slot_of"]]
    return (rows.view(torch.float8_e4m3fn).float() * _power(e[..., None].int() - 127)).bfloat16()


def _append_plain(st):
    q, k = None, st["k"].float()
    if "positions" in st:
        q, k = _turned(st, st["q"], "half").bfloat16(), _turned(st, k, "half")
    at = (st["page_of"], st["slot_of"])
    for x, rows in (("k", k), ("v", st["v"].float())):
        if st["c"]["cache"] == "e4m3":
            codes, e = _quantise(rows)
            st[x + "_pages"].index_put_(at, codes)
            st[x + "_scales"].transpose(1, 2).index_put_(at, e)
        else:
            st[x + "_pages"].index_put_(at, rows.bfloat16())
    return {"q": q, "k": _rows_back(st, "k"), "v": _rows_back(st, "v")}


def _attend_plain(st):
    """Sequences side by side, padded to the longest; every KV head's query heads share its keys."""
    c = st["c"]
    hkv, g, seqs = c["hkv"], c["hq"] // c["hkv"], len(st["lens"])
    new, top = max(a for a, _ in st["lens"]), max(n for _, n in st["lens"])
    table = st["table"].clamp(min=0).long()
    kv = [_values(st[x + "_pages"][table], None if x + "_scales" not in st else st[x + "_scales"][table])
          .flatten(1, 2)[:, :top].transpose(1, 2).reshape(seqs * hkv, top, DH) for x in "kv"]
    row = torch.arange(st["rows"], device="cuda") - st["row_start"].long()[st["seq"]]
    q = torch.zeros(seqs, new, c["hq"], DH, device="cuda")
    q[st["seq"], row] = st["q"].float()
    pos = torch.full((seqs, new), -1, device="cuda")
    pos[st["seq"], row] = st["pos"]
    q = q.view(seqs, new, hkv, g, DH).permute(0, 2, 3, 1, 4).reshape(seqs * hkv, g * new, DH)
    z = torch.bmm(q, kv[0].transpose(1, 2)).mul_(1.0 / math.sqrt(DH)).view(seqs, hkv * g, new, top)
    t = torch.arange(top, device="cuda")
    hidden = t > pos[..., None]
    if c["local"] >= 0:
        hidden |= (t < pos[..., None] - c["local"]) & (t >= c["sink"])
    z.masked_fill_(hidden[:, None], -math.inf)
    top_z = z.amax(-1, keepdim=True)
    z.sub_(top_z.clamp(min=-1e30)).exp_()
    total = z.sum(-1, keepdim=True)
    out = torch.bmm(z.view(seqs * hkv, g * new, top), kv[1]).view(seqs, hkv * g, new, DH)
    out /= total.clamp(min=1e-30)
    lse = (total.log() + top_z)[..., 0]
    return {"out": out.transpose(1, 2)[st["seq"], row].bfloat16(), "lse": lse.transpose(1, 2)[st["seq"], row]}


def run(state):
    if own:
        return _run_own(state)
    kind = state["c"]["kind"]
    if kind == "rope":
        order = state["c"]["order"]
        return {x: _turned(state, state[x], order).bfloat16() for x in "qk"}
    if kind == "append":
        return _append_plain(state)
    if kind == "read":
        return {x: _rows_back(state, x) for x in "kv"}
    return _attend_plain(state)


# ---------------------------------------------------------------- what a pass cannot do without


def _seen(c, pos):
    """Keys that the token at `pos` attends to."""
    lo = max(0, pos - c["local"]) if c["local"] >= 0 else 0
    return pos + 1 - lo + min(c["sink"], lo)


def work(case):
    c = dict(case)
    row = DH * 2
    if c["kind"] == "rope":
        rows = c["n"] * (c["hq"] + c["hkv"])
        return {"bytes": rows * 2 * row + c["n"] * c["axes"] * 4, "flops": rows * 64 * 6}
    lens = _lens(c)
    held = DH + 1 if c["cache"] == "e4m3" else row  # a row of the cache
    new = sum(a for a, _ in lens)
    if c["kind"] == "read":
        return {"bytes": new * c["hkv"] * 2 * (held + row), "flops": 0}
    if c["kind"] == "append":
        turned = c["hq"] * 2 * row if c["axes"] else 0
        return {"bytes": new * (turned + c["hkv"] * 2 * (row + 2 * held + row) + c["axes"] * 4),
                "flops": new * c["axes"] and new * (c["hq"] + c["hkv"]) * 64 * 6}
    pairs = keys = 0
    for a, n in lens:
        pairs += sum(_seen(c, p) for p in range(n - a, n))
        keys += min(n, _seen(c, n - a) + a - 1)
    return {"bytes": new * c["hq"] * (2 * row + 4) + keys * c["hkv"] * 2 * held, "flops": 4 * DH * c["hq"] * pairs}


# ---------------------------------------------------------------- in 64 bits


def _exact_turn(st, x, order):
    n = x.shape[0]
    angle = torch.empty(n, 64, dtype=torch.float64, device="cuda")
    for i, axis in enumerate(_axis_of_pair(st["positions"].shape[0])):
        angle[:, i] = st["positions"][axis].double() * st["inv_freq"][i]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    x = x.double()
    pairs = x.view(n, -1, 64, 2) if order == "adjacent" else x.view(n, -1, 2, 64).transpose(-1, -2)
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    return y.reshape(x.shape) if order == "adjacent" else y.transpose(-1, -2).reshape(x.shape)


def _exact_power(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_held(x, cache):
    """The values that the cache holds for rows x [..., 128] in 64 bits."""
    if cache != "e4m3":
        return x
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2((amax / E4M3_MAX).clamp(min=2.0 ** LOW_EXP))).long()
    e = e + (amax > E4M3_MAX * _exact_power(e)).long() - (amax <= E4M3_MAX * _exact_power(e - 1)).long()  # log2 rounds
    e = e.clamp(min=LOW_EXP)
    y = x * _exact_power(-e)
    step = _exact_power((y.abs().clamp(min=2.0 ** -6).view(torch.int64) >> 52) - 1023 - 3)  # 3 bits, exponents from -6
    return torch.round(y / step) * step * _exact_power(e)


def _exact_rows(st, x, b, n):
    """Keys or values [n][hkv][128] of sequence b, from the pages."""
    page = st["c"]["page"]
    pages = st["table"][b, : -(-n // page)].long()
    rows = st[x + "_pages"][pages]
    if st["c"]["cache"] == "e4m3":
        e = st[x + "_scales"][pages].long().transpose(1, 2)[..., None] - 127
        code = rows.long()
        power, low = (code >> 3) & 15, (code & 7).double()
        size = torch.where(power > 0, (8 + low) * _exact_power(power - 10), low * 2.0 ** -9)
        rows = torch.where(code > 127, -size, size) * _exact_power(e)
    return rows.double().flatten(0, 1)[:n]


def exact(case, seed):
    c = dict(case)
    if c["kind"] == "attend" and work(c)["flops"] > 9e12:
        return None
    st = prepare(case, seed)
    if c["kind"] == "rope":
        return {x: _exact_turn(st, st[x], c["order"]) for x in "qk"}
    if c["kind"] == "append":
        q, k = None, st["k"].double()
        if c["axes"]:
            q, k = _exact_turn(st, st["q"].double(), "half"), _exact_turn(st, k, "half")
        return {"q": q, "k": _exact_held(k, c["cache"]), "v": _exact_held(st["v"].double(), c["cache"])}
    got = {"k": [], "v": [], "out": [], "lse": []}
    at = 0
    for b, (a, n) in enumerate(st["lens"]):
        k, v = (_exact_rows(st, x, b, n) for x in "kv")
        if c["kind"] == "read":
            got["k"].append(k)
            got["v"].append(v)
            continue
        t, p = torch.arange(n, device="cuda"), torch.arange(n - a, n, device="cuda")[:, None]
        seen = t <= p
        if c["local"] >= 0:
            seen &= (t >= p - c["local"]) | (t < c["sink"])
        out = torch.empty(a, c["hq"], DH, dtype=torch.float64, device="cuda")
        lse = torch.empty(a, c["hq"], dtype=torch.float64, device="cuda")
        for h in range(c["hq"]):
            kvh = h // (c["hq"] // c["hkv"])
            z = st["q"][at: at + a, h].double() @ k[:, kvh].t() / math.sqrt(DH)
            z = torch.where(seen, z, -math.inf)
            lse[:, h] = torch.logsumexp(z, -1)
            out[:, h] = torch.softmax(z, -1) @ v[:, kvh]
        got["out"].append(out)
        got["lse"].append(lse)
        at += a
    return {x: torch.cat(y) for x, y in got.items() if y}

"""Drafted trees over a paged cache against plain references: positions and masks, attention, the walk, moved rows, and
a step of them together."""

import math
import random

import numpy as np
import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _branch import accept, apply_moves, as_words, attend_tree64, plan, random_parents, ways
from _cache import Batch
from paper_2609_31568_gb300 import scale as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    pkg.build()
    S.load()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same_bits(x, y):
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


def within(got, want, tol, what=""):
    got = got.double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    fine = torch.isfinite(want)
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or over.max() <= 0, f"{what}: over by {over.max():.3e} of {tol[fine].max():.3e}"


def trees(news, seed, **how):
    """Parents of every sequence."""
    rng = random.Random(seed)
    return [random_parents(rng, n, roots=min(n, rng.choice([1, 1, 2, 5])), **how) for n in news]


def batch_of(news, lens, n_rows=None, max_rows=None):
    """A batch without a cache."""
    starts = np.concatenate([[0], np.cumsum(news)])
    rows = int(starts[-1])
    return S.kv_batch(ints(starts), ints(lens), torch.zeros(len(news), 1, dtype=torch.int32, device="cuda"),
                      rows if n_rows is None else n_rows, max(max(news), 1) if max_rows is None else max_rows)


# ---------------------------------------------------------------- positions and masks

PLANS = [([1], [1]), ([1], [500]), ([8], [2048]), ([32, 33, 31], [32, 33, 40]), ([64], [64]), ([65], [100]), ([0, 3, 0, 17], [5, 9, 0, 300]),
         ([1024], [5000]), ([700, 1, 257], [100000, 1, 257]), ([5, 6, 7], [4, 6, 2]), ([3] * 200, list(range(3, 203)))]


@pytest.mark.parametrize("news,lens", PLANS)
@pytest.mark.parametrize("how", [dict(), dict(gone=0.2), dict(chain=0.97), dict(chain=1.0), dict(chain=0.0)])
@pytest.mark.parametrize("n_sink,n_local,more_words", [(0, -1, 0), (0, 0, 1), (2, 3, 0), (101, 1, 2), (0, 2 ** 31 - 1, 0)])
def test_plan(news, lens, how, n_sink, n_local, more_words):
    parents = trees(news, sum(news) + len(news), **how)
    rows = sum(news)
    words = min(32, (max(news) + 31) // 32 + more_words)
    b = batch_of(news, lens, n_rows=rows + 2)
    positions = torch.full((rows + 2,), -77, dtype=torch.int32, device="cuda")
    masks = torch.full((rows + 2, words), -77, dtype=torch.int32, device="cuda")
    tree = S.draft_tree(ints([p for x in parents for p in x] + [-1, -1]), positions, masks)
    S.scale_tree_plan(tree, b, n_sink, n_local)
    want_p, want_m = [], []
    for x, a, n in zip(parents, news, lens):
        p, seen = plan(x, n - a, n_sink, n_local)
        want_p += p
        want_m.append(as_words(seen, words))
    assert positions.tolist() == want_p + [-77, -77]  # rows behind the last sequence stay
    got = masks.cpu().numpy()
    assert (got[:rows] == np.concatenate(want_m)).all() and (got[rows:] == -77).all()


def test_plan_leaves_rows_past_max_rows():
    b = batch_of([9], [30], max_rows=4)
    positions, masks = ints([-77] * 9), ints([[-77]] * 9)
    S.scale_tree_plan(S.draft_tree(ints([-1, 0, 1, 2, 3, 4, 5, 6, 7]), positions, masks), b)
    assert positions.tolist() == [21, 22, 23, 24] + [-77] * 5
    assert masks.flatten().tolist() == [1, 3, 7, 15] + [-77] * 5


# ---------------------------------------------------------------- attention

ATTENDS = [  # new rows, lengths, query heads, KV heads, page
    ([1], [1], 1, 1, 16), ([1], [700], 4, 1, 16), ([4], [300], 4, 1, 64), ([2, 4, 1], [2, 130, 64], 16, 4, 48),
    ([16], [16], 1, 1, 16), ([17], [400], 1, 1, 16), ([24], [1000], 1, 1, 32), ([25], [25], 1, 1, 16),
    ([8], [2048], 4, 1, 64), ([25, 3, 0, 33], [700, 3, 9, 200], 32, 8, 64), ([60, 1, 17], [1300, 600, 17], 28, 4, 16),
    ([130], [390], 8, 1, 128), ([200, 33], [257, 4000], 6, 2, 48), ([65], [129], 32, 1, 64), ([300], [1000], 17, 1, 16),
    ([1024], [1500], 2, 2, 16), ([5, 6, 7], [3, 6, 20], 8, 2, 16),
]


def run_attend(bt, parents_or_seen, positions=None, n_sink=0, n_local=-1, scale=0.0, words=None, lse=True, masks=None):
    words = words or max(1, (max(bt.news) + 31) // 32)
    if masks is None:
        masks = torch.full((bt.n_rows, words), -1, dtype=torch.int32, device="cuda")
        masks[: bt.rows] = torch.from_numpy(as_words(parents_or_seen, words)).cuda()
    pos = torch.full((bt.n_rows,), 3, dtype=torch.int32, device="cuda")
    pos[: bt.rows] = ints(positions)
    tree = S.draft_tree(None, pos, masks)
    a = S.attend_params(num_q_heads=bt.hq, n_sink=n_sink, n_local=n_local, attn_scale=scale)
    ws = torch.empty(S.scale_cache_attend_workspace_size(a, bt.cache, bt.batch), dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(ws)
    out = torch.full((bt.n_rows, bt.hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    sums = torch.full((bt.n_rows, bt.hq), 7.0, device="cuda") if lse else None
    S.scale_cache_attend_tree(a, tree, bt.cache, bt.batch, bt.q, out, sums, ws)
    assert S.scale_get_device_status(ws) == S.SCALE_OK
    assert bool((out[bt.rows:] == 7.0).all()) and (sums is None or bool((sums[bt.rows:] == 7.0).all()))
    return out[: bt.rows], None if sums is None else sums[: bt.rows]


def check_attend(bt, seen, positions, n_sink=0, n_local=-1, scale=None, **how):
    out, lse = run_attend(bt, seen, positions, n_sink, n_local, scale or 0.0, **how)
    want, want_l, tol, tol_l = attend_tree64(bt, bt.q, seen, positions, n_sink, n_local, scale)
    within(lse, want_l, tol_l, "lse")
    assert torch.equal(lse == -math.inf, want_l == -math.inf)
    within(out, want, tol, "out")
    return out, lse


def planned(bt, parents, n_sink=0, n_local=-1):
    seen, positions = [], []
    for x, a, n in zip(parents, bt.news, bt.lens):
        p, s = plan(x, n - a, n_sink, n_local)
        positions += p
        seen += s
    return seen, positions


@pytest.mark.parametrize("news,lens,hq,hkv,page", ATTENDS)
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n_sink,n_local", [(0, -1), (5, 40), (0, 3)])
@pytest.mark.parametrize("wide", [False, True])
def test_attend_trees(news, lens, hq, hkv, page, e4m3, n_sink, n_local, wide):
    """`wide`: a table of 120,000 tokens, by which calls of few rows leave the route of few keys."""
    if wide and n_local >= 0 and n_sink + n_local < 40:
        pytest.skip("the window bounds the keys")
    bt = Batch(news, lens, hq=hq, hkv=hkv, page=page, e4m3=e4m3, seed=sum(lens) + hq, n_rows=sum(news) + 2,
               wider=120000 // page if wide else 0)
    seen, positions = planned(bt, trees(news, hq + sum(news)), n_sink, n_local)
    check_attend(bt, seen, positions, n_sink, n_local)


@pytest.mark.parametrize("news,lens,hq,hkv,page", ATTENDS[1:])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("wide", [False, True])
def test_attend_any_masks_and_absent_rows(news, lens, hq, hkv, page, e4m3, wide):
    """Masks that are no trees: later nodes, not the row itself, none at all; rows that are no nodes; nodes that nobody sees
    hold NaN, and bits of nodes past the sequence are set."""
    bt = Batch(news, lens, hq=hq, hkv=hkv, page=page, e4m3=e4m3, seed=sum(lens) + hkv, wider=120000 // page if wide else 0)
    rng = random.Random(hq + sum(lens))
    seen, positions = [], []
    for b, (a, n) in enumerate(zip(news, lens)):
        hidden = {c for c in range(a) if rng.random() < 0.3}
        for i in range(a):
            some = {c for c in range(a) if c not in hidden and rng.random() < rng.choice([0.1, 0.6])}
            seen.append(some)
            positions.append(rng.choice([-1, -2 ** 31]) if rng.random() < 0.25 else max(0, n - a) + rng.randrange(a))
        at = {c for i in range(a) if positions[len(positions) - a + i] >= 0 and n - a + i >= 0 for c in seen[len(seen) - a + i]}
        for c in range(a):
            t = n - a + c
            if c not in at and t >= 0:
                for x in range(2):
                    bt.pages[x][bt.table[b, t // page].long(), t % page] = 0x7F if e4m3 else math.nan
    past = [s | {c for c in range(a, 32 * ((max(news) + 31) // 32))} for s, a in
            zip(seen, [a for a in news for _ in range(a)])]
    check_attend(bt, past, positions)
    none = [set() for _ in seen]
    out, lse = check_attend(bt, none, [max(0, n - a) for a, n in zip(news, lens) for _ in range(a)]) if min(
        n - a for a, n in zip(news, lens) if a) > 0 else (None, None)
    out, lse = run_attend(bt, none, [-1] * bt.rows)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


MANY = [  # as ATTENDS, of so many keys that the SMs share them in equal runs; then of more sequences and pairs than SMs
    ([33, 1, 20, 64, 7], [60000, 30001, 129, 40000, 45003], 4, 1, 16), ([300, 70], [30000, 22222], 16, 4, 64),
    ([40] * 19, [5000 + 731 * i for i in range(19)], 4, 1, 64), ([30, 64] * 75, [700 + 13 * i for i in range(150)], 8, 2, 16),
    ([17 + i % 3 for i in range(700)], [20 + i % 211 for i in range(700)], 1, 1, 16),
]


@pytest.mark.parametrize("news,lens,hq,hkv,page", MANY)
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n_sink,n_local", [(0, -1), (130, 9000)])
def test_attend_trees_of_many_keys(news, lens, hq, hkv, page, e4m3, n_sink, n_local):
    bt = Batch(news, lens, hq=hq, hkv=hkv, page=page, e4m3=e4m3)
    seen, positions = planned(bt, trees(news, 3 + sum(lens), gone=0.1), n_sink, n_local)
    out, lse = check_attend(bt, seen, positions, n_sink, n_local)
    again, sums = run_attend(bt, seen, positions, n_sink, n_local)
    assert same_bits(out, again) and same_bits(lse, sums)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv,news,lens", [(4, 1, [4, 2], [700, 90]), (8, 2, [33, 70], [900, 300]), (4, 4, [16], [16])])
def test_a_chain_is_causal_attention(e4m3, hq, hkv, news, lens):
    """A tree of one branch is scale_cache_attend, windows and sinks included. Both are within the bounds of the 64-bit
    result, so at most twice those apart (calls of many rows cut a causal batch's keys elsewhere, so the bits differ); the
    route of few rows sums in the same order and gives the same bits."""
    bt = Batch(news, lens, hq=hq, hkv=hkv, page=16, e4m3=e4m3, seed=3)
    for n_sink, n_local in ((0, -1), (4, 25), (70, 0)):
        seen, positions = planned(bt, [[i - 1 for i in range(a)] for a in news], n_sink, n_local)
        out, lse = run_attend(bt, seen, positions, n_sink, n_local)
        a = S.attend_params(num_q_heads=hq, n_sink=n_sink, n_local=n_local)
        ws = torch.empty(S.scale_cache_attend_workspace_size(a, bt.cache, bt.batch), dtype=torch.uint8, device="cuda")
        S.scale_workspace_init(ws)
        want, want_l = torch.empty_like(out), torch.empty_like(lse)
        S.scale_cache_attend(a, bt.cache, bt.batch, bt.q, want, want_l, ws)
        _, _, tol, tol_l = attend_tree64(bt, bt.q, seen, positions, n_sink, n_local)
        within(out, want.double(), 2 * tol)
        within(lse, want_l.double(), 2 * tol_l)
        if max(news) * hq // hkv <= 16:
            assert same_bits(out, want) and same_bits(lse, want_l)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("news", [[3], [40]])
def test_attend_edges(e4m3, news):
    """A NaN query, logits far apart, another scale, no lse, strided rows, a workspace that holds anything, a long sequence
    that is cut among many CTAs, the same call twice."""
    bt = Batch(news, [20000], hq=8, hkv=2, page=32, e4m3=e4m3, seed=9)
    seen, positions = planned(bt, trees(news, 4))
    check_attend(bt, seen, positions, scale=0.5)
    first = run_attend(bt, seen, positions)
    again = run_attend(bt, seen, positions, lse=False)
    assert same_bits(first[0], again[0])
    wide = torch.full((bt.n_rows, 24, 128), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, 8:16] = bt.q
    q = bt.q
    bt.q = wide[:, 8:16]
    assert same_bits(run_attend(bt, seen, positions)[0], first[0])
    bt.q = q.clone()
    bt.q[news[0] - 1, 3, 5] = math.nan
    out, lse = run_attend(bt, seen, positions)
    assert bool(out[-1, 3].isnan().all()) and bool(lse[-1, 3].isnan())
    rest = torch.ones(bt.rows, 8, dtype=torch.bool, device="cuda")
    rest[-1, 3] = False
    # the other rows of its warp may take other references (a warp rescales together), so they are right, not the same bits
    want, _, tol, _ = attend_tree64(bt, q, seen, positions)
    within(out[rest], want[rest], tol[rest])
    bt.q = (q * 200).contiguous()
    check_attend(bt, seen, positions)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("nodes", [4, 60])
def test_attend_follows_its_lists_in_a_graph(e4m3, nodes):
    """Captured once, replayed with other trees, lengths and rows; another graph with a workspace of its own."""
    big = Batch([nodes, nodes], [900, 700], hq=4, hkv=1, page=16, e4m3=e4m3, seed=1)
    words = (nodes + 31) // 32
    pos, masks = ints([0] * big.rows), torch.zeros(big.rows, words, dtype=torch.int32, device="cuda")
    parents = ints([-1] * big.rows)
    tree = S.draft_tree(parents, pos, masks)
    a = S.attend_params(num_q_heads=4)

    def made():
        ws = torch.empty(S.scale_cache_attend_workspace_size(a, big.cache, big.batch), dtype=torch.uint8, device="cuda")
        S.scale_workspace_init(ws)
        return ws, torch.zeros(big.rows, 4, 128, dtype=torch.bfloat16, device="cuda")

    sides = [made(), made()]
    graphs = []
    for ws, out in sides:
        S.scale_tree_plan(tree, big.batch)
        S.scale_cache_attend_tree(a, tree, big.cache, big.batch, big.q, out, None, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            S.scale_tree_plan(tree, big.batch)
            S.scale_cache_attend_tree(a, tree, big.cache, big.batch, big.q, out, None, ws)
        graphs.append(g)
    for seed, cut in ((1, 0), (2, 300), (3, nodes)):
        news = [nodes - seed, nodes - 1]
        lens = [900 - cut, 700 - seed]
        big.row_start.copy_(ints([0, news[0], sum(news)]))
        big.kv_len.copy_(ints(lens))
        shapes = trees(news, seed)
        parents[: sum(news)] = ints([p for x in shapes for p in x])
        big.q.copy_(torch.randn(big.q.shape, device="cuda").bfloat16())
        for ws, out in sides:
            out.fill_(7.0)
        for g in graphs:
            g.replay()
        small = Batch.__new__(Batch)
        small.__dict__.update(big.__dict__, news=news, lens=lens, rows=sum(news),
                              values=[[v[:n] for v, n in zip(x, lens)] for x in big.values])
        seen, positions = planned(small, shapes)
        want, _, tol, _ = attend_tree64(small, big.q, seen, positions)
        within(sides[0][1][: small.rows], want, tol)
        assert same_bits(sides[0][1], sides[1][1]) and bool((sides[0][1][small.rows:] == 7.0).all())


# ---------------------------------------------------------------- the walk, and moved rows


def moved(bt, groups):
    """Copies of the caches' tensors after the moves, a list of (src, dst) rows for each group."""
    held = [x.clone() for x in bt.pages + [s for s in bt.scales if s is not None]]
    for x in held:
        for g in groups:
            apply_moves(x, g, bt.page)
    return held


@pytest.mark.parametrize("news,lens", [([1], [1]), ([5], [9]), ([16, 16], [300, 16]), ([0, 7, 0, 61], [4, 30, 0, 100]), ([1024], [1030]),
                                       ([6, 9], [4, 40]), ([3] * 70, list(range(3, 73)))])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hkv,page", [(1, 16), (3, 48), (8, 64)])
@pytest.mark.parametrize("given", [True, False])
def test_accept_and_move(news, lens, e4m3, hkv, page, given):
    bt = Batch(news, lens, hq=hkv, hkv=hkv, page=page, e4m3=e4m3, seed=7, n_rows=sum(news) + 2)
    for x in bt.pages:  # no NaN: rows are compared by their bits, and copied as they are
        x.copy_(torch.randint(0, 100, x.shape, device="cuda").to(x.dtype))
    rng = random.Random(sum(lens) + hkv + given)
    shapes = trees(news, sum(lens), gone=0.1, chain=0.5)
    tokens = [[rng.randrange(3) for _ in x] for x in shapes]
    choices = [[rng.randrange(3) for _ in x] for x in shapes]
    firsts = [rng.randrange(3) for _ in shapes]
    flat = lambda x: ints([v for y in x for v in y] + [0, 0])  # noqa: E731
    rows, seqs = bt.rows, len(news)
    n_rows = bt.n_rows
    src, dst, path = (ints([-77] * n_rows) for _ in range(3))
    count, after, length = (ints([-77] * seqs) for _ in range(3))
    tree = S.draft_tree(flat(shapes), ints([0] * n_rows), ints([[0] * 32] * n_rows))
    moves = S.cache_moves(src, dst, bt.row_start)
    layers = S.cache_layers([bt.cache])
    want = [accept(s, n - a, t, c, f if given else None) for s, a, n, t, c, f in zip(shapes, news, lens, tokens, choices, firsts)]
    groups = []
    for b, ((p, _), a, n) in enumerate(zip(want, news, lens)):
        place = lambda t: int(bt.table[b, t // page]) * page + t % page  # noqa: E731
        groups.append([(place(n - a + x), place(n - a + i)) for i, x in enumerate(p) if x != i])
    held = moved(bt, groups)
    S.scale_tree_accept(tree, layers, bt.batch, flat(tokens), flat(choices), ints(firsts) if given else None, count, path, after,
                        length, moves)
    S.scale_cache_move(layers, moves)
    assert count.tolist() == [len(p) for p, _ in want]
    assert after.tolist() == [x for _, x in want]
    assert length.tolist() == [n - a + len(p) if n >= a and a else n for (p, _), a, n in zip(want, news, lens)]
    assert path.tolist() == [v for (p, _), a in zip(want, news) for v in p + [-1] * (a - len(p))] + [-77, -77]
    got = bt.pages + [s for s in bt.scales if s is not None]
    assert all(same_bits(x, y) for x, y in zip(got, held))
    assert src[rows:].tolist() == dst[rows:].tolist() == [-77, -77]


def test_accept_without_pages_moves_nothing():
    """An entry of the page table outside the pool: the walk is as it was, and its rows stay."""
    bt = Batch([6], [40], hq=1, hkv=1, page=16, e4m3=False)
    bt.table[0, 2] = 10 ** 6
    out = [ints([-77] * 6) for _ in range(6)]
    moves = S.cache_moves(out[0], out[1], bt.row_start)
    tree = S.draft_tree(ints([-1, -1, 1, 1, 3, 4]), ints([0] * 6), ints([[0]] * 6))
    before = [x.clone() for x in bt.pages]
    S.scale_tree_accept(tree, S.cache_layers([bt.cache]), bt.batch, ints([1, 2, 3, 4, 5, 6]), ints([9, 4, 9, 5, 6, 7]), ints([2]),
                        out[2], out[3], out[4], out[5], moves)
    S.scale_cache_move(S.cache_layers([bt.cache]), moves)
    assert out[3].tolist() == [1, 3, 4, 5, -1, -1] and out[4][0] == 7 and out[5][0] == 38
    assert out[0].tolist() == [-1] * 6 and all(same_bits(x, y) for x, y in zip(bt.pages, before))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hkv", [1, 2, 3, 5, 8, 64])
@pytest.mark.parametrize("layers", [1, 3, 65])
def test_moves(e4m3, hkv, layers):
    """Groups of every size, in order: rows that an earlier move read are written by a later one; moves that are none."""
    page, pages, rng = 16, 40, random.Random(hkv)
    shape = (pages, page, hkv, 128)
    caches, tensors = [], []
    for _ in range(layers):
        kv = [torch.randint(0, 120, shape, device="cuda").to(torch.uint8 if e4m3 else torch.bfloat16) for _ in range(2)]
        kv += [torch.randint(27, 247, (pages, hkv, page), dtype=torch.uint8, device="cuda") for _ in range(2)] if e4m3 else []
        tensors.append(kv)
        caches.append(S.kv_cache(*kv))
    groups, at = [], 0
    for n in (0, 1, 200, 0, 33, 64, 7):
        mine = list(range(at, at + n + 4))
        at += n + 4
        src = sorted(rng.sample(mine, n))  # to the front, in order: no source behind its own place
        groups.append([(s, mine[i]) for i, s in enumerate(src)])
    swaps = list(range(at, at + 20))  # a row goes on after it was read
    groups.append([(swaps[i], swaps[i - 1]) for i in range(1, 20)])
    assert at + 20 <= page * pages
    flat = [m for g in groups for m in g]
    start = np.concatenate([[0], np.cumsum([len(g) for g in groups])])
    src, dst = ([m[i] for m in flat] for i in range(2))
    bad = rng.sample(range(len(flat)), 5)
    for i, x in zip(bad, (-1, page * pages, 2 ** 31 - 1, -2 ** 31, -5)):
        (src if i % 2 else dst)[i] = x
    held = [[x.clone() for x in kv] for kv in tensors]
    for kv in held:
        for x in kv:
            for g0, g1 in zip(start, start[1:]):
                apply_moves(x, [(src[i], dst[i]) for i in range(g0, g1) if i not in bad], page)
    S.scale_cache_move(S.cache_layers(caches), S.cache_moves(ints(src), ints(dst), ints(start)))
    for kv, want in zip(tensors, held):
        assert all(same_bits(x, y) for x, y in zip(kv, want))
    # lists that say less than nothing, or more than there is
    S.scale_cache_move(S.cache_layers(caches), S.cache_moves(ints(src)[:0], ints(dst)[:0], n_groups=1))
    S.scale_cache_move(S.cache_layers(caches), S.cache_moves(ints([-1] * 4), ints([-1] * 4), ints([-9, 2, 1, 10 ** 6])))
    for kv, want in zip(tensors, held):
        assert all(same_bits(x, y) for x, y in zip(kv, want))


def test_rows_past_max_rows_stay():
    """A bound below a sequence's rows: the rows past it are left as they were, and their nodes are none."""
    bt = Batch([9, 3], [60, 30], hq=4, hkv=1, page=16, e4m3=False)
    bt.batch = S.kv_batch(bt.row_start, bt.kv_len, bt.table, bt.n_rows, 4)
    parents = [[-1, 0, 0, 1, 3, 4, 0, 0, 1], [-1, 0, 1]]
    seen, positions = planned(bt, parents)
    masks = torch.from_numpy(as_words(seen, 1)).cuda()
    masks |= 1 << 7  # a node past max_rows
    a = S.attend_params(num_q_heads=4)
    ws = torch.empty(S.scale_cache_attend_workspace_size(a, bt.cache, bt.batch), dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(ws)
    out = torch.full((12, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    S.scale_cache_attend_tree(a, S.draft_tree(None, ints(positions), masks), bt.cache, bt.batch, bt.q, out, None, ws)
    want, _, tol, _ = attend_tree64(bt, bt.q, seen, positions)
    rows = [0, 1, 2, 3, 9, 10, 11]
    within(out[rows], want[rows], tol[rows])
    assert bool((out[4:9] == 7.0).all())
    path, src, dst = (ints([-77] * 12) for _ in range(3))
    out = [ints([-77] * 2) for _ in range(3)]
    tokens, choices = ints([1, 2, 9, 3, 4, 5, 6, 7, 8, 1, 2, 3]), ints([2, 3, 0, 4, 0, 0, 0, 0, 0, 2, 3, 6])
    moves = S.cache_moves(src, dst, bt.row_start)
    S.scale_tree_accept(S.draft_tree(ints([p for x in parents for p in x]), ints([0] * 12), ints([[0]] * 12)), S.cache_layers([bt.cache]),
                        bt.batch, tokens, choices, ints([1, 1]), out[0], path, out[1], out[2], moves)
    assert path.tolist() == [0, 1, 3, -1] + [-77] * 5 + [0, 1, 2]
    assert [x.tolist() for x in out] == [[3, 3], [4, 6], [54, 30]]
    assert src.tolist()[4:9] == [-77] * 5


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n_sink,n_local", [(0, -1), (3, 50)])
def test_long_trees_past_max_rows(e4m3, n_sink, n_local):
    """The same on the route of many rows: the nodes past the bound are neither rows nor seen."""
    news, lens, most = [100, 30, 71], [900, 200, 71], 70
    bt = Batch(news, lens, hq=8, hkv=2, page=16, e4m3=e4m3)
    bt.batch = S.kv_batch(bt.row_start, bt.kv_len, bt.table, bt.n_rows, most)
    seen, positions = planned(bt, trees(news, 17), n_sink, n_local)
    kept = [c < most for n in news for c in range(n)]
    masks = torch.from_numpy(as_words(seen, 4)).cuda()
    masks[:, 2] |= 0x7FFFFFC0  # nodes 70 to 94
    masks[:, 3] = -1
    a = S.attend_params(num_q_heads=8, n_sink=n_sink, n_local=n_local)
    ws = torch.empty(S.scale_cache_attend_workspace_size(a, bt.cache, bt.batch), dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(ws)
    out = torch.full((bt.rows, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    S.scale_cache_attend_tree(a, S.draft_tree(None, ints(positions), masks), bt.cache, bt.batch, bt.q, out, None, ws)
    assert S.scale_get_device_status(ws) == S.SCALE_OK
    want, _, tol, _ = attend_tree64(bt, bt.q, seen, positions, n_sink, n_local)
    kept = torch.tensor(kept, device="cuda")
    within(out[kept], want[kept], tol[kept])
    assert bool((out[~kept] == 7.0).all())


def test_a_captured_step_follows_its_lists_on_another_stream():
    """Plan, walk and moves captured once and replayed with other trees, beside eager calls on a stream of their own."""
    nodes, seqs, page, hkv = 24, 3, 16, 2
    table = torch.randperm(seqs * 8, device="cuda").int().view(seqs, 8)
    row_start, kv_len = ints(np.arange(seqs + 1) * nodes), ints([100, 40, 77])
    rows = seqs * nodes
    parents, tokens, choices, first = ints([-1] * rows), ints([0] * rows), ints([0] * rows), ints([0] * seqs)
    fresh = torch.randn(2, seqs * 8, page, hkv, 128, device="cuda").bfloat16()

    def side():
        pages = [fresh[i].clone() for i in range(2)]
        layers = S.cache_layers([S.kv_cache(*pages)])
        batch = S.kv_batch(row_start, kv_len, table, rows, nodes)
        tree = S.draft_tree(parents, ints([0] * rows), ints([[0]] * rows))
        moves = S.cache_moves(ints([0] * rows), ints([0] * rows), row_start)
        outs = [ints([0] * seqs), ints([0] * rows), ints([0] * seqs), ints([0] * seqs)]

        def call(stream=None):
            S.scale_tree_plan(tree, batch, stream=stream)
            S.scale_tree_accept(tree, layers, batch, tokens, choices, first, *outs, moves, stream=stream)
            S.scale_cache_move(layers, moves, stream=stream)

        return pages, list(tree.tensors[1:]) + outs + list(moves.tensors[:2]), call

    mine, other = side(), side()
    mine[2]()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        mine[2]()
    stream = torch.cuda.Stream()
    for seed in (1, 2, 3):
        rng = random.Random(seed)
        parents.copy_(ints([p for _ in range(seqs) for p in random_parents(rng, nodes, gone=0.1)]))
        tokens.copy_(ints([rng.randrange(2) for _ in range(rows)]))
        choices.copy_(ints([rng.randrange(2) for _ in range(rows)]))
        for pages, _, _ in (mine, other):
            for x, y in zip(pages, fresh):
                x.copy_(y)
        torch.cuda.synchronize()
        g.replay()
        other[2](stream)
        torch.cuda.synchronize()
        assert all(same_bits(x, y) for x, y in zip(mine[0] + mine[1], other[0] + other[1]))
        assert int(mine[1][2].sum()) > 0


def test_moves_beyond_32_bits():
    """A pool of more than 2^32 bytes of keys."""
    hkv, page = 64, 16
    pages = (1 << 32) // (hkv * 256 * page) + 100
    kv = [torch.zeros(pages, page, hkv, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    far = pages * page - 3
    for x in kv:
        x.view(-1, hkv, 128)[far] = torch.randn(hkv, 128, device="cuda").bfloat16()
    layers = S.cache_layers([S.kv_cache(*kv)])
    S.scale_cache_move(layers, S.cache_moves(ints([far, far]), ints([5, far - 40]), n_groups=2))
    for x in kv:
        rows = x.view(-1, hkv, 128)
        assert same_bits(rows[5], rows[far]) and same_bits(rows[far - 40], rows[far]) and bool((rows[far] != 0).any())
        assert not bool(rows[6: far - 40].any()) and not bool(rows[:5].any())


# ---------------------------------------------------------------- a step


@pytest.mark.parametrize("e4m3", [False, True])
def test_steps_of_trees_leave_the_cache_of_single_tokens(e4m3):
    """Two steps with drafted trees on one side, the accepted tokens one by one on the other: the same caches and, up to
    the accuracy of either route, the same attention."""
    hq, hkv, page, seqs = 8, 2, 16, 3
    rng = random.Random(5)
    gen = torch.Generator(device="cuda").manual_seed(6)
    starts = [37, 0, 15]
    inv = 500000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    table = torch.arange(3 * 8, dtype=torch.int32, device="cuda").view(3, 8)
    sides = [S.allocate_kv_cache(24, page, hkv, e4m3=e4m3) for _ in range(2)]
    embed = {x: torch.randn(50, h, 128, generator=gen, device="cuda").bfloat16() for x, h in (("q", hq), ("k", hkv), ("v", hkv))}
    a = S.attend_params(num_q_heads=hq)
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(ws)

    def push(cache, lens, news, tokens, positions, tree=None):
        b = S.kv_batch(ints(np.concatenate([[0], np.cumsum(news)])), ints(lens), table, sum(news), max(news))
        rows = ints(tokens).long()
        q, out = embed["q"][rows].clone(), torch.empty(sum(news), hq, 128, dtype=torch.bfloat16, device="cuda")
        S.scale_cache_append(cache, b, embed["k"][rows].contiguous(), embed["v"][rows].contiguous(),
                             S.rope_axes(inv, positions.view(1, -1)), q, q)
        assert S.scale_cache_attend_workspace_size(a, cache, b) <= ws.numel()
        if tree is None:
            S.scale_cache_attend(a, cache, b, q, out, None, ws)
        else:
            S.scale_cache_attend_tree(a, tree, cache, b, q, out, None, ws)
        return b, out

    text = [[rng.randrange(50) for _ in range(n)] for n in starts]
    for cache in sides:
        news = starts
        push(cache, starts, news, [t for x in text for t in x], ints([i for x in text for i in range(len(x))]))
    lens, first = list(starts), [rng.randrange(50) for _ in range(seqs)]
    for step in range(2):
        news = [rng.randrange(5, 30) for _ in range(seqs)]
        shapes = [random_parents(rng, n, chain=0.5) for n in news]
        tokens = [[f] + [rng.randrange(50) for _ in range(n - 1)] for f, n in zip(first, news)]
        choices = [[rng.choice([tokens[b][c] for c in range(n) if shapes[b][c] == i] or [rng.randrange(50)]) for i in range(n)]
                   for b, n in enumerate(news)]
        rows = sum(news)
        pos, masks = ints([0] * rows), ints([[0]] * rows)
        tree = S.draft_tree(ints([p for x in shapes for p in x]), pos, masks)
        total = [n + x for n, x in zip(lens, news)]
        b0 = S.kv_batch(ints(np.concatenate([[0], np.cumsum(news)])), ints(total), table, rows, max(news))
        S.scale_tree_plan(tree, b0)
        b, out = push(sides[0], total, news, [t for x in tokens for t in x], pos, tree)
        new = [ints([0] * seqs) for _ in range(3)]
        path = ints([0] * rows)
        moves = S.cache_moves(ints([0] * rows), ints([0] * rows), b.tensors[0])
        layers = S.cache_layers([sides[0]])
        S.scale_tree_accept(tree, layers, b, ints([t for x in tokens for t in x]), ints([t for x in choices for t in x]),
                            ints(first), new[0], path, new[1], new[2], moves)
        S.scale_cache_move(layers, moves)
        want = [accept(s, n, t, c, f) for s, n, t, c, f in zip(shapes, lens, tokens, choices, first)]
        assert [len(p) for p, _ in want] == new[0].tolist() and min(new[0].tolist()) >= 1
        at = np.concatenate([[0], np.cumsum(news)])
        seqs_rows = [[int(at[i]) + x for x in p] for i, (p, _) in enumerate(want)]
        counts = [len(p) for p, _ in want]
        lens2 = new[2].tolist()
        assert lens2 == [n + c for n, c in zip(lens, counts)]
        _, single = push(sides[1], lens2, counts, [tokens[i][x] for i, (p, _) in enumerate(want) for x in p],
                         ints([lens[i] + d for i, c in enumerate(counts) for d in range(c)]))
        # a bf16 output of either route is off by half a step and its weights' 8 bits, of values up to 5
        assert (out[[x for r in seqs_rows for x in r]].float() - single.float()).abs().max() < 2 * 5 * 2.0 ** -7
        first, lens = new[1].tolist(), lens2
    for b, n in enumerate(lens):
        for x, y in zip(sides[0].tensors, sides[1].tensors):
            if x is None:
                continue
            rows = [t[table[b].long()] for t in (x, y)]
            if x.dim() == 3:
                rows = [t.transpose(1, 2) for t in rows]
            assert same_bits(*[t.flatten(0, 1)[:n] for t in rows])

"""Beam search over a paged cache against plain references: the selection over beams and vocabulary, the reordering of the
beams' pages, and a run of them together."""

import math
import random

import numpy as np
import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _branch import apply_moves, best, reorder
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


def select(logits, scores, n_best, ws=None):
    """logits [groups * beams][vocab], scores [groups][beams]"""
    groups, beams = scores.shape
    p = S.beam_params(n_groups=groups, n_beams=beams, vocab=logits.shape[1], n_best=n_best)
    if ws is None:
        ws = torch.full((S.scale_beam_workspace_size(p),), 0xA5, dtype=torch.uint8, device="cuda")
    out = (torch.full((groups, n_best), math.nan, device="cuda"), torch.full((groups, n_best), -77, dtype=torch.int32, device="cuda"),
           torch.full((groups, n_best), -77, dtype=torch.int32, device="cuda"))
    S.scale_beam_select(p, logits, scores, *out, ws)
    return out


def check(logits, scores, n_best):
    """Against 64 bits. The sums are kept to 2^-22, so continuations whose scores are closer than that may change places
    across beams (never within one); none of these inputs has any that are not equal."""
    got = [x.cpu().numpy() for x in select(logits, scores, n_best)]
    groups, beams = scores.shape
    z = logits.double().cpu().numpy().reshape(groups, beams, -1)
    s = scores.cpu().numpy()
    for g in range(groups):
        want = best(z[g], s[g], n_best)
        gaps = [abs(a[0] - b[0]) for a, b in zip(want, want[1:]) if math.isfinite(b[0]) and a[1] != b[1]]
        assert all(x == 0 or x > 2.0 ** -22 for x in gaps), "the inputs decide too closely"
        assert got[1][g].tolist() == [b for _, b, _ in want], g
        assert got[2][g].tolist() == [t for _, _, t in want], g
        for x, (y, _, _) in zip(got[0][g], want):
            assert x == y or abs(x - y) <= 2.0 ** -22 + abs(y) * 2.0 ** -24


def random_logits(rows, vocab, seed, dtype, peaks=6):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(rows, vocab, generator=gen, device="cuda") * 2.5
    at = torch.randint(0, vocab, (rows, peaks), generator=gen, device="cuda")
    z.scatter_add_(1, at, torch.rand(rows, peaks, generator=gen, device="cuda") * 12)
    return z.to(dtype)


SIZES = [(1, 1, 1, 1), (1, 1, 7, 7), (1, 2, 1, 2), (2, 3, 33, 64), (1, 32, 2, 64), (3, 4, 1000, 8), (1, 4, 8192, 8), (2, 2, 8193, 64),
         (1, 1, 32000, 1), (5, 3, 20001, 6), (1, 32, 50000, 64), (40, 8, 700, 16), (1, 2, 160000, 33)]


@pytest.mark.parametrize("groups,beams,vocab,n_best", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_select(groups, beams, vocab, n_best, dtype):
    logits = random_logits(groups * beams, vocab, vocab + beams, dtype)
    scores = -20 * torch.rand(groups, beams, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    check(logits, scores, n_best)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset,stride", [(0, 5003), (1, 5001), (3, 5001), (5, 5006), (7, 5008), (2, 9000)])
def test_rows_that_begin_anywhere(dtype, offset, stride):
    """Rows off the 16-byte boundary, apart from each other, NaN and infinities between them; the same logits give the same
    bits wherever they lie."""
    vocab, rows = 5001, 6
    z = random_logits(rows, vocab, 5, dtype)
    scores = -5 * torch.rand(2, 3, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    want = select(z, scores, 12)
    buf = torch.full((offset + rows * stride + 8,), math.inf, dtype=dtype, device="cuda")
    view = buf[offset: offset + rows * stride].view(rows, stride)[:, :vocab]
    view.copy_(z)
    got = select(view, scores, 12)
    assert all(same_bits(x, y) for x, y in zip(got, want))
    if stride >= vocab:
        check(view, scores, 12)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["equal", "two", "masked", "sorted", "reversed", "few", "zeros", "huge"])
@pytest.mark.parametrize("vocab", [30, 9000, 40001])
def test_ties_and_masks(dtype, kind, vocab):
    """Equal logits go by the lower token; masked ones (-inf, the type's least) come last, in their order."""
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = torch.randn(6, vocab, generator=gen, device="cuda")
    if kind == "equal":
        z = torch.full_like(z, 1.5)
    elif kind == "two":
        z = (z > 0).float()
    elif kind == "masked":
        z[torch.rand(z.shape, generator=gen, device="cuda") < 0.99] = -math.inf
    elif kind == "few":  # fewer that are finite than are kept; the others -inf or the least
        keep = z[:, 20:23].clone()
        z[:3] = -math.inf
        z[3:] = torch.finfo(dtype).min
        z[:, 20:23] = keep
    elif kind == "sorted":
        z = z.sort(-1).values
    elif kind == "reversed":
        z = z.sort(-1, descending=True).values
    elif kind == "zeros":
        z = torch.where(z > 0, 0.0, -0.0)
    elif kind == "huge":
        z = z * 1e30
    # scores whose differences nothing of the sums' accuracy can turn around
    scores = torch.tensor([[0.0, -1.25, -2.5], [-3.0, -3.75, -50.0]], device="cuda")
    check(z.to(dtype), scores, 30)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [3, 500, 20001])
def test_beams_that_offer_nothing(dtype, vocab):
    """Scores and logits that are not finite, NaN logits, beams of one group that are the same."""
    z = random_logits(8, vocab, vocab, dtype, peaks=2)
    z[0, :] = math.nan
    z[1, vocab // 2] = math.inf
    z[2, :] = -math.inf
    z[3, ::2] = math.nan
    z[6] = z[5]
    z[7] = z[5]
    scores = torch.tensor([[0.0, -1.0, -2.0, -3.0], [math.nan, -1.0, -1.0, -math.inf]], device="cuda")
    check(z, scores, min(64, 4 * vocab))
    dead = torch.full((2, 4), -math.inf, device="cuda")
    score, beam, token = select(z, dead, min(64, 4 * vocab))
    assert bool((score == -math.inf).all())
    n = score.shape[1]
    assert beam[0].tolist() == [i // vocab for i in range(n)] and token[1].tolist() == [i % vocab for i in range(n)]


def test_the_same_beams_tie_wherever_their_rows_begin():
    """Rows of an odd length lie differently; equal beams still go by their number."""
    z = random_logits(1, 33333, 1, torch.bfloat16).repeat(8, 1)
    score, beam, token = select(z, torch.zeros(1, 8, device="cuda"), 24)
    assert beam[0].tolist() == list(range(8)) * 3 and len(set(token[0].tolist())) == 3


def test_choices_of_a_tree():
    """One beam and n_best 1: the model's token after every row."""
    z = random_logits(300, 5000, 9, torch.bfloat16)
    _, beam, token = select(z, torch.zeros(300, 1, device="cuda"), 1)
    assert bool((beam == 0).all()) and torch.equal(token[:, 0].long(), z.float().argmax(-1))


def test_select_in_a_graph_on_two_streams():
    """Captured once and replayed on new logits, beside eager calls on another stream with a workspace of their own."""
    z = random_logits(12, 30000, 1, torch.bfloat16)
    scores = torch.zeros(3, 4, device="cuda")
    p = S.beam_params(n_groups=3, n_beams=4, vocab=30000, n_best=8)
    made = lambda: (torch.empty(3, 8, device="cuda"), torch.empty(3, 8, dtype=torch.int32, device="cuda"),  # noqa: E731
                    torch.empty(3, 8, dtype=torch.int32, device="cuda"), torch.empty(S.scale_beam_workspace_size(p), dtype=torch.uint8, device="cuda"))
    mine, other = made(), made()
    S.scale_beam_select(p, z, scores, *mine)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.scale_beam_select(p, z, scores, *mine)
    side = torch.cuda.Stream()
    for seed in (2, 3):
        z.copy_(random_logits(12, 30000, seed, torch.bfloat16))
        scores.copy_(-torch.rand(3, 4, device="cuda"))
        torch.cuda.synchronize()
        g.replay()
        S.scale_beam_select(p, z, scores, *other, stream=side)
        torch.cuda.synchronize()
        assert all(same_bits(x, y) for x, y in zip(mine[:3], other[:3]))


def test_scores_that_round_alike_go_by_the_logit():
    """Logits far below 64 bits of the score: among equal scores of a beam the larger logit comes first."""
    z = torch.zeros(2, 300, device="cuda")
    z[0, 7], z[0, 200], z[1, 250] = 1e-30, 2e-30, 1e-30
    scores, beams, tokens = select(z, torch.zeros(1, 2, device="cuda"), 5)
    assert bool((scores == scores[0, 0]).all())
    assert beams.tolist() == [[0] * 5] and tokens.tolist() == [[200, 7, 0, 1, 2]]
    z[1] = -math.inf
    z[1, [3, 250]] = 1e-30
    z[1, 260] = 2e-30
    assert select(z[1:], torch.zeros(1, 1, device="cuda"), 4)[2].tolist() == [[260, 3, 250, 0]]


def test_rows_far_apart():
    """A stride by which the last rows lie more than 2^31 logits behind the first."""
    rows, vocab = 20, 5001
    buf = torch.empty(rows, 1 << 27, dtype=torch.bfloat16, device="cuda")
    view = buf[:, 77: 77 + vocab]
    view.copy_(random_logits(rows, vocab, 3, torch.bfloat16))
    scores = -5 * torch.rand(5, 4, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    want = select(view.contiguous(), scores, 9)
    assert all(same_bits(x, y) for x, y in zip(select(view, scores, 9), want))


# ---------------------------------------------------------------- reordering


def caches_of(layers, pages, page, hkv, e4m3):
    held = []
    for _ in range(layers):
        kv = [torch.randint(0, 120, (pages, page, hkv, 128), device="cuda").to(torch.uint8 if e4m3 else torch.bfloat16) for _ in range(2)]
        kv += [torch.randint(27, 247, (pages, hkv, page), dtype=torch.uint8, device="cuda") for _ in range(2)] if e4m3 else []
        held.append(kv)
    return held, S.cache_layers([S.kv_cache(*kv) for kv in held])


@pytest.mark.parametrize("groups,beams,page,stride", [(1, 1, 16, 1), (1, 4, 64, 3), (3, 5, 16, 130), (2, 32, 48, 9), (7, 2, 16, 300)])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(4))
def test_reorder(groups, beams, page, stride, e4m3, in_place, seed):
    rng = random.Random(seed * 100 + beams)
    n = groups * beams
    pages = min(n * stride, 400) + n * 4
    held, layers = caches_of(2, pages, page, 2, e4m3)
    kv_len, table, parents = [], [], []
    free = rng.sample(range(pages), pages)
    for _ in range(groups):
        length = rng.choice([0, 1, page - 1, page, rng.randrange(stride * page + 1), stride * page, stride * page + 5, -3])
        full = min(max(length, 0) // page, stride)
        shared = [rng.randrange(pages) for _ in range(full)]
        for _ in range(beams):
            kv_len.append(length)
            tail = [free.pop() if i == full else rng.choice([-1, 10 ** 6, 0]) for i in range(full, stride)]
            table.append([x if rng.random() < 0.8 else rng.randrange(pages) for x in shared] + tail)
        parents.append([rng.choice([rng.randrange(beams), rng.randrange(beams), i, -1, beams]) for i in range(beams)])
    t = ints(table)
    out = t if in_place else torch.full_like(t, -77)
    src, dst = (ints([-77] * (n * page)) for _ in range(2))
    moves = S.cache_moves(src, dst, n_groups=n)
    want_t, want_m = [], []
    for g in range(groups):
        rows, m = reorder(table[g * beams: (g + 1) * beams], parents[g], kv_len[g * beams], page)
        want_t += rows
        want_m += m
    want = [[x.clone() for x in kv] for kv in held]
    for kv in want:
        for x in kv:
            for m in want_m:
                apply_moves(x, m, page)
    S.scale_beam_reorder(layers, t, ints(kv_len), ints(parents), out, moves)
    S.scale_cache_move(layers, moves)
    assert out.tolist() == want_t
    assert in_place or t.tolist() == table
    flat = [m + [(-1, -1)] * (page - len(m)) for m in want_m]
    assert src.view(n, page).tolist() == [[x for x, _ in m] for m in flat]
    assert dst.view(n, page).tolist() == [[x for _, x in m] for m in flat]
    for kv, w in zip(held, want):
        assert all(same_bits(x, y) for x, y in zip(kv, w))


def test_a_captured_reordering_follows_its_lists():
    groups, beams, page, stride = 3, 4, 16, 5
    n = groups * beams
    held, layers = caches_of(2, n * stride, page, 2, True)
    fresh = [[x.clone() for x in kv] for kv in held]
    table = torch.randperm(n * stride, device="cuda").int().view(n, stride)
    kv_len, parents = ints([37] * n), torch.zeros(groups, beams, dtype=torch.int32, device="cuda")
    moves = S.cache_moves(ints([0] * (n * page)), ints([0] * (n * page)), n_groups=n)
    out = torch.empty_like(table)

    def call():
        S.scale_beam_reorder(layers, table, kv_len, parents, out, moves)
        S.scale_cache_move(layers, moves)

    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for seed in (1, 2, 3):
        rng = random.Random(seed)
        p = [[rng.randrange(beams) for _ in range(beams)] for _ in range(groups)]
        parents.copy_(ints(p))
        kv_len.fill_(20 + seed)
        want_t = []
        want = [[x.clone() for x in kv] for kv in fresh]
        for b in range(groups):
            rows, m = reorder(table[b * beams: (b + 1) * beams].tolist(), p[b], 20 + seed, page)
            want_t += rows
            for kv in want:
                for x in kv:
                    for y in m:
                        apply_moves(x, y, page)
        for kv, f in zip(held, fresh):
            for x, y in zip(kv, f):
                x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        assert out.tolist() == want_t
        assert all(same_bits(x, y) for kv, w in zip(held, want) for x, y in zip(kv, w))


def test_beam_search_over_the_cache_equals_copied_sequences():
    """Steps of append, attention, selection and reordering over shared pages against beams that each keep a sequence of
    their own, copied whole."""
    hq, hkv, page, groups, beams, vocab, steps = 4, 2, 16, 2, 3, 60, 20
    n = groups * beams
    gen = torch.Generator(device="cuda").manual_seed(2)
    k_of, v_of = (torch.randn(vocab, hkv, 128, generator=gen, device="cuda").bfloat16() for _ in range(2))
    q_of = torch.randn(vocab, hq, 128, generator=gen, device="cuda").bfloat16()
    head = torch.randn(hq * 128, vocab, generator=gen, device="cuda")
    pages_each = 4
    order = torch.randperm(n * pages_each, generator=gen, device="cuda").int()
    table = order.view(n, pages_each).clone()
    cache = S.allocate_kv_cache(n * pages_each, page, hkv)
    layers = S.cache_layers([cache])
    moves = S.cache_moves(ints([0] * (n * page)), ints([0] * (n * page)), n_groups=n)
    row_start = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    kv_len = torch.zeros(n, dtype=torch.int32, device="cuda")
    batch = S.kv_batch(row_start, kv_len, table, n, 1)
    a = S.attend_params(num_q_heads=hq)
    ws = torch.empty(S.scale_cache_attend_workspace_size(a, cache, batch), dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(ws)
    p = S.beam_params(n_groups=groups, n_beams=beams, vocab=vocab, n_best=beams)
    bws = torch.empty(S.scale_beam_workspace_size(p), dtype=torch.uint8, device="cuda")
    score = torch.tensor([[0.0, -math.inf, -math.inf]] * groups, device="cuda")
    token = torch.full((groups, beams), 5, dtype=torch.int32, device="cuda")
    out = torch.empty(n, hq, 128, dtype=torch.bfloat16, device="cuda")
    said = [[[5] for _ in range(beams)] for _ in range(groups)]
    for step in range(steps):
        kv_len += 1
        rows = token.flatten().long()
        S.scale_cache_append(cache, batch, k_of[rows].contiguous(), v_of[rows].contiguous())
        S.scale_cache_attend(a, cache, batch, q_of[rows].contiguous(), out, None, ws)
        for i in range(n):  # the beam's own tokens, as the pages hold them
            mine = said[i // beams][i % beams]
            page_of = table[i, torch.arange(len(mine), device="cuda") // page].long()
            held = cache.tensors[0][page_of, torch.arange(len(mine), device="cuda") % page]
            assert same_bits(held, k_of[torch.tensor(mine, device="cuda")]), (step, i)
        logits = (out.float().view(n, -1) @ head * 0.05).contiguous()
        new = torch.empty_like(score), torch.empty_like(token), torch.empty_like(token)
        S.scale_beam_select(p, logits, score, *new, bws)
        S.scale_beam_reorder(layers, table, kv_len, new[1], table, moves)
        S.scale_cache_move(layers, moves)
        score, token = new[0], new[2]
        said = [[said[g][b] + [t] for b, t in zip(new[1][g].tolist(), token[g].tolist())] for g in range(groups)]
    assert bool(torch.isfinite(score).all()) and len({tuple(x) for x in said[0]}) == beams


def test_select_of_random_groups_matches_sorting():
    """A larger batch by torch's stable sort in 64 bits."""
    groups, beams, vocab, k = 20, 6, 12345, 12
    z = random_logits(groups * beams, vocab, 77, torch.bfloat16)
    s = -10 * torch.rand(groups, beams, device="cuda", generator=torch.Generator(device="cuda").manual_seed(8))
    flat = (torch.log_softmax(z.double(), -1).view(groups, beams, vocab) + s.double()[..., None]).flatten(1)
    value, at = flat.sort(dim=-1, descending=True, stable=True)
    assert float((value[:, :k] - value[:, 1: k + 1])[value[:, :k] != value[:, 1: k + 1]].min()) > 2.0 ** -40
    score, beam, token = select(z, s, k)
    assert torch.equal(beam.long() * vocab + token, at[:, :k])
    assert ((score - value[:, :k]).abs() <= 2.0 ** -22 + value[:, :k].abs() * 2.0 ** -24).all()
    assert np.isfinite(score.cpu().numpy()).all()

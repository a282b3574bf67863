"""Beam selection at the ends of its range: logits below the normal numbers, sums of many logits far below the largest, scores
that lie next to each other, more rows of one beam than a group's beams may have."""

import math

import numpy as np
import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _branch import best
from paper_2609_31568_gb300 import scale as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    pkg.build()
    S.load()


def select(logits, scores, n_best):
    """(scores, beams, tokens) as numpy, from outputs that hold what no call writes."""
    groups, beams = scores.shape
    p = S.beam_params(n_groups=groups, n_beams=beams, vocab=logits.shape[1], n_best=n_best)
    ws = torch.full((S.scale_beam_workspace_size(p),), 0xA5, dtype=torch.uint8, device="cuda")
    out = (torch.full((groups, n_best), math.nan, device="cuda"), torch.full((groups, n_best), -77, dtype=torch.int32, device="cuda"),
           torch.full((groups, n_best), -77, dtype=torch.int32, device="cuda"))
    S.scale_beam_select(p, logits, scores, *out, ws)
    return [x.cpu().numpy() for x in out]


# ---------------------------------------------------------------- logits below the normal numbers


def subnormal(kind, rows, vocab, dtype):
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    sign = torch.randint(0, 2, (rows, vocab), generator=gen, device="cuda") * 2.0 - 1.0
    size = torch.randint(1, 90, (rows, vocab), generator=gen, device="cuda").float()
    if kind == "negative":
        z = torch.full((rows, vocab), -1.0, device="cuda")
    elif kind == "signs":  # of every size, zeros among them
        z = sign * torch.where(size > 60, 0.0, size)
    elif kind == "positive":
        z = size
    # 2^-133 is bf16's smallest; made from bits, so that no kernel on the way takes them for zeros
    bits = (z.abs().int() << (16 if dtype is torch.bfloat16 else 3)) | torch.where(z < 0, -2 ** 31, 0).int()
    z = bits.view(torch.float32)
    if dtype is torch.bfloat16:
        z = (bits >> 16).short().view(torch.bfloat16)
    return z


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["negative", "signs", "positive"])
@pytest.mark.parametrize("vocab", [30, 300, 9000, 32000, 100003])
@pytest.mark.parametrize("above", [0, 3])
def test_logits_below_the_normal_numbers(dtype, kind, vocab, above):
    """They count as zeros: equal ones go by the lower token, behind `above` tokens that are larger and before the smaller
    ones; every place of the outputs is written."""
    z = subnormal(kind, 6, vocab, dtype)
    if above:
        z[:, [vocab - 1, vocab // 2, 5]] = 0.5
        z[:, 7:vocab:11] = -0.5
    scores = torch.tensor([[0.0, -1.25, -2.5], [-3.0, -3.75, -50.0]], device="cuda")
    got = select(z, scores, 30)
    flat = z.float().cpu().numpy().astype(np.float64).reshape(2, 3, vocab)
    flat[np.abs(flat) < 2.0 ** -126] = 0.0
    for g in range(2):
        want = best(flat[g], scores[g].cpu().numpy(), 30)
        assert got[1][g].tolist() == [b for _, b, _ in want], g
        assert got[2][g].tolist() == [t for _, _, t in want], g
        for x, (y, _, _) in zip(got[0][g], want):
            assert abs(x - y) <= 2.0 ** -19 + abs(y) * 2.0 ** -24


def test_choices_of_rows_below_the_normal_numbers():
    """One beam and n_best 1, the choices of a tree's nodes."""
    z = subnormal("negative", 40, 32000, torch.bfloat16)
    z[1:, 9] = 0.0  # equal to the others
    _, beam, token = select(z, torch.zeros(40, 1, device="cuda"), 1)
    assert beam.tolist() == [[0]] * 40 and token.tolist() == [[0]] * 40


# ---------------------------------------------------------------- sums

# One logit of 0, all others `low`. The roundings of these sums, followed in 32 bits on the CPU with 2^x exact, come to 2^-24.7 of
# them or less, in any number of parts; of 2^x only those of the 31 logits beside the largest one are not 1, and 2^-22 of these
# is below 2^-30 of the sum. The logarithm is good to 2^-24, so a score to 2^-23, and it is rounded to 32 bits once.
FAR = [(32000, -5.625), (128000, -11.25), (128000, -5.625), (1 << 22, -11.25)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab,low", FAR)
@pytest.mark.parametrize("rows", [1, 100, 400])
def test_many_logits_far_below_the_largest(dtype, vocab, low, rows):
    if rows * vocab > 1 << 26:
        rows = 3
    z = torch.full((rows, vocab), low, dtype=dtype, device="cuda")
    at = [(7 + 4099 * i) % vocab for i in range(rows)]
    z[list(range(rows)), at] = 0.0
    score, _, token = select(z, torch.zeros(rows, 1, device="cuda"), 1)
    want = -math.log1p((vocab - 1) * math.exp(low))
    assert token[:, 0].tolist() == at
    assert np.abs(score.astype(np.float64) - want).max() <= 2.0 ** -23 + abs(want) * 2.0 ** -24


@pytest.mark.parametrize("rise", [1.5, 3.75, 4.25, 7.75, 12.0])
@pytest.mark.parametrize("rows,vocab", [(1, 1 << 24), (310, 1 << 22), (2, 1 << 20)])
def test_sums_whose_first_logits_are_the_smaller(rows, vocab, rise):
    """Now and then 8,192 logits of 0, all others `rise` above: the largest sums that there are, against what comes first."""
    z = torch.full((rows, vocab), rise, dtype=torch.bfloat16, device="cuda")
    z[:, : vocab // 8192 * 8192].view(rows, -1, 8192)[:, ::64] = 0.0
    score, _, token = select(z, torch.zeros(rows, 1, device="cuda"), 1)
    small = 8192 * len(range(0, vocab // 8192, 64))
    want = -math.log((vocab - small) + small * math.exp(-rise))
    assert (token == 8192).all()
    assert np.abs(score.astype(np.float64) - want).max() <= 2.0 ** -18 + abs(want) * 2.0 ** -24


@pytest.mark.parametrize("vocab,low", FAR[:3])
@pytest.mark.parametrize("gap", [1.5, -1.5])
def test_scores_next_to_each_other(vocab, low, gap):
    """Two beams whose best continuations are 1.5 * 2^-22 apart: one of a sum of many logits, one of a single logit."""
    z = torch.full((2, vocab), low, device="cuda")
    z[0, 11] = 0.0
    z[1] = -math.inf
    z[1, 13] = 0.0
    mine = -math.log1p((vocab - 1) * math.exp(low))
    ahead = 0.25 * math.floor(-4 * mine)  # the better it, the finer fp32 holds the other
    mine += ahead
    other = np.float32(mine + gap * 2.0 ** -22)
    assert abs((float(other) - mine) / (gap * 2.0 ** -22) - 1) < 0.2  # fp32 holds it closely enough
    score, beam, token = select(z, torch.tensor([[ahead, float(other)]], device="cuda"), 2)
    assert beam.tolist() == [[1, 0] if gap > 0 else [0, 1]] and token.tolist() == [[13, 11] if gap > 0 else [11, 13]]


def test_select_of_random_groups_far_enough_apart():
    """A larger batch by torch's stable sort in 64 bits, the groups whose neighbours of different beams lie 2^-17 apart (a sum's
    2^-18 for each); continuations of one beam may lie as close as they like."""
    groups, beams, vocab, k = 20, 6, 12345, 12
    gen = torch.Generator(device="cuda").manual_seed(5)
    z = (torch.randn(groups * beams, vocab, generator=gen, device="cuda") * 2.5)
    z.scatter_add_(1, torch.randint(0, vocab, (groups * beams, 6), generator=gen, device="cuda"),
                   torch.rand(groups * beams, 6, generator=gen, device="cuda") * 12)
    s = -10 * torch.rand(groups, beams, device="cuda", generator=gen)
    flat = (torch.log_softmax(z.double(), -1).view(groups, beams, vocab) + s.double()[..., None]).flatten(1)
    value, at = flat.sort(dim=-1, descending=True, stable=True)
    apart = (value[:, :k] - value[:, 1: k + 1]).cpu()
    across = (at[:, :k] // vocab != at[:, 1: k + 1] // vocab).cpu()
    sure = (apart > 2.0 ** -17) | ~across
    rows = sure.all(-1).nonzero()[:, 0].tolist()
    assert len(rows) >= groups - 2
    score, beam, token = select(z, s, k)
    for g in rows:
        assert (beam[g].astype(np.int64) * vocab + token[g]).tolist() == at[g, :k].tolist()
    assert (np.abs(score - value[:, :k].cpu().numpy()) <= 2.0 ** -18 + np.abs(score) * 2.0 ** -24).all()


# ---------------------------------------------------------------- rows of one beam


@pytest.mark.parametrize("rows,vocab,n_best", [(4097, 1000, 1), (12800, 301, 1), (12800, 301, 3), (70001, 40, 2)])
def test_rows_of_one_beam_are_not_bounded_as_beams_are(rows, vocab, n_best):
    """The choices after every node of a batch's trees."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    z = torch.randn(rows, vocab, generator=gen, device="cuda").bfloat16()
    score, beam, token = select(z, torch.zeros(rows, 1, device="cuda"), n_best)
    value, at = torch.log_softmax(z.double(), -1).sort(dim=-1, descending=True, stable=True)
    assert (beam == 0).all() and (token == at[:, :n_best].cpu().numpy()).all()
    want = value[:, :n_best].cpu().numpy()
    assert (np.abs(score - want) <= 2.0 ** -18 + np.abs(want) * 2.0 ** -24).all()


# ---------------------------------------------------------------- beams that begin from one prompt


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("prompt", [5, 16, 21])
@pytest.mark.parametrize("e4m3", [False, True])
def test_beams_begin_from_one_prompt(prompt, e4m3):
    """The prompt goes into beam 0's pages; the others share its complete pages, and what is in the page being filled is copied
    into theirs by a list of moves of the program's own. Every beam then holds its own tokens, step by step."""
    hkv, page, groups, beams, vocab, steps, pages_each = 2, 16, 2, 3, 50, 25, 4
    n = groups * beams
    gen = torch.Generator(device="cuda").manual_seed(prompt)
    k_of, v_of = (torch.randn(vocab, hkv, 128, generator=gen, device="cuda").bfloat16() for _ in range(2))
    table = torch.randperm(n * pages_each, generator=gen, device="cuda").int().view(n, pages_each).clone()
    cache = S.allocate_kv_cache(n * pages_each, page, hkv, e4m3=True) if e4m3 else S.allocate_kv_cache(n * pages_each, page, hkv)
    layers = S.cache_layers([cache])
    # ---- the prompts, a sequence for each group
    said = [[(7 * g + t) % vocab for t in range(prompt)] for g in range(groups)]
    rows = torch.tensor(said, device="cuda").flatten()
    first = S.kv_batch(ints([prompt * g for g in range(groups + 1)]), ints([prompt] * groups), table[::beams].contiguous(), groups * prompt, prompt)
    S.scale_cache_append(cache, first, k_of[rows].contiguous(), v_of[rows].contiguous())
    # ---- the beams
    full, rest = divmod(prompt, page)
    for i in range(n):
        table[i, :full] = table[i - i % beams, :full]
    src, dst = [], []
    for i in range(n):
        for t in range(page):
            copied = i % beams > 0 and t < rest
            src.append(int(table[i - i % beams, full]) * page + t if copied else -1)
            dst.append(int(table[i, full]) * page + t if copied else -1)
    S.scale_cache_move(layers, S.cache_moves(ints(src), ints(dst), n_groups=n))
    said = [list(said[i // beams]) for i in range(n)]
    # ---- steps
    moves = S.cache_moves(ints([0] * (n * page)), ints([0] * (n * page)), n_groups=n)
    kv_len = ints([prompt] * n)
    batch = S.kv_batch(torch.arange(n + 1, dtype=torch.int32, device="cuda"), kv_len, table, n, 1)
    p = S.beam_params(n_groups=groups, n_beams=beams, vocab=vocab, n_best=beams)
    ws = torch.empty(S.scale_beam_workspace_size(p), dtype=torch.uint8, device="cuda")
    score = torch.tensor([[0.0, -math.inf, -math.inf]] * groups, device="cuda")
    new = torch.empty_like(score), ints([[0] * beams] * groups), ints([[0] * beams] * groups)
    for _ in range(steps):
        logits = torch.randn(n, vocab, generator=gen, device="cuda") * 2
        S.scale_beam_select(p, logits, score, *new, ws)
        S.scale_beam_reorder(layers, table, kv_len, new[1], table, moves)
        S.scale_cache_move(layers, moves)
        score = new[0].clone()
        parent, token = new[1].flatten().tolist(), new[2].flatten().tolist()
        said = [said[i - i % beams + b] + [t] for i, (b, t) in enumerate(zip(parent, token))]
        kv_len += 1
        rows = new[2].flatten().long()
        S.scale_cache_append(cache, batch, k_of[rows].contiguous(), v_of[rows].contiguous())
    # ---- the same sequences, each on its own in a cache of its own
    length = prompt + steps
    alone = S.allocate_kv_cache(n * pages_each, page, hkv, e4m3=True) if e4m3 else S.allocate_kv_cache(n * pages_each, page, hkv)
    own = torch.arange(n * pages_each, dtype=torch.int32, device="cuda").view(n, pages_each)
    every = lambda t: S.kv_batch(ints([length * i for i in range(n + 1)]), ints([length] * n), t, n * length, length)  # noqa: E731
    rows = torch.tensor(said, device="cuda").flatten()
    S.scale_cache_append(alone, every(own), k_of[rows].contiguous(), v_of[rows].contiguous())
    out = [[torch.empty(n * length, hkv, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    S.scale_cache_read(cache, every(table), *out[0])
    S.scale_cache_read(alone, every(own), *out[1])
    assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(*out))
    assert len({tuple(x) for x in said[:beams]}) == beams

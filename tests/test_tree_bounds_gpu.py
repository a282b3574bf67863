"""Acceptance of drafted trees whose sequences have more rows than the batch's bound says: what becomes of the moves behind
it, and of the lengths."""

import random

import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _branch import accept, apply_moves, random_parents
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


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("most", [0, 1, 4, 20, 33, 200])
@pytest.mark.parametrize("seed", range(3))
def test_moves_behind_the_bound_are_none(e4m3, most, seed):
    """The lists hold another step's moves, rows of the pool all of them. After the walk only what it accepts moves."""
    rng = random.Random(seed)
    news, lens, page = [9, 0, 40, 3, 130], [60, 30, 41, 30, 200], 16
    bt = Batch(news, lens, hq=4, hkv=2, page=page, e4m3=e4m3)
    batch = S.kv_batch(bt.row_start, bt.kv_len, bt.table, bt.n_rows, most)
    parents = [random_parents(rng, n, roots=1, chain=0.5) for n in news]
    tokens = [[rng.randrange(3) for _ in x] for x in parents]
    choices = [[rng.randrange(3) for _ in x] for x in parents]
    first = [rng.randrange(3) for _ in news]
    pool = bt.pages[0].shape[0] * page
    stale = rng.sample(range(pool), 2 * bt.rows) if pool >= 2 * bt.rows else [rng.randrange(pool) for _ in range(2 * bt.rows)]
    src, dst, path = ints(stale[: bt.rows]), ints(stale[bt.rows:]), ints([-77] * bt.rows)
    moves = S.cache_moves(src, dst, bt.row_start)
    out = [ints([-77] * len(news)) for _ in range(3)]
    layers = S.cache_layers([bt.cache])
    held = [x for x in bt.pages + bt.scales if x is not None]
    want = [x.clone() for x in held]
    flat = lambda x: ints([y for z in x for y in z])  # noqa: E731
    tree = S.draft_tree(flat(parents), ints([0] * bt.rows), ints([[0] * 7] * bt.rows))
    S.scale_tree_accept(tree, layers, batch, flat(tokens), flat(choices), ints(first), out[0], path, out[1], out[2], moves)
    S.scale_cache_move(layers, moves)
    at = 0
    for b, (a, n) in enumerate(zip(news, lens)):
        looked = min(a, most)
        way, last = accept(parents[b][:looked], n - a, tokens[b][:looked], choices[b][:looked], first[b])
        assert (out[0][b].item(), out[1][b].item(), out[2][b].item()) == (len(way), last, n - a + len(way) if a else n), b
        assert path[at: at + a].tolist() == way + [-1] * (looked - len(way)) + [-77] * (a - looked)
        assert dst[at + looked: at + a].tolist() == [-1] * (a - looked)
        row = lambda t: int(bt.table[b, t // page]) * page + t % page  # noqa: E731
        mine = [(row(n - a + x), row(n - a + i)) for i, x in enumerate(way) if x != i]
        for x in want:
            apply_moves(x, mine, page)
        at += a
    assert all(same_bits(x, y) for x, y in zip(held, want))


def test_lengths_where_no_row_is_looked_at():
    """A bound of 0, and rows behind the tensors' end: nothing is accepted, and the drafted tokens do not count."""
    for starts, lens, n_rows, most in (([0, 5, 5, 9, 12], [20, 7, 3, 12], 12, 0), ([0, 4, 9], [30, 40], 4, 8), ([4, 6, 9], [30, 2], 4, 8)):
        seqs = len(lens)
        cache = S.allocate_kv_cache(8, 16, 1)
        batch = S.kv_batch(ints(starts), ints(lens), ints([[0] * 4] * seqs), n_rows, most)
        lists = [ints([-5] * n_rows) for _ in range(3)]
        out = [ints([-77] * seqs) for _ in range(3)]
        zeros = ints([0] * n_rows)
        tree = S.draft_tree(ints([-1] * n_rows), zeros, ints([[0]] * n_rows))
        moves = S.cache_moves(lists[0], lists[1], batch.tensors[0])
        S.scale_tree_accept(tree, S.cache_layers([cache]), batch, zeros + 6, zeros, ints([7] * seqs), out[0], lists[2], out[1], out[2], moves)
        rows = [y - x for x, y in zip(starts, starts[1:])]
        assert out[0].tolist() == [0] * seqs and out[1].tolist() == [7] * seqs
        assert out[2].tolist() == [n - a if n >= a else n for a, n in zip(rows, lens)], (starts, lens)

"""The calls over a batch's paged cache on the paths that only large, strided or shared calls take: rows of several steps
and warps of many rows, slices of joint rows, a pool shared with the selection path, threads."""

import concurrent.futures as cf
import math
import os
import subprocess
import sys

import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _cache import Batch
from paper_2609_31568_gb300 import scale as S
from test_cache_gpu import attend, check_attend, inv_freq, same_bits

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    pkg.build()
    S.load()


def all_pages(bt):
    return [*bt.pages, *(s for s in bt.scales if s is not None)]


# ---------------------------------------------------------------- many rows


def append_in_pieces(bt, k, v, rope=None, q=None, q_out=None, piece=97):
    """What one append of the batch does, by appends of at most `piece` rows of one sequence."""
    row = 0
    for b, (a, n) in enumerate(zip(bt.news, bt.lens)):
        for i in range(0, a, piece):
            m = min(piece, a - i)
            rows = slice(row + i, row + i + m)
            batch = S.kv_batch(torch.tensor([0, m], dtype=torch.int32, device="cuda"),
                               torch.tensor([n - a + i + m], dtype=torch.int32, device="cuda"),
                               bt.table[b: b + 1].contiguous(), m, m)
            if rope is None:
                S.scale_cache_append(bt.cache, batch, k[rows], v[rows])
            else:
                f, pos, axis, adjacent = rope
                S.scale_cache_append(bt.cache, batch, k[rows], v[rows], S.rope_axes(f, pos[:, rows].contiguous(), axis, adjacent),
                                     None if q is None else q[rows], None if q is None else q_out[rows])
        row += a


@pytest.mark.parametrize("hq,hkv,news,lens", [(32, 8, [3999, 0, 1501, 500], [4500, 7, 1501, 4000]),
                                              (1, 1, [60000, 9000, 0, 21001], [61000, 8990, 0, 21001])])
@pytest.mark.parametrize("adjacent,axes", [(False, 1), (True, 3)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_an_append_of_many_rows_is_as_many_small_ones(hq, hkv, news, lens, adjacent, axes, e4m3):
    """Rows of several steps, and warps of more rows than are looked up at a time; ten rows have no place."""
    whole, parts = (Batch(news, lens, hq=hq, hkv=hkv, page=64, e4m3=e4m3, fill=False, n_rows=sum(news) + 2) for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(11)
    k, v = whole.row_tensor(hkv, gen), whole.row_tensor(hkv, gen)
    pos = torch.randint(0, 1 << 20, (axes, whole.n_rows), generator=gen, device="cuda").int()
    f, axis = inv_freq(), [i % axes for i in range(64)]
    outs = [torch.full_like(whole.q, 7.0) for _ in range(2)]
    S.scale_cache_append(whole.cache, whole.batch, k, v, S.rope_axes(f, pos, axis, adjacent), whole.q, outs[0])
    append_in_pieces(parts, k, v, (f, pos, axis, adjacent), whole.q, outs[1], piece=97 if hq > 1 else 701)
    assert same_bits(*outs) and (outs[0][whole.rows:] == 7).all()
    for x, y in zip(all_pages(whole), all_pages(parts)):
        assert same_bits(x, y)
    turned = torch.full_like(whole.q, 7.0)
    S.scale_rope(S.rope_axes(f, pos, axis, adjacent), whole.q, None, turned, None)
    assert same_bits(turned[: whole.rows], outs[0][: whole.rows])


def held_rows(x):
    """(codes, scale bytes) of finite bf16 rows [n][heads][128]; torch's conversion rounds to nearest even."""
    top = x.abs().amax(-1).float()
    m, e = torch.frexp(top)
    e = torch.where(top > 0, torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-100), -100)
    down = ((127 - e) << 23).view(torch.float32)
    return (x.float() * down[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


@pytest.mark.parametrize("e4m3", [False, True])
def test_millions_of_rows(e4m3):
    """Rows beyond those that every warp of either kernel looks up at first (32 each of 2,432 and 77,824 warps), with
    empty sequences and rows without a place among them."""
    page, news = 64, [900000, 0, 1000001, 3, 699999]
    lens = [900000, 0, 1000500, 3, 699000]
    width = -(-max(lens) // page)
    used = [-(-n // page) for n in lens]
    pages = sum(used) + 3
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).int().cuda()
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = order[at: at + u]
        at += u
    table[2, 5000], table[0, 3] = pages, -7  # 128 rows without a page
    n = sum(news)
    gen = torch.Generator(device="cuda").manual_seed(2)
    rows = [torch.randn(n, 1, 128, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    cache = S.allocate_kv_cache(pages, page, 1, e4m3=e4m3)
    batch = S.kv_batch(torch.tensor([0, *torch.tensor(news).cumsum(0).tolist()], dtype=torch.int32, device="cuda"),
                       torch.tensor(lens, dtype=torch.int32, device="cuda"), table, n, max(news))
    S.scale_cache_append(cache, batch, *rows)
    outs = [torch.full_like(x, 7.0) for x in rows]
    S.scale_cache_read(cache, batch, *outs)
    seq = torch.repeat_interleave(torch.arange(len(news), device="cuda"), torch.tensor(news, device="cuda"))
    tok = torch.arange(n, device="cuda") - (batch.tensors[0][1:][seq].long() - batch.tensors[1][seq].long())
    at = torch.where(tok >= 0, table[seq, tok.clamp(min=0) // page].long(), -1)
    placed = (at >= 0) & (at < pages)
    assert int((~placed).sum()) == 999 + 128
    for x in range(2):
        want = rows[x].clone()
        pool = torch.zeros(pages * page, 128, dtype=cache.tensors[x].dtype, device="cuda")
        to = (at * page + tok % page)[placed]
        if e4m3:
            codes, e = held_rows(rows[x])
            pool[to] = codes[placed, 0]
            scales = torch.full((pages * page,), 127, dtype=torch.uint8, device="cuda")
            scales[to] = e[placed, 0]
            assert torch.equal(cache.tensors[2 + x].view(-1), scales)
            up = (e.int() << 23).view(torch.float32)
            want = (codes.view(torch.float8_e4m3fn).float() * up[..., None]).bfloat16()
        else:
            pool[to] = rows[x][placed, 0]
        assert same_bits(cache.tensors[x].view(-1, 128), pool)
        want[~placed] = 0
        assert same_bits(outs[x], want)


# ---------------------------------------------------------------- strides


@pytest.mark.parametrize("news,lens", [([5, 1], [40, 9]), ([900, 30], [900, 500]), ([5000], [6000])])
@pytest.mark.parametrize("hq,hkv,adjacent", [(8, 2, False), (7, 1, True)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_append_and_read_of_joint_rows(news, lens, hq, hkv, adjacent, e4m3):
    """q, k and v as slices of joint rows, q turned where it lies; rows read back into slices of joint rows."""
    flat, joint = (Batch(news, lens, hq=hq, hkv=hkv, page=32, e4m3=e4m3, fill=False, n_rows=sum(news) + 3) for _ in range(2))
    n = flat.n_rows
    gen = torch.Generator(device="cuda").manual_seed(4)
    k, v = flat.row_tensor(hkv, gen), flat.row_tensor(hkv, gen)
    wide = torch.randn(n, (hq + 2 * hkv) * 128 + 24, generator=gen, device="cuda").bfloat16()
    cut = [0, hq * 128, (hq + hkv) * 128, (hq + 2 * hkv) * 128]
    views = [wide[:, a:b].view(n, -1, 128) for a, b in zip(cut, cut[1:])]
    for x, y in zip(views, (flat.q, k, v)):
        x.copy_(y)
    before = wide.clone()
    pos = torch.arange(n, device="cuda").int()[None].contiguous()
    rope = S.rope_axes(inv_freq(), pos, None, adjacent)
    q_out = torch.empty_like(flat.q)
    S.scale_cache_append(flat.cache, flat.batch, k, v, rope, flat.q, q_out)
    S.scale_cache_append(joint.cache, joint.batch, views[1], views[2], rope, views[0], views[0])
    for x, y in zip(all_pages(flat), all_pages(joint)):
        assert same_bits(x, y)
    rows = flat.rows
    assert same_bits(views[0][:rows], q_out[:rows])
    assert same_bits(wide[:, cut[1]:], before[:, cut[1]:]) and same_bits(wide[rows:], before[rows:])
    # without rope
    S.scale_cache_append(flat.cache, flat.batch, k, v)
    S.scale_cache_append(joint.cache, joint.batch, views[1], views[2])
    for x, y in zip(all_pages(flat), all_pages(joint)):
        assert same_bits(x, y)
    back = torch.full((n, 2 * hkv * 128 + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    outs = [back[:, : hkv * 128].view(n, hkv, 128), back[:, hkv * 128 + 8: 2 * hkv * 128 + 8].view(n, hkv, 128)]
    want = [torch.full((n, hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    S.scale_cache_read(flat.cache, flat.batch, *want)
    S.scale_cache_read(joint.cache, joint.batch, *outs)
    assert all(same_bits(x, y) for x, y in zip(outs, want))
    assert (back[:, hkv * 128: hkv * 128 + 8] == 7).all() and (back[:, -8:] == 7).all()


@pytest.mark.parametrize("news,lens", [([1, 1, 1], [100, 1, 700]), ([80, 1], [300, 700])])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (7, 1)])
def test_strided_queries_over_an_8bit_cache(news, lens, hq, hkv):
    bt = Batch(news, lens, hq=hq, hkv=hkv, page=16, e4m3=True)
    want, want_l = attend(bt)
    joint = torch.full((bt.n_rows, (hq + 4) * 128 + 8), math.nan, dtype=torch.bfloat16, device="cuda")
    q = joint[:, 136: 136 + hq * 128].view(bt.n_rows, hq, 128)
    q.copy_(bt.q)
    out, lse = attend(bt, q=q)
    assert same_bits(out, want) and same_bits(lse, want_l)


# ---------------------------------------------------------------- one pool for both paths


@pytest.mark.parametrize("page,block", [(64, 64), (128, 64), (64, 1)])
def test_the_selection_path_reads_a_pool_that_was_appended_to(page, block):
    """Two sequences appended in pieces to one bf16 pool; each through the paged path, as from contiguous rows."""
    hq, hkv, total = 8, 2, [1500, 700]
    gen = torch.Generator(device="cuda").manual_seed(12)
    rows = [[torch.randn(n, h, 128, generator=gen, device="cuda").bfloat16() for h in (hq, hkv, hkv)] for n in total]
    cache = S.allocate_kv_cache(60, page, hkv)
    table = torch.randperm(60, generator=torch.Generator().manual_seed(4))[:48].int().view(2, 24).cuda()
    done = [0, 0]
    while done != total:
        news = [min(a, n - d) for a, n, d in zip((333, 200), total, done)]
        k, v = (torch.cat([rows[b][x][done[b]: done[b] + news[b]] for b in range(2)]) for x in (1, 2))
        done = [d + n for d, n in zip(done, news)]
        S.scale_cache_append(cache, S.kv_batch(torch.tensor([0, news[0], sum(news)], dtype=torch.int32, device="cuda"),
                                               torch.tensor(done, dtype=torch.int32, device="cuda"), table, sum(news), max(news)), k, v)
    for b, n in enumerate(total):
        p = S.params(num_q_heads=hq, num_kv_heads=hkv, sub_chunk=64, n_tokens=n, max_cluster_subchunks=4, block_size=block,
                     top_k=3 * 64 // block, n_sink=64, n_local=128)
        paged, flat = (S.allocate(p, S.SCALE_MODE_PER_CLUSTER) for _ in range(2))
        S.run_path_paged(p, S.SCALE_MODE_PER_CLUSTER, rows[b][0], S.kv_pages(*cache.tensors[:2], table[b].contiguous(), page), paged)
        S.run_path(p, S.SCALE_MODE_PER_CLUSTER, *rows[b], flat)
        assert S.scale_get_device_status(paged.ws) == S.SCALE_OK
        units = int(flat.n_units)
        assert int(paged.n_units) == units
        assert torch.equal(paged.sel_count[:units], flat.sel_count[:units])
        assert torch.equal(paged.sel_blocks[:units], flat.sel_blocks[:units])
        assert same_bits(paged.out, flat.out)


# ---------------------------------------------------------------- one workspace for batches of many sizes


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 1), (8, 2)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_the_largest_batch_sizes_the_workspace(hq, hkv, e4m3):
    """Batches of 25 rows of a sequence down to one, either route, in a workspace of the first's size."""
    bts = [Batch([n] * 3, [900, 30, 200], hq=hq, hkv=hkv, page=16, e4m3=e4m3) for n in (25, 24, 17, 16, 6, 4, 2, 1)]
    a = S.attend_params(num_q_heads=hq)
    ws = torch.empty(S.scale_cache_attend_workspace_size(a, bts[0].cache, bts[0].batch), dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(ws)
    for bt in bts:
        want, want_l = attend(bt)
        out, lse = attend(bt, ws=ws)
        assert same_bits(out, want) and same_bits(lse, want_l)


# ---------------------------------------------------------------- threads


def run_in_threads(works):
    """Each of the functions in a thread of its own; what any of them raises is raised here."""
    with cf.ThreadPoolExecutor(len(works)) as ex:
        for done in [ex.submit(w) for w in works]:
            done.result()


def test_every_thread_ends_with_its_results():
    """Calls of both routes and cache types, whose launches need different shared memory, from six threads."""
    bts = [Batch([1] * n, [20 + i % 50 for i in range(n)], hq=4, hkv=1, page=16, e4m3=True) for n in (1, 700)]
    bts += [Batch([40, 1], [300, 90], hq=8, hkv=2, page=16, e4m3=e4m3) for e4m3 in (False, True)]
    bts += [Batch([1] * n, [33 + i % 50 for i in range(n)], hq=4, hkv=1, page=16, e4m3=False) for n in (2, 600)]
    want = [attend(bt)[0] for bt in bts]
    torch.cuda.synchronize()
    rounds = []

    def work(bt, out):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(30):
                assert same_bits(attend(bt)[0], out)
                rounds.append(1)

    run_in_threads([lambda i=i: work(bts[i], want[i]) for i in range(6)])
    assert len(rounds) == 6 * 30


FIRST_CALLS = r'''
import sys, threading
sys.path[:0] = [%r, %r]
import torch
from _cache import Batch
from test_cache_gpu import attend, same_bits
from test_cache_paths_gpu import run_in_threads
bts = [Batch([40, 3], [100, 50], hq=8, hkv=2, page=16, e4m3=i %% 2 == 1) for i in range(8)]
streams = [torch.cuda.Stream() for _ in bts]
torch.cuda.synchronize()
gate = threading.Barrier(len(bts))
outs = [None] * len(bts)

def work(i):
    with torch.cuda.stream(streams[i]):
        gate.wait()
        outs[i] = attend(bts[i])[0]

run_in_threads([lambda i=i: work(i) for i in range(len(bts))])
torch.cuda.synchronize()
assert all(same_bits(outs[i], outs[i %% 2]) for i in range(len(bts)))
assert all(same_bits(attend(bts[i])[0], outs[i]) for i in range(2))
'''


def test_first_calls_of_a_process_come_from_threads():
    run = subprocess.run([sys.executable, "-c", FIRST_CALLS % (ROOT, os.path.join(ROOT, "tests"))], capture_output=True, text=True,
                         timeout=300)
    assert run.returncode == 0, run.stderr[-3000:]


# ---------------------------------------------------------------- the largest values


def test_8bit_rows_at_the_end_of_bf16():
    """Rows whose largest value lies above 448 * 2^119: what rounds to 256 * 2^120, beyond bf16, is held as 240 * 2^120."""
    n = 8
    bt = Batch([n], [n], hq=1, hkv=1, page=16, e4m3=True, fill=False)
    big = 2.0 ** 127
    x = torch.randn(n, 1, 128, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    for i, f in enumerate((1.9921875, 1.9375, 1.9296875, 1.890625, 1.8125, 1.7578125, 1.75, 1.0)):
        x[i, 0, 3], x[i, 0, 90] = f * big, -f * big
    x[0, 0, 50], x[1, 0, 51] = math.nan, math.inf
    S.scale_cache_append(bt.cache, bt.batch, x, x)
    out = [torch.empty_like(x) for _ in range(2)]
    S.scale_cache_read(bt.cache, bt.batch, *out)
    want = torch.tensor([240.0, 240, 240, 240, 224, 224, 224, 128], dtype=torch.float64, device="cuda") * 2.0 ** 120
    for y in out:
        assert torch.equal(y[:, 0, 3].double(), want) and torch.equal(y[:, 0, 90].double(), -want)
        assert y[0, 0, 50].isnan() and y[1, 0, 51].isinf()  # the largest code, 448, times 2^120
        assert torch.isfinite(y).sum() == n * 128 - 2
    page_of, slot = bt.table[0].long()[torch.arange(n, device="cuda") // 16], torch.arange(n, device="cuda") % 16
    assert bt.scales[0].transpose(1, 2)[page_of, slot][:, 0].tolist() == [247] * 6 + [246, 246]

"""How exact the attention over a batch's paged cache is, one part at a time: against 64-bit references whose bounds hold
only if that part keeps the bits it is said to keep."""

import math

import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _cache import Batch, attend64
from paper_2609_31568_gb300 import scale as S
from test_cache_gpu import attend, check_attend, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    pkg.build()
    S.load()


def weights64(bt, b, row):
    """Softmax weights fp64 [rows][hq][len] of sequence b's rows (the first of them row `row`), and by how much a weight's
    logarithm may be off: a logit of 128 exact products summed in fp32 (128 roundings, twice for sums that are cut,
    of at most their sum's size A), two roundings on its way into 2^x and 2^-21 for the exponential."""
    a, n = bt.news[b], bt.lens[b]
    k = bt.values[0][b].repeat_interleave(bt.hq // bt.hkv, 1).transpose(0, 1)
    x = bt.q[row: row + a].double().transpose(0, 1)
    seen = torch.arange(n, device="cuda") <= torch.arange(n - a, n, device="cuda")[:, None]
    z = x @ k.transpose(1, 2) / math.sqrt(128)
    big = (x.abs() @ k.abs().transpose(1, 2) / math.sqrt(128)).amax(-1)
    off = 2 * 128 * 2.0 ** -24 * big + 8 * 2.0 ** -24 * z.abs().amax(-1) + 2.0 ** -21
    return torch.softmax(torch.where(seen, z, -math.inf), -1).transpose(0, 1), off.t()


@pytest.mark.parametrize("hq,hkv,news", [(8, 1, 1), (4, 1, 2), (16, 1, 1), (16, 2, 2), (28, 4, 1)])
@pytest.mark.parametrize("most", [7, 90, 5000])
def test_weights_beside_bf16_values(hq, hkv, news, most):
    """Few rows: a weight has 16 bits in its product with a value, so values that nearly cancel leave what the weights do."""
    lens = [max(news, 2 + (most - 2) * i // 39) for i in range(40)]
    bt = Batch([news] * 40, lens, hq=hq, hkv=hkv, page=16, e4m3=False, seed=hq + most)
    bt.q *= 2.0 ** -4  # logits so small that their own roundings are
    for b, n in enumerate(lens):
        sign = torch.where(torch.arange(n, device="cuda") % 2 == 0, 1.0, -1.0).double()[:, None, None]
        bt.values[1][b] = bt._put(1, b, bt.values[1][b][:1] * sign)
    out, _ = attend(bt)
    for b, n in enumerate(lens):
        w, off = weights64(bt, b, news * b)
        v = bt.values[1][b].repeat_interleave(hq // hkv, 1)
        want, size = torch.einsum("rhn,nhd->rhd", w, v), torch.einsum("rhn,nhd->rhd", w, v.abs())
        # the output in bf16; the weights (and their sum) off by `off`, their products by 2^-16, n sums in fp32
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -16 + 2 * off[..., None] + 2 * n * 2.0 ** -24) * size
        within(out[news * b: news * (b + 1)], want, tol, f"{n} keys")


def own_logits(q, k, k_values, hq, rows):
    """lse of rows that see their own key only, which is its logit: (attend's, fp64, A = sum |q_i k_i| scale)."""
    bt = Batch([rows], [rows], hq=hq, hkv=1, page=16, e4m3=True)
    bt.q[:] = q
    bt.values[0][0] = bt._put(0, 0, k)
    assert torch.equal(bt.values[0][0], k_values)
    _, lse = attend(bt, n_sink=0, n_local=0)
    x, y = bt.q.double(), k_values.repeat_interleave(hq, 1)
    return lse.double(), (x * y).sum(-1) / math.sqrt(128), (x * y).abs().sum(-1) / math.sqrt(128)


@pytest.mark.parametrize("hq,rows", [(1, 100), (4, 33), (8, 60), (7, 41), (8, 2), (24, 1)])
@pytest.mark.parametrize("apart", [0, 1, 40])
def test_queries_beside_8bit_keys_keep_their_bits(hq, rows, apart):
    """A query is off by at most 2^-12 of the largest |q| of its own row, whatever the rows beside it (2^-17 where all
    of a warp's rows are of one size): keys that are zero where the row is largest show the rest of it."""
    gen = torch.Generator(device="cuda").manual_seed(hq + rows + apart)
    rand = lambda *n: torch.rand(*n, generator=gen, device="cuda")  # noqa: E731
    # the others from 2^-6 to 2^-22 of the largest, which is just above a power of two
    q = torch.exp2(-6 - 16 * rand(rows, hq, 128)) * torch.sign(rand(rows, hq, 128) - 0.5)
    q[..., 5] = 1 + 2.0 ** -7
    q = (q * torch.exp2((apart * (rand(rows, hq, 1) - 0.5)).round())).bfloat16()
    k = torch.where(rand(rows, 1, 128) < 0.5, -1.0, 1.0).double()
    k[..., 5] = 0
    got, want, size = own_logits(q, k * 256, k * 256, hq, rows)
    top = q.double().abs().amax(-1)
    lost = 2.0 ** (-17 if apart == 0 else -12) * top * 127 * 256 / math.sqrt(128)
    # and 2^-20, however small the logit: beside few rows the exponent of its value, 16 at most here, joins it in fp32 and
    # leaves it again (two roundings of half a step of 2^-20, times ln 2), and the sum's log2 is off by 2^-22
    within(got, want, lost + 2 * 128 * 2.0 ** -24 * size + 2.0 ** -21 * want.abs() + 2.0 ** -20)


@pytest.mark.parametrize("hq,hkv", [(8, 2), (7, 1), (32, 1)])
@pytest.mark.parametrize("sizes", [(-3.0, 0.0, 3.0, 4.0), (-12.0, 6.0, -3.0, 0.0), (0.0, 9.0, 11.0, 1.0)])
def test_neighbours_of_other_sizes(hq, hkv, sizes):
    """Rows of sizes up to 2^18 apart side by side, each as exact as alone."""
    bt = Batch([100, 30], [500, 90], hq=hq, hkv=hkv, page=16, e4m3=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    size = torch.tensor(sizes, device="cuda")[torch.randint(0, 4, (bt.rows, hq), generator=gen, device="cuda")]
    bt.q *= torch.exp2(size)[..., None].bfloat16()
    check_attend(bt)


@pytest.mark.parametrize("zero", [0.0, math.nan, math.inf])
def test_neighbours_that_are_zero_or_not_finite(zero):
    """They count for nothing in the size of the rows beside them."""
    bt = Batch([100], [300], hq=8, hkv=2, page=16, e4m3=True)
    bt.q[::3, ::2] = zero
    bad = torch.zeros(bt.rows, 8, dtype=torch.bool, device="cuda")
    bad[::3, ::2] = zero != 0.0
    out, lse = attend(bt)
    assert out[bad].isnan().all() and lse[bad].isnan().all()
    want, want_l, tol, tol_l = attend64(bt, torch.where(bad[..., None], 0.0, bt.q))
    within(out[~bad], want[~bad], tol[~bad], "out")
    within(lse[~bad].double(), want_l[~bad], tol_l[~bad], "lse")


@pytest.mark.parametrize("hq,news", [(8, 1), (4, 3), (24, 1)])
@pytest.mark.parametrize("gap", [10, 15, 19])
def test_small_weights_beside_8bit_values(hq, news, gap):
    """Few rows: weights of 2^-gap of a row's largest keep the 11 bits of f16, down to 2^-20, for the dimensions where
    the largest one's value is zero."""
    n = 40
    bt = Batch([news] * 5, [n] * 5, hq=hq, hkv=1, page=16, e4m3=True, seed=gap)
    for b in range(5):
        k, v = bt.values[0][b] * 0, bt.values[1][b].clone()
        k[0, :, 0] = 1.0
        v[0, :, 1:], v[1:, :, 0], v[:, :, 0] = 0, 0, 1.0
        v[1:] = v[1:] / v[1:].abs().amax(-1, keepdim=True) * 1.5  # scales alike
        bt.values[0][b], bt.values[1][b] = bt._put(0, b, k.bfloat16().double()), bt._put(1, b, v.bfloat16().double())
    bt.q[:] = 0
    gaps = gap + 0.9 * torch.rand(bt.q.shape[:2], generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    bt.q[..., 0] = gaps * math.log(2) * math.sqrt(128)  # key 0's logit; all others' are 0
    out, _ = attend(bt)
    for b in range(5):
        w, off = weights64(bt, b, news * b)
        assert 0.45 < float(w[0, 0, 1] / w[0, 0, 0]) * 2.0 ** gap < 1.05
        v = bt.values[1][b].repeat_interleave(hq, 1)
        want, size = torch.einsum("rhn,nhd->rhd", w, v), torch.einsum("rhn,nhd->rhd", w, v.abs())
        tol = 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2 * off[..., None] + 2 * n * 2.0 ** -24) * size
        within(out[news * b: news * (b + 1)], want, tol)

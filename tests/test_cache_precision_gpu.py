"""How exact the attention over a batch's paged cache is, one part at a time: against 64-bit references whose bounds hold
only if that part keeps the bits it is said to keep."""

import math

import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _cache import Batch
from paper_2609_31568_gb300 import scale as S
from test_cache_gpu import attend, within

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

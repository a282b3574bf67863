"""Batches over a paged cache for the GPU tests, and 64-bit references of the calls over it.

Everything that a call must not use holds NaN: spare pages, the places behind a sequence's end, the
rows behind the last sequence. Values that a cache holds are kept beside it in fp64."""

from __future__ import annotations

import math

import numpy as np
import torch

from paper_2609_31568_gb300 import scale as S

DH = 128
HALF_STEP = {torch.bfloat16: 2.0 ** -8}  # finfo.eps / 2


def e4m3_table() -> torch.Tensor:
    """fp64 [256]: the value of every e4m3 code, from its fields."""
    out = []
    for code in range(256):
        power, low = (code >> 3) & 15, code & 7
        x = math.nan if power == 15 and low == 7 else low * 2.0 ** -9 if power == 0 else (8 + low) * 2.0 ** (power - 10)
        out.append(-x if code & 128 else x)
    return torch.tensor(out, dtype=torch.float64)


def quantise64(x: torch.Tensor):
    """(codes, scale bytes) of fp64 rows [..., 128]: the nearest code by search, ties to the even one."""
    x = x.cpu()
    table = e4m3_table()[:127]  # 0 .. 448, ascending
    finite = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    amax = finite.amax(-1).numpy()
    _, p = np.frexp(amax)  # amax < 2^p
    e = np.where(amax <= 448.0 * np.ldexp(1.0, p - 9), p - 9, p - 8)
    e = torch.from_numpy(np.maximum(np.where(amax > 0, e, -100), -100))
    y = (x.abs() * torch.ldexp(torch.ones(1, dtype=torch.float64), -e)[..., None]).clamp(max=448.0)
    hi = torch.searchsorted(table, y.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = y - table[lo], table[hi] - y
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = torch.where(torch.isnan(x), torch.full_like(code, 127), code)
    return (code + 128 * torch.signbit(x)).to(torch.uint8), (e + 127).to(torch.uint8)


class Batch:
    """Sequences with `news` rows of `lens` tokens in a shuffled pool of pages."""

    def __init__(self, news, lens, *, hq, hkv, page, e4m3, seed=0, n_rows=None, fill=True, wider=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.news, self.lens, self.hq, self.hkv, self.page, self.e4m3 = list(news), list(lens), hq, hkv, page, e4m3
        self.rows = sum(news)
        self.n_rows = self.rows if n_rows is None else n_rows
        used = [max(0, -(-n // page)) for n in lens]
        pages = sum(used) + 3
        order = torch.randperm(pages, generator=gen, device="cuda").int()
        table = torch.full((len(lens), max(max(used), 1) + wider), -7, dtype=torch.int32, device="cuda")
        at = 0
        for b, u in enumerate(used):
            table[b, :u] = order[at: at + u]
            at += u
        self.table = table
        kind = torch.uint8 if e4m3 else torch.bfloat16
        bad = 0x7F if e4m3 else math.nan
        self.pages = [torch.full((pages, page, hkv, DH), bad, dtype=kind, device="cuda") for _ in range(2)]
        self.scales = [torch.full((pages, hkv, page), 130, dtype=torch.uint8, device="cuda") if e4m3 else None
                       for _ in range(2)]
        starts = np.concatenate([[0], np.cumsum(news)])
        self.row_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.values = [[], []]  # fp64 [len][hkv][128] of every sequence
        for b, n in enumerate(lens):
            for x in range(2):
                rows = torch.randn(max(n, 0), hkv, DH, generator=gen, device="cuda", dtype=torch.float64)
                rows = rows * (1.5 if x == 0 else 1.0) * torch.exp2(torch.randint(-2, 3, (max(n, 0), hkv, 1), generator=gen, device="cuda").double())
                self.values[x].append(self._put(x, b, rows.bfloat16().double()) if fill and n > 0 else rows * 0)
        self.q = self.row_tensor(hq, gen)
        self.cache = S.kv_cache(*self.pages, *self.scales) if e4m3 else S.kv_cache(*self.pages)
        self.batch = S.kv_batch(self.row_start, self.kv_len, self.table, self.n_rows, max(max(news), 1))

    def row_tensor(self, heads, gen):
        """bf16 [n_rows][heads][128], NaN behind the last sequence."""
        x = torch.full((self.n_rows, heads, DH), math.nan, dtype=torch.bfloat16, device="cuda")
        x[: self.rows] = torch.randn(self.rows, heads, DH, generator=gen, device="cuda").bfloat16()
        return x

    def _at(self, b, n):
        t = torch.arange(n, device="cuda")
        return self.table[b].long()[t // self.page], t % self.page

    def _put(self, x, b, rows):
        """Rows into the pages; the values that they hold."""
        page, slot = self._at(b, rows.shape[0])
        if not self.e4m3:
            self.pages[x][page, slot] = rows.bfloat16()
            return rows
        codes, e = quantise64(rows)
        self.pages[x][page, slot] = codes.cuda()
        self.scales[x].transpose(1, 2)[page, slot] = e.cuda()
        return (e4m3_table()[codes.long()] * torch.exp2(e.double() - 127)[..., None]).cuda()

    def held(self, x, b):
        """fp64 values [len][hkv][128] that the pages hold for sequence b."""
        page, slot = self._at(b, self.lens[b])
        rows = self.pages[x][page, slot]
        if not self.e4m3:
            return rows.double()
        e = self.scales[x].transpose(1, 2)[page, slot].double() - 127
        return e4m3_table().cuda()[rows.long()] * torch.exp2(e)[..., None]

    def positions(self):
        """(sequence, token) of every row."""
        return [(b, self.lens[b] - a + i) for b, a in enumerate(self.news) for i in range(a)]


def attend64(bt: Batch, q, n_sink=0, n_local=-1, scale=None, values=None):
    """(out, lse, bound of out, bound of lse) in fp64, [rows][hq][128] and [rows][hq].

    The bounds: products of bf16 values are exact in fp32, so a logit of 128 of them is off by at most
    128 roundings of their partial sums, at most A = sum |q_i k_i| scale each, twice 2^-24 for sums that are
    cut instead of rounded; then two roundings on its way into 2^x, and 2^-21 for the exponential. A weight is
    rounded to 11 or 8 bits before the product with V; n sums in fp32; the output is rounded to bf16."""
    scale = 1 / math.sqrt(DH) if scale is None else scale
    g = bt.hq // bt.hkv
    outs, lses, tol_o, tol_l = [], [], [], []
    row = 0
    for b, (a, n) in enumerate(zip(bt.news, bt.lens)):
        if a == 0:
            continue
        k, v = ((values or bt.values)[x][b].repeat_interleave(g, 1).transpose(0, 1) for x in range(2))  # [hq][n][128]
        x = q[row: row + a].double().transpose(0, 1)
        t, p = torch.arange(max(n, 0), device="cuda"), torch.arange(n - a, n, device="cuda")[:, None]
        seen = t <= p
        if n_local >= 0:
            seen &= (t >= p - n_local) | (t < n_sink)
        z = torch.where(seen, x @ k.transpose(1, 2) * scale, -math.inf)
        size = torch.where(seen, x.abs() @ k.abs().transpose(1, 2) * abs(scale), 0.0)
        top = z.amax(-1, keepdim=True) if n > 0 else torch.full((bt.hq, a, 1), -math.inf, device="cuda", dtype=torch.float64)
        w = torch.exp(z - top.clamp(min=-1e300))
        total = w.sum(-1, keepdim=True)
        w = w / total.clamp(min=1e-300)
        out = w @ v
        spread = w @ v.abs()
        big = size.amax(-1, keepdim=True) if n > 0 else torch.zeros_like(top)
        delta = 2 * 128 * 2.0 ** -24 * big + 8 * 2.0 ** -24 * z.abs().masked_fill(~seen, 0).amax(-1, keepdim=True) + 2.0 ** -21 if n > 0 else big
        sums = 2 * max(n, 1) * 2.0 ** -24
        outs.append(out.transpose(0, 1))
        lses.append((total.log() + top)[..., 0].t())
        tol_o.append((2.0 ** -8 * out.abs() + (2.0 ** -8 + 2 * delta + sums) * spread + 2.0 ** -130).transpose(0, 1))
        tol_l.append((delta + sums + 2.0 ** -22 * lses[-1].t()[..., None].abs().nan_to_num(posinf=0, neginf=0))[..., 0].t())
        row += a
    return tuple(torch.cat(x) for x in (outs, lses, tol_o, tol_l))


def turn64(x, positions, inv_freq, axis, adjacent):
    """Rows x [n][heads][128] turned, fp64; positions as whole numbers."""
    x = x.double()
    pairs = [(2 * i, 2 * i + 1) if adjacent else (i, i + 64) for i in range(64)]
    y = x.clone()
    for i, (a, b) in enumerate(pairs):
        angle = positions[axis[i]].double() * float(inv_freq[i])
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def pair_size(x, adjacent):
    """|x| + |its pair's other member|, fp64."""
    x = x.double().abs()
    if adjacent:
        s = x[..., 0::2] + x[..., 1::2]
        return torch.stack([s, s], -1).flatten(-2)
    s = x[..., :64] + x[..., 64:]
    return torch.cat([s, s], -1)

"""The calls over a batch's paged cache against 64-bit references: rotary positions, appending to and
reading from bf16 and 8-bit caches, attention; their edges, and a run of them together."""

import math

import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _cache import Batch, attend64, e4m3_table, pair_size, quantise64, turn64
from paper_2609_31568_gb300 import scale as S

pytestmark = pytest.mark.gpu

@pytest.fixture(scope="module", autouse=True)
def _built():
    pkg.build()
    S.load()


def inv_freq(base=500000.0):
    return base ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)


def within(got, want, tol, what=""):
    """got (any float type) within tol of want, both finite alike."""
    got = got.double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    fine = torch.isfinite(want)
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or over.max() <= 0, f"{what}: over by {over.max():.3e} of {tol[fine].max():.3e}"


def same_bits(x, y):
    return torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


# ---------------------------------------------------------------- rotary positions


@pytest.mark.parametrize("n,hq,hkv", [(1, 1, 0), (1, 32, 8), (7, 5, 1), (33, 28, 4), (500, 6, 2), (3001, 3, 3)])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("axes", [1, 3])
def test_rope(n, hq, hkv, adjacent, axes):
    gen = torch.Generator(device="cuda").manual_seed(n + hq)
    q = torch.randn(n, hq, 128, generator=gen, device="cuda").bfloat16()
    k = torch.randn(n, hkv, 128, generator=gen, device="cuda").bfloat16() if hkv else None
    pos = torch.randint(-5, 2 ** 31 - 1, (axes, n), generator=gen, device="cuda").int()
    pos[:, : n // 2] %= 5000
    axis = [0] * 64 if axes == 1 else [(0, 1, 2)[i % 3] if adjacent else (0 if i < 16 else 1 if i < 40 else 2) for i in range(64)]
    f = inv_freq()
    f[-1] = 0.0  # a pair that stays
    f[3] = -f[3]
    r = S.rope_axes(f, pos, axis, adjacent)
    outs = [torch.full_like(x, math.nan) if x is not None else None for x in (q, k)]
    S.scale_rope(r, q, k, *outs)
    for x, y in ((q, outs[0]), (k, outs[1])):
        if x is None:
            continue
        want = turn64(x, pos, f, axis, adjacent)
        # cos and sin within 2 ulp of at most 1, three roundings in fp32; the reference's angle (up to
        # 2^31 radians in 64 bits) is off by 2^-22 at most
        tol = 2.0 ** -8 * want.abs() + (6 * 2.0 ** -24 + 2.0 ** -21) * pair_size(x, adjacent)
        within(y, want, tol)
    in_place = q.clone()
    S.scale_rope(r, in_place, None, in_place, None)
    assert same_bits(in_place, outs[0])


def test_rope_of_joint_rows_in_place():
    """Queries and keys as slices of joint rows, turned where they lie; the values between stay."""
    n, hq, hkv = 37, 8, 2
    gen = torch.Generator(device="cuda").manual_seed(3)
    joint = torch.randn(n, (hq + 2 * hkv) * 128, generator=gen, device="cuda").bfloat16()
    before = joint.clone()
    q, k = joint[:, : hq * 128].view(n, hq, 128), joint[:, hq * 128: (hq + hkv) * 128].view(n, hkv, 128)
    r = S.rope_axes(inv_freq(), torch.arange(n, device="cuda").int()[None].contiguous())
    want = [torch.empty(n, h, 128, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv)]
    S.scale_rope(r, q, k, *want)
    S.scale_rope(r, q, k, q, k)
    assert same_bits(q, want[0]) and same_bits(k, want[1])
    assert same_bits(joint[:, (hq + hkv) * 128:], before[:, (hq + hkv) * 128:])


def test_rope_at_far_positions_keeps_differences():
    """Turning by p and by p + 1 differ by one step's angle, also where p has 31 bits."""
    f = inv_freq(10000.0)
    x = torch.zeros(2, 1, 128, device="cuda").bfloat16()
    x[..., :64] = 1.0
    for p in (0, 10 ** 6, 2 ** 31 - 2):
        y = torch.empty_like(x)
        S.scale_rope(S.rope_axes(f, torch.tensor([[p, p + 1]], dtype=torch.int32, device="cuda")), x, None, y, None)
        z = y[..., :64].double() + 1j * y[..., 64:].double()
        turn = torch.angle(z[1] / z[0])
        want = torch.remainder(f + math.pi, 2 * math.pi) - math.pi
        assert ((turn - want).abs() < 4 * 2.0 ** -8).all()  # each of the two members' bf16 roundings


# ---------------------------------------------------------------- append and read

SHAPES = [([1], [1]), ([3], [20]), ([1] * 33, list(range(1, 34))), ([5, 0, 40, 1], [300, 7, 40, 65]),
          ([0, 0, 17], [0, 9, 17]), ([700], [1500])]


@pytest.mark.parametrize("news,lens", SHAPES)
@pytest.mark.parametrize("hkv,page", [(1, 16), (8, 64), (3, 48)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_append_and_read(news, lens, hkv, page, e4m3):
    bt = Batch(news, lens, hq=hkv, hkv=hkv, page=page, e4m3=e4m3, n_rows=sum(news) + 3, fill=False)
    gen = torch.Generator(device="cuda").manual_seed(5)
    rows = [bt.row_tensor(hkv, gen) for _ in range(2)]
    before = [p.clone() for p in bt.pages], [s.clone() for s in bt.scales if s is not None]
    S.scale_cache_append(bt.cache, bt.batch, *rows)
    want_p, want_s = before
    at = bt.positions()
    seq, tok = (torch.tensor([x[i] for x in at], device="cuda") for i in range(2))
    page_of, slot = bt.table[seq, tok // page].long(), tok % page
    for x in range(2):
        if e4m3:
            codes, e = quantise64(rows[x][: bt.rows].double())
            want_p[x][page_of, slot] = codes.cuda()
            want_s[x].transpose(1, 2)[page_of, slot] = e.cuda()
            assert torch.equal(bt.scales[x], want_s[x])
        else:
            want_p[x][page_of, slot] = rows[x][: bt.rows]
        assert same_bits(bt.pages[x], want_p[x])  # every other place as it was
    outs = [torch.full((bt.n_rows, hkv, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    S.scale_cache_read(bt.cache, bt.batch, *outs)
    for x in range(2):
        want = torch.full_like(outs[x], 7.0)
        want[: bt.rows] = torch.cat([bt.held(x, b)[n - a: n] for b, (a, n) in enumerate(zip(news, lens))]).bfloat16()
        assert same_bits(outs[x], want)
    only = torch.full_like(outs[1], 7.0)
    S.scale_cache_read(bt.cache, bt.batch, None, only)
    assert same_bits(only, outs[1])


@pytest.mark.parametrize("news,lens", [([1] * 5, [9, 3, 700, 80, 1]), ([400, 3], [1000, 3])])
@pytest.mark.parametrize("hq,hkv,adjacent,axes", [(32, 8, False, 1), (7, 1, True, 3), (6, 2, False, 3)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_append_turns_keys_and_queries(news, lens, hq, hkv, adjacent, axes, e4m3):
    bt = Batch(news, lens, hq=hq, hkv=hkv, page=32, e4m3=e4m3, fill=False)
    gen = torch.Generator(device="cuda").manual_seed(6)
    k, v = bt.row_tensor(hkv, gen), bt.row_tensor(hkv, gen)
    pos = torch.randint(0, 1 << 20, (axes, bt.rows), generator=gen, device="cuda").int()
    axis = [i % axes for i in range(64)]
    f = inv_freq()
    r = S.rope_axes(f, pos, axis, adjacent)
    q_out = torch.empty_like(bt.q)
    S.scale_cache_append(bt.cache, bt.batch, k, v, r, bt.q, q_out)
    alone = torch.empty_like(bt.q), torch.empty_like(k)
    S.scale_rope(r, bt.q, k, *alone)
    assert same_bits(q_out, alone[0])
    held = [torch.cat([bt.held(x, b)[n - a: n] for b, (a, n) in enumerate(zip(news, lens))]) for x in range(2)]
    if not e4m3:
        assert same_bits(held[0].bfloat16(), alone[1])
        assert same_bits(held[1].bfloat16(), v)
        return
    # a value is within half a step (2^-4 of it; 2^-10 of the scale below the least normal code) of the
    # turned key in fp32, and the scale is the least that holds the row's largest value in fp32
    want = turn64(k, pos, f, axis, adjacent)
    off = (6 * 2.0 ** -24 + 2.0 ** -21) * pair_size(k, adjacent)
    at = bt.positions()
    e = torch.stack([bt.scales[0][bt.table[b, t // 32].long(), :, t % 32] for b, t in at]).double() - 127
    scale = torch.exp2(e)[..., None]
    within(held[0], want, torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * scale) + 2 * off)
    top = want.abs().amax(-1, keepdim=True)
    slack = 2 * off.amax(-1, keepdim=True)
    assert (top <= 448 * scale + slack).all() and (top + slack > 224 * scale).all()
    codes, sv = quantise64(v.double())
    assert torch.equal(held[1], (e4m3_table()[codes.long()] * torch.exp2(sv.double() - 127)[..., None]).cuda())


def test_8bit_rows_of_every_size():
    """Rows from the least to the largest bf16 magnitudes, zeros, and values that are not finite."""
    hkv, n = 2, 280
    bt = Batch([n], [n], hq=2, hkv=hkv, page=16, e4m3=True, fill=False)
    gen = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(n, hkv, 128, generator=gen, device="cuda").double()
    x *= torch.exp2(torch.linspace(-135, 126, n, device="cuda", dtype=torch.float64).round())[:, None, None]
    x = x.bfloat16()
    assert torch.isfinite(x).all()
    x[3], x[10, 0, 5], x[11, 1, :3], x[12, 0] = 0, math.inf, math.nan, -math.inf
    x[200, :, 100] = -math.inf
    x[40, 0] = 448.0 * 2.0 ** 5  # the largest code exactly, and just above it
    x[41, 0] = 450.0 * 2.0 ** 5
    S.scale_cache_append(bt.cache, bt.batch, x, x.flip(2).contiguous())
    codes, e = quantise64(x.double())
    page_of, slot = bt.table[0].long()[torch.arange(n, device="cuda") // 16], torch.arange(n, device="cuda") % 16
    got = bt.pages[0][page_of, slot].cpu()
    nan = torch.isnan(x).cpu()
    assert torch.equal(got[~nan], codes[~nan]) and ((got[nan] & 127) == 127).all()
    assert torch.equal(bt.scales[0].transpose(1, 2)[page_of, slot].cpu(), e)
    out = torch.empty_like(x)
    S.scale_cache_read(bt.cache, bt.batch, out, None)
    fine = ~nan.cuda()
    want = (e4m3_table()[codes.long()] * torch.exp2(e.double() - 127)[..., None]).cuda()
    assert torch.equal(out.double()[fine], want[fine]) and torch.isnan(out[~fine]).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_rows_without_a_place(e4m3):
    """Rows before a sequence's first token, pages outside the pool and past the table: nothing is written,
    and they read as zeros."""
    bt = Batch([6, 40, 30], [4, 100, 60], hq=2, hkv=2, page=16, e4m3=e4m3, fill=False)
    bt.table[1, 5] = bt.cache.num_pages  # tokens 80..95
    bt.table[1, 6] = -1                  # 96..99
    narrow = bt.table[:, :3].contiguous()  # sequence 2: tokens 48..59 lie past the table
    bt.batch = S.kv_batch(bt.row_start, bt.kv_len, narrow, bt.n_rows, 40)
    wide = S.kv_batch(bt.row_start, bt.kv_len, bt.table, bt.n_rows, 40)
    gen = torch.Generator(device="cuda").manual_seed(8)
    k, v = bt.row_tensor(2, gen), bt.row_tensor(2, gen)
    for batch, table in ((wide, bt.table), (bt.batch, narrow)):
        for p in bt.pages:
            p.fill_(0x7F if e4m3 else 1.0)
        S.scale_cache_append(bt.cache, batch, k, v)
        placed = [t >= 0 and t // 16 < table.shape[1] and 0 <= int(table[b, t // 16]) < bt.cache.num_pages
                  for b, t in bt.positions()]
        assert not all(placed) and any(placed)
        changed = (bt.pages[0].view(-1, 2, 128) != (0x7F if e4m3 else 1.0)).any(-1).any(-1).sum()
        assert int(changed) == sum(placed)
        out = torch.full_like(k, 5.0)
        S.scale_cache_read(bt.cache, batch, out, None)
        ok = torch.tensor(placed, device="cuda")
        assert (out[~ok] == 0).all() and (out[ok].double() - k[ok].double()).abs().max() <= 2.0 ** -4 * 8


# ---------------------------------------------------------------- attention


def attend(bt, q=None, n_sink=0, n_local=-1, attn_scale=0.0, lse=True, ws=None, batch=None):
    a = S.attend_params(num_q_heads=bt.hq, n_sink=n_sink, n_local=n_local, attn_scale=attn_scale)
    q = bt.q if q is None else q
    batch = bt.batch if batch is None else batch
    out = torch.full((bt.n_rows, bt.hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    l = torch.full((bt.n_rows, bt.hq), 7.0, device="cuda") if lse else None
    if ws is None:
        ws = torch.empty(S.scale_cache_attend_workspace_size(a, bt.cache, batch), dtype=torch.uint8, device="cuda")
        ws.fill_(0xFF)  # nothing in it but the header is read before it is written
        S.scale_workspace_init(ws)
    S.scale_cache_attend(a, bt.cache, batch, q, out, l, ws)
    assert S.scale_get_device_status(ws) == S.SCALE_OK
    return out, l


def check_attend(bt, **kw):
    out, lse = attend(bt, **kw)
    want, want_l, tol, tol_l = attend64(bt, kw.get("q", bt.q)[: bt.rows], kw.get("n_sink", 0), kw.get("n_local", -1),
                                        kw.get("attn_scale") or None)
    within(out[: bt.rows], want, tol, "out")
    got = lse[: bt.rows].double()
    assert torch.equal(torch.isinf(got), torch.isinf(want_l))
    within(got, want_l, tol_l, "lse")
    assert (out[bt.rows:] == 7).all() and (lse[bt.rows:] == 7).all()
    return out, lse


@pytest.mark.parametrize("hq,hkv", [(4, 1), (32, 8), (28, 4), (8, 1), (6, 2), (4, 4), (5, 1), (64, 2), (16, 1)])
@pytest.mark.parametrize("news,lens,page", [
    ([1], [1], 16), ([1], [2], 64), ([1, 1, 1], [17, 1, 300], 16), ([1] * 20, list(range(1, 1001, 50)), 48),
    ([1], [5000], 64), ([2, 0, 1], [129, 50, 128], 128)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_single_tokens(hq, hkv, news, lens, page, e4m3):
    check_attend(Batch(news, lens, hq=hq, hkv=hkv, page=page, e4m3=e4m3, n_rows=sum(news) + 2, seed=hq))


@pytest.mark.parametrize("hq,hkv", [(4, 1), (8, 2), (7, 1), (3, 3), (32, 1), (17, 1)])
@pytest.mark.parametrize("news,lens,page", [
    ([3], [3], 16), ([33], [40], 16), ([130], [130], 64), ([700], [1600], 48), ([1, 200, 5, 0, 64], [900, 200, 77, 3, 64], 32),
    ([257, 129], [1030, 129], 128)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_chunks(hq, hkv, news, lens, page, e4m3):
    check_attend(Batch(news, lens, hq=hq, hkv=hkv, page=page, e4m3=e4m3, n_rows=sum(news) + 5, seed=hq))


@pytest.mark.parametrize("n_sink,n_local", [(0, 0), (0, 5), (4, 0), (64, 100), (100, 64), (130, 513), (3000, 10), (0, 4000)])
@pytest.mark.parametrize("news,lens", [([1, 1], [1500, 70]), ([300, 1, 40], [1500, 600, 40])])
@pytest.mark.parametrize("hq,hkv,e4m3", [(8, 2, False), (8, 2, True), (5, 1, False)])
def test_sinks_and_window(n_sink, n_local, news, lens, hq, hkv, e4m3):
    check_attend(Batch(news, lens, hq=hq, hkv=hkv, page=32, e4m3=e4m3), n_sink=n_sink, n_local=n_local)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (32, 2)])
def test_rows_that_see_nothing(hq, hkv, e4m3):
    """Rows before a sequence's first token, of empty sequences and of a negative length: out 0, lse -inf."""
    bt = Batch([5, 3, 40, 1], [2, 0, 25, -4], hq=hq, hkv=hkv, page=16, e4m3=e4m3)
    out, lse = check_attend(bt)
    empty = torch.tensor([t < 0 for _, t in bt.positions()], device="cuda")
    assert int(empty.sum()) == 3 + 3 + 15 + 1
    assert (out[: bt.rows][empty] == 0).all() and (lse[: bt.rows][empty] == -math.inf).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("news", [[1, 1], [60, 1]])
def test_pages_outside_the_pool_read_as_zeros(news, e4m3):
    bt = Batch(news, [200, 90], hq=8, hkv=2, page=16, e4m3=e4m3)
    bt.table[0, 2], bt.table[0, 12], bt.table[1, 3] = bt.cache.num_pages, -1, 2 ** 31 - 1
    for b, lp in ((0, 2), (0, 12), (1, 3)):
        for x in range(2):
            bt.values[x][b][16 * lp: 16 * lp + 16] = 0
    check_attend(bt)
    narrow = bt.table[:, :7].contiguous()
    bt.batch = S.kv_batch(bt.row_start, bt.kv_len, narrow, bt.n_rows, max(news))
    for x in range(2):
        bt.values[x][0][112:] = 0
    check_attend(bt)


@pytest.mark.parametrize("news,lens", [([1], [3000]), ([90], [500])])
@pytest.mark.parametrize("e4m3", [False, True])
def test_logits_far_apart(news, lens, e4m3):
    """Logits of thousands, keys that outgrow the earlier ones along the sequence, and a scale of one's own."""
    bt = Batch(news, lens, hq=8, hkv=2, page=16, e4m3=e4m3)
    page, slot = bt._at(0, lens[0])
    for x in range(2):
        grow = torch.exp2(torch.linspace(-20, 6, lens[0], device="cuda", dtype=torch.float64).round())[:, None, None]
        rows = bt.values[x][0] * (grow if x == 0 else 1 / grow)
        bt.values[x][0] = bt._put(x, 0, rows.bfloat16().double())
    for scale in (0.0, 1.0, 1e-3):
        check_attend(bt, attn_scale=scale)


@pytest.mark.parametrize("news", [[1], [100]])
def test_8bit_scales_of_every_size(news):
    """Rows of 8-bit keys and values whose scales differ by 2^30 within a sequence: the values' size follows."""
    bt = Batch(news, [300], hq=4, hkv=1, page=16, e4m3=True)
    for x in range(2):
        grow = torch.exp2(torch.linspace(-24, 8, 300, device="cuda", dtype=torch.float64).round())[:, None, None]
        bt.values[x][0] = bt._put(x, 0, (bt.values[x][0] * (grow if x else grow.flip(0))).bfloat16().double())
    check_attend(bt)
    # and all values near the ends of fp32's range
    for shift in (-80, 100):
        small = Batch(news, [300], hq=4, hkv=1, page=16, e4m3=True)
        small.values[1][0] = small._put(1, 0, (small.values[1][0] * 2.0 ** shift).bfloat16().double())
        check_attend(small)


@pytest.mark.parametrize("news,lens", [([1, 1], [400, 37]), ([140, 1], [500, 37])])
@pytest.mark.parametrize("e4m3", [False, True])
def test_what_no_row_sees_may_be_anything(news, lens, e4m3):
    """NaN before the window and behind the sequence's end (spare places hold NaN in every test) reaches no row."""
    bt = Batch(news, lens, hq=8, hkv=2, page=32, e4m3=e4m3)
    clean = attend(bt, n_sink=10, n_local=100)
    page, slot = bt._at(0, lens[0])
    lo = lens[0] - news[0] - 100
    for x in range(2):
        bt.pages[x][page[10:lo], slot[10:lo]] = 0x7F if e4m3 else math.nan
        if not e4m3:
            bt.pages[x][page[20:lo], slot[20:lo]] = math.inf
    dirty = attend(bt, n_sink=10, n_local=100)
    assert same_bits(clean[0], dirty[0]) and same_bits(clean[1], dirty[1])


@pytest.mark.parametrize("news,lens", [([1, 1, 1], [100, 1, 700]), ([80, 1], [300, 700])])
def test_strided_rows_and_no_lse(news, lens):
    bt = Batch(news, lens, hq=8, hkv=2, page=16, e4m3=False)
    want, _ = attend(bt)
    joint = torch.full((bt.n_rows, 12 * 128), math.nan, dtype=torch.bfloat16, device="cuda")
    q = joint[:, 128: 9 * 128].view(bt.n_rows, 8, 128)
    q.copy_(bt.q)
    out, _ = attend(bt, q=q, lse=False)
    assert same_bits(out, want)
    a = S.attend_params(num_q_heads=8)
    ws = torch.empty(S.scale_cache_attend_workspace_size(a, bt.cache, bt.batch), dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(ws)
    wide = torch.full((bt.n_rows, 9 * 128 + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    S.scale_cache_attend(a, bt.cache, bt.batch, q, wide[:, : 8 * 128].view(bt.n_rows, 8, 128), None, ws)
    assert same_bits(wide[:, : 8 * 128], want.view(bt.n_rows, -1)) and (wide[:, 8 * 128:] == 7).all()


def test_rows_past_the_bound_are_left():
    bt = Batch([3, 200], [50, 300], hq=4, hkv=1, page=16, e4m3=False)
    want, _ = attend(bt)
    out, lse = attend(bt, batch=S.kv_batch(bt.row_start, bt.kv_len, bt.table, bt.n_rows, 70))
    assert same_bits(out[:73], want[:73]) and (out[73:] == 7).all() and (lse[73:] == 7).all()


def test_workspace_too_small_is_refused():
    bt = Batch([1], [50], hq=4, hkv=1, page=16, e4m3=False)
    a = S.attend_params(num_q_heads=4)
    size = S.scale_cache_attend_workspace_size(a, bt.cache, bt.batch)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    with pytest.raises(S.ScaleError) as e:
        S.scale_cache_attend(a, bt.cache, bt.batch, bt.q, torch.empty_like(bt.q), None, ws[: size - 1])
    assert e.value.rc == S.SCALE_ERR_WORKSPACE


def test_host_memory_is_refused():
    bt = Batch([1], [50], hq=4, hkv=1, page=16, e4m3=False)
    with pytest.raises(S.ScaleError) as e:
        S.scale_cache_read(bt.cache, bt.batch, torch.empty(1, 1, 128, dtype=torch.bfloat16), None)
    assert e.value.rc == S.SCALE_ERR_INVALID_ARG


# ---------------------------------------------------------------- streams, graphs, and a run of them together


def test_repeats_are_bit_equal_and_other_streams_work():
    bt = Batch([1, 130, 7, 1], [4000, 700, 300, 9], hq=16, hkv=2, page=16, e4m3=True)
    first = attend(bt)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            again = attend(bt)
            assert same_bits(first[0], again[0]) and same_bits(first[1], again[1])
    torch.cuda.current_stream().wait_stream(side)


def test_captured_step_follows_its_lists():
    """One captured step (append, attend, read), replayed on other lengths, rows and pages; two graphs
    that share a workspace, one after the other."""
    hq, hkv, page, n = 8, 2, 16, 4
    cache = S.allocate_kv_cache(64, page, hkv, e4m3=True)
    table = torch.randperm(60, generator=torch.Generator().manual_seed(1)).int().view(n, 15).cuda()
    kv_len = torch.ones(n, dtype=torch.int32, device="cuda")
    starts = [torch.arange(n + 1, device="cuda").int(), torch.tensor([0, 30, 31, 31, 40], dtype=torch.int32, device="cuda")]
    a = S.attend_params(num_q_heads=hq, n_sink=3, n_local=60)
    gen = torch.Generator(device="cuda").manual_seed(2)
    f = inv_freq()
    work = []
    for s, rows in zip(starts, (4, 40)):
        batch = S.kv_batch(s, kv_len, table, rows, 40)
        t = {x: torch.zeros(rows, h, 128, dtype=torch.bfloat16, device="cuda")
             for x, h in (("q", hq), ("k", hkv), ("v", hkv), ("qr", hq), ("out", hq), ("kb", hkv), ("vb", hkv))}
        pos = torch.zeros(1, rows, dtype=torch.int32, device="cuda")
        work.append((batch, t, S.rope_axes(f, pos), pos))
    size = max(S.scale_cache_attend_workspace_size(a, cache, w[0]) for w in work)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    S.scale_workspace_init(ws)

    def step(w, to):
        batch, t, rope, _ = w
        S.scale_cache_append(cache, batch, t["k"], t["v"], rope, t["q"], t["qr"])
        S.scale_cache_attend(a, cache, batch, t["qr"], to["out"], None, ws)
        S.scale_cache_read(cache, batch, to["kb"], to["vb"])

    for w in work:
        step(w, w[1])
    torch.cuda.synchronize()
    graphs = []
    for w in work:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(w, w[1])
        graphs.append(g)
    for lens in ([40, 9, 3, 200], [31, 100, 240, 9]):
        kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        for w in work:
            for x in ("q", "k", "v"):
                w[1][x].copy_(torch.randn(w[1][x].shape, generator=gen, device="cuda"))
            w[3].copy_(torch.randint(0, 1000, w[3].shape, generator=gen, device="cuda"))
        pages = [p.clone() for p in cache.tensors]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [{x: w[1][x].clone() for x in ("out", "kb", "vb")} for w in work]
        after = [p.clone() for p in cache.tensors]
        for p, old in zip(cache.tensors, pages):
            p.copy_(old)
        for w, want in zip(work, got):
            to = {x: torch.zeros_like(y) for x, y in want.items()}
            step(w, to)
            assert all(same_bits(to[x], want[x]) for x in to)
        assert all(same_bits(p, x) for p, x in zip(cache.tensors, after))
        assert S.scale_get_device_status(ws) == S.SCALE_OK


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (7, 1)])
def test_serving_run(hq, hkv, e4m3):
    """Two sequences prefilled in pieces of 100 and 61 tokens and decoded for five steps, with rotary positions; every output
    against the whole sequence in 64 bits, then the cache read back into the selection path's step (a)."""
    page, total = 32, [505, 310]
    gen = torch.Generator(device="cuda").manual_seed(9)
    full = [{x: torch.randn(n, h, 128, generator=gen, device="cuda").bfloat16() for x, h in (("q", hq), ("k", hkv), ("v", hkv))}
            for n in total]
    cache = S.allocate_kv_cache(40, page, hkv, e4m3=e4m3)
    table = torch.randperm(40, generator=torch.Generator().manual_seed(3))[:32].int().view(2, 16).cuda()
    f = inv_freq()
    a = S.attend_params(num_q_heads=hq)
    done, outs, turned = [0, 0], [[], []], [[], []]
    ws = None
    while done != total:
        prompt = [n - 5 for n in total]
        news = [min(100 if b == 0 else 61, prompt[b] - done[b]) if done[b] < prompt[b] else min(1, total[b] - done[b])
                for b in range(2)]
        rows = sum(news)
        parts = {x: torch.cat([full[b][x][done[b]: done[b] + news[b]] for b in range(2)]) for x in "qkv"}
        pos = torch.cat([torch.arange(done[b], done[b] + news[b], device="cuda") for b in range(2)]).int()[None].contiguous()
        done = [d + n for d, n in zip(done, news)]
        batch = S.kv_batch(torch.tensor([0, news[0], rows], dtype=torch.int32, device="cuda"),
                           torch.tensor(done, dtype=torch.int32, device="cuda"), table, rows, max(news))
        qr = torch.empty_like(parts["q"])
        S.scale_cache_append(cache, batch, parts["k"], parts["v"], S.rope_axes(f, pos), parts["q"], qr)
        need = S.scale_cache_attend_workspace_size(a, cache, batch)
        if ws is None or ws.numel() < need:
            ws = torch.empty(need, dtype=torch.uint8, device="cuda")
            S.scale_workspace_init(ws)
        out = torch.empty_like(qr)
        S.scale_cache_attend(a, cache, batch, qr, out, None, ws)
        for b in range(2):
            lo = 0 if b == 0 else news[0]
            outs[b].append(out[lo: lo + news[b]])
            turned[b].append(qr[lo: lo + news[b]])
    assert S.scale_get_device_status(ws) == S.SCALE_OK
    # read both sequences back whole
    rows = sum(total)
    whole = S.kv_batch(torch.tensor([0, total[0], rows], dtype=torch.int32, device="cuda"),
                       torch.tensor(total, dtype=torch.int32, device="cuda"), table, rows, max(total))
    kb, vb = (torch.empty(rows, hkv, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    S.scale_cache_read(cache, whole, kb, vb)
    step = 2.0 ** -4 if e4m3 else 2.0 ** -8
    bt = Batch([total[0], total[1]], total, hq=hq, hkv=hkv, page=page, e4m3=False, fill=False)
    for b, lo in ((0, 0), (1, total[0])):
        n = total[b]
        want = turn64(full[b]["k"], torch.arange(n, device="cuda")[None], f, [0] * 64, False)
        got = kb[lo: lo + n].double()
        floor = 2.0 ** -10 * 2 * want.abs().amax(-1, keepdim=True) / 448  # the 8-bit rows' least step
        within(got, want, step * want.abs() + 2.0 ** -20 * pair_size(full[b]["k"], False) + floor)
        bt.values[0][b], bt.values[1][b] = got, vb[lo: lo + n].double()
    q = torch.cat([torch.cat(t) for t in turned])
    want, _, tol, _ = attend64(bt, q)
    within(torch.cat([torch.cat(o) for o in outs]), want, tol)
    # step (a) of the selection path takes the keys as they were read
    p = S.params(num_q_heads=hq, num_kv_heads=hkv, sub_chunk=64, n_tokens=total[0], max_cluster_subchunks=2, block_size=32,
                 top_k=2, n_sink=32, n_local=64)
    buf = pkg.allocate(p, S.SCALE_MODE_PER_CLUSTER)
    q0 = q[: total[0]].contiguous()
    S.scale_build_reps(p, q0, kb[: total[0]], buf.reps, buf.fingerprints, buf.unit_start, buf.n_units, buf.ws)
    means = torch.stack([kb[: total[0]].double()[i: i + 32].mean(0) for i in range(0, total[0], 32)]).transpose(0, 1)
    assert (buf.reps.double() - means).abs().max() < 1e-5


# ---------------------------------------------------------------- how work is divided


@pytest.mark.parametrize("long_at", [0, 20, 47])
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_long_sequence_among_many_short(long_at, e4m3):
    """More query tiles than the SMs hold twice, one sequence of fifty times the keys of the others."""
    lens = [40 + 37 * i % 300 for i in range(48)]
    lens[long_at] = 19999
    check_attend(Batch([5] * 48, lens, hq=32, hkv=8, page=64, e4m3=e4m3))


@pytest.mark.parametrize("n_sink,n_local", [(0, -1), (64, 1500)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_more_query_tiles_than_sms(n_sink, n_local, e4m3):
    """Between one query tile pair per SM and two: some whole, the last ones in pieces that fill up the SMs."""
    check_attend(Batch([64 * 7, 1, 300, 64 * 9], [3000, 777, 2900, 3100], hq=16, hkv=8, page=32, e4m3=e4m3), n_sink=n_sink,
                 n_local=n_local)


# ---------------------------------------------------------------- queries of every kind


@pytest.mark.parametrize("news,lens", [([1, 2], [300, 70]), ([100, 3], [500, 90])])
@pytest.mark.parametrize("e4m3", [False, True])
def test_queries_that_are_not_finite(news, lens, e4m3):
    """A head with NaN or infinity in its query gets NaN; the rows beside it are as if it held zeros."""
    bt = Batch(news, lens, hq=8, hkv=2, page=16, e4m3=e4m3)
    bt.q[1, 2, 5], bt.q[-1, 6, 127], bt.q[0, 1, 0] = math.nan, math.inf, -math.inf
    out, lse = attend(bt)
    bad = torch.zeros(bt.rows, 8, dtype=torch.bool, device="cuda")
    bad[1, 2] = bad[-1, 6] = bad[0, 1] = True
    assert out[bad].isnan().all() and lse[bad].isnan().all()
    want, want_l, tol, tol_l = attend64(bt, torch.where(bad[..., None], 0.0, bt.q))
    within(out[~bad], want[~bad], tol[~bad], "out")
    within(lse[~bad].double(), want_l[~bad], tol_l[~bad], "lse")


@pytest.mark.parametrize("e4m3", [False, True])
def test_queries_of_every_size(e4m3):
    """Blocks of 32 (token, query head) rows whose queries are 2^18 apart, each as exact as alone."""
    bt = Batch([100], [500], hq=8, hkv=2, page=16, e4m3=e4m3)
    size = torch.tensor([-12.0, 6.0, -3.0, 0.0], device="cuda")[torch.arange(100, device="cuda") // 8 % 4]
    bt.q *= torch.exp2(size)[:, None, None].bfloat16()
    check_attend(bt)


# ---------------------------------------------------------------- the ends of the ranges


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("news,lens", [([1, 2], [41, 300]), ([50, 1], [90, 333])])
def test_pages_far_into_a_large_pool(news, lens, e4m3):
    """Rows beyond 2^31 and 2^32 bytes of a pool."""
    bt = Batch(news, lens, hq=64, hkv=64, page=16, e4m3=e4m3)
    extra = (600000 if e4m3 else 300000) // 16  # of 128 and 256 KB
    for x in range(2):
        pool = torch.empty((extra + bt.pages[x].shape[0], *bt.pages[x].shape[1:]), dtype=bt.pages[x].dtype, device="cuda")
        pool[extra:] = bt.pages[x]
        bt.pages[x] = pool
        if e4m3:
            scales = torch.empty((pool.shape[0], *bt.scales[x].shape[1:]), dtype=torch.uint8, device="cuda")
            scales[extra:] = bt.scales[x]
            bt.scales[x] = scales
    assert bt.pages[0].nbytes > 2 ** 32
    bt.table[bt.table >= 0] += extra
    bt.cache = S.kv_cache(*bt.pages, *bt.scales) if e4m3 else S.kv_cache(*bt.pages)
    check_attend(bt)
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows, outs = ([bt.row_tensor(64, gen) for _ in range(2)] for _ in range(2))
    S.scale_cache_append(bt.cache, bt.batch, *rows)
    S.scale_cache_read(bt.cache, bt.batch, *outs)
    for x in range(2):
        assert same_bits(outs[x], torch.cat([bt.held(x, b)[n - a: n] for b, (a, n) in enumerate(zip(news, lens))]).bfloat16())
        assert (outs[x].double() - rows[x].double()).abs().max() <= (2.0 ** -4 * 8 if e4m3 else 0)


@pytest.mark.parametrize("page", [272, 1024])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("news", [[1, 1], [70, 1]])
def test_large_pages(page, e4m3, news):
    check_attend(Batch(news, [1500, 271], hq=8, hkv=2, page=page, e4m3=e4m3))


@pytest.mark.parametrize("rows_of_one,e4m3", [(1, False), (1, True), (40, False)])
def test_4096_sequences(rows_of_one, e4m3):
    lens = [1 + 7 * i % 40 for i in range(4096)]
    news = [1] * 4096
    news[1000], lens[1000], news[77] = rows_of_one, 100, 0
    check_attend(Batch(news, lens, hq=2, hkv=1, page=16, e4m3=e4m3))


@pytest.mark.parametrize("max_rows", [1, 30])
def test_no_sequence_has_rows(max_rows):
    bt = Batch([0, 0], [5, 0], hq=8, hkv=2, page=16, e4m3=False, n_rows=4)
    out, lse = attend(bt, batch=S.kv_batch(bt.row_start, bt.kv_len, bt.table, 4, max_rows))
    assert (out == 7).all() and (lse == 7).all()


def test_calls_from_several_threads():
    """Batches of different sizes, whose launches need different amounts of shared memory, from four threads."""
    import threading

    bts = [Batch([1] * n, [20 + i % 50 for i in range(n)], hq=4, hkv=1, page=16, e4m3=True) for n in (1, 700)]
    want = [attend(bt)[0] for bt in bts]
    torch.cuda.synchronize()
    bad = []

    def work(bt, out):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(30):
                if not same_bits(attend(bt)[0], out):
                    bad.append(bt.rows)

    threads = [threading.Thread(target=work, args=(bts[i % 2], want[i % 2])) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_two_calls_at_once():
    """On two streams, each with a workspace of its own."""
    bts = [Batch([1] * 8, [3000 + 10 * i for i in range(8)], hq=16, hkv=2, page=16, e4m3=True),
           Batch([600], [3000], hq=16, hkv=2, page=64, e4m3=False)]
    want = [attend(bt) for bt in bts]
    streams = [torch.cuda.Stream() for _ in bts]
    a = S.attend_params(num_q_heads=16)
    work = []
    for bt in bts:
        ws = torch.empty(S.scale_cache_attend_workspace_size(a, bt.cache, bt.batch), dtype=torch.uint8, device="cuda")
        S.scale_workspace_init(ws)
        work.append((bt, ws, [torch.empty_like(bt.q) for _ in range(6)]))
    torch.cuda.synchronize()
    for i in range(6):
        for st, (bt, ws, outs) in zip(streams, work):
            S.scale_cache_attend(a, bt.cache, bt.batch, bt.q, outs[i], None, ws, stream=st)
    torch.cuda.synchronize()
    for (bt, ws, outs), (out, _) in zip(work, want):
        assert S.scale_get_device_status(ws) == S.SCALE_OK and all(same_bits(x, out) for x in outs)


@pytest.mark.parametrize("hq,hkv,new", [(17, 1, 1), (8, 1, 3), (24, 4, 4), (32, 8, 6), (32, 8, 5), (25, 1, 1)])
@pytest.mark.parametrize("n_sink,n_local", [(0, -1), (20, 90)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_around_the_rows_of_one_route(hq, hkv, new, n_sink, n_local, e4m3):
    """17 to 25 (token, query head) rows of a KV head: the last that the route of few rows takes, and the first that it leaves."""
    check_attend(Batch([new, 1, new], [700, 33, new], hq=hq, hkv=hkv, page=16, e4m3=e4m3, n_rows=2 * new + 3), n_sink=n_sink,
                 n_local=n_local)

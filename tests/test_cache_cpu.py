"""The calls over a batch's paged cache, without a GPU: struct layouts, refusals before any launch, the
binding's own checks, and the 8-bit reference of the GPU tests."""

import ctypes
import os
import subprocess

import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _cache import e4m3_table, quantise64
from paper_2609_31568_gb300 import scale as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    pkg.build()
    return S.load()


@pytest.mark.parametrize("name,cls", [("scale_cache_t", S.ScaleCache), ("scale_batch_t", S.ScaleBatch),
                                      ("scale_rope_t", S.ScaleRope), ("scale_attend_t", S.ScaleAttend)])
def test_struct_layouts_match_header(name, cls, tmp_path):
    fields = [f[0] for f in cls._fields_]
    prints = "".join(f'printf("{f} %zu\\n", offsetof({name}, {f}));' for f in fields)
    src = f'#include <stddef.h>\n#include <stdio.h>\n#include "scale.h"\nint main(void) {{ printf("size %zu\\n", sizeof({name})); {prints} return 0; }}\n'
    (tmp_path / "t.c").write_text(src)
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    out = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout
    got = dict(line.split() for line in out.strip().splitlines())
    assert int(got.pop("size")) == ctypes.sizeof(cls)
    assert got == {f: str(getattr(cls, f).offset) for f in fields}


def _cache(**over):
    return S.ScaleCache(**{**dict(dtype=S.SCALE_CACHE_BF16, num_kv_heads=8, page_size=64, num_pages=10), **over})


def _batch(**over):
    return S.ScaleBatch(**{**dict(n_seqs=2, table_stride=4, n_rows=10, max_rows=10), **over})


def _rope(**over):
    return S.ScaleRope(**{**dict(n_axes=1), **over})


def _calls(lib, c, b, a=None, r=None, hq=32, stride=0):
    """The return values of every call with these descriptors and no pointers but out-of-range ones."""
    a = a or S.ScaleAttend(hq, 0, -1, 0.0)
    r = r or _rope()
    qs, ks = stride or 4096, stride or 1024
    n = ctypes.c_size_t()
    ref = ctypes.byref
    return {
        "size": lib.scale_cache_attend_workspace_size(ref(a), ref(c), ref(b), ref(n)),
        "attend": lib.scale_cache_attend(ref(a), ref(c), ref(b), None, qs, None, qs, None, None, 0, None),
        "append": lib.scale_cache_append(ref(c), ref(b), None, ks, None, ks, ref(r), 0, None, 0, None, 0, None),
        "read": lib.scale_cache_read(ref(c), ref(b), 1 << 20, ks, 1 << 30, ks, None),
    }


@pytest.mark.parametrize("over,rc", [
    (dict(dtype=2), S.SCALE_ERR_INVALID_ARG),
    (dict(num_kv_heads=0), S.SCALE_ERR_INVALID_ARG),
    (dict(num_kv_heads=65), S.SCALE_ERR_UNSUPPORTED),
    (dict(page_size=0), S.SCALE_ERR_INVALID_ARG),
    (dict(page_size=24), S.SCALE_ERR_UNSUPPORTED),
    (dict(num_pages=0), S.SCALE_ERR_INVALID_ARG),
    (dict(num_pages=1 << 25), S.SCALE_ERR_UNSUPPORTED),      # 2^31 rows
    (dict(num_pages=(1 << 62)), S.SCALE_ERR_UNSUPPORTED),    # whose product wraps
])
def test_cache_is_checked(lib, over, rc):
    assert set(_calls(lib, _cache(**over), _batch()).values()) == {rc}


@pytest.mark.parametrize("over,rc", [
    (dict(n_seqs=0), S.SCALE_ERR_INVALID_ARG),
    (dict(n_seqs=4097), S.SCALE_ERR_UNSUPPORTED),
    (dict(table_stride=0), S.SCALE_ERR_INVALID_ARG),
    (dict(n_rows=-1), S.SCALE_ERR_INVALID_ARG),
    (dict(max_rows=-1), S.SCALE_ERR_INVALID_ARG),
])
def test_batch_is_checked(lib, over, rc):
    assert set(_calls(lib, _cache(), _batch(**over)).values()) == {rc}


def test_null_pointers_and_strides_are_refused(lib):
    got = _calls(lib, _cache(), _batch())
    assert got.pop("size") == S.SCALE_OK
    assert set(got.values()) == {S.SCALE_ERR_INVALID_ARG}
    for stride in (1000, 100, 1028):  # less than a row, not a multiple of 8
        got = _calls(lib, _cache(), _batch(), stride=stride)
        assert got.pop("size") == S.SCALE_OK
        assert set(got.values()) == {S.SCALE_ERR_INVALID_ARG}
    assert lib.scale_cache_read(ctypes.byref(_cache()), ctypes.byref(_batch()), None, 1024, None, 1024, None) \
        == S.SCALE_ERR_INVALID_ARG


@pytest.mark.parametrize("a,rc", [
    (S.ScaleAttend(0, 0, -1, 0.0), S.SCALE_ERR_INVALID_ARG),
    (S.ScaleAttend(12, 0, -1, 0.0), S.SCALE_ERR_INVALID_ARG),
    (S.ScaleAttend(264, 0, -1, 0.0), S.SCALE_ERR_UNSUPPORTED),  # 33 query heads per KV head
    (S.ScaleAttend(32, -1, -1, 0.0), S.SCALE_ERR_INVALID_ARG),
    (S.ScaleAttend(32, 0, -1, -1.0), S.SCALE_ERR_INVALID_ARG),
    (S.ScaleAttend(32, 0, -1, float("nan")), S.SCALE_ERR_INVALID_ARG),
    (S.ScaleAttend(32, 0, -1, float("inf")), S.SCALE_ERR_INVALID_ARG),
])
def test_attend_parameters_are_checked(lib, a, rc):
    got = _calls(lib, _cache(), _batch(), a=a, hq=max(a.num_q_heads, 1))
    assert got["size"] == rc and got["attend"] == rc


def test_rope_is_checked(lib):
    bad = _rope()
    bad.axis[5] = 1
    for r in (_rope(n_axes=0), _rope(n_axes=5), bad):
        assert lib.scale_rope(ctypes.byref(r), 4, 8, 16, 1024, 16, 1024, 0, None, 0, None, 0, None) == S.SCALE_ERR_INVALID_ARG
        assert _calls(lib, _cache(), _batch(), r=r)["append"] == S.SCALE_ERR_INVALID_ARG
    ok = ctypes.byref(_rope())
    at = 1 << 30  # addresses are compared before they are looked up
    call = lib.scale_rope
    assert call(ok, 4, 0, None, 0, None, 0, 0, None, 0, None, 0, None) == S.SCALE_ERR_INVALID_ARG
    assert call(ok, 4, 257, at, 65536, at, 65536, 0, None, 0, None, 0, None) == S.SCALE_ERR_UNSUPPORTED
    assert call(ok, -1, 8, at, 1024, at, 1024, 0, None, 0, None, 0, None) == S.SCALE_ERR_INVALID_ARG
    assert call(ok, 0, 8, at, 1024, at, 1024, 0, None, 0, None, 0, None) == S.SCALE_OK  # nothing to do
    assert call(ok, 4, 8, at, 1024, at + 2048, 1024, 0, None, 0, None, 0, None) == S.SCALE_ERR_INVALID_ARG  # a row later
    assert call(ok, 4, 8, at, 1024, at, 2048, 0, None, 0, None, 0, None) == S.SCALE_ERR_INVALID_ARG  # other strides
    # without rope, append turns no queries
    assert lib.scale_cache_append(ctypes.byref(_cache()), ctypes.byref(_batch()), at, 1024, at, 1024, None, 32, at, 4096,
                                  at, 4096, None) == S.SCALE_ERR_INVALID_ARG


def test_overlapping_outputs_are_refused(lib):
    at = 1 << 30
    a, c, b = S.ScaleAttend(32, 0, -1, 0.0), _cache(), _batch()
    assert lib.scale_cache_attend(ctypes.byref(a), ctypes.byref(c), ctypes.byref(b), at, 4096, at, 4096, None, None, 0,
                                  None) == S.SCALE_ERR_INVALID_ARG
    assert lib.scale_cache_read(ctypes.byref(c), ctypes.byref(b), at, 1024, at + 1024, 1024, None) == S.SCALE_ERR_INVALID_ARG


def test_nothing_to_do_is_ok(lib):
    at = 1 << 30
    c, b = _cache(), _batch(n_rows=0)
    a = S.ScaleAttend(32, 0, -1, 0.0)
    assert lib.scale_cache_read(ctypes.byref(c), ctypes.byref(b), at, 1024, None, 0, None) == S.SCALE_OK
    assert lib.scale_cache_append(ctypes.byref(c), ctypes.byref(b), at, 1024, at, 1024, None, 0, None, 0, None, 0,
                                  None) == S.SCALE_OK
    assert lib.scale_cache_attend(ctypes.byref(a), ctypes.byref(c), ctypes.byref(b), at, 4096, at, 4096, None, None, 0,
                                  None) == S.SCALE_OK


def test_binding_checks_shapes_and_types():
    pages = torch.zeros(3, 16, 2, 128, dtype=torch.bfloat16)
    codes = torch.zeros(3, 16, 2, 128, dtype=torch.uint8)
    scales = torch.zeros(3, 2, 16, dtype=torch.uint8)
    assert S.kv_cache(pages, pages.clone()).dtype == S.SCALE_CACHE_BF16
    c = S.kv_cache(codes, codes.clone(), scales, scales.clone())
    assert (c.dtype, c.num_kv_heads, c.page_size, c.num_pages) == (S.SCALE_CACHE_E4M3, 2, 16, 3)
    ints = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    for bad in (lambda: S.kv_cache(pages, codes), lambda: S.kv_cache(codes, codes), lambda: S.kv_cache(pages, pages, scales, scales),
                lambda: S.kv_cache(codes, codes, scales, None), lambda: S.kv_cache(codes, codes, scales[:2], scales),
                lambda: S.kv_cache(pages.float(), pages.float()), lambda: S.kv_cache(pages.transpose(0, 1), pages.transpose(0, 1)),
                lambda: S.kv_batch(ints(3), ints(3), ints(3, 4), 1, 1), lambda: S.kv_batch(ints(4), ints(3), ints(2, 4), 1, 1),
                lambda: S.kv_batch(ints(4).long(), ints(3), ints(3, 4), 1, 1),
                lambda: S.rope_axes(torch.zeros(64), ints(1, 5)), lambda: S.rope_axes(torch.zeros(64).double(), ints(5)),
                lambda: S.rope_axes(torch.zeros(64).double(), ints(2, 5), [2] * 64),
                lambda: S.rope_axes(torch.zeros(64).double(), ints(1, 5), [0] * 63)):
        with pytest.raises(ValueError):
            bad()
    joint = torch.zeros(5, 12 * 128, dtype=torch.bfloat16)
    assert S._rows(joint[:, 256: 768].view(5, 4, 128), 5, 4) == (joint.data_ptr() + 512, 12 * 128, 4)
    assert S._rows(joint[:1, 256: 768].view(1, 4, 128), 1) == (joint.data_ptr() + 512, 512, 4)  # one row: any stride does
    for x in (joint.view(5, 12, 128)[:, ::2], joint.view(5, 12, 128).float(), joint.view(5, 12, 128)[:3],
              joint.view(5, 24, 64), joint):
        with pytest.raises(ValueError):
            S._rows(x, 5)
    with pytest.raises(ValueError):
        S._rows(joint.view(5, 12, 128), 5, 8)


def test_e4m3_reference_against_torch():
    """The reference's table and rounding are those of torch's float8_e4m3fn where nothing saturates."""
    codes = torch.arange(256, dtype=torch.uint8)
    table = e4m3_table()
    assert torch.equal(table.nan_to_num(nan=1e3).abs(), codes.view(torch.float8_e4m3fn).double().nan_to_num(nan=1e3).abs())
    x = (torch.randn(300, 128, generator=torch.Generator().manual_seed(1)) * 3).bfloat16()
    x[0] = 0
    x[1, 5] = float("inf")
    x[2, 7] = float("nan")
    got, e = quantise64(x.double())
    scale = torch.exp2(127 - e.double())[:, None]
    fine = torch.isfinite(x)
    want = (x.double() * scale).float().to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(got[fine], want[fine])
    assert got[1, 5] == 126 and got[2, 7] == 127 and e[0] == 27
    top = x.double().abs().nan_to_num(nan=0, posinf=0).amax(-1)
    assert bool((top <= 448 / scale[:, 0]).all()) and bool((top[1:] > 224 / scale[1:, 0]).all())


def test_binding_refuses_other_types_of_the_same_size():
    half = torch.zeros(3, 16, 2, 128, dtype=torch.float16)
    codes, scales = torch.zeros(3, 16, 2, 128, dtype=torch.uint8), torch.zeros(3, 2, 16, dtype=torch.uint8)
    assert S.kv_cache(*(codes.view(torch.float8_e4m3fn) for _ in range(2)), scales, scales).dtype == S.SCALE_CACHE_E4M3
    for bad in (lambda: S.kv_cache(half, half), lambda: S._rows(half[0], 16), lambda: S._rows(half[0].view(torch.int16), 16),
                lambda: S.kv_cache(*(codes.view(torch.float8_e5m2) for _ in range(2)), scales, scales),
                lambda: S.kv_cache(*(codes.view(torch.int8) for _ in range(2)), scales, scales),
                lambda: S.kv_cache(codes, codes, scales.view(torch.int8), scales)):
        with pytest.raises(ValueError):
            bad()
    rows, ints = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.int32)
    b = S.kv_batch(ints[:3], ints[:2], ints.view(2, 4), 2, 1)
    with pytest.raises(ValueError):
        S.scale_cache_attend(S.attend_params(num_q_heads=4), S.kv_cache(codes, codes, scales, scales), b, rows, rows.clone(), ints, ints)


def _attend_size(lib, hq, hkv, e4m3, n_seqs, n_rows, max_rows):
    n = ctypes.c_size_t()
    c = _cache(dtype=S.SCALE_CACHE_E4M3 if e4m3 else S.SCALE_CACHE_BF16, num_kv_heads=hkv)
    assert lib.scale_cache_attend_workspace_size(ctypes.byref(S.ScaleAttend(hq, 0, -1, 0.0)), ctypes.byref(c),
                                                 ctypes.byref(_batch(n_seqs=n_seqs, n_rows=n_rows, max_rows=max_rows)),
                                                 ctypes.byref(n)) == S.SCALE_OK
    return n.value


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (32, 8), (28, 4), (17, 1), (25, 1), (64, 2), (64, 64)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_workspace_for_the_largest_batch_does_for_all(lib, hq, hkv, e4m3):
    """The size of a batch is at least that of every batch of no more sequences, rows and rows of a sequence."""
    sizes = {(s, r, m): _attend_size(lib, hq, hkv, e4m3, s, r, m)
             for s in (1, 7, 4096) for r in (1, 17, 40000) for m in (0, 1, 2, 3, 5, 16, 17, 24, 25, 129, 40000)}
    for x, big in sizes.items():
        for y, small in sizes.items():
            assert small <= big or any(a > b for a, b in zip(y, x)), (y, small, x, big)


def test_the_workspace_of_a_decode_step_follows_its_route(lib):
    """Partial results of as many warps as the route has: two of 520 bytes a row for each of 160 SMs' warps."""
    assert _attend_size(lib, 4, 1, False, 1, 1, 1) <= 2 * 160 * 8 * 8 * 520 + 4096
    assert _attend_size(lib, 32, 8, True, 64, 64, 1) <= 2 * 160 * 16 * 8 * 520 + 4096
    assert _attend_size(lib, 16, 1, False, 1, 1, 1) <= 2 * 160 * 8 * 16 * 520 + 4096


def test_pages_of_the_selection_path_are_checked():
    """Its kernels read bf16 pages of 128 values and do not see their type: an 8-bit cache's pages, half as large, are refused."""
    pages, table = torch.zeros(3, 64, 2, 128, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32)
    kv = S.kv_pages(pages, pages.clone(), table.clone(), 64)
    assert (kv.page_size, kv.num_pages) == (64, 3) and kv.tensors[2].data_ptr() == kv.page_table  # kept alive
    codes = torch.zeros(3, 64, 2, 128, dtype=torch.uint8)
    for bad in ((codes, codes, table, 64), (pages, codes, table, 64), (pages.half(), pages.half(), table, 64),
                (pages, pages[:2], table, 64), (pages[..., :64].contiguous(), pages[..., :64].contiguous(), table, 64),
                (pages, pages, table, 128), (pages[0], pages[0], table, 64), (pages, pages, table.long(), 64)):
        with pytest.raises(ValueError):
            S.kv_pages(*bad)


def test_numbers_beyond_32_bits_are_refused():
    """Not cut to their low bits: a window of 2^32 tokens would be one of none."""
    ints = torch.zeros(8, dtype=torch.int32)
    assert S.attend_params(num_q_heads=8, n_sink=2 ** 31 - 1, n_local=2 ** 31 - 1).n_local == 2 ** 31 - 1
    for bad in (lambda: S.attend_params(num_q_heads=8, n_local=2 ** 32), lambda: S.attend_params(num_q_heads=8, n_sink=2 ** 31),
                lambda: S.attend_params(num_q_heads=2 ** 32 + 8), lambda: S.attend_params(num_q_heads=8, n_local=-2 ** 31 - 1),
                lambda: S.kv_batch(ints[:3], ints[:2], ints.view(2, 4), 2 ** 32 + 2, 1),
                lambda: S.kv_batch(ints[:3], ints[:2], ints.view(2, 4), 2, 2 ** 32)):
        with pytest.raises(ValueError):
            bad()


def test_a_step_without_rows_enqueues_nothing(lib):
    """Empty tensors, whose address torch gives as 0, through every call of the binding."""
    pages, ints = torch.zeros(3, 16, 2, 128, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.int32)
    cache, batch = S.kv_cache(pages, pages.clone()), S.kv_batch(ints[:3], ints[:2], ints.view(2, 4), 0, 1)
    rope = S.rope_axes(torch.zeros(64).double(), torch.zeros(1, 0, dtype=torch.int32))
    q, k = torch.zeros(0, 4, 128, dtype=torch.bfloat16), torch.zeros(0, 2, 128, dtype=torch.bfloat16)
    S.scale_rope(rope, q, k, q, k, stream=0)
    S.scale_rope(rope, q, None, q, None, stream=0)
    S.scale_cache_append(cache, batch, k, k, stream=0)
    S.scale_cache_append(cache, batch, k, k, rope, q, q, stream=0)
    S.scale_cache_read(cache, batch, k, k, stream=0)
    S.scale_cache_read(cache, batch, None, k, stream=0)
    S.scale_cache_attend(S.attend_params(num_q_heads=4), cache, batch, q, q, None, ints, stream=0)
    # what is wrong without rows too
    at, ref = 1 << 30, ctypes.byref
    assert lib.scale_rope(ref(_rope()), 0, 257, at, 65536, at, 65536, 0, None, 0, None, 0, None) == S.SCALE_ERR_UNSUPPORTED
    assert lib.scale_rope(ref(_rope()), 0, 8, None, 1000, None, 1024, 0, None, 0, None, 0, None) == S.SCALE_ERR_INVALID_ARG
    assert lib.scale_cache_read(ref(_cache()), ref(_batch(n_rows=0)), at, 8, None, 0, None) == S.SCALE_ERR_INVALID_ARG

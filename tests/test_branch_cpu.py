"""The calls for drafted trees and beams, without a GPU: struct layouts, refusals before any launch, and the binding's own
checks."""

import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_31568_gb300 as pkg
from _branch import accept, as_words, best, plan, reorder
from paper_2609_31568_gb300 import scale as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 1 << 30  # no address: looked at after everything else
ref = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    pkg.build()
    return S.load()


@pytest.mark.parametrize("name,cls", [("scale_tree_t", S.ScaleTree), ("scale_moves_t", S.ScaleMoves),
                                      ("scale_beam_t", S.ScaleBeam)])
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


def _tree(**over):
    return S.ScaleTree(**{**dict(parents=AT, positions=AT, masks=AT, mask_words=1), **over})


def _moves(**over):
    return S.ScaleMoves(**{**dict(src=AT, dst=AT, n_groups=2, n_moves=10), **over})


def _plan(lib, t=None, b=None, sink=0):
    return lib.scale_tree_plan(ref(t or _tree()), ref(b or _batch()), sink, -1, None)


def _attend(lib, t=None, b=None, c=None, hq=32):
    return lib.scale_cache_attend_tree(ref(S.ScaleAttend(hq, 0, -1, 0.0)), ref(t or _tree()), ref(c or _cache()),
                                       ref(b or _batch()), None, 4096, None, 4096, None, None, 0, None)


def _accept(lib, t=None, b=None, c=None, m=None):
    b = b or _batch()
    return lib.scale_tree_accept(ref(t or _tree()), ref(c or _cache()), ref(b), AT, AT, None, AT, AT, AT, AT,
                                 ref(m or _moves(n_groups=b.n_seqs, n_moves=b.n_rows)), None)


@pytest.mark.parametrize("tree,batch,rc", [
    (dict(mask_words=-1), {}, S.SCALE_ERR_INVALID_ARG),
    (dict(mask_words=0), {}, S.SCALE_ERR_INVALID_ARG),
    (dict(mask_words=1), dict(max_rows=33), S.SCALE_ERR_INVALID_ARG),
    (dict(mask_words=33), {}, S.SCALE_ERR_UNSUPPORTED),
    (dict(mask_words=32), dict(max_rows=1025), S.SCALE_ERR_UNSUPPORTED),
    ({}, dict(n_seqs=4097), S.SCALE_ERR_UNSUPPORTED),
    ({}, dict(n_rows=-1), S.SCALE_ERR_INVALID_ARG),
    ({}, {}, S.SCALE_ERR_INVALID_ARG),  # lists that are no device memory
])
def test_trees_are_checked(lib, tree, batch, rc):
    t, b = _tree(**tree), _batch(**batch)
    assert _plan(lib, t, b) == rc
    assert _attend(lib, t, b) == rc


def test_plan_and_attention_of_nothing(lib):
    assert _plan(lib, b=_batch(n_rows=0)) == S.SCALE_OK
    assert _plan(lib, b=_batch(max_rows=0)) == S.SCALE_OK
    assert _plan(lib, sink=-1) == S.SCALE_ERR_INVALID_ARG
    assert lib.scale_tree_plan(None, ref(_batch()), 0, -1, None) == S.SCALE_ERR_INVALID_ARG
    at = ctypes.c_void_p(AT)
    call = lambda b, t: lib.scale_cache_attend_tree(ref(S.ScaleAttend(32, 0, -1, 0.0)), t, ref(_cache()), ref(b), at,  # noqa: E731
                                                    4096, at, 4096, None, None, 0, None)
    assert call(_batch(n_rows=0), ref(_tree())) == S.SCALE_OK
    assert call(_batch(n_rows=0), None) == S.SCALE_ERR_INVALID_ARG
    assert _attend(lib, c=_cache(page_size=24)) == S.SCALE_ERR_UNSUPPORTED
    assert _attend(lib, hq=264) == S.SCALE_ERR_UNSUPPORTED


def test_accept_is_checked(lib):
    assert _accept(lib) == S.SCALE_ERR_INVALID_ARG  # lists that are no device memory
    assert _accept(lib, b=_batch(max_rows=1025)) == S.SCALE_ERR_UNSUPPORTED
    assert _accept(lib, c=_cache(page_size=8)) == S.SCALE_ERR_UNSUPPORTED
    for m in (_moves(n_groups=3), _moves(n_moves=9), _moves(start=AT), _moves(n_groups=0)):
        assert _accept(lib, m=m) == S.SCALE_ERR_INVALID_ARG
    assert lib.scale_tree_accept(None, ref(_cache()), ref(_batch()), AT, AT, None, AT, AT, AT, AT, ref(_moves()),
                                 None) == S.SCALE_ERR_INVALID_ARG


def test_moves_are_checked(lib):
    def call(caches, m, n=None):
        layers = (S.ScaleCache * len(caches))(*caches)
        return lib.scale_cache_move(layers, len(caches) if n is None else n, ref(m), None)

    start = _moves(start=AT)
    assert call([_cache()], start) == S.SCALE_ERR_INVALID_ARG  # pages that are no device memory
    assert call([_cache()], _moves(start=AT, n_moves=0)) == S.SCALE_OK
    assert call([_cache()], start, 0) == S.SCALE_ERR_INVALID_ARG
    assert call([_cache()] * 1025, start) == S.SCALE_ERR_UNSUPPORTED
    assert call([_cache()], _moves(start=AT, n_groups=4097)) == S.SCALE_ERR_UNSUPPORTED
    assert call([_cache()], _moves(n_moves=(1 << 28) + 2)) == S.SCALE_ERR_UNSUPPORTED
    assert call([_cache()], _moves(start=AT, n_moves=2**31 - 1)) == S.SCALE_ERR_UNSUPPORTED
    assert call([_cache()], _moves(n_groups=0)) == S.SCALE_ERR_INVALID_ARG
    assert call([_cache()], _moves(n_moves=-1)) == S.SCALE_ERR_INVALID_ARG
    assert call([_cache()], _moves(n_moves=9)) == S.SCALE_ERR_INVALID_ARG  # not the same for both groups
    for over in (dict(num_pages=11), dict(page_size=32), dict(num_kv_heads=4), dict(dtype=S.SCALE_CACHE_E4M3)):
        assert call([_cache(), _cache(**over)], _moves(start=AT, n_moves=0)) == S.SCALE_ERR_INVALID_ARG
    assert lib.scale_cache_move(None, 1, ref(start), None) == S.SCALE_ERR_INVALID_ARG


@pytest.mark.parametrize("over,rc", [
    ((0, 1, 10, 1, 0), S.SCALE_ERR_INVALID_ARG),
    ((1, 0, 10, 1, 0), S.SCALE_ERR_INVALID_ARG),
    ((1, 1, 0, 1, 0), S.SCALE_ERR_INVALID_ARG),
    ((1, 1, 10, 0, 0), S.SCALE_ERR_INVALID_ARG),
    ((1, 1, 10, 1, 2), S.SCALE_ERR_INVALID_ARG),
    ((1, 2, 10, 21, 0), S.SCALE_ERR_INVALID_ARG),   # more than there are
    ((1, 33, 10, 1, 0), S.SCALE_ERR_UNSUPPORTED),
    ((1, 2, 100, 65, 0), S.SCALE_ERR_UNSUPPORTED),
    ((1, 1, (1 << 24) + 1, 1, 0), S.SCALE_ERR_UNSUPPORTED),
    ((513, 8, 10, 1, 0), S.SCALE_ERR_UNSUPPORTED),
])
def test_beams_are_checked(lib, over, rc):
    n = ctypes.c_size_t()
    b = S.ScaleBeam(*over)
    assert lib.scale_beam_workspace_size(ref(b), ref(n)) == rc
    assert lib.scale_beam_select(ref(b), AT, 1 << 25, AT, AT, AT, AT, AT, 1 << 40, None) == rc


def test_beam_calls_refuse_bad_pointers(lib):
    b = S.ScaleBeam(2, 2, 100, 4, 0)
    assert lib.scale_beam_select(ref(b), AT, 99, AT, AT, AT, AT, AT, 1 << 40, None) == S.SCALE_ERR_INVALID_ARG
    assert lib.scale_beam_select(ref(b), AT, 100, AT, AT, AT, AT, AT, 1 << 40, None) == S.SCALE_ERR_INVALID_ARG
    assert lib.scale_beam_workspace_size(ref(b), None) == S.SCALE_ERR_INVALID_ARG
    m = _moves(n_groups=4, n_moves=4 * 64)
    call = lambda g, n, m, table=AT, out=AT, stride=3: lib.scale_beam_reorder(ref(_cache()), g, n, AT, AT, table, stride, out,  # noqa: E731
                                                                             ref(m), None)
    assert call(2, 2, m) == S.SCALE_ERR_INVALID_ARG
    assert call(1, 33, m) == S.SCALE_ERR_UNSUPPORTED and call(4096, 2, m) == S.SCALE_ERR_UNSUPPORTED
    assert call(0, 2, m) == S.SCALE_ERR_INVALID_ARG and call(2, 2, m, stride=0) == S.SCALE_ERR_INVALID_ARG
    assert call(2, 2, _moves(n_groups=4, n_moves=255)) == S.SCALE_ERR_INVALID_ARG
    assert call(2, 2, m, stride=2**31 - 1) == S.SCALE_ERR_INVALID_ARG  # (the pointers: any width will do)
    assert call(2, 2, m, out=AT + 16) == S.SCALE_ERR_INVALID_ARG  # tables that overlap


def test_a_beam_workspace_grows_with_the_call(lib):
    size = lambda *x: S.scale_beam_workspace_size(S.beam_params(**dict(zip(("n_groups", "n_beams", "vocab", "n_best"), x))))  # noqa: E731
    assert size(1, 1, 1, 1) >= 16
    assert size(64, 8, 128000, 16) >= 64 * 8 * (16 * 8 + 8)


def test_binding_checks_shapes_and_types():
    ints = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    pages = torch.zeros(3, 16, 2, 128, dtype=torch.bfloat16)
    layers = S.cache_layers([S.kv_cache(pages, pages.clone()), S.kv_cache(pages.clone(), pages.clone())])
    assert len(layers) == 2 and layers[1].page_size == 16 and len(layers.tensors) == 2
    tree = S.draft_tree(ints(5), ints(5), ints(5, 2))
    assert (tree.mask_words, tree.n_rows) == (2, 5) and S.draft_tree(None, ints(5), ints(5, 2)).parents is None
    moves = S.cache_moves(ints(6), ints(6), n_groups=3)
    assert (moves.n_groups, moves.n_moves, moves.start) == (3, 6, None)
    assert S.cache_moves(ints(6), ints(6), ints(4)).n_groups == 3
    batch = S.kv_batch(ints(3), ints(2), ints(2, 4), 6, 1)
    logits, f = torch.zeros(4, 10), torch.zeros(8)
    beam = S.beam_params(n_groups=2, n_beams=2, vocab=10, n_best=3)
    for bad in (lambda: S.draft_tree(ints(4), ints(5), ints(5, 2)), lambda: S.draft_tree(ints(5), ints(5), ints(4, 2)),
                lambda: S.draft_tree(ints(5).long(), ints(5), ints(5, 2)), lambda: S.draft_tree(ints(5), ints(5), ints(2, 5).t()),
                lambda: S.draft_tree(ints(5), ints(5).float(), ints(5, 2)), lambda: S.cache_moves(ints(6), ints(5), n_groups=3),
                lambda: S.cache_moves(ints(6), ints(6)), lambda: S.cache_moves(ints(6), ints(6), ints(4), 3),
                lambda: S.cache_moves(ints(6), ints(6).long(), n_groups=3), lambda: S.cache_moves(ints(6), ints(6), n_groups=2 ** 32),
                lambda: S.beam_params(n_groups=2 ** 31, n_beams=1, vocab=1, n_best=1),
                lambda: S.scale_tree_plan(tree, batch),  # 6 rows, 5 in the tree
                lambda: S.scale_beam_select(beam, logits.double(), f, f, ints(8), ints(8), f),
                lambda: S.scale_beam_select(beam, logits[:3], f, f, ints(8), ints(8), f),
                lambda: S.scale_beam_select(beam, torch.zeros(10, 4).t(), f, f, ints(8), ints(8), f),
                lambda: S.scale_beam_select(beam, logits, f[:3], f, ints(8), ints(8), f),
                lambda: S.scale_beam_select(beam, logits, f, f, ints(5), ints(8), f),
                lambda: S.scale_beam_select(beam, logits, f, f, ints(8).long(), ints(8), f),
                lambda: S.scale_beam_reorder(layers, ints(4, 3), ints(4), ints(4), ints(4, 3), moves),
                lambda: S.scale_beam_reorder(layers, ints(4, 3), ints(4), ints(2, 2), ints(4, 4), moves),
                lambda: S.scale_beam_reorder(layers, ints(4, 3), ints(3), ints(2, 2), ints(4, 3), moves)):
        with pytest.raises(ValueError):
            bad()


def test_a_step_without_rows_enqueues_nothing(lib):
    ints = lambda *n: torch.zeros(*n, dtype=torch.int32)  # noqa: E731
    pages = torch.zeros(3, 16, 2, 128, dtype=torch.bfloat16)
    cache, batch = S.kv_cache(pages, pages.clone()), S.kv_batch(ints(3), ints(2), ints(2, 4), 0, 1)
    tree = S.draft_tree(ints(0), ints(0), ints(0, 1))
    q = torch.zeros(0, 4, 128, dtype=torch.bfloat16)
    S.scale_tree_plan(tree, batch, stream=0)
    S.scale_cache_attend_tree(S.attend_params(num_q_heads=4), tree, cache, batch, q, q, None, ints(8), stream=0)
    S.scale_cache_move(S.cache_layers([cache]), S.cache_moves(ints(0), ints(0), ints(3)), stream=0)


def test_references_by_hand():
    """A root, its children 1 and 2, 3 below 2, 4 below 3, a row that is none and one below it."""
    parents = [-1, 0, 0, 2, 3, 7, 5]
    positions, seen = plan(parents, 10)
    assert positions == [10, 11, 11, 12, 13, -1, -1]
    assert seen == [{0}, {0, 1}, {0, 2}, {0, 2, 3}, {0, 2, 3, 4}, set(), set()]
    assert plan(parents, 10, n_local=1)[1][4] == {3, 4} and plan(parents, 10, n_sink=11, n_local=1)[1][4] == {0, 3, 4}
    assert as_words([{0, 33}, {31}], 2).tolist() == [[1, 2], [-2 ** 31, 0]]
    assert accept(parents, 10, [5, 8, 8, 9, 4, 8, 9], [8, 1, 9, 3, 2, 0, 0], 5) == ([0, 1], 1)  # the lower of two eights
    assert accept(parents, 10, [5, 7, 8, 9, 4, 8, 9], [8, 1, 9, 3, 2, 0, 0], 5) == ([0, 2, 3], 3)
    assert accept(parents, 10, [5] * 7, [0] * 7, 6) == ([], 6) and accept(parents, 10, [5] * 7, [0] * 7, None) == ([0], 0)
    assert accept(parents, -1, [5] * 7, [0] * 7, 5) == ([], 5)
    table = [[1, 2, 3], [1, 4, 5], [1, 6, 7]]
    new, moves = reorder(table, [2, 2, 0], 18, 16)  # 0 goes on in beam 2's place, beam 1's pages become a copy
    assert new == [[1, 6, 7], [1, 4, 5], [1, 2, 3]]
    assert moves[0] == [] and moves[2] == [] and moves[1] == [(96, 64), (97, 65)]
    got = best(np.log(np.array([[0.5, 0.25, 0.25], [0.8, 0.1, 0.1]])), np.array([0.0, -1.0]), 4)
    assert [(b, t) for _, b, t in got] == [(0, 0), (1, 0), (0, 1), (0, 2)]

"""Sizes of the calls for drafted trees and beams, without a GPU: workspaces, bounds."""

import ctypes

import pytest

import paper_2609_31568_gb300 as pkg
from paper_2609_31568_gb300 import scale as S

AT = 1 << 30  # no address: looked at after everything else


@pytest.fixture(scope="module")
def lib():
    pkg.build()
    return S.load()


def size(groups, beams, vocab, n_best):
    return S.scale_beam_workspace_size(S.beam_params(n_groups=groups, n_beams=beams, vocab=vocab, n_best=n_best))


@pytest.mark.parametrize("beams,n_best", [(1, 1), (1, 8), (3, 2), (8, 16), (32, 64)])
@pytest.mark.parametrize("vocab", [70, 8192, 8193, 32000, 128000, 1 << 24])
def test_a_workspace_does_for_every_smaller_call(lib, beams, n_best, vocab):
    """A batch's finished groups leave; the workspace stays the largest batch's."""
    sizes = [size(g, beams, vocab, n_best) for g in range(1, min(700, 4096 // beams) + 1)]
    assert sizes == sorted(sizes)


def test_a_workspace_does_for_fewer_beams_tokens_and_continuations(lib):
    for groups in (1, 9, 37, 38, 100):
        for at, values in ((1, range(1, 33)), (2, [64, 100, 8191, 8192, 8193, 16384, 16385, 50000, 100003, 128000, 2 ** 20, 2 ** 24]), (3, range(1, 65))):
            for call in ([groups, 8, 128000, 16], [groups, 2, 40000, 4], [groups, 32, 64, 64]):
                sizes = [size(*call[:at], x, *call[at + 1:]) for x in values]
                assert sizes == sorted(sizes), (call, at)


def test_rows_of_one_beam(lib):
    """Choices of a batch's nodes: as many rows as its trees can have."""
    n = ctypes.c_size_t()
    ask = lambda groups, beams: lib.scale_beam_workspace_size(ctypes.byref(S.ScaleBeam(groups, beams, 100, 1, 0)), ctypes.byref(n))  # noqa: E731
    assert ask(64 * 200, 1) == S.SCALE_OK and ask(4096 * 1024, 1) == S.SCALE_OK
    assert ask(4096 * 1024 + 1, 1) == S.SCALE_ERR_UNSUPPORTED
    assert ask(2048, 2) == S.SCALE_OK and ask(2049, 2) == S.SCALE_ERR_UNSUPPORTED
    b = S.ScaleBeam(12800, 1, 100, 1, 0)
    # past the bounds, at pointers that are no device memory
    assert lib.scale_beam_select(ctypes.byref(b), AT, 100, AT, AT, AT, AT, AT, 1 << 40, None) == S.SCALE_ERR_INVALID_ARG

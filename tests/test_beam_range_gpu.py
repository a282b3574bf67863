"""Beam selection at the ends of its range: logits below the normal numbers."""

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

"""Gradients of the dense head over several tiles of tokens and several pieces of the vocabulary, added to what dw holds.
Inputs and bounds as in test_gpu_loss.py."""

import pytest

from paper_2608_02703_gb300 import archead

from .test_gpu_loss import HALF_STEP, U, _build, _draw, _exact, _near, _torch  # noqa: F401 - a fixture among them

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("M,V,d,ldx,ldw", [
    (700, 3001, 200, 200, 200),  # three tiles of tokens, one piece
    (700, 200000, 40, 40, 40),  # and two pieces
    (200, 600000, 16, 16, 16),  # two pieces, x read where it lies
    (200, 600000, 13, 15, 16),  # gathered; rows of dw by single values
    (40, 600000, 16, 16, 24),  # G in two parts
    (50, 600000, 13, 13, 16),
], ids=str)
def test_accumulation_over_tiles_and_pieces(M, V, d, ldx, ldw, dtype):
    torch = _torch()
    x, w, t, g = _draw(M, V, d, dtype, seed=71, ignored=0.2, ldx=ldx, ldw=ldw)
    loss, ce, lse = archead.archead_loss_create(M, V, d), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    archead.archead_linear_ce(loss, x, w, t, ce, lse=lse)
    whole = torch.randn((V, ldw), device="cuda").to(w.dtype)
    before, more = whole.clone(), whole[:, :d]
    dx = torch.empty((M, d), dtype=x.dtype, device="cuda")
    archead.archead_linear_ce_backward(loss, x, w, t, lse, g, dx=dx, dw=more, accumulate=True)
    fresh, alone = torch.empty_strided(w.shape, w.stride(), dtype=w.dtype, device="cuda"), torch.empty_like(dx)
    archead.archead_linear_ce_backward(loss, x, w, t, lse, g, dw=fresh)
    archead.archead_linear_ce_backward(loss, x, w, t, lse, g, dx=alone)
    assert archead.archead_loss_sync_status(loss) == archead.OK
    # (V of some 2^19 adds that many terms of one sum: what the terms of the loss's sum cost is added to the bound)
    exact_dx, exact_dw, dx_off, dw_off = _exact(x, w, t, g, dtype, sums=V / 4096 * U)[2:]
    tiny = 2.0 ** -25 if dtype == "fp16" else 2.0 ** -126
    for got in (dx, alone):
        _near(got, exact_dx, dx_off + HALF_STEP[dtype] * (exact_dx.abs() + dx_off) + tiny, "dx")
    _near(fresh, exact_dw, dw_off + HALF_STEP[dtype] * (exact_dw.abs() + dw_off) + tiny, "dw")
    want = exact_dw + before[:, :d].double()
    _near(more, want, dw_off + U * want.abs() + HALF_STEP[dtype] * (want.abs() + dw_off) + tiny, "dw, added")
    assert torch.equal(whole[:, d:], before[:, d:])
    # Added to nothing it is the gradient.
    more.zero_()
    archead.archead_linear_ce_backward(loss, x, w, t, lse, g, dw=more, accumulate=True)
    assert torch.equal(more, fresh)

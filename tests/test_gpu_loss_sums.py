"""Sums of the dense head's loss and its gradient, where their rounding shows.

Tensor cores add to a running sum and cut what does not fit into fp32: by less than a unit in the last place, 2^-23 of
the sum so far, for every 16 products, and always toward zero.  A logit is cut into parts of 1024 products for that, which
are added to one another by ordinary additions, each within 2^-24: it is within 64 * 2^-23 of its absolute terms beside
these.  The gradients' own sums are of 2000 products at most here.  The gradient computes a logit as the loss does, in the same parts: what it is off by is the same
in l and in lse, and exp(l - lse) does not see what both have.
"""

import pytest

from paper_2608_02703_gb300 import archead

from .test_gpu_loss import HALF_STEP, IGNORED, U, _build, _draw, _dtype, _near, _torch  # noqa: F401 - a fixture among them

pytestmark = pytest.mark.gpu

LOGIT = 64 * 2.0 ** -23
CHAIN = 512 * 2.0 ** -23
TINY = {"bf16": 2.0 ** -126, "fp16": 2.0 ** -25}


def _run(x, w, t, g, loss=None, **kw):
    torch = _torch()
    (M, d), V = x.shape, w.shape[0]
    loss = loss or archead.archead_loss_create(M, V, d)
    ce, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_strided(w.shape, w.stride(), dtype=w.dtype, device="cuda")
    archead.archead_linear_ce(loss, x, w, t, ce, lse=lse, **kw)
    archead.archead_linear_ce_backward(loss, x, w, t, lse, g, dx=dx, dw=dw, **kw)
    assert archead.archead_loss_sync_status(loss) == archead.OK
    return ce, lse, dx, dw


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("M,d,ldx", [(40, 4096, 4096), (40, 4096, 4099), (300, 4096, 4096), (40, 16384, 16384),
                                     (130, 16384, 16384)], ids=str)
def test_tokens_that_the_model_is_sure_of(M, d, ldx, dtype):
    """1 - p from 1e-1 to 1e-5, of values that are no whole numbers.  Of a logit all but its difference to the others
    cancels: p of the other columns, and 1 - p of the target's, are within twice the logits' error of themselves.  What is
    left of the target's p itself: lse's rounding (2^-20 between 16 and 32), the sum's (some 20 additions of 2^-24 of 1), the
    exponential's (2^-22): together less than 2^-17."""
    torch = _torch()
    V = 2000
    gen = torch.Generator(device="cuda").manual_seed(d + M)
    w = (torch.randn((V, d), generator=gen, device="cuda") * (2.5 / d ** 0.5)).to(_dtype(dtype))
    t = torch.randint(0, V, (M,), generator=gen, device="cuda").to(torch.int32)
    x = torch.empty((M, ldx), dtype=_dtype(dtype), device="cuda")[:, :d]
    of_target, free = w[t.long()].float(), torch.randn((M, d), generator=gen, device="cuda")
    want = 12 + 11 * torch.rand((M, 1), generator=gen, device="cuda")
    gain = (want - (free * of_target).sum(dim=1, keepdim=True)) / of_target.square().sum(dim=1, keepdim=True)
    x.copy_(free + gain * of_target)
    g = 0.5 + torch.rand(M, generator=gen, device="cuda")
    _, lse, dx, dw = _run(x, w, t, g)
    xx, ww, gg, at = x.double(), w.double(), g.double()[:, None], t.long()[:, None]
    logits = xx @ ww.t()
    exact_lse = torch.logsumexp(logits, dim=1, keepdim=True)
    assert exact_lse.max() < 32
    G = torch.exp(logits - exact_lse)
    sure = -torch.expm1(logits - exact_lse).gather(1, at)
    assert sure.min() < 3e-5 and sure.max() > 3e-2
    delta = (LOGIT + 16 * U) * (xx.abs() @ ww.abs().t()).max()
    assert delta < 2.0 ** -7
    assert (lse[:, None] - exact_lse).abs().max() <= delta + 2.0 ** -18
    G.scatter_(1, at, -sure)
    off = (2 * delta + 2.0 ** -15 + HALF_STEP[dtype]) * G.abs() + 2.0 ** -126
    off.scatter_add_(1, at, torch.full_like(sure, 2.0 ** -17))
    off, G = off * gg, G * gg
    if dtype == "fp16":
        off += 2.0 ** -25 * 2.0 ** -14 * gg.max()
    for got, exact, bound in ((dx, G @ ww, (off + CHAIN * G.abs()) @ ww.abs()),
                              (dw, G.t() @ xx, (off + CHAIN * G.abs()).t() @ xx.abs())):
        _near(got, exact, bound + HALF_STEP[dtype] * (exact.abs() + bound) + TINY[dtype], "gradient")
    # The whole row of a token, held against its own size: 1e-4 of the target's p would be all of it for the surest.
    rows = (dx.double() - G @ ww).norm(dim=1) / (G @ ww).norm(dim=1)
    assert (rows <= 2 * delta + 2.0 ** -15 + 2 * HALF_STEP[dtype] + 2.0 ** -16 / sure[:, 0]).all()

"""Logits at the ends of fp32's range in the dense head's loss."""

import pytest

from paper_2608_02703_gb300 import archead

from .test_gpu_loss import U, _build, _near, _torch  # noqa: F401 - a fixture among them

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,V,d", [(4, 300, 64), (4, 9000, 64), (60, 3000, 4096), (300, 3000, 64)], ids=str)
def test_infinite_logits(M, V, d):
    """lse is infinite with a logit, ce as its definition has it; what is -infinity adds nothing; no other token changes."""
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(51)
    x = torch.randn((M, d), generator=gen, device="cuda").to(torch.bfloat16)
    w = (torch.randn((V, d), generator=gen, device="cuda") * 0.2).to(torch.bfloat16)
    t = torch.randint(V // 2, V, (M,), generator=gen, device="cuda").to(torch.int32)
    w[:, 0], x[:, 0] = 0, 0
    w[7, 0], w[V // 3, 0] = 2.0 ** 40, -2.0 ** 40
    loss = archead.archead_loss_create(M, V, d)
    want, want_lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    archead.archead_linear_ce(loss, x, w, t, want, lse=want_lse)
    x[0, 0] = 2.0 ** 100  # l[7] infinite, l[V / 3] -infinite
    x[1, 0], t[1] = -2.0 ** 100, V // 3  # the other way round, and the infinite one the target
    x[2, 0], t[2] = 2.0 ** 100, V // 3  # the target -infinite
    ce, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    archead.archead_linear_ce(loss, x, w, t, ce, lse=lse)
    archead.archead_linear_ce_backward(loss, x, w, t, lse, torch.ones(M, device="cuda"), dx=dx, dw=dw)
    assert archead.archead_loss_sync_status(loss) == archead.OK
    inf = float("inf")
    assert lse[:3].tolist() == [inf] * 3 and ce[0] == inf and ce[1].isnan() and ce[2] == inf
    assert torch.equal(ce[3:], want[3:]) and torch.equal(lse[3:], want_lse[3:])
    # exp(inf - inf) is no number: of these tokens' rows, and of the weight's rows with infinite logits.
    rows = torch.ones(V, dtype=torch.bool, device="cuda")
    rows[7] = rows[V // 3] = False
    assert dx[:3].isnan().all() and dx[3:].isfinite().all() and dw[~rows].isnan().all() and dw[rows][:, 1:].isfinite().all()


def test_logits_of_minus_infinity():
    torch = _torch()
    M, V, d = 5, 700, 64
    gen = torch.Generator(device="cuda").manual_seed(52)
    x = torch.randint(-2, 3, (M, d), generator=gen, device="cuda").to(torch.bfloat16)
    w = torch.randint(-1, 2, (V, d), generator=gen, device="cuda").to(torch.bfloat16)
    t = torch.randint(0, 300, (M,), generator=gen, device="cuda").to(torch.int32)
    x[:, 0], w[:, 0] = 2.0 ** 100, 0
    w[300:, 0] = -2.0 ** 40
    loss, ce, lse = archead.archead_loss_create(M, V, d), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    archead.archead_linear_ce(loss, x, w, t, ce, lse=lse)
    logits = x.double() @ w[:300].double().t()
    want = torch.logsumexp(logits, dim=1)
    _near(lse, want, 2.0 ** -16 + 2 * U * want.abs(), "lse")
    want = want - logits.gather(1, t.long()[:, None])[:, 0]
    _near(ce, want, 2.0 ** -16 + 2 * U * want.abs(), "ce")

"""Waits that give up in each form of the dense head's loss: x read where it lies, and gathered with the weights' first loads
ahead; sums in parts, with registers handed on.  Test of the gradient's products with many tokens: test_gpu_loss.py.

A wait of one cycle gives up if it outlasts the time that the hardware suspends a probe.  Sums over 16384 of few tokens
wait for the weights' way from memory that long in about every call or every other one; a call is repeated until one has
reported it, of 60 at most."""

import pytest

from paper_2608_02703_gb300 import archead

from .test_gpu_loss import IGNORED, _build, _torch  # noqa: F401 - a fixture among them

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,ldx", [(40, 16384), (200, 16384), (200, 16387)])
def test_every_form_gives_up_and_recovers(M, ldx):
    torch = _torch()
    V, d = 65536, 16384
    gen = torch.Generator(device="cuda").manual_seed(61)
    x = torch.randn((M, ldx), generator=gen, device="cuda").to(torch.bfloat16)[:, :d]
    w = (torch.randn((V, d), generator=gen, device="cuda") * 0.02).to(torch.bfloat16)
    t = torch.randint(0, V, (M,), generator=gen, device="cuda").to(torch.int32)
    t[::9] = IGNORED
    g = torch.rand(M, generator=gen, device="cuda")
    loss, ce, lse = archead.archead_loss_create(M, V, d), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)

    def forward():
        archead.archead_linear_ce(loss, x, w, t, ce, lse=lse)

    def backward(lse, **kw):
        archead.archead_linear_ce_backward(loss, x, w, t, lse, g, **kw)

    forward()
    backward(lse, dx=dx, dw=dw)
    assert archead.archead_loss_sync_status(loss) == archead.OK
    want = [v.clone() for v in (ce, lse, dx, dw)]
    for call in (forward, lambda: backward(want[1], dw=dw), lambda: backward(want[1], dx=dx)):
        archead.archead_loss_set_wait_budget(loss, 1)
        said = archead.OK
        for _ in range(60):
            call()
            said = archead.archead_loss_sync_status(loss)
            assert archead.archead_loss_sync_status(loss) == archead.OK
            if said != archead.OK:
                break
        assert said == archead.ERR_DEVICE_TIMEOUT
        archead.archead_loss_set_wait_budget(loss, 2_000_000_000)
        for v in (ce, lse, dx, dw):
            v.zero_()
        forward()
        backward(lse, dx=dx, dw=dw)
        assert archead.archead_loss_sync_status(loss) == archead.OK
        assert all(torch.equal(a, b) for a, b in zip((ce, lse, dx, dw), want))

"""Sums of the dense head's loss and its gradient, where their rounding shows.

Tensor cores add to a running sum and cut what does not fit into fp32: by less than a unit in the last place, 2^-23 of
the sum so far, for every 16 products, and always toward zero.  A sum is cut into parts for that (of 1024 products for
a logit, of 16384 for an element of a gradient) and the parts are added to one another by ordinary additions, each within
2^-24.  So a logit is within 64 * 2^-23 of its absolute terms beside its additions, a gradient's element within
1024 * 2^-23 of them.  The gradient computes a logit as the loss does, in the same parts: what it is off by is the same
in l and in lse, and exp(l - lse) does not see what both have.
"""

import pytest

from paper_2608_02703_gb300 import archead

from .test_gpu_loss import HALF_STEP, IGNORED, U, _build, _draw, _dtype, _near, _torch  # noqa: F401 - a fixture among them

pytestmark = pytest.mark.gpu

LOGIT = 64 * 2.0 ** -23
CHAIN = 1024 * 2.0 ** -23
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


def _mean_off(got, want):
    """The mean of the errors relative to the values, with their signs: roundings to nearest cancel in it."""
    return ((got.double() - want) / want).mean().item()


@pytest.mark.parametrize("M,wide", [(1 << 18, 64), (40000, 300)], ids=str)
def test_sums_over_many_tokens_are_not_cut_short(M, wide):
    """Terms of one sign.  Logits are 0 and factors powers of two: p is 1 / V and G exact.  fp16's rounding of an element
    of dw is 2^-11 at most and 2^-12.5 in the mean square or less, either way: of 60 * 64 elements 2^-18 in the mean, and
    four times that at most."""
    torch = _torch()
    V = 64
    gen = torch.Generator(device="cuda").manual_seed(41)
    x = (0.5 + torch.rand((M, wide), generator=gen, device="cuda")).half()
    w = torch.zeros((V, (wide + 7) // 8 * 8), dtype=torch.float16, device="cuda")[:, :wide]
    t = torch.full((M,), V - 1, dtype=torch.int32, device="cuda")
    g = torch.full((M,), 2.0 ** -10, device="cuda")
    dw = _run(x, w, t, g)[3]
    want = (x.double().sum(dim=0) * 2.0 ** -16).expand(V - 1, wide)
    assert abs(_mean_off(dw[:V - 1], want)) <= CHAIN + (M / 16384 + 1) * U + 2.0 ** -16
    assert abs(_mean_off(dw[V - 1:], -want[:1] * (V - 1))) <= CHAIN + (M / 16384 + 1) * U + 2.0 ** -13.5


@pytest.mark.parametrize("M,V", [(40, 1 << 18), (200, 1 << 18), (2500, 1 << 17)], ids=str)
def test_sums_over_a_large_vocabulary_are_not_cut_short(M, V):
    """The same for dx: the targets' row of w is 0, the others are positive.  Of 8192 columns, the same for every token,
    roundings are 2^-19 in the mean, and four times that at most; p, a power of two but for 2^-20 of itself, may be
    rounded to one in G."""
    torch = _torch()
    d = 8192
    gen = torch.Generator(device="cuda").manual_seed(42)
    w = torch.empty((V, d), dtype=torch.float16, device="cuda")
    for part in w.split(1 << 14):
        part.copy_(0.5 + torch.rand(part.shape, generator=gen, device="cuda"))
    w[5] = 0
    x = torch.zeros((M, d), dtype=torch.float16, device="cuda")
    t = torch.full((M,), 5, dtype=torch.int32, device="cuda")
    dx = _run(x, w, t, torch.ones(M, device="cuda"))[2]
    want = sum(part.double().sum(dim=0) for part in w.split(1 << 14)) / V
    assert (dx == dx[0]).all()
    assert abs(_mean_off(dx[0], want)) <= CHAIN + (V / 16384 + 32) * U + 2.0 ** -17 + 2.0 ** -20


@pytest.mark.parametrize("M,V,d", [(1 << 20, 40, 8), (2, 1 << 24, 8), (3, 300, 1 << 16)], ids=str)
def test_largest_sizes_within_their_chains(M, V, d):
    """Bounds that go by how long a sum on the tensor cores is.  Targets of the vocabulary's first half, states and factors
    of one sign: gradients are large beside the bounds."""
    torch = _torch()
    x, w, t, g = _draw(M, V, d, "bf16", seed=43)
    x, t, g = x.abs(), t % (V // 2), g.abs()
    _, _, dx, dw = _run(x, w, t, g)
    x, w, g = x.double(), w.double(), g.double()
    at = t.long()[:, None]
    G = torch.softmax(x @ w.t(), dim=1)
    off = (2.0 ** -15 + 2 * V / 4096 * U) * G + 2.0 ** -126
    G.scatter_add_(1, at, torch.full((M, 1), -1.0, dtype=torch.float64, device="cuda"))
    off = (off + HALF_STEP["bf16"] * G.abs()) * g.abs()[:, None]
    G *= g[:, None]
    for got, exact, bound in ((dx, G @ w, (off + (CHAIN + (V / 16384 + 32) * U) * G.abs()) @ w.abs()),
                              (dw, G.t() @ x, (off + (CHAIN + (M / 16384 + 32) * U) * G.abs()).t() @ x.abs())):
        _near(got, exact, bound + HALF_STEP["bf16"] * (exact.abs() + bound) + 2.0 ** -126, "gradient")
        assert exact.norm() > 4 * bound.norm() or V == 1 << 24 and got is dw


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("M,V,d,ignored", [(1, 3000, 512, 0), (4, 4096, 512, 0), (33, 3001, 200, 0.3), (64, 3000, 1500, 0),
                                           (32, 2000, 77, 0.1), (50, 600000, 64, 0)], ids=str)
def test_gradients_of_few_tokens_are_rounded_once(M, V, d, ignored, dtype):
    """Up to 64 tokens G is held in two parts: of an element half a step of half a step is lost, in fp16 no less than half of
    2^-24 of its scale.  So what dx and dw are off by is, but for these errors, the rounding of their values: a distance
    to the nearest number of the type changes by no more than the value does."""
    torch = _torch()
    gen = torch.Generator(device="cuda").manual_seed(V + d)
    x = torch.randn((M, d), generator=gen, device="cuda").to(_dtype(dtype))
    w = torch.empty((V, (d + 7) // 8 * 8), dtype=_dtype(dtype), device="cuda")[:, :d]
    w.copy_(torch.randn((V, d), generator=gen, device="cuda") * (2.5 / d ** 0.5))
    t = torch.randint(0, V, (M,), generator=gen, device="cuda").to(torch.int32)
    t[torch.rand(M, generator=gen, device="cuda") < ignored] = IGNORED
    g = 0.5 + torch.rand(M, generator=gen, device="cuda")
    _, _, dx, dw = _run(x, w, t, g)
    live = (t != IGNORED).double()[:, None]
    xx, ww, gg, at = x.double(), w.double(), g.double()[:, None] * live, t.clamp_min(0).long()[:, None]
    logits = xx @ ww.t()
    delta = (LOGIT + 16 * U) * (xx.abs() @ ww.abs().t()).max()
    G = torch.softmax(logits, dim=1)
    off = (2 * delta + 2.0 ** -15) * G + 2.0 ** -126
    G.scatter_add_(1, at, torch.full((M, 1), -1.0, dtype=torch.float64, device="cuda"))
    G, off = G * gg, (off + HALF_STEP[dtype] ** 2 * G.abs()) * gg
    if dtype == "fp16":
        off += 2.0 ** -25 * 2.0 ** -14 * gg.max()
    chain = min(CHAIN, V / 16 * 2.0 ** -23)
    for got, exact, bound in ((dx, G @ ww, (off + chain * G.abs()) @ ww.abs()), (dw, G.t() @ xx, (off + CHAIN / 64 * G.abs()).t() @ xx.abs())):
        rounding = (exact.to(got.dtype).double() - exact).norm()
        assert (got.double() - exact).norm() <= rounding + 2 * (bound + TINY[dtype]).norm()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("M,d,ldx", [(65, 512, 512), (200, 513, 514), (300, 510, 510), (1000, 768, 768)], ids=str)
def test_dx_of_more_tokens_keeps_what_its_targets_weigh(M, d, ldx, dtype):
    """Logits of 0: p is 1 / 4096 in all columns, and G the same but at the target, where nearly all of its weight is.  G is
    rounded to 16 bits: alike in the other columns, half a step of what they sum up to; at the target what rounding took
    is added to dx.  So dx is off by its own rounding, but for that (see the test before)."""
    torch = _torch()
    V = 4096
    gen = torch.Generator(device="cuda").manual_seed(81)
    x = torch.zeros((M, ldx), dtype=_dtype(dtype), device="cuda")[:, :d]
    w = torch.empty((V, (d + 7) // 8 * 8), dtype=_dtype(dtype), device="cuda")[:, :d]
    w.copy_(torch.randn((V, d), generator=gen, device="cuda"))
    t = torch.randint(0, V, (M,), generator=gen, device="cuda").to(torch.int32)
    t[::5] = IGNORED
    t[1], t[2] = 0, V - 1
    g = 0.5 + torch.rand(M, generator=gen, device="cuda")
    dx = _run(x, w, t, g)[2]
    live = (t != IGNORED).double()[:, None]
    ww, gg = w.double(), g.double()[:, None] * live
    at_target, even = ww[t.clamp_min(0).long()], ww.sum(dim=0, keepdim=True) / V
    exact = gg * (even - at_target)
    # p within 2^-15 of itself; sums of 4096 products in one, cut short by 256 * 2^-23 of their absolute terms at most,
    # and added with some 40 roundings.
    bound = gg * ((2.0 ** -15 + HALF_STEP[dtype]) * even.abs()
                  + (2.0 ** -15 + 40 * U) * (ww.abs().sum(dim=0, keepdim=True) / V + at_target.abs()) + 2.0 ** -24 * at_target.abs())
    rounding = (exact.to(dx.dtype).double() - exact).norm()
    assert (dx.double() - exact).norm() <= rounding + 2 * (bound + TINY[dtype]).norm()

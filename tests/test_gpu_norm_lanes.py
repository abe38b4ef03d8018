"""All threads of a row use the factor that is written.

A row's sum of squares is carried as two floats through a butterfly of its 32 lanes.  The order in which the low parts
are added is not the same in the two lanes of an exchange, and they can end a unit in the last place of the low
part apart: some 2^-47 of the sum, in one row of 300.  Where the factor is next to a border between two floats, that decides
which of them a lane takes.  Rows whose lanes differ are found here by the same additions in numpy, and eps moves their
factors over a border in small steps."""

from fractions import Fraction

import numpy as np
import pytest

from paper_2608_02703_gb300 import archead

from .test_gpu_norm import _build, _torch  # noqa: F401 - a fixture among them

pytestmark = pytest.mark.gpu

F = np.float32


def _add(hi, lo, v, rest):
    """A sum in two floats and one more, the low parts from the right."""
    s = hi + v
    b = s - hi
    e = (hi - (s - b)) + (v - b)
    return s, lo + (e + rest)


def _lanes(rows):
    """Sums of the 32 lanes, for rows of 512 values of 16 bits: a lane has eight neighbours of each half, two sums."""
    v = rows.reshape(-1, 2, 32, 8).transpose(0, 2, 1, 3).reshape(-1, 32, 8, 2)
    hi, lo = np.zeros(v.shape[:2] + (2,), F), np.zeros(v.shape[:2] + (2,), F)
    for i in range(8):
        s = hi + v[:, :, i] ** 2
        b = s - hi
        lo = lo + ((hi - (s - b)) + (v[:, :, i] ** 2 - b))
        hi = s
    h, l = np.zeros(v.shape[:2], F), np.zeros(v.shape[:2], F)
    for j in range(2):
        h, l = _add(h, l, hi[:, :, j], lo[:, :, j])
    for o in (16, 8, 4, 2, 1):
        other = np.arange(32) ^ o
        h, l = _add(h, l, h[:, other], l[:, other])
    return h, l


def test_lanes_agree_next_to_a_border():
    torch = _torch()
    rng = np.random.default_rng(1)
    rows = torch.from_numpy(rng.standard_normal((40000, 512)).astype(F)).to(torch.bfloat16)
    values = rows.float().numpy()
    h, l = _lanes(values)
    spread = (l.max(axis=1) - l.min(axis=1)) / h[:, 0]
    weight = torch.ones(512, device="cuda")
    steps = 1024
    y, rstd = torch.empty((steps, 512), device="cuda"), torch.empty(steps, device="cuda")
    for i in np.argsort(spread)[-24:]:
        assert spread[i] > 2.0 ** -49
        mean = sum(Fraction(float(v)) ** 2 for v in values[i]) / 512
        # The border below the factor without eps, and the eps that leads to it.
        r = F(1 / np.sqrt(float(mean) + 1e-6))
        border = (Fraction(float(r)) + Fraction(float(np.nextafter(r, F(0))))) / 2
        eps = 1 / border ** 2 - mean
        assert 0 < eps < Fraction(1, 100000)
        x = rows[i:i + 1].cuda()
        for k in range(steps):
            archead.archead_rms_norm(x, weight, float(eps + mean * Fraction(k - steps // 2, 2 ** 50)), y=y[k:k + 1],
                                     rstd=rstd[k:k + 1])
        assert len(rstd.unique()) == 2  # (the border is within the steps)
        assert torch.equal(y, x.float() * rstd[:, None])

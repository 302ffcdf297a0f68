"""The lower tail of GELU, g times the normal distribution function, where 1 + erf would cancel: relative to the value, however small it is."""
import math

import numpy as np
import pytest
import torch

from oracle import feed_forward as F
from paper_2502_08145_amd import binding as B

TAIL = -np.arange(16.0, 97.0) / 8   # -2 to -12, bf16 numbers


def test_oracle_gelu_keeps_its_digits_in_the_lower_tail():
    """Against the integral of the density from g down, by Simpson's rule on exp(-t^2 / 2) / exp(-g^2 / 2): nothing there cancels."""
    t = np.linspace(0.0, 12.0, 24001)
    weights = np.where(np.arange(t.size) % 2 == 1, 4.0, 2.0)
    weights[[0, -1]] = 1.0
    for g in TAIL:
        density = math.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        below = density * float((weights * np.exp(g * t - t * t / 2)).sum()) * (t[1] - t[0]) / 3
        value, slope = (float(v[0]) for v in F.activation(np.array([g]), "gelu"))
        assert abs(value - g * below) <= 1e-11 * abs(g * below), g
        assert abs(slope - (below + g * density)) <= 1e-11 * abs(slope), g


# The kernels, relative to the value.  Distribution function and density have an exponential whose exponent g^2 / 2 is rounded three times, by 2^-24 each:
# g^2 2^-23 <= 2^-15 of themselves here; 2^-19 for what multiplies it: below 2^-14 together.  In the slope p + g density(g), p takes at most
# 1.67 of the difference's magnitude: 2^-13.  Then one rounding to bf16, U.
U, ACT, SLOPE = 2.0 ** -8, 2.0 ** -14, 2.0 ** -13


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16).cuda()


def _near(got, ref, bound, what):
    off = np.abs(got.float().cpu().numpy().astype(np.float64) - ref) / np.abs(ref)
    assert off.max() <= bound, f"{what}: {off.max():.3e} of the value, {bound:.3e} allowed"


@pytest.mark.gpu
@pytest.mark.parametrize("F_", [81, 88])
@pytest.mark.parametrize("kept", ["bf16", "8 bits"])
def test_gelu_gradients_in_the_lower_tail(F_, kept):
    M = 5
    g = np.tile(np.resize(TAIL, F_), (M, 1))
    if kept == "8 bits":   # all of these are e4m3 numbers
        g = np.tile(np.resize([-2.0, -2.5, -3.0, -3.5, -4.0, -5.0, -6.0, -7.0, -8.0, -9.0, -10.0, -11.0, -12.0], F_), (M, 1))
    gu = np.concatenate([g, np.ones_like(g)], 1)
    dgu, h = (torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda") for shape in ((M, 2 * F_), (M, F_)))
    how = (M, F_, 8, "NN", "gelu")
    dh = _dev(np.full_like(g, 0.5))
    if kept == "bf16":
        B.axonn_gated_bwd(*how, dh, _dev(gu), None, None, dgu, h, None, None)
    else:
        q = B.q8_empty(M, 2 * F_)
        B.axonn_q8_quantize(M, 2 * F_, _dev(gu), *q)
        B.axonn_gated_bwd_q8(*how, dh, *q, None, None, None, dgu, h, None, None, None)
    act, slope = F.activation(g, "gelu")
    _near(h, act, U + ACT, "h")
    _near(dgu[:, F_:], 0.5 * act, U + ACT, "dU")
    _near(dgu[:, :F_], 0.5 * slope, U + SLOPE, "dG")


@pytest.mark.gpu
@pytest.mark.parametrize("M, F_, D", [(3, 81, 64), (16, 81, 72), (81, 96, 64), (81, 512, 128), (300, 2048, 128), (2048, 4096, 128), (7, 5, 4)])
@pytest.mark.parametrize("layout", ["NN", "NT"])
def test_gelu_projection_in_the_lower_tail(M, F_, D, layout):
    """x and W hold g in one row of the product and a one for U: both sums are exact, on whichever kernel the sizes choose."""
    x, w = np.zeros((M, D)), np.zeros((D, 2 * F_))
    g = TAIL[np.round(np.linspace(0, TAIL.size - 1, M)).astype(int)][:, None]
    x[:, :1], x[:, 1] = g, 1.0
    w[0, :F_], w[1, F_:] = 1.0, 1.0
    h = torch.full((M, F_), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.axonn_gated_fwd(M, F_, D, layout, "gelu", _dev(x), _dev(w if layout == "NN" else w.T), h)
    _near(h, np.broadcast_to(F.activation(g, "gelu")[0], (M, F_)), U + ACT, "h")

"""The norm's 8-bit output to the bit: the least exponent that does not saturate, and one rounding from the unrounded y.

Inputs whose y is exact in fp32 and has more digits than bf16: every eight values of a row are 35, 28, 6, 1, 1, 1, 0, 0 sixteenths in some order, with signs, whose
mean square is one; times a power of two for each row, with eps = 0, rstd is that power's inverse, and every sum on the way is a whole number below 2^24 of
one unit.  Weights have eight digits.  In each block one column's makes its values 448 where z is 28 sixteenths (the largest that exponent 0 holds), or 448 (1 + 2^-10)
where it is 35, which takes exponent 1 and would be 448 again if it were rounded to bf16 before."""
import numpy as np
import pytest
import torch

from oracle import feed_forward as F
from paper_2502_08145_amd import binding as B

SIZES = [(64, 7), (70, 8), (70, 128), (70, 136), (65, 511), (70, 1000), (40, 1001), (33, 2048), (20, 2056), (12, 4096), (10, 5120), (9, 8200), (9, 16384), (9, 20001), (8, 32768)]


def exact_inputs(rows, cols):
    """(x, residual, weight) in float64, bf16 numbers"""
    rng = np.random.default_rng(rows + cols)
    z = np.full((rows, cols), 16.0)
    for c in range(0, cols // 8 * 8, 8):
        z[:, c:c + 8] = rng.permuted(np.tile([35.0, 28.0, 6.0, 1.0, 1.0, 1.0, 0.0, 0.0], (rows, 1)), axis=1)
    z *= rng.choice([-1.0, 1.0], z.shape)
    residual = rng.integers(-100, 101, z.shape).astype(np.float64)
    power = np.exp2(rng.integers(-10, 11, (rows, 1)) - 4.0)
    weight = rng.integers(128, 256, cols) / 16.0
    for block, c in enumerate(range(0, cols, 128)):
        weight[c + rng.integers(0, min(128, cols - c))] = 256.0 if block % 2 else 205.0
    return (z - residual) * power, residual * power, weight


def test_the_inputs_tell_one_rounding_from_two():
    x, r, w = exact_inputs(70, 1000)
    assert all(np.array_equal(F.bf16_round(v), v) for v in (x, r, w))
    z, y, rstd = F.rmsnorm(x, r, w, 0.0)
    assert np.array_equal(np.exp2(np.round(np.log2(rstd))), rstd)
    for v in (z * rstd[:, None], y):
        assert np.array_equal(v.astype(np.float32).astype(np.float64), v)
    codes, e = F.q8_quantize(y)
    twice, e_twice = F.q8_quantize(F.bf16_round(y))
    assert (e != e_twice).sum() > 20 and (codes != twice)[np.repeat(e == e_twice, 128, 1)].sum() > 20
    most = np.abs(F.q8_values(codes, np.zeros_like(e), 1000)).max()
    assert most == 448.0 and (np.abs(y) == 448.0).any() and (np.abs(y) == 448.4375).any()


@pytest.mark.gpu
@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm_to_8_bits_is_the_quantised_y_to_the_bit(rows, cols, residual):
    x, r, w = exact_inputs(rows, cols)
    if not residual:
        x, r = x + r, None
    z, y, rstd = F.rmsnorm(x, r, w, 0.0)
    dev = [None if v is None else torch.from_numpy(v.astype(np.float32)).to(torch.bfloat16).cuda() for v in (x, r, w)]
    codes, e = F.q8_quantize(y)
    for both in (False, True):
        q, s = (t.fill_(0xA5) for t in B.q8_empty(rows, cols))
        got = torch.full((rows, cols), float("nan"), dtype=torch.bfloat16, device="cuda") if both else None
        rs = torch.full((rows,), float("nan"), device="cuda")
        B.axonn_rmsnorm_fwd(rows, cols, *dev, 0.0, None, got, q, s, rs)
        assert np.array_equal(rs.cpu().numpy(), rstd)
        assert np.array_equal(s.cpu().numpy()[:, :rows], (e.T + 127).astype(np.uint8))
        assert np.array_equal(F.E4M3[q.cpu().numpy()], F.E4M3[codes])   # a zero's sign aside
        if both:
            assert np.array_equal(got.float().cpu().numpy(), F.bf16_round(y))

"""The operators around a feed-forward block's products where a launch holds all the workgroups that it may, and where a kernel's loop runs more than once."""
import pytest
import torch

from paper_2502_08145_amd import binding as B

pytestmark = pytest.mark.gpu


def filled(*shape, dtype=torch.bfloat16):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def test_product_with_more_columns_than_the_kernel_for_few_rows_takes():
    M, N, K = 4, (1 << 26) + 70, 128
    gen = torch.Generator(device="cuda").manual_seed(1)
    values, scales = [], []
    for rows in (M, N):   # ones and twos (0x38, 0x40), times 1/2, 1 or 2: sums are exact
        values.append(torch.randint(0, 2, (rows, K), generator=gen, device="cuda", dtype=torch.uint8).mul_(8).add_(0x38))
        scales.append(torch.randint(126, 129, (1, B.axonn_q8_scale_row(rows)), generator=gen, device="cuda", dtype=torch.uint8))
    c = filled(M, N)
    B.axonn_q8_linear(M, N, K, values[0], scales[0], values[1], scales[1], c)

    def stands_for(i, lo, hi):
        return values[i][lo:hi].view(torch.float8_e4m3fn).float() * torch.exp2(scales[i][0, lo:hi].float() - 127.0)[:, None]

    a = stands_for(0, 0, M)
    for lo in range(0, N, 1 << 22):
        hi = min(N, lo + (1 << 22))
        assert torch.equal(c[:, lo:hi], (a @ stands_for(1, lo, hi).t()).to(torch.bfloat16)), lo


@pytest.mark.parametrize("M, F, D, layout", [(1, (1 << 28) + 70, 1, "NT"), ((1 << 28) + 70, 3, 8, "NN")])
def test_gated_projection_of_more_blocks_than_a_launch_takes(M, F, D, layout):
    """U is G negated: whole numbers, so that the sums are exact."""
    gen = torch.Generator(device="cuda").manual_seed(M)

    def numbers(*shape):
        return torch.randint(-2, 3, shape, generator=gen, device="cuda", dtype=torch.int8).to(torch.bfloat16)

    x, half = numbers(M, D), numbers(D, F)
    w = torch.cat([half, -half], 1) if layout == "NN" else torch.cat([half.t(), -half.t()], 0).contiguous()
    h, gu = filled(M, F), filled(M, 2 * F)
    B.axonn_gated_fwd(M, F, D, layout, "silu", x, w, h, gu)
    step = 1 << 24
    for lo in range(0, max(M, F), step):   # along the axis that is long
        rows, columns = (slice(lo, lo + step), slice(None)) if M > F else (slice(None), slice(lo, lo + step))
        g = (x[rows].float()[:, :, None] * half[:, columns].float()[None]).sum(1)
        assert torch.equal(gu[rows][:, :F][:, columns], g.to(torch.bfloat16)) and torch.equal(gu[rows][:, F:][:, columns], (-g).to(torch.bfloat16)), lo
        ref = g / (1 + torch.exp(-g)) * -g
        assert bool(((h[rows][:, columns].float() - ref).abs() <= 2.0 ** -8 * ref.abs()).all()), lo

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


# ---- loops over more than one piece of work, and offsets beyond 2^31: the same bits as from calls on slices, which need neither ---------------


def random(gen, *shape):
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for part in x.view(-1).split(1 << 28):
        part.normal_(generator=gen)
    return x


def slices(rows, step):
    return [(lo, min(rows, lo + step)) for lo in range(0, rows, step)]


def test_norm_of_more_rows_than_workgroups():
    rows, cols = 3 * (1 << 20) + 5, 712   # up to four rows a workgroup of two waves, and 2.2e9 values
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, r, w = random(gen, rows, cols), random(gen, rows, cols), random(gen, cols)
    total, y, rstd, (q, s) = filled(rows, cols), filled(rows, cols), filled(rows, dtype=torch.float32), B.q8_empty(rows, cols)
    B.axonn_rmsnorm_fwd(rows, cols, x, r, w, 1e-5, total, y, q, s, rstd)
    for lo, hi in slices(rows, 1 << 19):
        n = hi - lo
        total2, y2, rstd2, (q2, s2) = filled(n, cols), filled(n, cols), filled(n, dtype=torch.float32), B.q8_empty(n, cols)
        B.axonn_rmsnorm_fwd(n, cols, x[lo:hi], r[lo:hi], w, 1e-5, total2, y2, q2, s2, rstd2)
        assert torch.equal(total[lo:hi], total2) and torch.equal(y[lo:hi], y2) and torch.equal(rstd[lo:hi], rstd2)
        assert torch.equal(q[lo:hi], q2) and torch.equal(s[:, lo:hi], s2[:, :n])
    z = x[-1000:].double() + r[-1000:].double()
    ref = z / (z.square().mean(1, keepdim=True) + 1e-5).sqrt() * w.double()
    assert bool(((y[-1000:].double() - ref).abs() <= (2.0 ** -8 + (cols + 16) * 2.0 ** -23) * ref.abs()).all())


def test_norm_gradients_beyond_32_bits():
    rows, cols = 270000, 8200
    gen = torch.Generator(device="cuda").manual_seed(3)
    dy, z, w = random(gen, rows, cols), random(gen, rows, cols), random(gen, cols)
    rstd = torch.rand(rows, generator=gen, device="cuda") + 0.5
    scratch = torch.empty(B.axonn_rmsnorm_bwd_scratch_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    dx, dw = filled(rows, cols), filled(cols, dtype=torch.float32)
    B.axonn_rmsnorm_bwd(rows, cols, dy, z, w, rstd, None, dx, dw, scratch)
    ref, sums = (torch.zeros(cols, dtype=torch.float64, device="cuda") for _ in range(2))
    for lo, hi in slices(rows, 30000):
        dx2, dw2 = filled(hi - lo, cols), filled(cols, dtype=torch.float32)
        B.axonn_rmsnorm_bwd(hi - lo, cols, dy[lo:hi], z[lo:hi], w, rstd[lo:hi], None, dx2, dw2, scratch)
        assert torch.equal(dx[lo:hi], dx2), lo
        terms = dy[lo:hi].double() * (z[lo:hi].double() * rstd[lo:hi].double()[:, None])
        ref += terms.sum(0)
        sums += terms.abs().sum(0)
    assert bool(((dw.double() - ref).abs() <= (rows + 8) * 2.0 ** -23 * sums).all())


def test_quantize_by_rows_of_more_tiles_than_workgroups():
    rows, cols = 16 * ((1 << 20) + 3) - 5, 136
    x = random(torch.Generator(device="cuda").manual_seed(4), rows, cols)
    q, s = B.q8_empty(rows, cols)
    B.axonn_q8_quantize(rows, cols, x, q, s)
    back = filled(rows, cols)
    B.axonn_q8_restore(rows, cols, q, s, back)
    for lo, hi in slices(rows, 1 << 22):
        n = hi - lo
        (q2, s2), back2 = B.q8_empty(n, cols), filled(n, cols)
        B.axonn_q8_quantize(n, cols, x[lo:hi], q2, s2)
        B.axonn_q8_restore(n, cols, q2, s2, back2)
        assert torch.equal(q[lo:hi], q2) and torch.equal(s[:, lo:hi], s2[:, :n]) and torch.equal(back[lo:hi], back2), lo


@pytest.mark.parametrize("tiles, cols, both", [((1 << 20) + 3, 17, True), (3 * (1 << 20) + 2, 8, False)])
def test_quantize_by_columns_of_more_tiles_than_workgroups(tiles, cols, both):
    rows = 128 * tiles - 37
    x = random(torch.Generator(device="cuda").manual_seed(5), rows, cols)
    q, s = B.q8_empty(rows, cols) if both else (None, None)
    qt, st = B.q8_empty(cols, rows)
    B.axonn_q8_quantize(rows, cols, x, q, s, qt, st)
    for lo, hi in slices(rows, 1 << 25):
        n = hi - lo
        q2, s2 = B.q8_empty(n, cols) if both else (None, None)
        qt2, st2 = B.q8_empty(cols, n)
        B.axonn_q8_quantize(n, cols, x[lo:hi], q2, s2, qt2, st2)
        assert torch.equal(qt[:, lo:lo + qt2.shape[1]], qt2) and torch.equal(st[lo // 128:lo // 128 + st2.shape[0], :cols], st2[:, :cols]), lo
        if both:
            assert torch.equal(q[lo:hi], q2) and torch.equal(s[:, lo:hi], s2[:, :n]), lo


@pytest.mark.parametrize("F", [65544, 65541])
def test_gradients_of_the_activation_beyond_32_bits(F):
    M, step = 33000, 1504   # slices on 16 bytes
    gen = torch.Generator(device="cuda").manual_seed(F)
    dh, gu = random(gen, M, F), random(gen, M, 2 * F)
    q, s = B.q8_empty(M, 2 * F)
    B.axonn_q8_quantize(M, 2 * F, gu, q, s)
    dgu, h, dgu8, h8 = filled(M, 2 * F), filled(M, F), filled(M, 2 * F), filled(M, F)
    how = F, 8, "NN", "silu"
    B.axonn_gated_bwd(M, *how, dh, gu, None, None, dgu, h, None, None)
    B.axonn_gated_bwd_q8(M, *how, dh, q, s, None, None, None, dgu8, h8, None, None, None)
    for lo, hi in slices(M, step):
        n = hi - lo
        part = torch.zeros((s.shape[0], B.axonn_q8_scale_row(n)), dtype=torch.uint8, device="cuda")
        part[:, :n] = s[:, lo:hi]
        dgu2, h2 = filled(n, 2 * F), filled(n, F)
        B.axonn_gated_bwd(n, *how, dh[lo:hi], gu[lo:hi], None, None, dgu2, h2, None, None)
        assert torch.equal(dgu[lo:hi], dgu2) and torch.equal(h[lo:hi], h2), lo
        B.axonn_gated_bwd_q8(n, *how, dh[lo:hi], q[lo:hi], part, None, None, None, dgu2, h2, None, None, None)
        assert torch.equal(dgu8[lo:hi], dgu2) and torch.equal(h8[lo:hi], h2), lo


def numbers(gen, *shape):
    return torch.randint(-2, 3, shape, generator=gen, device="cuda", dtype=torch.int8).to(torch.bfloat16)


def test_product_beyond_32_bits():
    M, N, K = 70000, 32770, 128
    gen = torch.Generator(device="cuda").manual_seed(6)
    a, b = numbers(gen, M, K), numbers(gen, N, K)
    qa, qb, c = B.q8_empty(M, K), B.q8_empty(N, K), filled(M, N)
    B.axonn_q8_quantize(M, K, a, *qa)
    B.axonn_q8_quantize(N, K, b, *qb)
    B.axonn_q8_linear(M, N, K, *qa, *qb, c)
    for lo, hi in slices(M, 10000):
        assert torch.equal(c[lo:hi], (a[lo:hi].float() @ b.float().t()).to(torch.bfloat16)), lo


@pytest.mark.parametrize("layout, F", [("NN", 65544), ("NT", 65544), ("NN", 65541), ("NT", 65541)])
def test_gated_projection_beyond_32_bits(layout, F):
    M, D = 33000, 72
    gen = torch.Generator(device="cuda").manual_seed(7)
    x, w = numbers(gen, M, D), numbers(gen, D, 2 * F)
    h, gu = filled(M, F), filled(M, 2 * F)
    B.axonn_gated_fwd(M, F, D, layout, "silu", x, w if layout == "NN" else w.t().contiguous(), h, gu)
    for lo, hi in slices(M, 3000):
        ref = x[lo:hi].float() @ w.float()
        assert torch.equal(gu[lo:hi], ref.to(torch.bfloat16)), lo
        g, u = ref[:, :F], ref[:, F:]
        ref = torch.sigmoid(g) * g * u
        assert bool(((h[lo:hi].float() - ref).abs() <= 2.0 ** -8 * ref.abs()).all()), lo

"""Every kernel that the 8-bit products and the gated projections choose among, against 64 bits at a size that chooses it; and that the sizes do choose them."""
import pytest
import torch

from paper_2502_08145_amd import binding as B
from tests import host_runtime
from tests import test_feed_forward_gpu as small

U, FINE = 2.0 ** -8, 2.0 ** -18

# M, F, D, layout: whole and moved-back tiles, D of 64 and off it, D long enough for every stage and for the loads by lines (beyond 768)
GATED = {
    "gated_tile_kernel<256, 256, 4, false, 0, false>": [(540, 6872, 832, "NN")],
    "gated_tile_kernel<256, 256, 4, false, 0, true>": [(524, 6976, 784, "NN")],
    "gated_tile_kernel<256, 256, 4, true, 1, false>": [(520, 6944, 832, "NT")],
    "gated_tile_kernel<256, 256, 4, true, 1, true>": [(532, 6704, 776, "NT")],
    "gated_group_kernel<256, 128, 1, false, false>": [(256, 8200, 128, "NN"), (667, 2736, 832, "NN"), (512, 8192, 4096, "NN")],
    "gated_group_kernel<256, 128, 1, false, true>": [(3834, 520, 72, "NN"), (716, 5392, 800, "NN")],
    "gated_group_kernel<256, 128, 1, true, false>": [(2048, 1032, 128, "NT"), (495, 4128, 1088, "NT")],
    "gated_group_kernel<256, 128, 1, true, true>": [(2048, 1032, 72, "NT"), (391, 4928, 792, "NT")],
    "gated_group_kernel<128, 256, 1, false, false>": [(279, 5872, 832, "NN")],
    "gated_group_kernel<128, 256, 1, false, true>": [(267, 5752, 800, "NN")],
    "gated_group_kernel<128, 256, 1, true, false>": [(290, 6632, 832, "NT")],
    "gated_group_kernel<128, 256, 1, true, true>": [(281, 6824, 776, "NT")],
    "gated_group_kernel<128, 128, 1, false, false>": [(140, 5712, 832, "NN")],
    "gated_group_kernel<128, 128, 1, false, true>": [(132, 5592, 784, "NN")],
    "gated_group_kernel<128, 128, 1, true, false>": [(131, 6376, 832, "NT")],
    "gated_group_kernel<128, 128, 1, true, true>": [(137, 5544, 776, "NT")],
    "gated_group_kernel<128, 64, 1, false, false>": [(3433, 272, 128, "NN"), (2175, 456, 832, "NN")],
    "gated_group_kernel<128, 64, 1, false, true>": [(593, 1632, 72, "NN"), (331, 2720, 784, "NN")],
    "gated_group_kernel<128, 64, 1, true, false>": [(2048, 200, 128, "NT"), (205, 2408, 896, "NT")],
    "gated_group_kernel<128, 64, 1, true, true>": [(200, 2056, 72, "NT"), (218, 2072, 776, "NT")],
    "gated_group_kernel<64, 128, 1, false, false>": [(64, 2056, 128, "NN"), (69, 4272, 832, "NN")],
    "gated_group_kernel<64, 128, 1, false, true>": [(68, 4472, 784, "NN")],
    "gated_group_kernel<64, 128, 1, true, false>": [(520, 512, 128, "NT"), (65, 4896, 832, "NT")],
    "gated_group_kernel<64, 128, 1, true, true>": [(65, 4208, 792, "NT")],
    "gated_group_kernel<64, 64, 2, false, false>": [(256, 512, 1024, "NN"), (64, 32, 1408, "NN")],
    "gated_group_kernel<64, 64, 2, false, true>": [(65, 32, 1560, "NN")],
    "gated_group_kernel<64, 64, 2, true, false>": [(64, 2056, 256, "NT"), (1654, 72, 832, "NT")],
    "gated_group_kernel<64, 64, 2, true, true>": [(163, 504, 784, "NT")],
    "gated_wavek_kernel<false, 2, 1, false>": [(20, 2056, 256, "NN")],
    "gated_wavek_kernel<false, 4, 2, false>": [(192, 4099, 64, "NN"), (391, 1001, 777, "NN"), (849, 1217, 1352, "NN")],
    "gated_wavek_kernel<true, 4, 2, false>": [(192, 4099, 64, "NT"), (391, 1001, 777, "NT"), (849, 1217, 1352, "NT")],
    "gated_wavek_kernel<true, 1, 2, true>": [(8, 4099, 4096, "NT")],
    "gated_wavek_kernel<true, 2, 2, true>": [(20, 4099, 4096, "NT")],
}
# M, N, K: real numbers, K up to 16384
PRODUCTS = {
    "q8_tile_kernel<256, 256, 2, 4, 2, true>": [(3840, 3850, 128), (2050, 4100, 1000), (2300, 4300, 3000), (2048, 6144, 16384)],
    "q8_tile_kernel<256, 128, 4, 2, 2, true>": [(1024, 4099, 64), (1024, 4099, 640), (1030, 4100, 4096), (2048, 4096, 16384)],
    "q8_tile_kernel<128, 128, 2, 4, 2, true>": [(1000, 3000, 1000), (513, 4099, 2000), (1000, 2100, 16384)],
    "q8_tile_kernel<64, 64, 2, 2, 4, false>": [(65, 130, 640), (64, 200, 16384), (500, 1000, 16384)],
    "q8_rows_kernel<1>": [(1, 4096, 16384), (13, 1001, 1300)],
    "q8_rows_kernel<2>": [(30, 4000, 16384), (17, 300, 1000)],
}


def cases(table):
    return [pytest.param(*size, id=" ".join(map(str, size))) for sizes in table.values() for size in sizes]


def gated_call(M, F, D, layout):
    return "axonn_gated_fwd", [M, F, D, B._layout(layout), 0, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 0]


def product_call(M, N, K):
    return "axonn_q8_linear", [M, N, K] + [1 << 20] * 5 + [0]


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    return host_runtime.build_runtime(tmp_path_factory.mktemp("runtime"))


@pytest.mark.parametrize("table, call", [(GATED, gated_call), (PRODUCTS, product_call)], ids=["gated", "products"])
def test_the_sizes_choose_the_kernels_that_they_stand_for(so, table, call):
    sizes = [(name, size) for name, of in table.items() for size in of]
    answers = host_runtime.run(so, [call(*size) for _, size in sizes])
    names = host_runtime.readable(x.kernel for a in answers for x in a.launches)
    assert [(size, [names[x.kernel] for x in a.launches]) for (_, size), a in zip(sizes, answers)] == [(size, [name]) for name, size in sizes]


def test_every_kernel_is_compared_somewhere(so):
    plain = [getattr(p, "values", p) for p in small.GATED]
    calls = ([gated_call(*size) for of in GATED.values() for size in of] + [product_call(*size) for of in PRODUCTS.values() for size in of]
             + [gated_call(*p, layout) for p in plain for layout in ("NN", "NT")])
    there = host_runtime.readable(k for k in host_runtime.kernels_of_the_library(so))
    there = {name for name in there.values() if name.startswith(("gated_", "q8_"))}
    assert len(there) > 40
    reached = host_runtime.readable(x.kernel for a in host_runtime.run(so, calls) for x in a.launches)
    assert there == set(reached.values())


# ---- on the GPU, the references there too ---------------------------------------------------------------------------------------


def normal(gen, shape, sigma=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * sigma).to(torch.bfloat16)


def close(got, ref, bound, what):
    over = (got.double() - ref).abs() - bound
    assert bool(got.isfinite().all()) and float(over.max()) <= 0, f"{what}: {float(over.max()):.3e} over the bound"


def act(g, name):
    return g * torch.sigmoid(g) if name == "silu" else g * 0.5 * torch.special.erfc(g * -(0.5 ** 0.5))


@pytest.mark.gpu
@pytest.mark.parametrize("M, F, D, layout", cases(GATED))
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_gated(M, F, D, layout, name):
    """The bounds of test_feed_forward_gpu.py: sums in fp32, one rounding, |act'| <= 1.13."""
    gen = torch.Generator(device="cuda").manual_seed(M + F + D)
    x, w = normal(gen, (M, D)), normal(gen, (D, 2 * F), D ** -0.5)
    room = torch.full((M * F + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    h, gu = room[:M * F].view(M, F), torch.full((M, 2 * F), float("nan"), dtype=torch.bfloat16, device="cuda")
    h.fill_(float("nan"))
    B.axonn_gated_fwd(M, F, D, layout, name, x, w if layout == "NN" else w.t().contiguous(), h, gu)
    ref, e = x.double() @ w.double(), (x.double().abs() @ w.double().abs()) * (D * 2.0 ** -23)
    close(gu, ref, U * ref.abs() + e, "gu")
    (g, u), (eg, eu) = ref.split(F, 1), e.split(F, 1)
    a = act(g, name)
    close(h, a * u, U * (a * u).abs() + (1.13 * eg + FINE * (a.abs() + g.abs())) * (u.abs() + eu) + (a.abs() + 1.13 * eg) * eu, "h")
    assert bool((room[M * F:] == 7.0).all())


def in_8_bits(x):
    rows, cols = x.shape
    q, s = B.q8_empty(rows, cols)
    q.fill_(0xA5), s.fill_(0xA5)
    B.axonn_q8_quantize(rows, cols, x, q, s)
    values = q.view(torch.float8_e4m3fn).double().view(rows, -1, 128) * torch.exp2(s[:, :rows].t().double() - 127.0)[:, :, None]
    return (q, s), values.view(rows, -1)


@pytest.mark.gpu
@pytest.mark.parametrize("M, N, K", cases(PRODUCTS))
def test_product(M, N, K):
    """The bound that follows from the scaled instruction: of each group of eight neighbouring k, what is below 2^-13 of the largest product is dropped, for
    each of the eight; everything between the groups is fp32; one rounding.  Rows and blocks of very different sizes, so that a scale from another
    one shows, and b's rows nearly orthogonal to a's first, so that sums cancel and the bits show."""
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)

    def sizes(n, lo, hi):
        return torch.exp2(torch.randint(lo, hi, (n,), generator=gen, device="cuda").float())

    blocks = sizes(-(-K // 128), -3, 3).repeat_interleave(128)[:K]
    a, b = normal(gen, (M, K)).float() * blocks, normal(gen, (N, K)).float() / blocks
    b -= torch.outer(b @ a[0] / (a[0] @ a[0]), a[0])
    a, b = (a * sizes(M, -6, 6)[:, None]).to(torch.bfloat16), (b * sizes(N, -6, 6)[:, None]).to(torch.bfloat16)
    (qa, a), (qb, b) = in_8_bits(a), in_8_bits(b)
    room = torch.full((M * N + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    c = room[:M * N].view(M, N)
    c.fill_(float("nan"))
    B.axonn_q8_linear(M, N, K, *qa, *qb, c)
    bound = (a.abs() @ b.abs().t()) * (K * 2.0 ** -23)
    ref = a @ b.t()
    a, b = a.abs().float().t().contiguous(), b.abs().float().t().contiguous()   # exact
    dropped = torch.zeros((M, N), device="cuda")
    for k in range(0, a.shape[0], 8):
        most = torch.outer(a[k], b[k])
        for i in range(k + 1, k + 8):
            torch.maximum(most, torch.outer(a[i], b[i]), out=most)
        dropped += most
    bound += dropped.double() * (8 * 2.0 ** -13 * (1 + U))
    close(c, ref, U * ref.abs() + bound, f"{M} x {N} x {K}")
    assert bool((room[M * N:] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("M, N, K", [(2048, 6144, 16384), (2048, 4096, 16384), (1030, 4100, 4000), (1000, 2100, 16384), (500, 1000, 16384), (1, 4096, 16384), (13, 1001, 16300), (30, 4000, 16384)])
def test_product_of_whole_numbers_over_a_long_k_is_exact(M, N, K):
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    a, b = (torch.randint(-2, 3, (n, K), generator=gen, device="cuda").to(torch.bfloat16) for n in (M, N))
    (qa, _), (qb, _) = in_8_bits(a), in_8_bits(b)
    c = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.axonn_q8_linear(M, N, K, *qa, *qb, c)
    assert torch.equal(c, (a.double() @ b.double().t()).float().to(torch.bfloat16))   # sums below 2^24

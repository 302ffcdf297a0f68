// The gated projections  h = act(x Wg) * (x Wu)  in one kernel: g = x Wg and u = x Wu of an output are two sums of the same lane, so the activation and the
// product cost no trip to memory.  x is [M, D]; Wg and Wu are the two halves of W, [D, 2F] (NN) or [2F, D] (NT); h is [M, F].  For the backward
// pass the two sums can be stored too, rounded to bf16 as [M, 2F]; h is always computed from the unrounded ones.
#pragma once
#include "gemm_mfma16_k64.hpp"
#include "gemm_mfma16_k64g.hpp"
#include "gemm_wavek.hpp"
#include "row_ops.hpp"

namespace axonn {

// ---- activations -------------------------------------------------------------------------------------------------------------
enum { kSilu = 0, kGelu = 1 };

// act(g), and its derivative.  The fast path's exponential rounds its argument times log2(e), so that it is off by up to |g| 2^-23 of itself (the density's
// by g^2 2^-23), 2^-15 at the ends of the range, against the 2^-9 of the result's rounding.
//
// GELU's distribution function below -|g| is density(g) P(t) with t = 1 / (1 + 0.36 |g|), which has its digits however small the value is; 1 + erf has none
// left there (at -5.5 half of the value, at -6 all of it).  P, a polynomial without constant term, was fitted to exp(g^2 / 2) times the function over
// 0 <= |g| <= 14 for the least relative error, 2^-20.  The exponential is the slope's too.  (Gradients of 2048 x 8192: 29.9 us, with erfc 33.4,
// with 1 + erf 30.9.)
__device__ __forceinline__ float normal_below(float g, float exponential) {   // exponential: exp(-g^2 / 2)
    const float t = __builtin_amdgcn_rcpf(1.f + 0.36f * fabsf(g));
    const float tail = exponential * t * (0.14371304f + t * (0.14177249f + t * (0.13971901f + t * (0.02655006f + t * (0.18095289f + t * (-0.17976384f + t * 0.04705604f))))));
    return g < 0.f ? tail : 1.f - tail;
}
__device__ __forceinline__ float activation(int act, float g) {
    if (act == kSilu) return g / (1.f + __expf(-g));
    return g * normal_below(g, __expf(-0.5f * g * g));
}
__device__ __forceinline__ float activation(int act, float g, float* slope) {
    if (act == kSilu) {
        const float p = 1.f / (1.f + __expf(-g));
        *slope = p * (1.f + g * (1.f - p));
        return g * p;
    }
    const float exponential = __expf(-0.5f * g * g), p = normal_below(g, exponential);
    *slope = p + g * (exponential * 0.39894228f);
    return g * p;
}

struct GatedOut {
    uint16_t* h;
    uint16_t* gu;   // nullptr: not kept
    int64_t F;
    int act;
};

// ---- tiles: the bf16 tile kernels with another order of b's columns ------------------------------------------------------------------
// Of the TN columns of b that a wave multiplies the first half comes from Wg and the other half, the same columns, from Wu; the order is made where the
// direct loads fetch, and everything between them and the sums is the tile kernels' own.  A tile of BM x BN gives BM x BN/2 of h.
// Bound by what bounds the product of the same sizes, whose time it takes: 2048 x 8192 x 4096 NN with the sums kept 218 us, 1260 TFLOP/s, at the board's power limit;
// 299 x 2088 x 1608 12.8 us, a chain of 26 steps on 165 of the 256 units.
template <int BN, int TN>
struct GatedKind {
    static constexpr bool kOwn = true;
    static constexpr int kColumns = BN / 2, HALF = TN / 2;
    GatedOut out;

    // column of W behind column p of the tile, beyond the tile's first
    __device__ __forceinline__ int64_t column(int p) const { return HALF * (p / TN) + p % HALF + (p % TN >= HALF ? out.F : 0); }

    // 64-k kernel, K-contiguous: a load is eight rows of W, all in one half
    template <int ROWS, int REGION, int NW>
    __device__ __forceinline__ void place(OperandK64KContig<ROWS, REGION, NW>& op, const uint16_t* W, int64_t n0, uint32_t ld_bytes, int, int wave) const {
#pragma unroll
        for (int c = 0; c < op.QL; ++c) op.base[c] = reinterpret_cast<const uint8_t*>(W) + (size_t)(n0 + column(8 * (op.QL * wave + c))) * ld_bytes;
    }
    // ... MN-contiguous: a lane's 16 bytes are eight columns, all in one half
    template <int ROWS, int REGION, int NW, int NB>
    __device__ __forceinline__ void place(OperandK64MNContig<ROWS, REGION, NW, NB>& op, const uint16_t*, int64_t, uint32_t ld_bytes, int lane, int) const {
        using In = typename OperandK64MNContig<ROWS, REGION, NW, NB>::Inner;
#pragma unroll
        for (int c = 0; c < op.QH; ++c) {
            const uint32_t moved = moved_to(op.in.voff[c], (uint32_t)(In::KR * c + lane / In::CPR) * ld_bytes);
            op.voff_hi[c] += moved - op.in.voff[c];
            op.in.voff[c] = moved;
        }
    }
    // eight-wave kernel, the same two.  K-contiguous: the rows of a wave lie in either half, so a lane's offset holds all of its row's (below 4 GB)
    template <int ROWS, int REGION, int NW, int NB>
    __device__ __forceinline__ void place(GroupKContig<ROWS, REGION, NW, NB>& op, const uint16_t* W, int64_t n0, uint32_t ld_bytes, int lane, int wave, int, int,
                                          uint32_t) const {
        op.base = reinterpret_cast<const uint8_t*>(W) + (size_t)n0 * ld_bytes;
        place_rows(op.voff, ld_bytes, lane, wave, ROWS / NW);
    }
    // loaded by lines: where a row starts in its line does not change, F rows on is a multiple of 128 bytes (D and F are multiples of 8)
    template <int ROWS, int REGION, int NW, int NB>
    __device__ __forceinline__ void place(GroupKLines<ROWS, REGION, NW, NB>& op, const uint16_t* W, int64_t n0, uint32_t ld_bytes, int lane, int wave, int, int,
                                          uint32_t) const {
        op.base = reinterpret_cast<const uint8_t*>(W) + (size_t)n0 * ld_bytes - 128;
        place_rows(op.voff, ld_bytes, lane, wave, ROWS / NW);
    }
    template <int QL>
    __device__ __forceinline__ void place_rows(uint32_t (&voff)[QL], uint32_t ld_bytes, int lane, int wave, int rows) const {
#pragma unroll
        for (int x = 0; x < QL; ++x) {
            const int row = 8 * x + (lane >> 3);   // of the wave's
            voff[x] += (uint32_t)column(rows * wave + row) * ld_bytes - (uint32_t)row * ld_bytes;
        }
    }
    // Here the order is made where the fragments are read: a k-row of the tile is BN/2 columns of Wg and then of Wu, whole lines.  (In the waves' order it is
    // pieces of 32 bytes by turns: 256 x 4096 x 4096 26 us.)
    template <int ROWS, int REGION, int NW, int NB>
    __device__ __forceinline__ void place(GroupMNContig<ROWS, REGION, NW, NB>& op, const uint16_t*, int64_t, uint32_t ld_bytes, int lane, int, int group, int wn,
                                          uint32_t lds0) const {
        using Op = GroupMNContig<ROWS, REGION, NW, NB>;
#pragma unroll
        for (int x = 0; x < Op::QL; ++x) {
            const uint32_t k_row = (uint32_t)(Op::KR * x + lane / Op::CPR) * ld_bytes;
            if ((op.voff[x] - k_row) / 2 >= BN / 2) op.voff[x] += 2u * (uint32_t)(out.F - BN / 2);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i)
            op.raddr[i] = Op::row_address(lds0 + REGION, HALF * wn + (i < NB / 2 ? 16 * i : BN / 2 + 16 * (i - NB / 2)), group, lane);
    }
    // an offset of a k-row's and a column's bytes, with the column of W in place of the tile's
    __device__ __forceinline__ uint32_t moved_to(uint32_t voff, uint32_t k_row) const { return k_row + 2u * (uint32_t)column((int)(voff - k_row) / 2); }

    // a wave's MI block rows from row0 on; `epi`: LDS of its own
    template <int MI, int NI>
    __device__ __forceinline__ void store(f32x4 (&acc)[MI][NI], uint8_t* epi, int64_t row0, int64_t n0, int wn, int lane) const {
        constexpr int NH = NI / 2;
        static_assert(16 * NI == TN, "a wave's columns");
        const int64_t col0 = n0 + HALF * wn;
        auto rows16 = [&](f32x4 (&row)[NH], uint16_t* p, int64_t ld) __attribute__((always_inline)) {
            if constexpr (NH >= 2) {
                store_block_row16<HALF, NH>(row, epi, p, (int)ld, lane);
            } else {   // 32 bytes a row: left to the L2 to put together
                *reinterpret_cast<u32x2*>(p + (int64_t)(lane & 15) * ld + 4 * (lane >> 4)) = u32x2{pack2_bf16(row[0][0], row[0][1]), pack2_bf16(row[0][2], row[0][3])};
            }
        };
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            f32x4 part[NH];
            if (out.gu) {
                uint16_t* const gu = out.gu + (row0 + 16 * i) * (2 * out.F) + col0;
#pragma unroll
                for (int j = 0; j < NH; ++j) part[j] = acc[i][j];
                rows16(part, gu, 2 * out.F);
#pragma unroll
                for (int j = 0; j < NH; ++j) part[j] = acc[i][NH + j];
                rows16(part, gu + out.F, 2 * out.F);
            }
#pragma unroll
            for (int j = 0; j < NH; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) part[j][e] = activation(out.act, acc[i][j][e]) * acc[i][NH + j][e];
            rows16(part, out.h + (row0 + 16 * i) * out.F + col0, out.F);
        }
    }
};

// Requires M >= BM, F >= BN/2, D > 64, D and F multiples of 8, 16-byte aligned matrices; K: D up to the next multiple of 64.
template <int BM, int BN, int WN, bool B_KC, int SCHED, bool KTAIL>
__global__ __launch_bounds__(128 * WN) void gated_tile_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, int K, int ldx, int ldw, TileGrid grid,
                                                              int group_m, GatedOut out) {
    tile_k64<BM, BN, WN, true, B_KC, false, SCHED, KTAIL>(X, W, nullptr, K, ldx, ldw, 0, grid, group_m, SplitK{}, GatedKind<BN, BN / WN>{out});
}
// The eight-wave kernel.  The same, and W below 4 GB in NT.
template <int BM, int BN, int G, bool B_KC, bool KTAIL>
__global__ __launch_bounds__(512, (GroupCfg<BM, BN, G>::WAVES_PER_SIMD)) void gated_group_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, int K, int ldx,
                                                                                                int ldw, TileGrid grid, int group_m, GatedOut out) {
    using Kind = GatedKind<BN, BN / GroupCfg<BM, BN, G>::WN>;
    const TileWork work = map_workgroup<false, false>(blockIdx.x, grid.tiles_m * grid.tiles_n, K, grid.tiles_m, grid.tiles_n, group_m, SplitK{});
    const int64_t m0 = min(work.tile_m * BM, grid.m_last), n0 = min(work.tile_n * Kind::kColumns, grid.n_last);
    if constexpr (KTAIL && group_lines(BM, BN, true, B_KC)) {
        if (K > kGroupLinesK) {
            group_tile<BM, BN, G, true, B_KC, true, true, false, Kind>(X, W, nullptr, K, ldx, ldw, 0, m0, n0, grid.k_tail, GroupSplit{}, 0, 0, Kind{out});
            return;
        }
    }
    group_tile<BM, BN, G, true, B_KC, KTAIL, false, false, Kind>(X, W, nullptr, K, ldx, ldw, 0, m0, n0, grid.k_tail, GroupSplit{}, 0, 0, Kind{out});
}

// ---- few rows, few tiles, rows at any address: the waves of a workgroup split K ---------------------------------------------------------
// As gemm_wavek_kernel, with two operands in b's place: 16 NB columns of Wg and of Wu.  blockDim.x = 64 * (waves per tile).
// STREAM: W is read by one row of tiles and is larger than the caches hold from one call to the next.
// Requires D >= 8, leading dimensions below 2^24; M >= 16 MI if MI > 2; F >= 16 NB in NN.
template <bool B_KC, int MI, int NB, bool STREAM = false>
__global__ __launch_bounds__(64 * WaveKCfg::max_waves(MI, 2 * NB)) void gated_wavek_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, int64_t M, int64_t D,
                                                                                           int tiles_m, int tiles_n, int group_m, GatedOut out) {
    constexpr int TM = 16 * MI, TN = 16 * NB, BLOCKS = MI * 2 * NB;
    using OpX = WaveKContig<MI>;
    using OpW = typename std::conditional<B_KC, WaveKContig<NB, STREAM>, WaveMNContig<NB>>::type;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int64_t F = out.F;
    const TileWork work = map_workgroup<false, false>(blockIdx.x, gridDim.x, 0, tiles_m, tiles_n, group_m, SplitK{});
    int64_t m0 = (int64_t)work.tile_m * TM, n0 = (int64_t)work.tile_n * TN;
    m0 = m0 + TM <= M ? m0 : M > TM ? M - TM : 0;
    n0 = n0 + TN <= F ? n0 : F > TN ? F - TN : 0;

    OpX opx;
    OpW opw[2];
    opx.init(X, m0, M, D, lane);
    opw[0].init(W, n0, F, B_KC ? D : 2 * F, lane);
    opw[1].init(W + (B_KC ? F * D : F), n0, F, B_KC ? D : 2 * F, lane);
    uint8_t* const lx = smem + wave * (OpX::LDS_BYTES + 2 * OpW::LDS_BYTES);
    uint8_t* const lw[2] = {lx + OpX::LDS_BYTES, lx + OpX::LDS_BYTES + OpW::LDS_BYTES};

    f32x4 acc[MI][2 * NB];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    typename OpX::Regs rx;
    typename OpW::Regs rw[2];
    auto load = [&](int64_t k0) __attribute__((always_inline)) {
        opx.load(rx, k0);
        opw[0].load(rw[0], k0);
        opw[1].load(rw[1], k0);
    };
    auto multiply_half = [&](int h) __attribute__((always_inline)) {
        bf16x8 fx[MI], fw[2 * NB];
#pragma unroll
        for (int i = 0; i < MI; ++i) fx[i] = opx.fragment(lx, i, h);
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) fw[j] = opw[j / NB].fragment(lw[j / NB], j % NB, h);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < 2 * NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[j], fx[i], acc[i][j], 0, 0, 0);
    };
    // whole chunks of 64 k: wave, wave + waves, ...; a shorter one at the end is the first of the wave that has the fewest
    const int64_t step = (int64_t)waves * WaveKCfg::KC, whole = D & ~(int64_t)(WaveKCfg::KC - 1);
    const int left = (int)(D - whole);
    int64_t k0 = (int64_t)wave * WaveKCfg::KC;
    if (left != 0 && wave == (int)((whole / WaveKCfg::KC) % waves)) {
        opx.load_tail(rx, whole, left, lane);
        opw[0].load_tail(rw[0], whole, left, lane);
        opw[1].load_tail(rw[1], whole, left, lane);
        k0 -= step;   // counts as the chunk before the first
    } else if (k0 < whole) {
        load(k0);
    }
    for (; k0 < whole; k0 += step) {
        opx.stage(rx, lx);
        opw[0].stage(rw[0], lw[0]);
        opw[1].stage(rw[1], lw[1]);
        wave_order();
        if (k0 + step < whole) load(k0 + step);
        multiply_half(0);
        if (k0 >= 0 || left > 32) multiply_half(1);   // the second half of a tail of up to 32 k is zeros
        wave_order();
    }

    // this lane's four outputs of a pair of blocks, row 16 i + lane % 16, column 16 j + 4 (lane / 16) ..
    auto store4 = [&](uint16_t* p, const f32x4& v, int count) __attribute__((always_inline)) {
        const u32x2 w{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
        if (count >= 4) {
            *reinterpret_cast<u32x2_any*>(p) = w;
        } else {
            p[0] = (uint16_t)w[0];
            if (count > 1) p[1] = (uint16_t)(w[0] >> 16);
            if (count > 2) p[2] = (uint16_t)w[1];
        }
    };
    auto store = [&](int i, int j, const f32x4& g, const f32x4& u) __attribute__((always_inline)) {
        const int64_t m = m0 + 16 * i + (lane & 15), n = n0 + 16 * j + 4 * (lane >> 4);
        if (m >= M || n >= F) return;
        const int count = (int)min((int64_t)4, F - n);
        f32x4 h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = activation(out.act, g[e]) * u[e];
        store4(out.h + m * F + n, h, count);
        if (out.gu) {
            store4(out.gu + m * 2 * F + n, g, count);
            store4(out.gu + m * 2 * F + F + n, u, count);
        }
    };
    if (waves == 1) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j) store(i, j, acc[i][j], acc[i][NB + j]);
        return;
    }
    // partial sums to LDS, 1 KB per (wave, block); then wave w adds up the pairs of blocks w, w + waves, ... over the waves in their order
    __syncthreads();   // the staging regions are free
    f32x4* const part = reinterpret_cast<f32x4*>(smem);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) part[((wave * MI + i) * (2 * NB) + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    for (int b = wave; b < MI * NB; b += waves) {
        const int i = b / NB, j = b % NB, at = i * (2 * NB) + j;
        f32x4 g = part[at * 64 + lane], u = part[(at + NB) * 64 + lane];
        for (int w = 1; w < waves; ++w) {
            g += part[(w * BLOCKS + at) * 64 + lane];
            u += part[(w * BLOCKS + at + NB) * 64 + lane];
        }
        store(i, j, g, u);
    }
}

// ---- up to four rows, NT: W is read once, straight to the registers of the products ---------------------------------------------------------------
// A workgroup has four columns of h, its waves take turns along D.  128 k of four rows of W are one load, four pieces of 256 bytes: a lane's sixteen bytes,
// k 8 (lane / 4) .. of row lane % 4, are what it gives to two products of 16 independent blocks, 4 x 4 x 4 each, and x's rows are loaded the same way.
// So no value goes through LDS, no lane waits for another, and the vector unit has no arithmetic to do; the 16 blocks' sums are added up once, behind
// the last k, in a fixed order.
// Bound by the way from memory: 1 x 8192 x 4096 23.2 us, 5.8 TB/s (the wave-K kernel 30.1), 1 x 13824 x 5120 43.5 (49.2), each call with a W that no cache holds.  Only D of multiples of 8: with rows at
// any address the pieces cross lines, and 4 x 4096 x 1001 took 10 us where the wave-K kernel takes 7.  Nor more rows: every workgroup loads all of x, and
// 8 x 8192 x 4096 took 33.
// Requires D % 8 == 0, M <= 4.
template <bool STREAM>
__global__ __launch_bounds__(1024) void gated_rows_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, int64_t M, int64_t D, GatedOut out) {
    constexpr int U = 4;   // loads of a row that are under way together
    typedef short i16x4 __attribute__((ext_vector_type(4)));
    __shared__ float part[16][2][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int64_t F = out.F, f0 = 4 * (int64_t)blockIdx.x;
    const uint16_t* const w[2] = {W + min(f0 + (lane & 3), F - 1) * D, W + (F + min(f0 + (lane & 3), F - 1)) * D};
    const uint16_t* const x = X + min((int64_t)(lane & 3), M - 1) * D;
    f32x4 acc[2] = {};
    for (int64_t k0 = (int64_t)wave * (128 * U); k0 < D; k0 += (int64_t)waves * (128 * U)) {
        u32x4 vw[2][U], vx[U];
        const int64_t k = k0 + 8 * (lane >> 2);
        auto load = [&](auto whole) __attribute__((always_inline)) {   // whole: all 128 U of these k exist
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool there = decltype(whole)::value || k + 128 * u < D;
                const u32x4 none = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int half = 0; half < 2; ++half) vw[half][u] = there ? load16<STREAM>(w[half] + k + 128 * u) : none;
                vx[u] = there ? load16<false>(x + k + 128 * u) : none;
            }
        };
        if (k0 + 128 * U <= D) load(std::true_type{});
        else load(std::false_type{});
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < 4; q += 2)
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    acc[half] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(i16x4, u32x2{vx[u][q], vx[u][q + 1]}),
                                                                       __builtin_bit_cast(i16x4, u32x2{vw[half][u][q], vw[half][u][q + 1]}), acc[half], 0, 0, 0);
    }
    // acc[half][e]: row e, column lane % 4, of the k of block lane / 4
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v = acc[half][e];
#pragma unroll
            for (int step = 4; step < 64; step *= 2) v += __shfl_xor(v, step);
            if (lane < 4) part[wave][half][4 * e + lane] = v;
        }
    __syncthreads();
    const int m = threadIdx.x >> 2;
    const int64_t f = f0 + (threadIdx.x & 3);
    if (m >= M || f >= F) return;
    float g = 0.f, u = 0.f;
    for (int i = 0; i < waves; ++i) {
        g += part[i][0][threadIdx.x];
        u += part[i][1][threadIdx.x];
    }
    out.h[m * F + f] = (uint16_t)pack2_bf16(activation(out.act, g) * u, 0.f);
    if (out.gu) {
        out.gu[m * 2 * F + f] = (uint16_t)pack2_bf16(g, 0.f);
        out.gu[m * 2 * F + F + f] = (uint16_t)pack2_bf16(u, 0.f);
    }
}

// ---- what none of the others takes (D < 8, F < 16 in NN, leading dimensions of 2^24 and more) ---------------------------------------------------------------------------------------------------
// Blocks from `first` on, 64 x 64 of h each by 2 x 2 waves, 32 k at a time: what a thread stages of the next 32 k is on its way to registers while this one's is multiplied from LDS,
// where both operands lie K-contiguous in rows of 32 k and 16 bytes more (sixteen rows then start in different banks).
template <bool B_KC>
__global__ __launch_bounds__(256) void gated_any_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ W, int64_t M, int64_t D, int64_t first, int64_t blocks_n,
                                                        GatedOut out) {
    constexpr int LD = 40;   // bf16 of an LDS row
    __shared__ __attribute__((aligned(16))) uint16_t panel[3][64][LD];   // x, Wg, Wu
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, wm = wave >> 1, wn = wave & 1, r16 = lane & 15, quad = lane >> 4;
    const int64_t block = first + blockIdx.x, m0 = block / blocks_n * 64, n0 = block % blocks_n * 64, F = out.F;
    const int row = t >> 2, chunk = 8 * (t & 3);      // of a K-contiguous panel
    const int k_row = t >> 3, n_chunk = 8 * (t & 7);  // of W as [D, 2F]
    const u32x4 none = {0u, 0u, 0u, 0u};
    u32x4 vx, vw[2];
    auto fetch = [&](int64_t k0) __attribute__((always_inline)) {
        vx = m0 + row < M ? load8<true>(X + (m0 + row) * D + k0 + chunk, k0 + chunk, D) : none;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if constexpr (B_KC) vw[half] = n0 + row < F ? load8<true>(W + (half * F + n0 + row) * D + k0 + chunk, k0 + chunk, D) : none;
            else vw[half] = k0 + k_row < D ? load8<true>(W + (k0 + k_row) * (2 * F) + half * F + n0 + n_chunk, n0 + n_chunk, F) : none;
        }
    };
    f32x4 acc[2][2][2] = {};   // [half][row block][column block]
    fetch(0);
    for (int64_t k0 = 0; k0 < D; k0 += 32) {
        __syncthreads();
        *reinterpret_cast<u32x4*>(&panel[0][row][chunk]) = vx;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if constexpr (B_KC) {
                *reinterpret_cast<u32x4*>(&panel[1 + half][row][chunk]) = vw[half];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) panel[1 + half][n_chunk + i][k_row] = (uint16_t)(vw[half][i / 2] >> (16 * (i & 1)));
            }
        }
        __syncthreads();
        if (k0 + 32 < D) fetch(k0 + 32);
        bf16x8 fx[2], fw[2][2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            fx[b] = *reinterpret_cast<const bf16x8*>(&panel[0][32 * wm + 16 * b + r16][8 * quad]);
#pragma unroll
            for (int half = 0; half < 2; ++half) fw[half][b] = *reinterpret_cast<const bf16x8*>(&panel[1 + half][32 * wn + 16 * b + r16][8 * quad]);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[half][i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[half][j], fx[i], acc[half][i][j], 0, 0, 0);
    }
    // acc[half][i][j][e]: row 16 i + r16, column 16 j + 4 quad + e
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t m = m0 + 32 * wm + 16 * i + r16, n = n0 + 32 * wn + 16 * j + 4 * quad;
            if (m >= M) continue;
            uint32_t g01 = pack2_bf16(acc[0][i][j][0], acc[0][i][j][1]), g23 = pack2_bf16(acc[0][i][j][2], acc[0][i][j][3]);
            uint32_t u01 = pack2_bf16(acc[1][i][j][0], acc[1][i][j][1]), u23 = pack2_bf16(acc[1][i][j][2], acc[1][i][j][3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (n + e >= F) continue;
                const float h = activation(out.act, acc[0][i][j][e]) * acc[1][i][j][e];
                out.h[m * F + n + e] = (uint16_t)pack2_bf16(h, 0.f);
                if (out.gu) {
                    out.gu[m * 2 * F + n + e] = (uint16_t)((e < 2 ? g01 : g23) >> (16 * (e & 1)));
                    out.gu[m * 2 * F + F + n + e] = (uint16_t)((e < 2 ? u01 : u23) >> (16 * (e & 1)));
                }
            }
        }
}

// ---- the gradients of the activation and the product ------------------------------------------------------------------------------
// dg = dh u act'(g), du = dh act(g), side by side as [M, 2F], and h again, eight columns a thread.  dg and du are rounded to bf16 because they are operands of
// two products on the bf16 matrix unit, whose gradients are then 0.0023 of their norm off (0.0017 with their own rounding alone); in fp32 they would be twice
// the bytes and a sixteenth of the unit's rate.  Q8: g and u come from the 8-bit
// format, rows of 2F.  RAGGED: F is no multiple of 8 (u's pieces then start at any byte).  Bound by memory: 10 or 8 bytes an element and 2 for h;
// 2048 x 4096 18 to 20 us (101 MB), from 8 bits 17 to 18 (84 MB).
// Q8: workgroups from slope_groups on restore the other matrix that was kept, which the products want (a launch of its own took 3.5 us where all of it is small).
struct KeptQ8 {
    const uint8_t *q, *qs;
    uint16_t* x;
    int64_t D;
};
namespace rows {   // kernels that are no product and have no layout
template <bool Q8, bool RAGGED>
__global__ __launch_bounds__(256) void gated_slope_kernel(int slope_groups, KeptQ8 kept, int64_t M, int64_t F, int act, const uint16_t* __restrict__ dh, const uint16_t* __restrict__ gu,
                                                          const uint8_t* __restrict__ guq, const uint8_t* __restrict__ gus, uint16_t* __restrict__ dgu, uint16_t* __restrict__ h) {
    if constexpr (Q8) {
        if ((int)blockIdx.x >= slope_groups) {
            q8_restore(blockIdx.x - slope_groups, gridDim.x - slope_groups, M, kept.D, kept.q, kept.qs, kept.x);
            return;
        }
    }
    const int64_t pieces = (F + 7) / 8, total = M * pieces, row_bytes = q8_row_bytes(2 * F), scale_row = q8_scale_row(M);
    for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < total; p += (int64_t)slope_groups * 256) {
        int64_t row, col;
        row_of(p, pieces, &row, &col);
        col *= 8;
        float d[8], g[8], u[8];
        unpack8(load8<RAGGED>(dh + row * F + col, col, F), d);
        auto decode = [&](int64_t at, float (&f)[8]) __attribute__((always_inline)) {
            const uint8_t* const q = guq + row * row_bytes;
            if (!RAGGED) {
                q8_unpack8(*reinterpret_cast<const u32x2*>(q + at), f);
                const float scale = q8_scale(gus[(at / kQ8Block) * scale_row + row]);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= scale;
            } else {   // eight bytes from anywhere, of up to two blocks; what is behind the row's end belongs to no column
                typedef u32x2 __attribute__((aligned(1))) u32x2_bytes;
                const int64_t from = min(at, row_bytes - 8), block = at / kQ8Block, next = min((at + 7) / kQ8Block, row_bytes / kQ8Block - 1);
                const uint64_t v = __builtin_bit_cast(uint64_t, *reinterpret_cast<const u32x2_bytes*>(q + from)) >> (8 * (at - from));
                const float scale[2] = {q8_scale(gus[block * scale_row + row]), q8_scale(gus[next * scale_row + row])};
                q8_unpack8(__builtin_bit_cast(u32x2, v), f);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= scale[(at + i) / kQ8Block != block];
            }
        };
        if constexpr (Q8) {
            decode(col, g);
            decode(F + col, u);
        } else {
            unpack8(load8<RAGGED>(gu + row * 2 * F + col, col, F), g);
            unpack8(load8<RAGGED>(gu + row * 2 * F + F + col, col, F), u);
        }
        float dg[8], du[8], a[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float slope;
            a[i] = activation(act, g[i], &slope);
            dg[i] = d[i] * u[i] * slope;
            du[i] = d[i] * a[i];
            a[i] *= u[i];
        }
        store8<RAGGED>(dgu + row * 2 * F + col, pack8(dg), col, F);
        store8<RAGGED>(dgu + row * 2 * F + F + col, pack8(du), col, F);
        if (h) store8<RAGGED>(h + row * F + col, pack8(a), col, F);
    }
}
}  // namespace rows
using namespace rows;

}  // namespace axonn

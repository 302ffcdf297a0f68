// The gated projections and their gradients: which kernel, and the entry points.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/axonn_linear.h"
#include "gemm_gated.hpp"
#include "kernels.hpp"

namespace axonn {

typedef void (*gated_tile_t)(const uint16_t*, const uint16_t*, int, int, int, TileGrid, int, GatedOut);
struct GatedTile {
    int bm, bn, groups, threads, lds_bytes;   // groups 0: the 64-k kernel on its large tile
    gated_tile_t fn[2][2];                     // [NN, NT][D a multiple of 64, or not]
};
// load schedules as in kernels_k64.hip
template <int SCHED_NN, int SCHED_NT>
static GatedTile gated_large() {
    return GatedTile{256, 256, 0, 512, std::max(k64_lds_bytes(256, 256, SCHED_NN), k64_lds_bytes(256, 256, SCHED_NT)),
                     {{gated_tile_kernel<256, 256, 4, false, SCHED_NN, false>, gated_tile_kernel<256, 256, 4, false, SCHED_NN, true>},
                      {gated_tile_kernel<256, 256, 4, true, SCHED_NT, false>, gated_tile_kernel<256, 256, 4, true, SCHED_NT, true>}}};
}
template <int BM, int BN, int G>
static GatedTile gated_group() {
    return GatedTile{BM, BN, G, 512, group_lds<BM, BN, G>(),
                     {{gated_group_kernel<BM, BN, G, false, false>, gated_group_kernel<BM, BN, G, false, true>},
                      {gated_group_kernel<BM, BN, G, true, false>, gated_group_kernel<BM, BN, G, true, true>}}};
}
static const GatedTile kGatedTiles[] = {gated_large<0, 1>(), gated_group<256, 128, 1>(), gated_group<128, 256, 1>(), gated_group<128, 128, 1>(), gated_group<128, 64, 1>(),
                                        gated_group<64, 128, 1>(), gated_group<64, 64, 2>()};

typedef void (*gated_wavek_t)(const uint16_t*, const uint16_t*, int64_t, int64_t, int, int, int, GatedOut);
struct GatedWaveK {
    int mi, nb;
    gated_wavek_t fn[2];
    gated_wavek_t past;   // NT, W past the caches
};
// A W of 64 MB and more, read once, goes past the caches: with a few such layers none of it is still there at the next call.  Eight layers' W in turn:
// 16 x 8192 x 4096 30.2 -> 26.7 us, 1 x 8192 x 4096 26.2 -> 23.2, 16 x 4096 x 4096 14.7 -> 13.2; one W again and again, which a program of one layer would
// do, 21.0 -> 25.9, 21.1 -> 22.4, 12.1 -> 12.9.  32 MB: 8.6 and 8.7, with all of it in the caches 7.2 and 7.3.  (NN gains nothing.)
static bool gated_past(int64_t F, int64_t D) { return 2 * F * D >= (int64_t)1 << 25; }
// NN: the blocks of either half are 32 bytes of a k-row each.  One doubles the workgroups where there are few (1 x 2048 x 4096 18.2 us with two, 16.0 with one)
// and costs the way from memory where there are enough (16 x 8192 x 4096 35 and 52, 48 x 4096 x 4096 19 and 26): up to F = 4096 and 32 rows.  Four are
// whole lines: 33 x 8192 x 4096 57 -> 39 us, 8 x 16384 x 4096 67 -> 55.
static const GatedWaveK kGatedWaveK[] = {{1, 1, {gated_wavek_kernel<false, 1, 1>, gated_wavek_kernel<true, 1, 1>}, gated_wavek_kernel<true, 1, 1, true>},
                                         {1, 2, {gated_wavek_kernel<false, 1, 2>, gated_wavek_kernel<true, 1, 2>}, gated_wavek_kernel<true, 1, 2, true>},
                                         {2, 1, {gated_wavek_kernel<false, 2, 1>, gated_wavek_kernel<true, 2, 1>}, gated_wavek_kernel<true, 2, 1, true>},
                                         {2, 2, {gated_wavek_kernel<false, 2, 2>, gated_wavek_kernel<true, 2, 2>}, gated_wavek_kernel<true, 2, 2, true>},
                                         {4, 2, {gated_wavek_kernel<false, 4, 2>, gated_wavek_kernel<true, 4, 2>}, nullptr},
                                         {1, 4, {gated_wavek_kernel<false, 1, 4>, nullptr}, nullptr},
                                         {2, 4, {gated_wavek_kernel<false, 2, 4>, nullptr}, nullptr}};
static int gated_wavek_lds(const GatedWaveK& t, int waves, bool nt) {
    const int staged = waves * (WaveKCfg::stage_bytes(true, t.mi) + 2 * WaveKCfg::stage_bytes(nt, t.nb)), sums = waves > 1 ? waves * t.mi * 2 * t.nb * 1024 : 0;
    return std::max(staged, sums);
}

// the most waves that LDS and registers have room for
static int gated_wavek_waves(const GatedWaveK& t, bool nt) {
    int waves = WaveKCfg::max_waves(t.mi, 2 * t.nb);
    while (gated_wavek_lds(t, waves, nt) > 160 * 1024) waves /= 2;
    return waves;
}

void gated_raise_lds_limit() {
    for (const GatedTile& t : kGatedTiles)
        for (const auto& layout : t.fn)
            for (const gated_tile_t fn : layout)
                (void)hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, t.lds_bytes);
    for (const GatedWaveK& t : kGatedWaveK)
        for (const gated_wavek_t fn : {t.fn[0], t.fn[1], t.past})
            if (fn) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize,
                                              gated_wavek_lds(t, gated_wavek_waves(t, fn != t.fn[0]), fn != t.fn[0]));
}

struct GatedChoice {
    const GatedTile* tile = nullptr;
    const GatedWaveK* wavek = nullptr;
    int waves = 0;
    double us = 0.0;
    void consider(double t, const GatedTile* a, const GatedWaveK* b, int w) {
        if (t < 0.0 || ((tile || wavek) && t >= us)) return;
        tile = a;
        wavek = b;
        waves = w;
        us = t;
    }
};

constexpr int64_t kMaxWorkgroups = (int64_t)1 << 22;   // of a launch: times 512 threads below 2^32

// The kernel with the shortest modelled time; the models are those of a product with an output of M x 2F, which takes as long, but for NN tiles
// whose halves are not whole lines (1.1 and 1.03, by the choices on 30 products of 1 to 299 rows).
static GatedChoice gated_choose(int64_t M, int64_t F, int64_t D, bool nt) {
    const int layout = nt ? AXONN_NT : AXONN_NN;
    const int64_t ldw = nt ? D : 2 * F;
    GatedChoice best;
    if (D % 8 == 0 && F % 8 == 0 && D > 64 && D < (1 << 23) && F < (1 << 22) && (!nt || (F + 256) * D * 2 < ((int64_t)1 << 32))) {
        for (const GatedTile& t : kGatedTiles) {
            if (M < t.bm || 2 * F < t.bn || ((M + t.bm - 1) / t.bm) * ((F + t.bn / 2 - 1) / (t.bn / 2)) >= kMaxWorkgroups) continue;
            if (t.groups) {
                best.consider((nt || t.bn > 64 ? 1.0 : 1.1) * group_us(t.bm, t.bn, t.groups, layout, M, 2 * F, D, D, ldw, 2 * F), &t, nullptr, 0);
            } else {
                // a round of 256 tiles: 1.44 us for 64 k and 6 us beside it; the last one takes half as long and more as it has more tiles
                const double tiles = (double)((M + 255) / 256) * (double)((F + 127) / 128), rest = tiles / 256.0 - std::floor(tiles / 256.0);
                const double rounds = std::floor(tiles / 256.0) + (rest > 0.0 ? 0.6 + 0.4 * rest : 0.0);
                best.consider(2.0 + rounds * ((double)((D + 63) / 64) * 1.44 + 6.0), &t, nullptr, 0);
            }
        }
    }
    if (D >= 8 && D < WaveKCfg::MAX_LD && ldw < WaveKCfg::MAX_LD) {
        for (const GatedWaveK& t : kGatedWaveK) {
            if (!t.fn[nt] || (t.mi > 2 && M < 16 * t.mi) || (!nt && (F < 16 * t.nb || (t.nb == 1 && (F > 4096 || M > 32))))) continue;
            const double lines = nt || t.nb == 4 ? 1.0 : t.nb == 2 ? 1.03 : 1.0;
            const int64_t tiles = ((M + 16 * t.mi - 1) / (16 * t.mi)) * ((F + 16 * t.nb - 1) / (16 * t.nb));
            for (int w = 1; w <= gated_wavek_waves(t, nt) && (w == 1 || (int64_t)(w - 1) * WaveKCfg::KC < D); w *= 2)
                if (tiles * 64 * w < ((int64_t)1 << 31)) best.consider(lines * wavek_us(t.mi, 2 * t.nb, w, layout, M, 2 * F, D, D, ldw), nullptr, &t, w);
        }
    }
    return best;
}

// Up to four rows, NT: enough waves along D to fill the chip eight times over, no more than D has loads for
static bool gated_takes_rows(int64_t M, int64_t F, int64_t D, bool nt) { return nt && M <= 4 && F < (1 << 26) && D % 8 == 0 && D > 0; }
static int gated_rows_waves(int64_t F, int64_t D) {
    int waves = 1;
    while (waves < 16 && (F + 3) / 4 * waves < 8192 && waves * 512 < D) waves *= 2;
    return waves;
}

// sizes and layout; the pointers of what holds at least one element are looked at by the callers
static bool gated_sizes(int64_t M, int64_t F, int64_t D, int layout, int activation) {
    constexpr int64_t kMaxDim = (int64_t)1 << 30, kMaxElems = (int64_t)1 << 40;
    return M >= 0 && F >= 0 && D >= 0 && M < kMaxDim && F < kMaxDim && D < kMaxDim && M * D < kMaxElems && 2 * F * D < kMaxElems && 2 * M * F < kMaxElems &&
           (layout == AXONN_NN || layout == AXONN_NT) && (activation == kSilu || activation == kGelu);
}
static bool at16(const void* p) { return p && !(reinterpret_cast<uintptr_t>(p) & 15); }

static int gated_forward(int64_t M, int64_t F, int64_t D, int layout, const uint16_t* X, const uint16_t* W, const GatedOut& out, hipStream_t s) {
    const bool nt = layout == AXONN_NT;
    (void)hipGetLastError();
    if (gated_takes_rows(M, F, D, nt)) {
        hipLaunchKernelGGL((gated_past(F, D) ? gated_rows_kernel<true> : gated_rows_kernel<false>), dim3((unsigned)((F + 3) / 4)), dim3(64 * gated_rows_waves(F, D)), 0, s, X, W,
                           M, D, out);
        return hipGetLastError() == hipSuccess ? AXONN_OK : AXONN_ERR_LAUNCH;
    }
    const GatedChoice how = gated_choose(M, F, D, nt);
    if (how.tile || how.wavek) raise_lds_limits_once();
    if (how.tile) {
        const GatedTile& t = *how.tile;
        const int64_t tiles_m = (M + t.bm - 1) / t.bm, tiles_n = (F + t.bn / 2 - 1) / (t.bn / 2);
        const int k_tail = (int)(D % 64);
        hipLaunchKernelGGL(t.fn[nt][k_tail != 0], dim3((unsigned)(tiles_m * tiles_n)), dim3(t.threads), t.lds_bytes, s, X, W, (int)(D - k_tail + (k_tail ? 64 : 0)), (int)D,
                           (int)(nt ? D : 2 * F), TileGrid{(int)tiles_m, (int)tiles_n, (int)(M - t.bm), (int)(F - t.bn / 2), k_tail}, (int)std::min<int64_t>(tiles_m, 8), out);
    } else if (how.wavek) {
        const GatedWaveK& t = *how.wavek;
        const int64_t tiles_m = (M + 16 * t.mi - 1) / (16 * t.mi), tiles_n = (F + 16 * t.nb - 1) / (16 * t.nb);
        hipLaunchKernelGGL((t.past && nt && tiles_m == 1 && gated_past(F, D) ? t.past : t.fn[nt]), dim3((unsigned)(tiles_m * tiles_n)), dim3(64 * how.waves), gated_wavek_lds(t, how.waves, nt), s, X, W, M, D, (int)tiles_m, (int)tiles_n,
                           (int)std::min<int64_t>(tiles_m, 8), out);
    } else {
        const int64_t blocks_n = (F + 63) / 64, blocks = blocks_n * ((M + 63) / 64);
        for (int64_t first = 0; first < blocks; first += kMaxWorkgroups)
            hipLaunchKernelGGL((nt ? gated_any_kernel<true> : gated_any_kernel<false>), dim3((unsigned)std::min(blocks - first, kMaxWorkgroups)), dim3(256), 0, s, X, W, M, D, first,
                               blocks_n, out);
    }
    return hipGetLastError() == hipSuccess ? AXONN_OK : AXONN_ERR_LAUNCH;
}

// dGU and h from dh and what was saved, then the two products on the library's own kernels: dx sums over both halves at once
static int gated_backward(int64_t M, int64_t F, int64_t D, int layout, int activation, const void* dH, const void* gu, const void* guq, const void* gus, const KeptQ8& kept,
                          const void* X, const void* W, void* dGU, void* H, void* dX, void* dW, void* stream) {
    if (M > 0 && F > 0) {
        auto groups = [](int64_t pieces) { return (int)std::min<int64_t>((pieces + 255) / 256, 1 << 16); };
        const int slope = groups(M * ((F + 7) / 8)), restore = kept.x ? groups(M * (q8_row_bytes(D) / 8)) : 0;
        const bool ragged = F % 8 != 0;
        (void)hipGetLastError();
        hipLaunchKernelGGL((guq ? (ragged ? gated_slope_kernel<true, true> : gated_slope_kernel<true, false>) : ragged ? gated_slope_kernel<false, true> : gated_slope_kernel<false, false>),
                           dim3((unsigned)(slope + restore)), dim3(256), 0, static_cast<hipStream_t>(stream), slope, kept, M, F, activation, (const uint16_t*)dH, (const uint16_t*)gu,
                           (const uint8_t*)guq, (const uint8_t*)gus, (uint16_t*)dGU, (uint16_t*)H);
        if (hipGetLastError() != hipSuccess) return AXONN_ERR_LAUNCH;
    }
    const bool nt = layout == AXONN_NT;
    if (dX) {
        const int rc = axonn_linear_bwd_data(M, D, 2 * F, nt ? AXONN_NN : AXONN_NT, dGU, W, dX, 1, stream);
        if (rc != AXONN_OK) return rc;
    }
    if (!dW) return AXONN_OK;
    return nt ? axonn_linear_bwd_weight(2 * F, D, M, AXONN_TN, dGU, X, dW, 1, stream) : axonn_linear_bwd_weight(D, 2 * F, M, AXONN_TN, X, dGU, dW, 1, stream);
}

// what both backward entry points ask of the rest of their arguments
static bool gated_backward_args(int64_t M, int64_t F, int64_t D, const void* dH, const void* W, const void* dGU, const void* H, const void* dX, const void* dW) {
    auto is = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    if (!is(dH) || !is(W) || !is(dGU) || !is(H) || !is(dX) || !is(dW)) return false;
    if (M > 0 && F > 0 && (!dH || !dGU)) return false;
    return !(dX && M > 0 && D > 0 && F > 0 && !W);
}

}  // namespace axonn

extern "C" {

int axonn_gated_fwd(int64_t M, int64_t F, int64_t D, int layout, int activation, const void* X, const void* W, void* H, void* GU, void* stream) {
    using namespace axonn;
    if (!gated_sizes(M, F, D, layout, activation)) return AXONN_ERR_INVALID_ARG;
    if (M == 0 || F == 0) return AXONN_OK;
    if (!at16(H) || (GU && !at16(GU)) || (D > 0 && (!at16(X) || !at16(W)))) return AXONN_ERR_INVALID_ARG;
    return gated_forward(M, F, D, layout, (const uint16_t*)X, (const uint16_t*)W, GatedOut{(uint16_t*)H, (uint16_t*)GU, F, activation}, static_cast<hipStream_t>(stream));
}

int axonn_gated_bwd(int64_t M, int64_t F, int64_t D, int layout, int activation, const void* dH, const void* GU, const void* X, const void* W, void* dGU, void* H, void* dX,
                    void* dW, void* stream) {
    using namespace axonn;
    if (!gated_sizes(M, F, D, layout, activation) || !gated_backward_args(M, F, D, dH, W, dGU, H, dX, dW)) return AXONN_ERR_INVALID_ARG;
    if (M > 0 && F > 0 && (!at16(GU) || (dW && D > 0 && !at16(X)))) return AXONN_ERR_INVALID_ARG;
    return gated_backward(M, F, D, layout, activation, dH, GU, nullptr, nullptr, KeptQ8{nullptr, nullptr, nullptr, 0}, X, W, dGU, H, dX, dW, stream);
}

int axonn_gated_bwd_q8(int64_t M, int64_t F, int64_t D, int layout, int activation, const void* dH, const void* GU, const void* GU_scale, const void* X, const void* X_scale,
                       const void* W, void* dGU, void* H, void* dX, void* dW, void* scratch, size_t scratch_bytes, void* stream) {
    using namespace axonn;
    if (!gated_sizes(M, F, D, layout, activation) || !gated_backward_args(M, F, D, dH, W, dGU, H, dX, dW)) return AXONN_ERR_INVALID_ARG;
    if (M > 0 && F > 0 && (!at16(GU) || !at16(GU_scale))) return AXONN_ERR_INVALID_ARG;
    KeptQ8 kept = {nullptr, nullptr, nullptr, 0};
    if (M > 0 && F > 0 && D > 0 && dW) {
        if (!at16(X) || !at16(X_scale) || !at16(scratch)) return AXONN_ERR_INVALID_ARG;
        if (scratch_bytes < (size_t)(M * D) * 2) return AXONN_ERR_WORKSPACE;
        kept = KeptQ8{(const uint8_t*)X, (const uint8_t*)X_scale, (uint16_t*)scratch, D};   // exact: the product below is that of the 8-bit values
    }
    return gated_backward(M, F, D, layout, activation, dH, nullptr, GU, GU_scale, kept, scratch, W, dGU, H, dX, dW, stream);
}

}  // extern "C"

// Products of matrices in the 8-bit format: which kernel, and the entry point.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/axonn_linear.h"
#include "gemm_q8.hpp"
#include "kernels.hpp"

namespace axonn {

typedef void (*q8_tile_t)(Q8Operand, Q8Operand, uint16_t*, int64_t, int, int, int);
struct Q8Variant {
    int bm, bn, threads, lds_bytes;
    q8_tile_t fn;
    int per_unit;              // workgroups that fit on a compute unit
    double step, step_alone;   // us for 128 k: with so many on every unit, and with one on each (or on some)
    double fixed;              // us of a round beside that
};
template <int BM, int BN, int WM, int WN, int NS, bool HALVES>
static Q8Variant q8_variant(double step, double step_alone, double fixed) {
    using T = Q8Tile<BM, BN, WM, WN, NS, HALVES>;
    return Q8Variant{BM, BN, T::NT, T::LDS_BYTES, q8_tile_kernel<BM, BN, WM, WN, NS, HALVES>, 160 * 1024 / T::LDS_BYTES, step, step_alone, fixed};
}
// Times over K and over the number of tiles.  More buffers than two gain nothing on the larger tiles (4096^3 on 128 x 128: 66 us with two, 77 with three,
// which leave room for one workgroup a unit); on 64 x 64 reading a whole stage ahead, with four, takes 256 x 4096 x 4096 from 12.0 us to 10.1.
static const Q8Variant kQ8Tiles[] = {q8_variant<256, 256, 2, 4, 2, true>(1.30, 1.15, 6.0), q8_variant<256, 128, 4, 2, 2, true>(0.93, 0.75, 3.0),
                                     q8_variant<128, 128, 2, 4, 2, true>(0.98, 0.57, 3.0), q8_variant<64, 64, 2, 2, 4, false>(0.40, 0.25, 2.0)};

void q8_raise_lds_limit() {
    for (const Q8Variant& v : kQ8Tiles) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(v.fn), hipFuncAttributeMaxDynamicSharedMemorySize, v.lds_bytes);
}

namespace rows {
__global__ __launch_bounds__(256) void q8_zero_kernel(uint16_t* c, int64_t count) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) c[i] = 0;
}
}  // namespace rows
using namespace rows;

constexpr int64_t kMaxWorkgroups = (int64_t)1 << 22;   // of a launch: times 512 threads below 2^32
struct Q8Choice {
    const Q8Variant* tile = nullptr;
    bool few_rows = false;   // neither: no kernel takes that many workgroups
};
// The tile with the shortest modelled time: whole rounds, and what is left of one; or the kernel for few rows.  Both are bound by reading b where there
// are few rows of a: tiles at 6.7 MB/us (33 x 16384 x 4096 12.5 us), the other kernel at 5.6 to 2.9 as a gets more rows (4, 16 and 32 rows: 14.4, 17.9 and
// 25.8 us), but over few rows of b its workgroups share K where a tile takes it all (32 x 4096 x 4096 9.0 us and 9.8, 8 x 4096 x 16384 18 and 34).
static Q8Choice q8_choose(int64_t M, int64_t N, int64_t steps) {
    constexpr int64_t kUnits = 256;
    const double b_bytes = (double)N * (double)steps * 128.0;
    Q8Choice best;
    double best_us = 0.0;
    if (M <= 32 && (N + 15) / 16 < kMaxWorkgroups) {
        best.few_rows = true;
        best_us = 2.5 + b_bytes / (M <= 4 ? 5.6e6 : M <= 16 ? 4.4e6 : 2.9e6);
    }
    for (const Q8Variant& v : kQ8Tiles) {
        const int64_t tiles = ((M + v.bm - 1) / v.bm) * ((N + v.bn - 1) / v.bn), round = kUnits * v.per_unit, rest = tiles % round;
        if (tiles >= kMaxWorkgroups) continue;
        double us = (double)(tiles / round) * ((double)steps * v.step + v.fixed);
        if (rest) us += (double)steps * (rest > kUnits ? v.step : v.step_alone) + v.fixed;
        us = std::max(us, 2.5 + b_bytes / 6.7e6);
        if ((!best.tile && !best.few_rows) || us < best_us) {
            best = Q8Choice{&v, false};
            best_us = us;
        }
    }
    return best;
}

}  // namespace axonn

extern "C" int axonn_q8_linear(int64_t M, int64_t N, int64_t K, const void* a, const void* a_scale, const void* b, const void* b_scale, void* c, void* stream) {
    using namespace axonn;
    constexpr int64_t kMaxDim = (int64_t)1 << 31, kMaxElems = (int64_t)1 << 40;
    if (M < 0 || N < 0 || K < 0 || M >= kMaxDim || N >= kMaxDim || K >= kMaxDim || M * K >= kMaxElems || K * N >= kMaxElems || M * N >= kMaxElems)
        return AXONN_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return AXONN_OK;
    auto at16 = [](const void* p) { return p && !(reinterpret_cast<uintptr_t>(p) & 15); };
    if (!c || (reinterpret_cast<uintptr_t>(c) & 1)) return AXONN_ERR_INVALID_ARG;
    if (K > 0 && (!at16(a) || !at16(a_scale) || !at16(b) || !at16(b_scale))) return AXONN_ERR_INVALID_ARG;
    if (K > ((int64_t)1 << 24)) return AXONN_ERR_UNSUPPORTED;   // a tile's rows are addressed with 32 bits
    const Q8Operand A{(const uint8_t*)a, (const uint8_t*)a_scale, M}, B{(const uint8_t*)b, (const uint8_t*)b_scale, N};
    const int64_t row_bytes = q8_row_bytes(K);
    hipStream_t s = static_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    if (K == 0) {
        hipLaunchKernelGGL(q8_zero_kernel, dim3((unsigned)std::min<int64_t>((M * N + 255) / 256, 1 << 16)), dim3(256), 0, s, (uint16_t*)c, M * N);
        return hipGetLastError() == hipSuccess ? AXONN_OK : AXONN_ERR_LAUNCH;
    }
    const Q8Choice how = q8_choose(M, N, row_bytes / 128);
    if (how.few_rows) {   // at most 32
        hipLaunchKernelGGL((M <= 16 ? q8_rows_kernel<1> : q8_rows_kernel<2>), dim3((unsigned)((N + 15) / 16)), dim3(512), 0, s, A, B, (uint16_t*)c, row_bytes);
    } else if (!how.tile) {
        return AXONN_ERR_UNSUPPORTED;
    } else {
        raise_lds_limits_once();
        const Q8Variant& v = *how.tile;
        const int64_t tiles_m = (M + v.bm - 1) / v.bm, tiles_n = (N + v.bn - 1) / v.bn;
        hipLaunchKernelGGL(v.fn, dim3((unsigned)(tiles_m * tiles_n)), dim3(v.threads), v.lds_bytes, s, A, B, (uint16_t*)c, row_bytes, (int)tiles_m, (int)tiles_n,
                           (int)std::min<int64_t>(tiles_m, 8));
    }
    return hipGetLastError() == hipSuccess ? AXONN_OK : AXONN_ERR_LAUNCH;
}

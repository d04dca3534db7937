// Products of rows sorted by expert with each expert's weights: the projection's kernels
// (qlinear_fwd.h), each workgroup on the rows and weights of one expert.  Few rows are
// bound by reading the weights of the experts that have any (32 on 64, 2048 -> 4096
// channels of 8 bits: 48 us, 4.4 TB/s), many by the matrix cores (16384 on 8, 4096 -> 4096:
// 287 us, 1.92 POP/s; one product of 8192 x 8192 x 8192 of the library 2.10).
#include <algorithm>

#include "qlinear_experts.h"
#include "qlinear_fwd.h"
#include "qlinear_plan.h"

namespace qconv {

namespace {

template <class T, int WB, int FJ, int FI>
__global__ void __launch_bounds__(512) experts_rows(LinearArgs a, ExpertArg ex) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    ExpertRows p;
    if (!expert_tile<16 * FI>(ex, (int)blockIdx.y, p)) return;
    few_product<T, WB, FJ, FI, false>(of_expert(a, p), (int)blockIdx.x, p.tile, smem);
}
template <class T, int WB, int TJ, int TI, int WJ, int WI, int KS>
__global__ void __launch_bounds__(KS *WJ *WI * 64, TJ == 64 ? 4 : 2) experts_tiles(LinearArgs a, ExpertArg ex) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    ExpertRows p;
    int tj;
    if (!expert_place<TI>(ex, a.tiles_j, p, tj)) return;
    tile_product<T, WB, TJ, TI, WJ, WI, KS, false>(of_expert(a, p), tj, p.tile, smem);
}

template <auto Kernel, int LDS>
hipError_t start(const LinearArgs &a, const ExpertArg &ex, dim3 grid, int threads, hipStream_t stream) {
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(Kernel), LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(Kernel, grid, dim3((unsigned)threads), LDS, stream, a, ex);
    return hipGetLastError();
}
template <class T, int WB, int FJ, int FI>
hipError_t few(const LinearArgs &a, const ExpertArg &ex, hipStream_t stream) {
    const dim3 grid((unsigned)((a.k + 16 * FJ - 1) / (16 * FJ)), (unsigned)most_tiles(a.m, ex.count, 16 * FI));
    return start<experts_rows<T, WB, FJ, FI>, few_lds(FJ, FI, false)>(a, ex, grid, 512, stream);
}
template <class T, int WB, int SIZE, int WJ, int WI, int KS>
hipError_t tile(LinearArgs a, const ExpertArg &ex, hipStream_t stream) {
    a.tiles_j = (a.k + SIZE - 1) / SIZE;
    const dim3 grid((unsigned)most_tiles(a.m, ex.count, SIZE) * (unsigned)a.tiles_j);
    return start<experts_tiles<T, WB, SIZE, SIZE, WJ, WI, KS>, tile_lds<T, SIZE, SIZE, WJ * WI * 64, KS, false>()>(
        a, ex, grid, KS * WJ * WI * 64, stream);
}

template <class T, int WB>
hipError_t product(const LinearArgs &a, const ExpertArg &ex, hipStream_t stream) {
    // 4-bit rows of many experts of up to 8 rows each: a wave for each 16 x 16 results, so
    // that the weights stream (64 experts, 2048 -> 4096 channels: 32 rows 28.0 us, by the
    // kernels below 37.7, 128 rows 43.6 and 79.4, 512 rows 62.4 and 80.3).  Fewer results
    // than 12 waves for each CU take a share of the channels each, which those do as well
    // or better (32 experts, 2048 -> 1024: 32 rows 11.4 and 9.5), and more rows are theirs
    // (8 experts, 4096 -> 4096: 128 rows 22.7 and 20.2, 256 rows 33.2 and 20.9).
    if constexpr (WB == 4)
        if (expected_rows(a.m, ex.count) <= 8 && (a.k + 15) / 16 * expected_tiles(a.m, ex.count, 16) >= 12 * 256)
            return launch_expert_rows4(a, ex, __is_same(T, BF16) ? QCONV_BF16 : QCONV_F16, stream);
    switch (plan_linear(a, WB, [&](int size) { return expected_tiles(a.m, ex.count, size); })) {
        case Kind::FEW_1x1: return few<T, WB, 1, 1>(a, ex, stream);
        case Kind::FEW_2x1: return few<T, WB, 2, 1>(a, ex, stream);
        case Kind::FEW_2x2: return few<T, WB, 2, 2>(a, ex, stream);
        case Kind::TILE_64x4: return tile<T, WB, 64, 1, 4, 4>(a, ex, stream);
        case Kind::TILE_64x2: return tile<T, WB, 64, 1, 4, 2>(a, ex, stream);
        case Kind::TILE_128: return tile<T, WB, 128, 2, 2, 1>(a, ex, stream);
        case Kind::TILE_256: return tile<T, WB, 256, 4, 2, 1>(a, ex, stream);
        default: return tile<T, WB, 64, 1, 4, 1>(a, ex, stream);
    }
}

}  // namespace

hipError_t launch_experts(const LinearArgs &a, const ExpertArg &ex, int w_bits, int dtype, hipStream_t stream) {
    if (dtype == QCONV_BF16) return w_bits == 4 ? product<BF16, 4>(a, ex, stream) : product<BF16, 8>(a, ex, stream);
    return w_bits == 4 ? product<F16, 4>(a, ex, stream) : product<F16, 8>(a, ex, stream);
}

}  // namespace qconv

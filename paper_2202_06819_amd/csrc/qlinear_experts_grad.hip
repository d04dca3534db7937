// Gradients of the experts' products: the gradients' tile product (qlinear_grad.h), each
// workgroup on the rows of one expert.  Bound by the matrix cores where the experts have
// many rows (16384 on 8, 4096 x 4096: both products 1.04 ms, 1.06 PFLOP/s), by writing dw
// where they have few (1999 on 24, 1411 -> 1003: dw 54 us in tiles of 256, 66 of 64).
#include <algorithm>

#include "qlinear_experts.h"
#include "qlinear_grad.h"
#include "qlinear_plan.h"

namespace qconv {

namespace {

// dx of the experts' rows: a tile's rows are one expert's, its sum runs over that
// expert's output channels.
template <class T, int WB, bool COPY, int GS, int TJ, int TI, int WJ, int WI, int KS>
__global__ void __launch_bounds__(KS *WJ *WI * 64, GS == 0 ? 1 : TJ == 64 ? 4 : 2) experts_back_rows(GradArgs a, GroupArg g, ExpertArg ex) {
    extern __shared__ __attribute__((aligned(16))) uint8_t all_smem[];
    ExpertRows p;
    int tj;
    if (!expert_place<TI>(ex, a.tiles_j, p, tj)) return;
    a.p = static_cast<const uint16_t *>(a.p) + (int64_t)p.row0 * a.ldp;
    a.b.codes += (int64_t)p.expert * a.nt * a.b.pitch;
    if (GS == 0) a.b.scale += (int64_t)p.expert * a.nt;
    a.out = static_cast<uint16_t *>(a.out) + (int64_t)p.row0 * a.ldo;
    a.ni = p.rows;
    grad_product<T, WB, false, COPY, GS, TJ, TI, WJ, WI, KS>(a, of_expert<GS>(g, p, a.nt), 0, p.tile, tj, all_smem);
}

// dw of each expert: the sum runs over its rows, none of them for some.
template <class T, bool COPY, int TJ, int TI, int WJ, int WI, int KS>
__global__ void __launch_bounds__(KS *WJ *WI * 64) experts_back_weights(GradArgs a, ExpertArg ex) {
    extern __shared__ __attribute__((aligned(16))) uint8_t all_smem[];
    const int tiles = a.tiles_i * a.tiles_j, e = (int)blockIdx.x / tiles;
    int ti, tj;
    tile_at(xcd_run((int)blockIdx.x - e * tiles, tiles), a.tiles_i, a.tiles_j, ti, tj);
    const ExpertRows p = expert_rows(ex, e);
    a.out = static_cast<float *>(a.out) + (int64_t)e * a.ni * a.ldo;
    if (p.rows == 0) {
        for (int n = (int)threadIdx.x; n < TI * TJ / 4; n += KS * WJ * WI * 64) {
            const int row = ti * TI + n / (TJ / 4), col = tj * TJ + n % (TJ / 4) * 4;
            if (row < a.ni) store4(static_cast<float *>(a.out) + (int64_t)row * a.ldo + col, f32x4{0, 0, 0, 0}, a.nj - col);
        }
        return;
    }
    a.p = static_cast<const uint16_t *>(a.p) + (int64_t)p.row0 * a.ldp;
    a.b.codes += (int64_t)p.row0 * a.b.pitch;
    a.b.scale += p.row0;
    a.nt = p.rows;
    a.steps = a.steps_per_split = (p.rows + 63) / 64;
    grad_product<T, 8, true, COPY, 0, TJ, TI, WJ, WI, KS>(a, GroupArg{}, 0, ti, tj, all_smem);
}

template <auto Kernel, int LDS, class... Args>
hipError_t start(int64_t blocks, int threads, hipStream_t stream, Args... args) {
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(Kernel), LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(Kernel, dim3((unsigned)blocks), dim3((unsigned)threads), LDS, stream, args...);
    return hipGetLastError();
}

template <class T, int WB, bool COPY, int GS, int SIZE, int WJ, int WI, int KS>
hipError_t rows_tile(GradArgs a, const GroupArg &g, const ExpertArg &ex, hipStream_t stream) {
    a.tiles_j = (a.nj + SIZE - 1) / SIZE;
    return start<experts_back_rows<T, WB, COPY, GS, SIZE, SIZE, WJ, WI, KS>, KS * grad_lds(SIZE, GS)>(
        most_tiles(a.ni, ex.count, SIZE) * a.tiles_j, KS * WJ * WI * 64, stream, a, g, ex);
}
template <class T, int WB, bool COPY, int GS>
hipError_t rows_product(const GradArgs &a, const GroupArg &g, const ExpertArg &ex, const GradPlan &plan, hipStream_t stream) {
    if (plan.tile == 256) return rows_tile<T, WB, COPY, GS, 256, 8, 1, 1>(a, g, ex, stream);
    if (plan.tile == 128) return rows_tile<T, WB, COPY, GS, 128, 4, 1, 1>(a, g, ex, stream);
    if (plan.groups == 4) return rows_tile<T, WB, COPY, GS, 64, 2, 2, 4>(a, g, ex, stream);
    if (plan.groups == 2) return rows_tile<T, WB, COPY, GS, 64, 2, 2, 2>(a, g, ex, stream);
    return rows_tile<T, WB, COPY, GS, 64, 2, 2, 1>(a, g, ex, stream);
}
template <class T>
hipError_t rows(GradArgs a, GroupArg g, const ExpertArg &ex, int w_bits, int scale_bytes, hipStream_t stream) {
    const bool copies = whole_vectors(a, false);
    const GradPlan plan = plan_expert_grad(
        [&](int size) { return expected_tiles(a.ni, ex.count, size) * ((a.nj + size - 1) / size); }, (a.nt + 63) / 64);
    a.splits = 1;
    a.steps = a.steps_per_split = plan.steps;
    if (w_bits == 8)
        return copies ? rows_product<T, 8, true, 0>(a, g, ex, plan, stream) : rows_product<T, 8, false, 0>(a, g, ex, plan, stream);
    if (scale_bytes == 0)   // one scale a row: any value too, so a group of all channels
        g = {a.b.scale, 1, 0, 0};
    if (scale_bytes == 2)
        return copies ? rows_product<T, 4, true, 2>(a, g, ex, plan, stream) : rows_product<T, 4, false, 2>(a, g, ex, plan, stream);
    return copies ? rows_product<T, 4, true, 4>(a, g, ex, plan, stream) : rows_product<T, 4, false, 4>(a, g, ex, plan, stream);
}

template <class T, bool COPY, int SIZE, int WJ, int WI, int KS>
hipError_t weights_tile(GradArgs a, const ExpertArg &ex, hipStream_t stream) {
    a.tiles_i = (a.ni + SIZE - 1) / SIZE;
    a.tiles_j = (a.nj + SIZE - 1) / SIZE;
    return start<experts_back_weights<T, COPY, SIZE, SIZE, WJ, WI, KS>, KS * grad_lds(SIZE)>(
        (int64_t)ex.count * a.tiles_i * a.tiles_j, KS * WJ * WI * 64, stream, a, ex);
}
template <class T, bool COPY>
hipError_t weights_product(const GradArgs &a, const ExpertArg &ex, const GradPlan &plan, hipStream_t stream) {
    if (plan.tile == 256) return weights_tile<T, COPY, 256, 8, 1, 1>(a, ex, stream);
    if (plan.tile == 128) return weights_tile<T, COPY, 128, 4, 1, 1>(a, ex, stream);
    if (plan.groups == 4) return weights_tile<T, COPY, 64, 4, 1, 4>(a, ex, stream);
    if (plan.groups == 2) return weights_tile<T, COPY, 64, 4, 1, 2>(a, ex, stream);
    return weights_tile<T, COPY, 64, 4, 1, 1>(a, ex, stream);
}
template <class T>
hipError_t weights(GradArgs a, const ExpertArg &ex, hipStream_t stream) {
    const GradPlan plan = plan_expert_grad(
        [&](int size) { return (int64_t)ex.count * ((a.ni + size - 1) / size) * ((a.nj + size - 1) / size); },
        (expected_rows(a.nt, ex.count) + 63) / 64);
    a.splits = 1;
    return whole_vectors(a, true) ? weights_product<T, true>(a, ex, plan, stream)
                                  : weights_product<T, false>(a, ex, plan, stream);
}

}  // namespace

hipError_t launch_expert_grad_input(const GradArgs &a, const GroupArg &g, const ExpertArg &ex, int w_bits, int scale_bytes,
                                    int dtype, hipStream_t stream) {
    return dtype == QCONV_BF16 ? rows<BF16>(a, g, ex, w_bits, scale_bytes, stream)
                               : rows<F16>(a, g, ex, w_bits, scale_bytes, stream);
}
hipError_t launch_expert_grad_weight(const GradArgs &a, const ExpertArg &ex, int dtype, hipStream_t stream) {
    return dtype == QCONV_BF16 ? weights<BF16>(a, ex, stream) : weights<F16>(a, ex, stream);
}

}  // namespace qconv

// The input gradient through 4-bit weights with scales of groups of channels: the
// gradient's tile product (qlinear_grad.h) with a scale for each t and 32 columns.
#include <algorithm>

#include "qlinear_grad.h"

namespace qconv {

namespace {

template <class T, bool COPY, int GS, int TJ, int TI, int WJ, int WI, int KS>
__global__ void __launch_bounds__(KS *WJ *WI * 64, TJ == 64 ? 4 : 2) groups_back(GradArgs a, GroupArg groups) {
    extern __shared__ __attribute__((aligned(16))) uint8_t all_smem[];
    const GradPlace p = grad_place(a);
    grad_product<T, 4, false, COPY, GS, TJ, TI, WJ, WI, KS>(a, groups, p.split, p.ti, p.tj, all_smem);
}

template <auto Kernel, int LDS, int THREADS>
hipError_t tile(const GradArgs &a, const GroupArg &g, hipStream_t stream) {
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(Kernel), LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(Kernel, dim3((unsigned)(a.tiles_i * a.tiles_j * a.splits)), dim3(THREADS), LDS, stream, a, g);
    return hipGetLastError();
}

template <class T, bool COPY, int GS>
hipError_t product(const GradArgs &a, const GroupArg &g, const GradPlan &plan, hipStream_t stream) {
    if (plan.tile == 256) return tile<groups_back<T, COPY, GS, 256, 256, 8, 1, 1>, grad_lds(256, GS), 512>(a, g, stream);
    if (plan.tile == 128) return tile<groups_back<T, COPY, GS, 128, 128, 4, 1, 1>, grad_lds(128, GS), 256>(a, g, stream);
    if (plan.groups == 4) return tile<groups_back<T, COPY, GS, 64, 64, 2, 2, 4>, 4 * grad_lds(64, GS), 1024>(a, g, stream);
    if (plan.groups == 2) return tile<groups_back<T, COPY, GS, 64, 64, 2, 2, 2>, 2 * grad_lds(64, GS), 512>(a, g, stream);
    return tile<groups_back<T, COPY, GS, 64, 64, 2, 2, 1>, grad_lds(64, GS), 256>(a, g, stream);
}

template <class T>
hipError_t grad(GradArgs a, const GroupArg &g, int scale_bytes, hipStream_t stream) {
    const bool copies = whole_vectors(a, false);
    const GradPlan plan = plan_grad(a.ni, a.nj, a.nt);
    a.tiles_i = (a.ni + plan.tile - 1) / plan.tile;
    a.tiles_j = (a.nj + plan.tile - 1) / plan.tile;
    a.splits = plan.splits;
    a.steps = plan.steps;
    a.steps_per_split = plan.steps_per_split;
    hipError_t e;
    if (scale_bytes == 4)
        e = copies ? product<T, true, 4>(a, g, plan, stream) : product<T, false, 4>(a, g, plan, stream);
    else
        e = copies ? product<T, true, 2>(a, g, plan, stream) : product<T, false, 2>(a, g, plan, stream);
    return e != hipSuccess || a.splits == 1 ? e : launch_grad_sum(a, false, __is_same(T, BF16) ? QCONV_BF16 : QCONV_F16, stream);
}

}  // namespace

hipError_t launch_group_grad(const GradArgs &a, const GroupArg &g, int scale_bytes, int dtype, hipStream_t stream) {
    return dtype == QCONV_BF16 ? grad<BF16>(a, g, scale_bytes, stream) : grad<F16>(a, g, scale_bytes, stream);
}

}  // namespace qconv

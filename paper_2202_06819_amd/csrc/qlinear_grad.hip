// Launches of the products of the linear layer's backward pass.
#include "qlinear_grad.h"

namespace qconv {

namespace {

template <auto Kernel, int LDS, int THREADS>
hipError_t tile(const GradArgs &a, hipStream_t stream) {
    static const hipError_t set =
        hipFuncSetAttribute(reinterpret_cast<const void *>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (set != hipSuccess) return set;
    hipLaunchKernelGGL(Kernel, dim3((unsigned)(a.tiles_i * a.tiles_j * a.splits)), dim3(THREADS), LDS, stream, a);
    return hipGetLastError();
}

// Copies only: three steps in LDS.
constexpr int copy_lds(int size) { return 3 * (size * 64 + size * 128 + 256); }
template <class T, PForm P>
hipError_t copied(const GradArgs &a, int size, hipStream_t stream) {
    if (size == 256) return tile<grad_tile<T, P, 256, 256, 8, 1>, copy_lds(256), 512>(a, stream);
    if (size == 128) return tile<grad_tile<T, P, 128, 128, 4, 1>, copy_lds(128), 256>(a, stream);
    return tile<grad_tile<T, P, 64, 64, 2, 2>, copy_lds(64), 256>(a, stream);
}

// Through registers: two steps in LDS, and no tile of 256, which they would not hold.
template <class T, int WB, PForm P>
hipError_t held(const GradArgs &a, int size, hipStream_t stream) {
    if (size == 128) return tile<grad_regs<T, WB, P, 128, 128, 2, 2>, 4 * 128 * kStepBytes, 256>(a, stream);
    return tile<grad_regs<T, WB, P, 64, 64, 1, 4>, 4 * 64 * kStepBytes, 256>(a, stream);
}

template <class Out>
hipError_t sum(const GradArgs &a, hipStream_t stream) {
    const int64_t threads = (int64_t)a.ni * (a.ldpart / 4);
    launch_slices((threads + 255) / 256, 256, [&](long long first, unsigned count) {
        hipLaunchKernelGGL((grad_sum<Out>), dim3(count), dim3(256), 0, stream, a, (int64_t)first);
    });
    return hipGetLastError();
}

template <class T>
hipError_t grad(GradArgs a, bool transposed, int w_bits, hipStream_t stream) {
    const bool copies = w_bits == 8 && whole_vectors(a, transposed);
    const GradPlan plan = plan_grad(a.ni, a.nj, a.nt, copies);
    a.tiles_i = (a.ni + plan.tile - 1) / plan.tile;
    a.tiles_j = (a.nj + plan.tile - 1) / plan.tile;
    a.splits = plan.splits;
    a.steps = plan.steps;
    a.steps_per_split = plan.steps_per_split;
    hipError_t e;
    if (copies)
        e = transposed ? copied<T, PForm::COLUMNS_COPY>(a, plan.tile, stream) : copied<T, PForm::ROWS_COPY>(a, plan.tile, stream);
    else if (transposed)
        e = held<T, 8, PForm::COLUMNS>(a, plan.tile, stream);
    else if (w_bits == 8)
        e = held<T, 8, PForm::ROWS>(a, plan.tile, stream);
    else if (whole_vectors(a, false))
        e = held<T, 4, PForm::ROWS_COPY>(a, plan.tile, stream);
    else
        e = held<T, 4, PForm::ROWS>(a, plan.tile, stream);
    if (e != hipSuccess || a.splits == 1) return e;
    return transposed ? sum<float>(a, stream) : sum<typename T::elem>(a, stream);
}

}  // namespace

GradPlan plan_grad(int64_t ni, int64_t nj, int64_t nt, bool copies) {
    GradPlan p{64, 1, 0, 0};
    p.steps = (int)((nt + 63) / 64);
    auto tiles = [&](int64_t t) { return ((ni + t - 1) / t) * ((nj + t - 1) / t); };
    if (copies && tiles(256) >= 192) p.tile = 256;
    else if (tiles(128) * (p.steps / 4 + 1) >= 192) p.tile = 128;
    // split the sum until the chip is full, eight steps a split at least
    int64_t splits = (256 + tiles(p.tile) - 1) / tiles(p.tile);
    if (p.tile == 256) splits = 1;
    if (splits > (p.steps + 7) / 8) splits = (p.steps + 7) / 8;
    if (splits > 32) splits = 32;
    if (splits < 1) splits = 1;
    p.steps_per_split = (int)((p.steps + splits - 1) / splits);
    p.splits = p.steps_per_split ? (p.steps + p.steps_per_split - 1) / p.steps_per_split : 1;
    return p;
}

hipError_t launch_grad(const GradArgs &a, bool transposed, int w_bits, int dtype, hipStream_t stream) {
    return dtype == QCONV_BF16 ? grad<BF16>(a, transposed, w_bits, stream) : grad<F16>(a, transposed, w_bits, stream);
}

}  // namespace qconv

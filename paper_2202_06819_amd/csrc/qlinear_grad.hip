// Launches of the products of the linear layer's backward pass.
#include <algorithm>

#include "qlinear_grad.h"
#include "qlinear_plan.h"

namespace qconv {

namespace {

template <auto Kernel, int LDS, int THREADS>
hipError_t tile(const GradArgs &a, hipStream_t stream) {
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(Kernel), LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(Kernel, dim3((unsigned)(a.tiles_i * a.tiles_j * a.splits)), dim3(THREADS), LDS, stream, a);
    return hipGetLastError();
}

template <class T, int WB, bool TRANSPOSED, bool COPY>
hipError_t product(const GradArgs &a, const GradPlan &plan, hipStream_t stream) {
    const int size = plan.tile, groups = plan.groups;
    if (size == 256) return tile<grad_tile<T, WB, TRANSPOSED, COPY, 256, 256, 8, 1, 1>, grad_lds(256), 512>(a, stream);
    if (size == 128) return tile<grad_tile<T, WB, TRANSPOSED, COPY, 128, 128, 4, 1, 1>, grad_lds(128), 256>(a, stream);
    // (waves of 16 x 64 convert no code twice, waves of 32 x 32 read p from LDS less often:
    // a step takes 0.46 against 0.52 us transposed, 0.56 against 0.52 in rows)
    constexpr int WJ = TRANSPOSED ? 4 : 2, WI = TRANSPOSED ? 1 : 2;
    if (groups == 4)
        return tile<grad_tile<T, WB, TRANSPOSED, COPY, 64, 64, WJ, WI, 4>, 4 * grad_lds(64), 1024>(a, stream);
    if (groups == 2) return tile<grad_tile<T, WB, TRANSPOSED, COPY, 64, 64, WJ, WI, 2>, 2 * grad_lds(64), 512>(a, stream);
    return tile<grad_tile<T, WB, TRANSPOSED, COPY, 64, 64, WJ, WI, 1>, grad_lds(64), 256>(a, stream);
}

template <class Out>
hipError_t sum(const GradArgs &a, hipStream_t stream) {
    const unsigned threads = (unsigned)a.ni * (unsigned)(a.ldpart / 4);
    hipLaunchKernelGGL((grad_sum<Out>), dim3((threads + 255) / 256), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <class T>
hipError_t grad(GradArgs a, bool transposed, int w_bits, hipStream_t stream) {
    // (of no rows nothing is read, and copies then read nothing)
    const bool copies = a.nt == 0 || whole_vectors(a, transposed);
    const GradPlan plan = plan_grad(a.ni, a.nj, a.nt);
    a.tiles_i = (a.ni + plan.tile - 1) / plan.tile;
    a.tiles_j = (a.nj + plan.tile - 1) / plan.tile;
    a.splits = plan.splits;
    a.steps = plan.steps;
    a.steps_per_split = plan.steps_per_split;
    hipError_t e;
    if (transposed)
        e = copies ? product<T, 8, true, true>(a, plan, stream) : product<T, 8, true, false>(a, plan, stream);
    else if (w_bits == 8)
        e = copies ? product<T, 8, false, true>(a, plan, stream) : product<T, 8, false, false>(a, plan, stream);
    else
        e = copies ? product<T, 4, false, true>(a, plan, stream) : product<T, 4, false, false>(a, plan, stream);
    if (e != hipSuccess || a.splits == 1) return e;
    return launch_grad_sum(a, transposed, __is_same(T, BF16) ? QCONV_BF16 : QCONV_F16, stream);
}

}  // namespace

hipError_t launch_grad_sum(const GradArgs &a, bool to_float, int dtype, hipStream_t stream) {
    if (to_float) return sum<float>(a, stream);
    return dtype == QCONV_BF16 ? sum<BF16::elem>(a, stream) : sum<F16::elem>(a, stream);
}

// The tile, its groups of waves and the split that a model of the kernels' times (us)
// finds fastest.  The constants are measured: a step of 64 of the summed axis takes 1.35
// in a tile of 256 (one workgroup fits a CU), 0.83 alone and 1.25 for two on a CU in one
// of 128, 0.5 to 1.1 for one to four in one of 64; two groups of a tile of 64 take a step
// each in 0.57, four in 1.0; a split adds a launch and its partial sums' way through
// memory.  E.g. (the fastest of some replays; calls one by one take a few percent
// longer) 1024 x 1024 from 32768 rows: 79 us in 16 tiles of 256 split 16 ways, 101 in 64
// of 128 split 8 ways, 133 in 256 of 64 split 8 ways, 141 of four groups; from 2560
// rows: 14.2 in tiles of 64 with four groups, 14.7 with two, 21.6 with one, 22.4 in 128
// split 4 ways, 28.4 in 256 split 8 ways; from 1024: 8.3 with two groups, 9.2 with four,
// 10.6 with one, 18.6 in 128.  512 x 1024 from 4096: 17.2 with four groups split 2 ways.
GradPlan plan_grad(int64_t ni, int64_t nj, int64_t nt) {
    GradPlan best{64, 1, 1, 0, (int)((nt + 63) / 64)};
    double best_us = 0;
    const int64_t steps = best.steps;
    for (const auto &k : kGradKinds) {
        const int64_t tiles = ((ni + k.tile - 1) / k.tile) * ((nj + k.tile - 1) / k.tile);
        for (int64_t want = 1; want <= 32; want *= 2) {
            const int64_t per = (steps + want - 1) / want, splits = per ? (steps + per - 1) / per : 1;
            if (want > 1 && (splits < want || splits * tiles > 4096)) break;
            double us = grad_time(k, splits * tiles, per);
            if (splits > 1) us += 4 + 0.1 * splits + 8e-6 * splits * ni * nj / 5.0;
            if (best_us == 0 || us < best_us) {
                best_us = us;
                best.tile = k.tile;
                best.groups = k.groups;
                best.splits = (int)splits;
                best.steps_per_split = (int)per;
            }
        }
    }
    return best;
}

hipError_t launch_grad(const GradArgs &a, bool transposed, int w_bits, int dtype, hipStream_t stream) {
    return dtype == QCONV_BF16 ? grad<BF16>(a, transposed, w_bits, stream) : grad<F16>(a, transposed, w_bits, stream);
}

}  // namespace qconv

// Launches of the projection with adapters.
#include "qlinear_fwd.h"

namespace qconv {

namespace {

template <class T, int WB, int FI>
void few(const LinearArgs &a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.k + 15) / 16));
    if (a.ad.count)
        hipLaunchKernelGGL((linear_few<T, WB, FI, true>), grid, dim3(512), 0, stream, a);
    else
        hipLaunchKernelGGL((linear_few<T, WB, FI, false>), grid, dim3(512), 0, stream, a);
}

template <auto Kernel, int TJ, int TI, int THREADS>
hipError_t tile(LinearArgs a, hipStream_t stream) {
    constexpr int kLds = 2 * (TJ + TI) * kStepBytes;
    static const hipError_t set =
        hipFuncSetAttribute(reinterpret_cast<const void *>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (set != hipSuccess) return set;
    a.tiles_j = (a.k + TJ - 1) / TJ;
    a.tiles_i = (a.m + TI - 1) / TI;
    hipLaunchKernelGGL(Kernel, dim3((unsigned)a.tiles_i * (unsigned)a.tiles_j), dim3(THREADS), kLds, stream, a);
    return hipSuccess;
}

template <class T, int WB, bool AD>
hipError_t many(const LinearArgs &a, hipStream_t stream) {
    const int64_t big = (int64_t)((a.k + 255) / 256) * ((a.m + 255) / 256);
    if (big >= 192) return tile<linear_tile<T, WB, 256, 256, 4, 2, AD>, 256, 256, 512>(a, stream);
    return tile<linear_tile<T, WB, 128, 128, 2, 2, AD>, 128, 128, 256>(a, stream);
}

template <class T, int RF>
void rows(const LinearArgs &a, hipStream_t stream) {
    const int steps = (a.c + 31) / 32, per = (steps + a.ad.splits - 1) / a.ad.splits;
    hipLaunchKernelGGL((adapter_rows<T, RF>), dim3((unsigned)((a.m + 15) / 16), (unsigned)a.ad.splits), dim3(512), 0,
                       stream, a, per);
}

template <class T, int WB>
hipError_t linear(const LinearArgs &a, hipStream_t stream) {
    if (a.ad.count) {
        if (a.ad.rank <= 16) rows<T, 1>(a, stream);
        else if (a.ad.rank <= 32) rows<T, 2>(a, stream);
        else if (a.ad.rank <= 64) rows<T, 4>(a, stream);
        else rows<T, 8>(a, stream);
    }
    hipError_t e = hipSuccess;
    if (a.m <= 16) few<T, WB, 1>(a, stream);
    else if (a.m <= 32) few<T, WB, 2>(a, stream);
    else if (a.m <= 64) few<T, WB, 4>(a, stream);
    else e = a.ad.count ? many<T, WB, true>(a, stream) : many<T, WB, false>(a, stream);
    return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace

int linear_adapter_splits(int64_t m, int64_t c) {
    const int64_t tiles = (m + 15) / 16, steps = (c + 31) / 32;
    int64_t splits = 256 / tiles;
    if (splits > (steps + 7) / 8) splits = (steps + 7) / 8;
    return (int)(splits < 1 ? 1 : splits > 8 ? 8 : splits);
}

hipError_t launch_linear(const LinearArgs &a, int w_bits, int dtype, hipStream_t stream) {
    if (dtype == QCONV_BF16) return w_bits == 4 ? linear<BF16, 4>(a, stream) : linear<BF16, 8>(a, stream);
    return w_bits == 4 ? linear<F16, 4>(a, stream) : linear<F16, 8>(a, stream);
}

}  // namespace qconv

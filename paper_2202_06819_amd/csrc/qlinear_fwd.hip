// Launches of the projection with adapters.
#include "qlinear_fwd.h"

namespace qconv {

namespace {

// A launch with LDS of any size up to the CU's.
template <auto Kernel, int LDS>
hipError_t start(const LinearArgs &a, dim3 grid, int threads, hipStream_t stream) {
    static const hipError_t set =
        hipFuncSetAttribute(reinterpret_cast<const void *>(Kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (set != hipSuccess) return set;
    hipLaunchKernelGGL(Kernel, grid, dim3((unsigned)threads), LDS, stream, a);
    return hipSuccess;
}

template <class T, int WB, int FJ, int FI>
hipError_t few(const LinearArgs &a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.k + 16 * FJ - 1) / (16 * FJ)), (unsigned)((a.m + 16 * FI - 1) / (16 * FI)));
    if (a.ad.count) return start<linear_few<T, WB, FJ, FI, true>, few_lds(FJ, FI, true)>(a, grid, 512, stream);
    return start<linear_few<T, WB, FJ, FI, false>, few_lds(FJ, FI, false)>(a, grid, 512, stream);
}
template <class T, int WB, int FI>
hipError_t few_channels(const LinearArgs &a, hipStream_t stream) {
    return a.k >= 32 * 192 ? few<T, WB, 2, FI>(a, stream) : few<T, WB, 1, FI>(a, stream);
}

template <auto Kernel, int TJ, int TI, int THREADS>
hipError_t tile(LinearArgs a, hipStream_t stream) {
    a.tiles_j = (a.k + TJ - 1) / TJ;
    a.tiles_i = (a.m + TI - 1) / TI;
    return start<Kernel, 2 * (TJ + TI) * kStepBytes>(a, dim3((unsigned)a.tiles_i * (unsigned)a.tiles_j), THREADS, stream);
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
    hipError_t e;
    if (a.m <= 16) e = few_channels<T, WB, 1>(a, stream);
    else if (a.m <= 32) e = few_channels<T, WB, 2>(a, stream);
    else if (a.m <= 64) e = few_channels<T, WB, 4>(a, stream);
    else e = a.ad.count ? many<T, WB, true>(a, stream) : many<T, WB, false>(a, stream);
    return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace

int linear_adapter_splits(int64_t m, int64_t c) {
    // about 128 workgroups of 16 rows, each with a step of 32 channels for every wave
    const int64_t tiles = (m + 15) / 16, steps = (c + 31) / 32;
    int64_t splits = 128 / tiles;
    if (splits > (steps + 7) / 8) splits = (steps + 7) / 8;
    return (int)(splits < 1 ? 1 : splits > 16 ? 16 : splits);
}

hipError_t launch_linear(const LinearArgs &a, int w_bits, int dtype, hipStream_t stream) {
    if (dtype == QCONV_BF16) return w_bits == 4 ? linear<BF16, 4>(a, stream) : linear<BF16, 8>(a, stream);
    return w_bits == 4 ? linear<F16, 4>(a, stream) : linear<F16, 8>(a, stream);
}

}  // namespace qconv

// Launches of the projection with adapters.
#include <algorithm>

#include "qlinear_fwd.h"
#include "qlinear_plan.h"

namespace qconv {

namespace {

// A launch with LDS of any size up to the CU's.
template <auto Kernel, int LDS>
hipError_t start(const LinearArgs &a, dim3 grid, int threads, hipStream_t stream) {
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(Kernel), LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(Kernel, grid, dim3((unsigned)threads), LDS, stream, a);
    return hipSuccess;
}

template <class T, int WB, int FJ, int FI, bool AD>
hipError_t few(const LinearArgs &a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.k + 16 * FJ - 1) / (16 * FJ)), (unsigned)((a.m + 16 * FI - 1) / (16 * FI)));
    return start<linear_few<T, WB, FJ, FI, AD>, few_lds(FJ, FI, AD)>(a, grid, 512, stream);
}

template <class T, auto Kernel, int TJ, int TI, int KS, int THREADS, bool AD>
hipError_t tile(LinearArgs a, hipStream_t stream) {
    a.tiles_j = (a.k + TJ - 1) / TJ;
    a.tiles_i = (a.m + TI - 1) / TI;
    return start<Kernel, tile_lds<T, TJ, TI, THREADS / KS, KS, AD>()>(a, dim3((unsigned)a.tiles_i * (unsigned)a.tiles_j),
                                                                      THREADS, stream);
}

template <class T, int WB, bool AD>
hipError_t product(const LinearArgs &a, hipStream_t stream) {
    switch (plan_linear(a, WB, [&](int rows) { return (a.m + rows - 1) / rows; })) {
        case Kind::FEW_1x1: return few<T, WB, 1, 1, AD>(a, stream);
        case Kind::FEW_2x1: return few<T, WB, 2, 1, AD>(a, stream);
        case Kind::FEW_2x2: return few<T, WB, 2, 2, AD>(a, stream);
        case Kind::FEW_2x4:
            if constexpr (AD) return few<T, WB, 2, 4, AD>(a, stream);
            [[fallthrough]];
        case Kind::TILE_64x4: return tile<T, linear_tile<T, WB, 64, 64, 1, 4, 4, AD>, 64, 64, 4, 1024, AD>(a, stream);
        case Kind::TILE_64x2: return tile<T, linear_tile<T, WB, 64, 64, 1, 4, 2, AD>, 64, 64, 2, 512, AD>(a, stream);
        case Kind::TILE_64: return tile<T, linear_tile<T, WB, 64, 64, 1, 4, 1, AD>, 64, 64, 1, 256, AD>(a, stream);
        case Kind::TILE_128: return tile<T, linear_tile<T, WB, 128, 128, 2, 2, 1, AD>, 128, 128, 1, 256, AD>(a, stream);
        default: return tile<T, linear_tile<T, WB, 256, 256, 4, 2, 1, AD>, 256, 256, 1, 512, AD>(a, stream);
    }
}

template <class T, int RF, int NI>
hipError_t rows_of(const LinearArgs &a, hipStream_t stream) {
    constexpr auto kKernel = adapter_rows<T, RF, NI>;
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(kKernel), adapter_lds(RF, NI));
    if (e != hipSuccess) return e;
    const int steps = (a.c + 31) / 32, per = (steps + a.ad.splits - 1) / a.ad.splits, tiles = (a.m + 16 * NI - 1) / (16 * NI);
    const int z = std::min({256 / (tiles * a.ad.splits) + 1, a.ad.count, 4});
    hipLaunchKernelGGL(kKernel, dim3((unsigned)tiles, (unsigned)a.ad.splits, (unsigned)z), dim3(adapter_waves(RF) * 64),
                       adapter_lds(RF, NI), stream, a, per);
    return hipSuccess;
}
template <class T, int RF>
hipError_t rows(const LinearArgs &a, hipStream_t stream) {
    return a.m > 512 ? rows_of<T, RF, 2>(a, stream) : rows_of<T, RF, 1>(a, stream);
}

template <class T, int WB>
hipError_t linear(const LinearArgs &a, hipStream_t stream) {
    if (a.ad.count) {
        const hipError_t e = a.ad.rank <= 16 ? rows<T, 1>(a, stream) : a.ad.rank <= 32 ? rows<T, 2>(a, stream)
                             : a.ad.rank <= 64 ? rows<T, 4>(a, stream) : rows<T, 8>(a, stream);
        if (e != hipSuccess) return e;
    }
    const hipError_t e = a.ad.count ? product<T, WB, true>(a, stream) : product<T, WB, false>(a, stream);
    return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace

int linear_adapter_splits(int64_t m, int64_t c) {
    // about 256 workgroups of 16 rows, with eight steps of 32 channels each at least;
    // fewer partial sums for more rows, since every workgroup of the product adds them
    const int64_t tiles = (m + 15) / 16, steps = (c + 31) / 32;
    // (565 rows, 6144 -> 272 channels: 14.6 us with four runs, 20.9 with two; 2003 rows,
    // 2048 -> 8192 channels: the product 48.7 us with two, 55 with four)
    int64_t splits = 256 / tiles;
    int64_t most = m <= 16 ? 4 : m <= 64 ? 16 : m <= 512 ? 1024 / m : 2;
    if (m > 256 && c > 4096) splits = 512 / tiles, most = 4;
    if (splits > most) splits = most;
    if (splits > (steps + 7) / 8) splits = (steps + 7) / 8;
    return (int)(splits < 1 ? 1 : splits);
}

hipError_t launch_linear(const LinearArgs &a, int w_bits, int dtype, hipStream_t stream) {
    if (dtype == QCONV_BF16) return w_bits == 4 ? linear<BF16, 4>(a, stream) : linear<BF16, 8>(a, stream);
    return w_bits == 4 ? linear<F16, 4>(a, stream) : linear<F16, 8>(a, stream);
}

}  // namespace qconv

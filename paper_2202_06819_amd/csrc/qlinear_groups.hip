// Launches of the projection by 4-bit weights with scales of groups of channels, dense
// and of experts.
#include <algorithm>

#include "qlinear_experts.h"
#include "qlinear_groups.h"
#include "qlinear_plan.h"

namespace qconv {

namespace {

template <int GS, int NG, int FJ, int RB>
__global__ void __launch_bounds__(512) groups_rows(LinearArgs a, GroupArg g, int bf16) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    groups_few<GS, NG, FJ, RB>(a, g, bf16, (int)blockIdx.x, (int)blockIdx.y, smem);
}
template <int GS, int NG, int TJ, int TI, int WJ, int WI, int KS>
__global__ void __launch_bounds__(KS *WJ *WI * 64, TJ == 64 ? 4 : 2) groups_tiles(LinearArgs a, GroupArg g, int bf16) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    int ti, tj;
    tile_at(xcd_run((int)blockIdx.x, a.tiles_i * a.tiles_j), a.tiles_i, a.tiles_j, ti, tj);
    groups_tile<GS, NG, TJ, TI, WJ, WI, KS>(a, g, bf16, tj, ti, smem);
}
template <int GS, int NG, int FJ, int RB>
__global__ void __launch_bounds__(512) expert_groups_rows(LinearArgs a, GroupArg g, ExpertArg ex, int bf16) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    constexpr int kSize = 16 / NG * RB;
    if ((int)blockIdx.y >= expert_tiles<kSize>(ex)) return;
    const ExpertRows p = expert_tile<kSize>(ex, (int)blockIdx.y);
    groups_few<GS, NG, FJ, RB>(of_expert(a, p), of_expert<GS>(g, p, a.k), bf16, (int)blockIdx.x, p.tile, smem);
}
template <int GS, int NG, int TJ, int TI, int WJ, int WI, int KS>
__global__ void __launch_bounds__(KS *WJ *WI * 64, TJ == 64 ? 4 : 2)
    expert_groups_tiles(LinearArgs a, GroupArg g, ExpertArg ex, int bf16) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    ExpertRows p;
    int tj;
    if (!expert_place<TI>(ex, a.tiles_j, p, tj)) return;
    groups_tile<GS, NG, TJ, TI, WJ, WI, KS>(of_expert(a, p), of_expert<GS>(g, p, a.k), bf16, tj, p.tile, smem);
}

template <auto Kernel, int LDS, class... Args>
hipError_t start(dim3 grid, int threads, hipStream_t stream, Args... args) {
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(Kernel), LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(Kernel, grid, dim3((unsigned)threads), LDS, stream, args...);
    return hipGetLastError();
}

struct Call {
    LinearArgs a;
    GroupArg g;
    ExpertArg ex;
    bool experts;
    int bf16;
    hipStream_t stream;
    // tiles of `size` rows that a launch has to have
    int64_t row_tiles(int size) const { return experts ? most_tiles(a.m, ex.count, size) : (a.m + size - 1) / size; }
};

template <int GS, int NG, int FJ, int RB>
hipError_t few(const Call &c) {
    constexpr int kLds = groups_few_lds(FJ, RB, NG);
    const dim3 grid((unsigned)((c.a.k + 16 * FJ - 1) / (16 * FJ)), (unsigned)c.row_tiles(16 / NG * RB));
    if (c.experts) return start<expert_groups_rows<GS, NG, FJ, RB>, kLds>(grid, 512, c.stream, c.a, c.g, c.ex, c.bf16);
    return start<groups_rows<GS, NG, FJ, RB>, kLds>(grid, 512, c.stream, c.a, c.g, c.bf16);
}
template <int GS, int NG, int SIZE, int WJ, int WI, int KS>
hipError_t tile(Call c) {
    constexpr int kLds = groups_tile_lds(SIZE, SIZE, KS, NG);
    c.a.tiles_j = (c.a.k + SIZE - 1) / SIZE;
    c.a.tiles_i = (int32_t)c.row_tiles(SIZE);
    const dim3 grid((unsigned)c.a.tiles_i * (unsigned)c.a.tiles_j);
    if (c.experts)
        return start<expert_groups_tiles<GS, NG, SIZE, SIZE, WJ, WI, KS>, kLds>(grid, KS * WJ * WI * 64, c.stream, c.a, c.g,
                                                                               c.ex, c.bf16);
    return start<groups_tiles<GS, NG, SIZE, SIZE, WJ, WI, KS>, kLds>(grid, KS * WJ * WI * 64, c.stream, c.a, c.g, c.bf16);
}

template <int GS, int NG>
hipError_t product(const Call &c) {
    const int64_t each = c.experts ? expected_rows(c.a.m, c.ex.count) : c.a.m;
    if (each <= 16) {
        if (NG == 4 && each > 8) return few<GS, NG, 1, NG == 4 ? 4 : 1>(c);
        if (NG >= 2 && each > 16 / NG) return few<GS, NG, 1, NG >= 2 ? 2 : 1>(c);
        return few<GS, NG, 1, 1>(c);
    }
    const Kind kind = plan_linear(c.a, 4, [&](int size) {
        return c.experts ? expected_tiles(c.a.m, c.ex.count, size) : (c.a.m + size - 1) / size;
    });
    switch (kind) {
        case Kind::TILE_64x4: return tile<GS, NG, 64, 1, 4, 4>(c);
        case Kind::TILE_64: return tile<GS, NG, 64, 1, 4, 1>(c);
        case Kind::TILE_128: return tile<GS, NG, 128, 2, 2, 1>(c);
        case Kind::TILE_256: return tile<GS, NG, 256, 4, 2, 1>(c);
        default: return tile<GS, NG, 64, 1, 4, 2>(c);
    }
}

hipError_t run(const Call &c, int scale_bytes, int group) {
    if (scale_bytes == 4)
        return group % 128 == 0 ? product<4, 1>(c) : group % 64 == 0 ? product<4, 2>(c) : product<4, 4>(c);
    return group % 128 == 0 ? product<2, 1>(c) : group % 64 == 0 ? product<2, 2>(c) : product<2, 4>(c);
}

}  // namespace

hipError_t launch_groups(const LinearArgs &a, const GroupArg &g, int scale_bytes, int group, int dtype, hipStream_t stream) {
    return run({a, g, ExpertArg{}, false, dtype == QCONV_BF16, stream}, scale_bytes, group);
}
hipError_t launch_expert_groups(const LinearArgs &a, const GroupArg &g, const ExpertArg &ex, int scale_bytes, int group,
                                int dtype, hipStream_t stream) {
    return run({a, g, ex, true, dtype == QCONV_BF16, stream}, scale_bytes, group);
}

}  // namespace qconv

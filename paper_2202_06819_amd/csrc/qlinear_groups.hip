// Launches of the projection by 4-bit weights with scales of groups of channels, dense
// and of experts.
#include <algorithm>
#include <cmath>

#include "qlinear_experts.h"
#include "qlinear_groups.h"
#include "qlinear_plan.h"

namespace qconv {

namespace {

template <int GS, int NG, bool EVEN, int RB>
__global__ void __launch_bounds__(512) groups_rows(LinearArgs a, GroupArg g, int bf16, int share, int chunk) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    groups_few<GS, NG, EVEN, RB>(a, g, bf16, share, chunk, (int)blockIdx.x, (int)blockIdx.y, smem);
}
template <int GS, int NG, int TJ, int TI, int WJ, int WI, int KS>
__global__ void __launch_bounds__(KS *WJ *WI * 64, TJ == 64 ? 4 : 2) groups_tiles(LinearArgs a, GroupArg g, int bf16) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    int ti, tj;
    tile_at(xcd_run((int)blockIdx.x, a.tiles_i * a.tiles_j), a.tiles_i, a.tiles_j, ti, tj);
    groups_tile<GS, NG, TJ, TI, WJ, WI, KS>(a, g, bf16, tj, ti, smem);
}
template <int GS, int NG, bool EVEN, int RB>
__global__ void __launch_bounds__(512) expert_groups_rows(LinearArgs a, GroupArg g, ExpertArg ex, int bf16, int share, int chunk) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    ExpertRows p;
    if (!expert_tile<16 / NG * RB>(ex, (int)blockIdx.y, p)) return;
    groups_few<GS, NG, EVEN, RB>(of_expert(a, p), of_expert<GS>(g, p, a.k), bf16, share, chunk, (int)blockIdx.x, p.tile, smem);
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

// A launch with `lds` bytes, LDS at most.
template <auto Kernel, int LDS, class... Args>
hipError_t start(dim3 grid, int threads, int lds, hipStream_t stream, Args... args) {
    const hipError_t e = allow_lds(reinterpret_cast<const void *>(Kernel), LDS);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(Kernel, grid, dim3((unsigned)threads), (unsigned)lds, stream, args...);
    return hipGetLastError();
}

struct Call {
    LinearArgs a;
    GroupArg g;
    ExpertArg ex;
    bool experts;
    int bf16;
    hipStream_t stream;
    // rows of a product, of an expert that has any
    int64_t rows() const { return experts ? expected_rows(a.m, ex.count) : a.m; }
    // tiles of `size` rows that a launch has to have
    int64_t row_tiles(int size) const { return experts ? most_tiles(a.m, ex.count, size) : (a.m + size - 1) / size; }
};

template <int GS, int NG, bool EVEN, int RB>
hipError_t few(const Call &c) {
    constexpr int kSize = 16 / NG * RB, kMost = groups_few_lds(16, 32, RB, NG);
    // waves to a tile: enough to fill the chip with 24 for each CU, of a block at least
    // (32 rows on 25 experts, 2048 -> 4096 channels, 6400 tiles: 29.0 us with one, 31.2 with
    // two, 36.6 with four; 128 rows on 31, 4096 -> 2048, 3968 tiles: 40.7, 35.2 and 36.5; a
    // row, 4096 -> 8192, 512 tiles: 14.1, 9.3, 7.2 and 7.2 with eight)
    const int64_t tiles = (c.a.k + 15) / 16, all = tiles * (c.experts ? expected_tiles(c.a.m, c.ex.count, kSize) : c.row_tiles(kSize));
    int share = 1;
    while (share < kGroupWaves && all * share < 6144 && c.a.steps > share * kBlock) share *= 2;
    // rows in LDS: 64 KiB of them at most (a chunk is whole turns of the waves), or all
    const int rows = std::min(kSize, c.a.m);
    int chunk = kGroupWaves * kBlock;
    while (chunk < c.a.steps && rows * few_pitch(2 * chunk) <= 16 * few_pitch(kGroupWaves * kBlock)) chunk *= 2;
    const dim3 grid((unsigned)((tiles * share + kGroupWaves - 1) / kGroupWaves), (unsigned)c.row_tiles(kSize));
    const int lds = groups_few_lds(rows, chunk, RB, NG);
    if constexpr (GS > 0)
        if (!c.experts) return start<groups_rows<GS, NG, EVEN, RB>, kMost>(grid, 512, lds, c.stream, c.a, c.g, c.bf16, share, chunk);
    return start<expert_groups_rows<GS, NG, EVEN, RB>, kMost>(grid, 512, lds, c.stream, c.a, c.g, c.ex, c.bf16, share, chunk);
}
template <int GS, int NG, int SIZE, int WJ, int WI, int KS>
hipError_t tile(Call c) {
    constexpr int kLds = groups_tile_lds(SIZE, SIZE, KS, NG);
    c.a.tiles_j = (c.a.k + SIZE - 1) / SIZE;
    c.a.tiles_i = (int32_t)c.row_tiles(SIZE);
    const dim3 grid((unsigned)c.a.tiles_i * (unsigned)c.a.tiles_j);
    if (c.experts)
        return start<expert_groups_tiles<GS, NG, SIZE, SIZE, WJ, WI, KS>, kLds>(grid, KS * WJ * WI * 64, kLds, c.stream, c.a, c.g,
                                                                               c.ex, c.bf16);
    return start<groups_tiles<GS, NG, SIZE, SIZE, WJ, WI, KS>, kLds>(grid, KS * WJ * WI * 64, kLds, c.stream, c.a, c.g, c.bf16);
}

// A model of the kernels' times (us), its constants measured: a tile takes `start` in its
// turn on a CU and step[n] for each 128 channels (of each of its groups of waves) with n + 1
// on it, by the slices of a step (1, 2 or 4).  E.g. 2048 -> 8192 channels in groups of 128:
// 24 rows 7.0, as a tile of 64 with four groups 8.9; 64 rows 9.4 as that tile, 12.4 as rows;
// 300 rows, 4096 -> 4096: 22.5 (tile of 64, two groups; four 26.9, one 31.8, tile of 128 36);
// 4096 rows 93 (tile of 256; of 128 99, of 64 140), in groups of 32 167 (176, 209).
struct Tile {
    Kind kind;
    int size, groups, resident;
    double start, step[3][4];
};
constexpr Tile kTiles[] = {
    {Kind::TILE_64x4, 64, 4, 1, 3.5, {{1.3}, {1.45}, {2.05}}},
    {Kind::TILE_64x2, 64, 2, 2, 3.4, {{0.95, 1.0}, {1.05, 1.12}, {1.4, 1.56}}},
    {Kind::TILE_64, 64, 1, 4, 2.9, {{0.87, 0.9, 0.95, 1.0}, {0.91, 0.96, 1.05, 1.14}, {1.12, 1.17, 1.35, 1.55}}},
    {Kind::TILE_128, 128, 1, 2, 4.2, {{0.98, 1.43}, {1.16, 1.7}, {1.82, 2.6}}},
    {Kind::TILE_256, 256, 1, 1, 6.0, {{2.5}, {3.15}, {4.9}}}};
// Of the few-row kernel: for each 16 channels by 128 of a tile's rows, and what its blocks of
// 16 / slices rows past the first add; but a wave's turn for each block at least, however few
// the channels (20 rows, 128 -> 1024: 4.9 in groups of 128, 5.8 of 64, 7.9 of 32; tiles 3.7
// to 3.9).
constexpr double kFewStart = 3.5, kFewUnit = 0.24e-3, kFewBlock = 0.08e-3, kFewTurn = 1.0;

// Blocks of rows of a tile of the few-row kernel, for so many rows.
int few_blocks(int slices, int64_t rows) {
    const int64_t block = 16 / slices;
    return slices == 1 || rows <= block ? 1 : slices == 2 || rows <= 2 * block ? 2 : 4;
}

// The fastest, and its time; FEW_1x1: the few-row kernel, of few_slices.
Kind plan(const Call &c, int slices, int few_slices, double &best_us) {
    const int n = slices == 1 ? 0 : slices == 2 ? 1 : 2;
    const auto row_tiles = [&](int size) {
        return c.experts ? expected_tiles(c.a.m, c.ex.count, size) : (c.a.m + size - 1) / size;
    };
    const int blocks = few_blocks(few_slices, c.rows()), few_rows = 16 / few_slices * blocks;
    const double units = (double)((c.a.k + 15) / 16) * row_tiles(few_rows) * c.a.steps;
    Kind best = Kind::FEW_1x1;
    best_us = kFewStart + std::max((kFewUnit + kFewBlock * (blocks - 1)) * units, kFewTurn * blocks);
    if (c.row_tiles(few_rows) > 65535) best_us = INFINITY;   // (a grid's second axis)
    for (const Tile &t : kTiles) {
        const int64_t on_cu = ((c.a.k + t.size - 1) / t.size * (int64_t)row_tiles(t.size) + 255) / 256, rest = on_cu % t.resident;
        const double step = (on_cu / t.resident) * t.step[n][t.resident - 1] + (rest ? t.step[n][rest - 1] : 0.0);
        const double us = (on_cu + t.resident - 1) / t.resident * t.start + (c.a.steps + t.groups - 1) / t.groups * step;
        if (us < best_us) best = t.kind, best_us = us;
    }
    return best;
}

template <int GS, int NG, bool EVEN>
hipError_t few_of(const Call &c) {
    const int blocks = few_blocks(NG, c.rows());
    if constexpr (NG == 4)
        if (blocks == 4) return few<GS, NG, EVEN, 4>(c);
    if constexpr (NG >= 2)
        if (blocks == 2) return few<GS, NG, EVEN, 2>(c);
    return few<GS, NG, EVEN, 1>(c);
}

template <int GS, int NG>
hipError_t product(const Call &c, int group) {
    const bool even = group == 128 / NG;
    const int few_slices = even ? NG : 4;
    double us;
    const Kind kind = plan(c, NG, few_slices, us);
    // A last tile of few rows may cost a turn of all CUs: those rows by a launch of their own
    // (1543 rows, 2824 -> 5003 channels in groups of 32: 520 tiles of 128 where 512 fit at
    // once; 7 rows apart 82.5 us, with them 88.9).
    if (!c.experts && kind != Kind::FEW_1x1 && c.a.m % 64 && c.a.m % 64 <= 16) {
        Call whole = c, rest = c;
        rest.a.m = c.a.m % 64;
        whole.a.m -= rest.a.m;
        double whole_us, rest_us;
        plan(whole, NG, few_slices, whole_us);
        if (plan(rest, NG, few_slices, rest_us) == Kind::FEW_1x1 && whole_us + rest_us + 2.0 < us) {
            rest.a.x.codes += (int64_t)whole.a.m * c.a.x.pitch;
            rest.a.x.scale += whole.a.m;
            rest.a.y = static_cast<uint16_t *>(c.a.y) + (int64_t)whole.a.m * c.a.ldy;
            const hipError_t e = product<GS, NG>(whole, group);
            return e != hipSuccess ? e : product<GS, NG>(rest, group);
        }
    }
    switch (kind) {
        case Kind::FEW_1x1: return even ? few_of<GS, NG, true>(c) : few_of<GS, 4, false>(c);
        case Kind::TILE_64x4: return tile<GS, NG, 64, 1, 4, 4>(c);
        case Kind::TILE_64x2: return tile<GS, NG, 64, 1, 4, 2>(c);
        case Kind::TILE_128: return tile<GS, NG, 128, 2, 2, 1>(c);
        case Kind::TILE_256: return tile<GS, NG, 256, 4, 2, 1>(c);
        default: return tile<GS, NG, 64, 1, 4, 1>(c);
    }
}

hipError_t run(const Call &c, int scale_bytes, int group) {
    if (scale_bytes == 4)
        return group % 128 == 0 ? product<4, 1>(c, group) : group % 64 == 0 ? product<4, 2>(c, group) : product<4, 4>(c, group);
    return group % 128 == 0 ? product<2, 1>(c, group) : group % 64 == 0 ? product<2, 2>(c, group) : product<2, 4>(c, group);
}

}  // namespace

hipError_t launch_expert_rows4(const LinearArgs &a, const ExpertArg &ex, int dtype, hipStream_t stream) {
    return few<0, 1, true, 1>({a, GroupArg{}, ex, true, dtype == QCONV_BF16, stream});
}

hipError_t launch_groups(const LinearArgs &a, const GroupArg &g, int scale_bytes, int group, int dtype, hipStream_t stream) {
    return run({a, g, ExpertArg{}, false, dtype == QCONV_BF16, stream}, scale_bytes, group);
}
hipError_t launch_expert_groups(const LinearArgs &a, const GroupArg &g, const ExpertArg &ex, int scale_bytes, int group,
                                int dtype, hipStream_t stream) {
    return run({a, g, ex, true, dtype == QCONV_BF16, stream}, scale_bytes, group);
}

}  // namespace qconv

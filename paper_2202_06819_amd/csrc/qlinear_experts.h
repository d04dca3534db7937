// Which rows of which expert a workgroup takes.  How the rows are dealt to the experts
// is known on the device only: a launch has workgroups for the most tiles that its rows
// can make (ceil(m_e / T) summed over the experts is at most m / T + min(experts, m)), and
// each finds its own tile from the offsets, in a few instructions of one wave: 64 experts
// at a time, a lane each, and a running sum over the lanes.  Those past the last tile end.
#pragma once

#include "qlinear_device.h"

namespace qconv {

// Workgroups of tiles of `size` rows that cover m rows dealt to `experts` in any way.
inline int64_t most_tiles(int64_t m, int64_t experts, int64_t size) { return m / size + (experts < m ? experts : m); }

struct ExpertRows {
    int expert, row0, rows;   // the expert's rows, of all
    int tile;                 // of the expert's own tiles
};

__device__ __forceinline__ int within(int v, int most) { return min(max(v, 0), most); }

// The lane's expert e: its rows, and the sum of the tiles of the experts up to it in the
// lanes of this wave.
template <int SIZE>
__device__ __forceinline__ void lane_expert(const ExpertArg &ex, int e, int &row0, int &rows, int &tiles, int &sum) {
    const bool in = e < ex.count;
    row0 = in ? within(ex.offsets[e], ex.rows) : 0;
    rows = in ? max(within(ex.offsets[e + 1], ex.rows) - row0, 0) : 0;
    tiles = (rows + SIZE - 1) / SIZE;
    sum = tiles;
    const int lane = (int)threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int before = __shfl_up(sum, d);
        sum += lane >= d ? before : 0;
    }
}

// Tiles of SIZE rows of all experts.
template <int SIZE>
__device__ __forceinline__ int expert_tiles(const ExpertArg &ex) {
    int total = 0;
    for (int e0 = 0; e0 < ex.count; e0 += 64) {
        int row0, rows, tiles, sum;
        lane_expert<SIZE>(ex, e0 + ((int)threadIdx.x & 63), row0, rows, tiles, sum);
        total += __builtin_amdgcn_readlane(sum, 63);
    }
    return total;
}
// Which rows the `which`-th of them holds; false: there are not so many.
template <int SIZE>
__device__ __forceinline__ bool expert_tile(const ExpertArg &ex, int which, ExpertRows &p) {
    for (int e0 = 0; e0 < ex.count; e0 += 64) {
        int row0, rows, tiles, sum;
        lane_expert<SIZE>(ex, e0 + ((int)threadIdx.x & 63), row0, rows, tiles, sum);
        const uint64_t past = __ballot(sum > which);
        if (past) {
            const int lane = __builtin_ctzll(past);
            p = {e0 + lane, __builtin_amdgcn_readlane(row0, lane), __builtin_amdgcn_readlane(rows, lane),
                 which - (__builtin_amdgcn_readlane(sum, lane) - __builtin_amdgcn_readlane(tiles, lane))};
            return true;
        }
        which -= __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// The rows of expert e alone.
__device__ __forceinline__ ExpertRows expert_rows(const ExpertArg &ex, int e) {
    const int row0 = within(ex.offsets[e], ex.rows);
    return {e, row0, max(within(ex.offsets[e + 1], ex.rows) - row0, 0), 0};
}

// Tile n of tiles_j columns and all experts' rows for this workgroup, in an order that
// keeps neighbours on one XCD; false: none.
template <int SIZE>
__device__ __forceinline__ bool expert_place(const ExpertArg &ex, int tiles_j, ExpertRows &rows, int &tj) {
    const int total = expert_tiles<SIZE>(ex), id = (int)blockIdx.x;
    if (id >= total * tiles_j) return false;
    int ti;
    tile_at(xcd_run(id, total * tiles_j), total, tiles_j, ti, tj);
    return expert_tile<SIZE>(ex, ti, rows);
}

// A product's operands for those rows.
__device__ __forceinline__ LinearArgs of_expert(LinearArgs a, const ExpertRows &p) {
    a.x.codes += (int64_t)p.row0 * a.x.pitch;
    a.x.scale += p.row0;
    a.w.codes += (int64_t)p.expert * a.k * a.w.pitch;
    a.w.scale += (int64_t)p.expert * a.k;
    a.y = static_cast<uint16_t *>(a.y) + (int64_t)p.row0 * a.ldy;
    a.m = p.rows;
    return a;
}
template <int GS>
__device__ __forceinline__ GroupArg of_expert(GroupArg g, const ExpertRows &p, int k) {
    if constexpr (GS > 0) g.scale = static_cast<const uint8_t *>(g.scale) + (int64_t)p.expert * k * g.pitch * GS;
    return g;
}

}  // namespace qconv

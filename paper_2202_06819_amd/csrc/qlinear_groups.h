// The projection of 8-bit rows by 4-bit weights with a scale for each group of channels:
//   y[i][j] = xs[i] sum_g ws[j][g] sum_{c in g} x[i][c] w[j][c]
// A group's sum of codes runs on the int8 matrix cores, exact in int32 (weights widened
// to 16 times their value); it is scaled and added up in 32-bit floats.  Groups hold a
// multiple of 32 channels.  NG is how many slices of a 128-channel step a scale of its own
// may begin in: 1 (groups of a multiple of 128), 2 (of 64) or 4 (of 32).  GS: a scale's bytes.
#pragma once

#include "qlinear_device.h"
#include "qlinear_scales.h"

namespace qconv {

// --------------------------------------------------------------- few rows

// 16 / NG * RB rows against 16 output channels a wave, or, where there are few channels,
// a run of `share` waves that take blocks of four 128-channel steps in turn and whose sums
// meet in LDS.  Weights go straight from memory into registers, a block ahead; rows are
// staged in LDS, `chunk` steps of them at a time.  (Bound by reading the weights, 8192 x
// 4096 of one row in 5.3 us; rows and scales read from memory beside each step's weights
// add 2.2 and 1.3 us to that, loads that give nothing among them: hence LDS, and a block's
// scales in one or two loads.)
//
// A lane has 16 bytes of weights of one channel, 32 values: they belong to one group,
// whichever the groups' size, but the matrix instruction adds up what four lanes hold.
// So the rows of its other operand are NG copies of 16 / NG rows of x, each zero but for
// the lanes of its own slice: a product then gives the slices' sums apart, at no cost in
// reading weights.  A result's lane holds one channel, so that one scale serves its four
// results.  EVEN: groups of 128 / NG channels; others are served by NG 4, whose scales are
// loaded one by one.  GS 0: no groups but a scale for each row of weights, with the sum of
// all channels exact (for experts' 4-bit rows).
constexpr int kGroupWaves = 8, kBlock = 4;   // waves of a workgroup; steps of a block
constexpr int kZeros = kBlock * kStepBytes;  // LDS that lanes of other slices read
constexpr int few_pitch(int chunk) { return chunk * kStepBytes + 16; }
constexpr int groups_few_lds(int rows, int chunk, int rb, int ng) {
    const int x = rows * few_pitch(chunk), sums = kGroupWaves * rb * (64 / ng) * 16;
    return kZeros + (x > sums ? x : sums);
}
template <int GS>
struct GroupsSum {
    using type = f32x4;
};
template <>
struct GroupsSum<0> {
    using type = i32x4;
};
template <int GS, int NG, bool EVEN, int RB>
__device__ __forceinline__ void groups_few(LinearArgs a, GroupArg groups, bool bf16, int share, int chunk, int tile_j,
                                           int tile_i, uint8_t *smem) {
    static_assert(GS ? EVEN || NG == 4 : EVEN && NG == 1);
    using Sum = typename GroupsSum<GS>::type;
    constexpr int kRows = 16 / NG, kLanes = 64 / NG, kScales = kBlock * NG;   // a row's scales of a block
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = lane & 15, g = lane >> 4;
    const int turn = wave & (share - 1);
    const int ch0 = (tile_j * kGroupWaves + wave) / share * 16, row0 = tile_i * kRows * RB;
    const int rows = min(a.m - row0, kRows * RB);
    const __amdgpu_buffer_rsrc_t rx = range_of(a.x.codes + (int64_t)row0 * a.x.pitch,
                                               (int64_t)(rows - 1) * a.x.pitch + a.x.used);
    const __amdgpu_buffer_rsrc_t rw = range_of(a.w.codes + (int64_t)ch0 * a.w.pitch,
                                               (int64_t)(a.k - 1 - ch0) * a.w.pitch + a.w.used);
    const int channel = min(ch0 + r, a.k - 1);
    const int last = (a.c - 1) / 32, held = GS ? group_of(groups, last) + 1 : 0;   // the row's last 32 channels, its groups
    const uint8_t *const scales = static_cast<const uint8_t *>(groups.scale) + (int64_t)channel * groups.pitch * GS;
    const int slice = g * NG / 4;   // of the lane's weights, and of its results

    // Steps from `from` on of the rows of x into LDS, zeros past the row's end.  Waves are
    // dealt to the rows.  meanwhile(): what else to load while the first vectors are on
    // their way.
    const int per_row = rows >= 8 ? 1 : rows >= 4 ? 2 : rows >= 2 ? 4 : 8;
    const auto stage = [&](int from, int count, auto meanwhile) {
        constexpr int kDeep = 4;
        const int stride = per_row * 64, ends = count * 8;
        u32x4_t q[kDeep];
        const auto fetch = [&](int row, int v) {
#pragma unroll
            for (int e = 0; e < kDeep; ++e) {
                const int at = (from * 8 + v + e * stride) * 16;
                q[e] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                    rx, (int)(row < rows && at < a.x.used ? (uint32_t)row * (uint32_t)a.x.pitch + (uint32_t)at : kNowhere), 0, 0));
            }
        };
        const auto put = [&](int row, int v) {
#pragma unroll
            for (int e = 0; e < kDeep; ++e)
                if (row < rows && v + e * stride < ends)
                    *reinterpret_cast<u32x4_t *>(smem + kZeros + row * few_pitch(chunk) + (v + e * stride) * 16) = q[e];
        };
        int row = wave / per_row, v = (wave % per_row) * 64 + lane;
        fetch(row, v);
        __builtin_amdgcn_sched_barrier(0);
        meanwhile();
        __builtin_amdgcn_sched_barrier(0);
        put(row, v);
        while (row < rows) {
            v += kDeep * stride;
            if (v - lane >= ends) row += kGroupWaves / per_row, v = (wave % per_row) * 64 + lane;
            if (row >= rows) break;
            fetch(row, v);
            put(row, v);
        }
    };
    // (what lies past a row of weights meets zeros of x; past the last row nothing is read)
    u32x4_t w[kBlock];
    const uint32_t w_at = (uint32_t)r * (uint32_t)a.w.pitch + (uint32_t)g * 16;
    const auto load = [&](int s, u32x4_t &q) {
        q = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(s < a.steps ? w_at + (uint32_t)s * 64u : kNowhere), 0, 0));
    };
    // The scales of a block's slices, as they lie in memory: all of them, or (one by one)
    // the lane's own.
    struct Scales {
        uint32_t q[EVEN ? GS ? kScales * GS / 4 : 1 : kBlock];
    };
    const auto load_scales = [&](int block, Scales &q) {
        if constexpr (GS == 0) {
            q.q[0] = 0;
        } else if constexpr (EVEN) {
            const int at = block * kScales;
            if (at + kScales <= held) {
                __builtin_memcpy(q.q, scales + at * GS, kScales * GS);
            } else {   // the row's end: one by one, all of them on their way at once
                uint32_t v[kScales];
#pragma unroll
                for (int n = 0; n < kScales; ++n) {
                    const int from = min(at + n, held - 1);
                    v[n] = GS == 4 ? reinterpret_cast<const uint32_t *>(scales)[from] : reinterpret_cast<const uint16_t *>(scales)[from];
                }
#pragma unroll
                for (int n = 0; n < kScales * GS / 4; ++n) q.q[n] = 0;
#pragma unroll
                for (int n = 0; n < kScales; ++n)
                    q.q[n * GS / 4] |= (at + n < held ? v[n] : 0u) << (GS == 2 ? n % 2 * 16 : 0);
            }
        } else {
#pragma unroll
            for (int e = 0; e < kBlock; ++e) {
                const int unit = (block * kBlock + e) * 4 + g;
                const uint32_t v = load_scale<GS>(groups, (int64_t)channel * groups.pitch + group_of(groups, min(unit, last)));
                q.q[e] = unit <= last ? v : 0u;
            }
        }
    };
    const auto scale_of = [&](const Scales &q, int e) {   // of the lane's slice in step e
        if constexpr (GS == 0) return 0.0f;
        if constexpr (!EVEN) return scale_value<GS>(groups, q.q[e]);
        // (by masks: a choice between two of an array's places would put it into memory)
        const uint32_t odd = slice & 1 ? ~0u : 0u, high = slice & 2 ? ~0u : 0u;
        const auto either = [](uint32_t mask, uint32_t yes, uint32_t no) { return (yes & mask) | (no & ~mask); };
        uint32_t v;
        if constexpr (GS == 4) {
            if constexpr (NG == 1) v = q.q[e];
            else if constexpr (NG == 2) v = either(odd, q.q[2 * e + 1], q.q[2 * e]);
            else v = either(high, either(odd, q.q[4 * e + 3], q.q[4 * e + 2]), either(odd, q.q[4 * e + 1], q.q[4 * e]));
        } else {
            if constexpr (NG == 1) v = q.q[e / 2] >> (e % 2 * 16);
            else if constexpr (NG == 2) v = q.q[e] >> (odd & 16);
            else v = either(high, q.q[2 * e + 1], q.q[2 * e]) >> (odd & 16);
            v &= 0xffffu;
        }
        return scale_value<GS>(groups, v);
    };
    // Lanes of x's operand: their row in LDS, or zeros.
    uint32_t x_at[RB], moves[RB];   // moves: all ones where the address moves on with the block
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int row = b * kRows + r % kRows;
        const bool mine = r / kRows == slice && row < rows;
        moves[b] = mine ? ~0u : 0u;
        x_at[b] = mine ? (uint32_t)(kZeros + row * few_pitch(chunk) + g * 32) : 0u;
    }
    Sum acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b] = Sum{0, 0, 0, 0};
    const auto multiply = [&](const u32x4_t &q, float scale, const uint8_t *const (&from)[RB], int e) {
        i32x4 ww[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint2 p = widen8(q[2 * h]), t = widen8(q[2 * h + 1]);
            ww[h] = i32x4{(int)p.x, (int)p.y, (int)t.x, (int)t.y};
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            i32x4 t{0, 0, 0, 0};
            if constexpr (GS == 0) t = acc[b];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                t = MmaI8::mma(*reinterpret_cast<const i32x4 *>(from[b] + e * kStepBytes + h * 16), ww[h], t);
            if constexpr (GS == 0) {
                acc[b] = t;
            } else {
#pragma unroll
                for (int n = 0; n < 4; ++n) acc[b][n] = __builtin_fmaf((float)t[n], scale, acc[b][n]);
                asm volatile("" : "+v"(acc[b]));   // here, not where the sum is next used
            }
        }
    };

    if ((int)threadIdx.x < kZeros / 16) reinterpret_cast<u32x4_t *>(smem)[threadIdx.x] = u32x4_t{0, 0, 0, 0};
    const int blocks = (a.steps + kBlock - 1) / kBlock, turns = (blocks + share - 1) / share;   // a wave's
    const int chunk_turns = chunk / (kBlock * share);
    Scales scale{};
    stage(0, min(chunk, turns * share * kBlock), [&] {
        if (turn < blocks) load_scales(turn, scale);
#pragma unroll
        for (int e = 0; e < kBlock; ++e) load(turn * kBlock + e, w[e]);
    });
    // (LDS alone is waited for: the weights stay on their way)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const __amdgpu_buffer_rsrc_t rxs = range_of(a.x.scale + row0, (int64_t)rows * 4);
    float xs[RB][4];   // of the lane's results, wanted at the end
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            xs[b][e] = __builtin_bit_cast(float, (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rxs, (b * kRows + g * 4 + e) * 4, 0, 0));
    for (int n = 0, left = chunk_turns; n < turns; ++n, --left) {
        if (left == 0) {   // the next chunk
            left = chunk_turns;
            __syncthreads();
            stage(n * share * kBlock, min(chunk, (turns - n) * share * kBlock), [] {});
            __syncthreads();
        }
        const uint32_t off = (uint32_t)((chunk_turns - left) * share + turn) * (kBlock * kStepBytes);
        const uint8_t *from[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) from[b] = smem + x_at[b] + (off & moves[b]);
        const int next = (n + 1) * share + turn;
        Scales then{};
        if (next < blocks) load_scales(next, then);
#pragma unroll
        for (int e = 0; e < kBlock; ++e) {
            multiply(w[e], scale_of(scale, e), from, e);
            __builtin_amdgcn_sched_barrier(0);
            load(next * kBlock + e, w[e]);
            __builtin_amdgcn_sched_barrier(0);
        }
        scale = then;
    }
    // the slices' sums of a row and channel meet: lanes 16 and 32 apart
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (NG == 4) acc[b][e] += __shfl_xor(acc[b][e], 16);
            if constexpr (NG >= 2) acc[b][e] += __shfl_xor(acc[b][e], 32);
        }
    if (share > 1) {
        auto part = reinterpret_cast<Sum(*)[RB][kLanes]>(smem + kZeros);
        __syncthreads();   // everyone is done with the rows
        if (lane < kLanes)
#pragma unroll
            for (int b = 0; b < RB; ++b) part[wave][b][lane] = acc[b];
        __syncthreads();
        if (turn) return;
        if (lane < kLanes)
            for (int n = 1; n < share; ++n)
#pragma unroll
                for (int b = 0; b < RB; ++b) acc[b] += part[wave + n][b][lane];
    }
    // four rows of one channel a lane
    const int ch = ch0 + r;
    if (lane >= kLanes || ch >= a.k) return;
    float ws = 1.0f;
    if constexpr (GS == 0) ws = a.w.scale[ch];
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = row0 + b * kRows + g * 4 + e;
            if (row >= a.m) break;
            float y = (float)acc[b][e] * (xs[b][e] * 0.0625f);
            if constexpr (GS == 0) y *= ws;
            const int64_t to = (int64_t)row * a.ldy + ch;
            if (bf16) static_cast<BF16::elem *>(a.y)[to] = (BF16::elem)y;
            else static_cast<F16::elem *>(a.y)[to] = (F16::elem)y;
        }
}

// --------------------------------------------------------------- many rows

// The products of a slice: 64 channels deep, or 32.
template <int NG>
struct GroupsMma : MmaI8 {};
template <>
struct GroupsMma<4> {
    using frag = long;
    static __device__ __forceinline__ i32x4 mma(frag a, frag b, i32x4 c) {
        return __builtin_amdgcn_mfma_i32_16x16x32_i8(a, b, c, 0, 0, 0);
    }
};

// A step's products for FJ x FI fragments, each slice's scaled and added to d.  While two
// fragments are multiplied the two before them are converted, scaled and added, so that
// the vector instructions (two a result and slice) run beside the matrix cores; the units
// are fenced off from each other, or the scheduler brings forth all whole numbers first
// and has no registers for them.  `scales`: NG x TJ floats.
template <int NG, int TJ, int FJ, int FI>
__device__ __forceinline__ void groups_step(const uint8_t *lj, const uint8_t *li, const float *scales, int jrow0, int irow0,
                                            int lane, f32x4 (&d)[FJ][FI]) {
    static_assert(FJ == 4, "a lane holds 16 consecutive rows of the product");
    constexpr int kHalves = NG == 1 ? 2 : 1;   // products of a slice
    typedef typename GroupsMma<NG>::frag frag;
    const int r = lane & 15, g = lane >> 4;
    // the lane's part of row `row`, product h of a slice
    const auto read = [&](const uint8_t *l, int row, int slice, int h) {
        if constexpr (NG < 4)
            return *reinterpret_cast<const frag *>(l + row * kStepBytes + ((((slice + h) * 4 + g) ^ slot(row)) << 4));
        else   // 32 channels: eight a lane
            return *reinterpret_cast<const frag *>(l + row * kStepBytes + (((slice * 2 + (g >> 1)) ^ slot(row)) << 4) + (g & 1) * 8);
    };
#pragma unroll
    for (int slice = 0; slice < NG; ++slice) {
        frag w[kHalves][FJ], x[2][kHalves];
        f32x4 ws[FJ];
#pragma unroll
        for (int j = 0; j < FJ; ++j) ws[j] = *reinterpret_cast<const f32x4 *>(scales + slice * TJ + jrow0 + g * 16 + 4 * j);
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int j = 0; j < FJ; ++j) w[h][j] = read(lj, jrow0 + j_row(j, r), slice, h);
#pragma unroll
        for (int h = 0; h < kHalves; ++h) x[0][h] = read(li, irow0 + r, slice, h);
        i32x4 t[2][2];
        // unit u: fragments 2 (u % 2) and the one after it of row fragment u / 2
        const auto fold = [&](int u) {
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int j = u % 2 * 2 + n;
#pragma unroll
                for (int e = 0; e < 4; ++e) d[j][u / 2][e] = __builtin_fmaf((float)t[u & 1][n][e], ws[j][e], d[j][u / 2][e]);
                asm volatile("" : "+v"(d[j][u / 2]));   // here, not where the sum is next used
            }
        };
#pragma unroll
        for (int u = 0; u < 2 * FI; ++u) {
            const int i = u / 2;
            if (u % 2 == 0 && i + 1 < FI)   // (a fragment ahead)
#pragma unroll
                for (int h = 0; h < kHalves; ++h) x[~i & 1][h] = read(li, irow0 + (i + 1) * 16 + r, slice, h);
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    t[u & 1][n] = GroupsMma<NG>::mma(w[h][u % 2 * 2 + n], x[i & 1][h], h ? t[u & 1][n] : i32x4{0, 0, 0, 0});
            if (u) fold(u - 1);
#pragma unroll
            for (int n = 0; n < 2 * kHalves; ++n) {
                __builtin_amdgcn_sched_group_barrier(8, 1, 0);                 // a matrix instruction,
                __builtin_amdgcn_sched_group_barrier(2, 16 / (2 * kHalves), 0);   // its share of vector instructions
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        fold(2 * FI - 1);
    }
}

// The tile product of whole rows' scales (qlinear_fwd.h: TJ output channels by TI rows,
// two LDS buffers, KS groups of waves), with a step's scales beside its operands.
constexpr int groups_tile_lds(int tj, int ti, int ks, int ng) { return ks * 2 * ((tj + ti) * kStepBytes + ng * tj * 4); }
template <int GS, int NG, int TJ, int TI, int WJ, int WI, int KS>
__device__ __forceinline__ void groups_tile(LinearArgs a, GroupArg groups, bool bf16, int tj, int ti,
                                            uint8_t *smem) {
    constexpr int FJ = 4, FI = TI / (16 * WI), kThreads = WJ * WI * 64, kRowsBytes = (TJ + TI) * kStepBytes;
    constexpr int kBuffer = kRowsBytes + NG * TJ * 4;
    static_assert(TJ == WJ * 64);
    static_assert(KS == 1 || FI == 1);
    const int group = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kThreads), thread = (int)threadIdx.x % kThreads;
    const int wave = __builtin_amdgcn_readfirstlane(thread >> 6), lane = threadIdx.x & 63;
    const int i0 = ti * TI, j0 = tj * TJ;
    const u32x4_t rx = range_words(a.x.codes + (int64_t)i0 * a.x.pitch, (int64_t)(a.m - 1 - i0) * a.x.pitch + a.x.used);
    const __amdgpu_buffer_rsrc_t rw = range_of(a.w.codes + (int64_t)j0 * a.w.pitch,
                                               (int64_t)(a.k - 1 - j0) * a.w.pitch + a.w.used);
    const int last = (a.c - 1) / 32;
    const __amdgpu_buffer_rsrc_t rs = range_of(static_cast<const uint8_t *>(groups.scale) + (int64_t)j0 * groups.pitch * GS,
                                               ((int64_t)(a.k - 1 - j0) * groups.pitch + group_of(groups, last) + 1) * GS);
    constexpr int kUnits = TJ * 4 / kThreads, kScales = (NG * TJ + kThreads - 1) / kThreads;
    u32x4_t held[kUnits];
    uint32_t scale[kScales];
    const auto fetch = [&](int s, uint8_t *buf) {
        copy_rows<TI, kThreads>(buf + TJ * kStepBytes, rx, (uint32_t)a.x.pitch, s * 128, a.x.used, wave, lane);
#pragma unroll
        for (int n = 0; n < kUnits; ++n) {
            const int unit = n * kThreads + thread, row = unit >> 2, at = s * 64 + (unit & 3) * 16;
            held[n] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                rw, (int)(at < a.w.used ? (uint32_t)row * (uint32_t)a.w.pitch + (uint32_t)at : kNowhere), 0, 0));
        }
#pragma unroll
        for (int n = 0; n < kScales; ++n) {
            const int at = n * kThreads + thread, row = at % TJ, unit = s * 4 + at / TJ * (4 / NG);
            const int to = (int)(at < NG * TJ && unit <= last
                                     ? ((uint32_t)row * (uint32_t)groups.pitch + (uint32_t)group_of(groups, unit)) * GS : kNowhere);
            if constexpr (GS == 4) scale[n] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, to, 0, 0);
            else scale[n] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, to, 0, 0);
        }
    };
    const auto settle = [&](uint8_t *buf) {
#pragma unroll
        for (int n = 0; n < kUnits; ++n) {
            const int unit = n * kThreads + thread, row = unit >> 2, v = (unit & 3) * 2;
            const uint2 p = widen8(held[n][0]), q = widen8(held[n][1]);
            const uint2 s = widen8(held[n][2]), t = widen8(held[n][3]);
            *reinterpret_cast<uint4 *>(buf + row * kStepBytes + ((v ^ slot(row)) << 4)) = uint4{p.x, p.y, q.x, q.y};
            *reinterpret_cast<uint4 *>(buf + row * kStepBytes + (((v + 1) ^ slot(row)) << 4)) = uint4{s.x, s.y, t.x, t.y};
        }
#pragma unroll
        for (int n = 0; n < kScales; ++n)
            if (n * kThreads + thread < NG * TJ)
                reinterpret_cast<float *>(buf + kRowsBytes)[n * kThreads + thread] = scale_value<GS>(groups, scale[n]);
        copies_done();
    };
    const int jrow0 = (wave / WI) * 64, irow0 = (wave % WI) * FI * 16;
    f32x4 d[FJ][FI];
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int i = 0; i < FI; ++i) d[j][i] = f32x4{0, 0, 0, 0};
    // (a group's step past the last one is all zeros)
    uint8_t *const own = smem + group * 2 * kBuffer;
    fetch(group, own);
    settle(own);
    __syncthreads();
    int buf = 0;
    for (int s = 0; s < a.steps; s += KS) {
        uint8_t *cur = own + buf * kBuffer, *next = own + (buf ^ 1) * kBuffer;
        if (s + KS < a.steps) fetch(s + KS + group, next);
        groups_step<NG, TJ, FJ, FI>(cur, cur + TJ * kStepBytes, reinterpret_cast<const float *>(cur + kRowsBytes), jrow0,
                                    irow0, lane, d);
        if (s + KS < a.steps) settle(next);
        __syncthreads();
        buf ^= 1;
    }
    // lane (r, g): channels ch .. ch + 15 of one row of each fragment i
    const int r = lane & 15, g = lane >> 4;
    const int ch = j0 + jrow0 + g * 16;
    if constexpr (KS > 1) {
        auto sums = [&](int from, int j) {
            return reinterpret_cast<f32x4 *>(smem + from * 2 * kBuffer) + (wave * FJ + j) * 64 + lane;
        };
        if (group)
#pragma unroll
            for (int j = 0; j < FJ; ++j) *sums(group, j) = d[j][0];
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int from = 1; from < KS; ++from)
#pragma unroll
            for (int j = 0; j < FJ; ++j) d[j][0] += *sums(from, j);
    }
    const auto give = [&](auto type) {
        using T = decltype(type);
#pragma unroll
        for (int i = 0; i < FI; ++i) {
            const int row = i0 + irow0 + i * 16 + r;
            if (row >= a.m) continue;
            const float xs = a.x.scale[row] * 0.0625f;
            typename T::elem *out = static_cast<typename T::elem *>(a.y) + (int64_t)row * a.ldy + ch;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 lo = d[2 * h][i] * xs, hi = d[2 * h + 1][i] * xs;
                if (ch + 8 * h + 8 <= a.k) {
                    const u32x4_t w{pack2<T>(lo[0], lo[1]), pack2<T>(lo[2], lo[3]), pack2<T>(hi[0], hi[1]), pack2<T>(hi[2], hi[3])};
                    __builtin_memcpy(out + 8 * h, &w, 16);   // of any alignment
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (ch + 8 * h + e < a.k) out[8 * h + e] = (typename T::elem)(e < 4 ? lo[e & 3] : hi[e & 3]);
                }
            }
        }
    };
    if (bf16) give(BF16{});
    else give(F16{});
}

}  // namespace qconv

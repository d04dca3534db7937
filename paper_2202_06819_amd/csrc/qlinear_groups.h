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

// Up to 16 / NG * RB rows against 16 FJ output channels a workgroup, eight waves taking
// the 128-channel steps in turn, as in the few-row kernel of whole rows' scales.  A lane
// has 16 bytes of weights of one channel, 32 values: they belong to one group, whichever
// the groups' size, but the matrix instruction adds up what four lanes hold.  So the
// rows of its other operand are NG copies of 16 / NG rows of x, each zero but for the
// lanes of its own slice: a product then gives the slices' sums apart, at no cost in
// reading weights, which bounds this kernel.  A result's lane holds one channel, so that
// one scale serves its four results.
constexpr int kGroupWaves = 8;
constexpr int groups_few_lds(int fj, int rb, int ng) { return kGroupWaves * fj * rb * (64 / ng) * 16; }
template <int GS, int NG, int FJ, int RB>
__device__ __forceinline__ void groups_few(const LinearArgs &a, const GroupArg &groups, bool bf16, int tile_j, int tile_i,
                                           uint8_t *smem) {
    constexpr int kRows = 16 / NG, kFlight = 4, kLanes = 64 / NG;
    auto part = reinterpret_cast<f32x4(*)[FJ * RB][kLanes]>(smem);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = lane & 15, g = lane >> 4;
    const int ch0 = tile_j * 16 * FJ, row0 = tile_i * kRows * RB;
    const __amdgpu_buffer_rsrc_t rx = range_of(a.x.codes + (int64_t)row0 * a.x.pitch,
                                               (int64_t)(a.m - 1 - row0) * a.x.pitch + a.x.used);
    const __amdgpu_buffer_rsrc_t rw = range_of(a.w.codes + (int64_t)ch0 * a.w.pitch,
                                               (int64_t)(a.k - 1 - ch0) * a.w.pitch + a.w.used);
    const int last = (a.c - 1) / 32;   // the row's last 32 channels
    const __amdgpu_buffer_rsrc_t rs = range_of(static_cast<const uint8_t *>(groups.scale) + (int64_t)ch0 * groups.pitch * GS,
                                               ((int64_t)(a.k - 1 - ch0) * groups.pitch + group_of(groups, last) + 1) * GS);
    const int slice = g * NG / 4;             // of the lane's weights, and of its results
    const bool mine = r / kRows == slice;     // the lane's row of x is its slice's copy
    struct Step {
        u32x4_t w[FJ], x[RB][2];
        uint32_t scale[FJ];
    };
    const auto load = [&](int s, Step &q) {
        const int at = s * 64 + g * 16;
        const bool in = at < a.w.used;
        const int unit = s * 4 + slice * (4 / NG);
        const uint32_t group = (uint32_t)group_of(groups, min(unit, last));
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            q.w[j] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                rw, (int)(in ? (uint32_t)(j * 16 + r) * (uint32_t)a.w.pitch + (uint32_t)at : kNowhere), 0, 0));
            const int to = (int)(unit <= last ? ((uint32_t)(j * 16 + r) * (uint32_t)groups.pitch + group) * GS : kNowhere);
            if constexpr (GS == 4) q.scale[j] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, to, 0, 0);
            else q.scale[j] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, to, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int from = s * 128 + g * 32 + h * 16;
                q.x[b][h] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                    rx, (int)(mine && from < a.x.used
                                  ? (uint32_t)(b * kRows + r % kRows) * (uint32_t)a.x.pitch + (uint32_t)from : kNowhere), 0, 0));
            }
    };
    f32x4 acc[FJ][RB];
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[j][b] = f32x4{0, 0, 0, 0};
    const auto multiply = [&](const Step &q) {
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            i32x4 w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint2 p = widen8(q.w[j][2 * h]), t = widen8(q.w[j][2 * h + 1]);
                w[h] = i32x4{(int)p.x, (int)p.y, (int)t.x, (int)t.y};
            }
            const float scale = scale_value<GS>(groups, q.scale[j]);
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                i32x4 t{0, 0, 0, 0};
                t = MmaI8::mma(__builtin_bit_cast(i32x4, q.x[b][0]), w[0], t);
                t = MmaI8::mma(__builtin_bit_cast(i32x4, q.x[b][1]), w[1], t);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][b][e] = __builtin_fmaf((float)t[e], scale, acc[j][b][e]);
            }
        }
    };
    Step q[kFlight];
#pragma unroll
    for (int e = 0; e < kFlight; ++e)
        if (wave + e * kGroupWaves < a.steps) load(wave + e * kGroupWaves, q[e]);
    for (int s = wave; s < a.steps; s += kFlight * kGroupWaves) {
#pragma unroll
        for (int e = 0; e < kFlight; ++e) {
            if (s + e * kGroupWaves < a.steps) multiply(q[e]);
            if (s + (kFlight + e) * kGroupWaves < a.steps) load(s + (kFlight + e) * kGroupWaves, q[e]);
        }
    }
    // the slices' sums of a row and channel meet: lanes 16 and 32 apart
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int b = 0; b < RB; ++b) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (NG == 4) acc[j][b][e] += __shfl_xor(acc[j][b][e], 16);
                if (NG >= 2) acc[j][b][e] += __shfl_xor(acc[j][b][e], 32);
            }
            if (lane < kLanes) part[wave][j * RB + b][lane] = acc[j][b];
        }
    __syncthreads();
    // four rows of one channel a thread
    for (int o = (int)threadIdx.x; o < FJ * RB * kLanes; o += kGroupWaves * 64) {
        const int f = o / kLanes, l = o % kLanes, j = f / RB, b = f % RB;
        f32x4 t = part[0][f][l];
#pragma unroll
        for (int w = 1; w < kGroupWaves; ++w) t += part[w][f][l];
        const int ch = ch0 + j * 16 + (l & 15), row = row0 + b * kRows + (l >> 4) * 4;
        if (ch >= a.k) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (row + e >= a.m) break;
            const float y = t[e] * (a.x.scale[row + e] * 0.0625f);
            const int64_t to = (int64_t)(row + e) * a.ldy + ch;
            if (bf16) static_cast<BF16::elem *>(a.y)[to] = (BF16::elem)y;
            else static_cast<F16::elem *>(a.y)[to] = (F16::elem)y;
        }
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
        frag w[kHalves][FJ], x[kHalves];
        f32x4 ws[FJ];
#pragma unroll
        for (int j = 0; j < FJ; ++j) ws[j] = *reinterpret_cast<const f32x4 *>(scales + slice * TJ + jrow0 + g * 16 + 4 * j);
#pragma unroll
        for (int h = 0; h < kHalves; ++h)
#pragma unroll
            for (int j = 0; j < FJ; ++j) w[h][j] = read(lj, jrow0 + j_row(j, r), slice, h);
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
            if (u % 2 == 0)
#pragma unroll
                for (int h = 0; h < kHalves; ++h) x[h] = read(li, irow0 + u / 2 * 16 + r, slice, h);
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    t[u & 1][n] = GroupsMma<NG>::mma(w[h][u % 2 * 2 + n], x[h], h ? t[u & 1][n] : i32x4{0, 0, 0, 0});
            if (u) fold(u - 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        fold(2 * FI - 1);
    }
}

// The tile product of whole rows' scales (qlinear_fwd.h: TJ output channels by TI rows,
// two LDS buffers, KS groups of waves), with a step's scales beside its operands.
constexpr int groups_tile_lds(int tj, int ti, int ks, int ng) { return ks * 2 * ((tj + ti) * kStepBytes + ng * tj * 4); }
template <int GS, int NG, int TJ, int TI, int WJ, int WI, int KS>
__device__ __forceinline__ void groups_tile(const LinearArgs &a, const GroupArg &groups, bool bf16, int tj, int ti,
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

// The shared projection on 8-bit rows with low-rank adapters:
//   y[i][j] = xs[i] ws[j] sum_c x[i][c] w[j][c] + alpha_a sum_r u[i][r] B_a[j][r]
//   u[i][r] = xs[i] sum_c x[i][c] A_a[r][c],   a = the adapter of row i (or none)
// The first sum runs on the int8 matrix cores, exact in int32 (the host bounds
// it); 4-bit weights are widened to 16 times their value.  The adapters' first
// products (adapter_rows) come from their own launch as partial sums; their
// second ones are added to the float result before its only rounding.
#pragma once

#include "qlinear_device.h"

namespace qconv {

// ---------------------------------------------------------- adapters, part one

// 8 codes of a row as eight 16-bit floats (exact).
template <class T>
__device__ __forceinline__ typename T::v8 codes_to_v8(uint2 q) {
    u32x4_t out;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w = (h ? q.y : q.x) ^ 0x80808080u;   // code + 128, unsigned bytes
        out[2 * h] = pack2<T>((float)(w & 255u) - 128.0f, (float)((w >> 8) & 255u) - 128.0f);
        out[2 * h + 1] = pack2<T>((float)((w >> 16) & 255u) - 128.0f, (float)(w >> 24) - 128.0f);
    }
    return __builtin_bit_cast(typename T::v8, out);
}

// The lowest row of `left` (a mask of 16 rows) gives the next adapter; its rows
// leave the mask.  `id` is the lane's row's adapter (row = lane & 15).
__device__ __forceinline__ int next_adapter(uint32_t &left, int id) {
    const int a = __builtin_amdgcn_readlane(id, __builtin_ctz(left));
    left &= ~(uint32_t)__ballot(id == a);
    return a;
}

// Partial sums of u over one of `splits` runs of channels, without the row
// scale: sum of codes times A for the row's own adapter.  A workgroup takes 16
// rows and a run; its waves take the run's 32-channel steps in turn, and for
// each adapter that the rows name, multiply its A (RF fragments of 16 ranks) by
// all of them and keep the rows that asked for it.
template <class T, int RF>
__global__ void __launch_bounds__(512) adapter_rows(LinearArgs a, int steps_per_split) {
    constexpr int kWaves = 8;
    __shared__ f32x4 part[kWaves][RF][64];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = lane & 15, g = lane >> 4;
    const int row0 = (int)blockIdx.x * 16, row = row0 + r;
    const int all = (a.c + 31) / 32;
    const int begin = (int)blockIdx.y * steps_per_split, end = min(begin + steps_per_split, all);
    int id = row < a.m ? a.ad.row[row] : -1;
    if (id < 0 || id >= a.ad.count) id = -1;
    f32x4 sum[RF];
#pragma unroll
    for (int f = 0; f < RF; ++f) sum[f] = f32x4{0, 0, 0, 0};
    const uint8_t *x = a.x.codes + (int64_t)min(row, a.m - 1) * a.x.pitch;
    uint32_t left = (uint32_t)__ballot(id >= 0) & 0xffffu;
    while (left) {
        const int ad = next_adapter(left, id);
        const typename T::elem *A = static_cast<const typename T::elem *>(a.ad.a) + (int64_t)ad * a.ad.rank * a.c;
        f32x4 d[RF];
#pragma unroll
        for (int f = 0; f < RF; ++f) d[f] = f32x4{0, 0, 0, 0};
        for (int s = begin + wave; s < end; s += kWaves) {
            const int at = s * 32 + g * 8;      // c is a multiple of 8: a vector is whole or absent
            const bool in = at < a.c;
            const uint2 q = in ? *reinterpret_cast<const uint2 *>(x + at) : uint2{0u, 0u};
            const typename T::v8 b = codes_to_v8<T>(q);
#pragma unroll
            for (int f = 0; f < RF; ++f) {
                u32x4_t w{0, 0, 0, 0};
                if (in && f * 16 + r < a.ad.rank)
                    w = *reinterpret_cast<const u32x4_t *>(A + (int64_t)(f * 16 + r) * a.c + at);
                d[f] = T::mma(__builtin_bit_cast(typename T::v8, w), b, d[f]);
            }
        }
        if (id == ad)
#pragma unroll
            for (int f = 0; f < RF; ++f) sum[f] = d[f];
    }
#pragma unroll
    for (int f = 0; f < RF; ++f) part[wave][f][lane] = sum[f];
    __syncthreads();
    // lane (r, g) of fragment f holds ranks 16 f + 4 g + 0..3 of row r
    for (int f = wave; f < RF; f += kWaves) {
        f32x4 t = part[0][f][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) t += part[w][f][lane];
        const int rank = f * 16 + g * 4;
        if (row < a.m && rank < a.ad.rank)
            *reinterpret_cast<f32x4 *>(a.ad.u + ((int64_t)blockIdx.y * a.m + row) * a.ad.rank + rank) = t;
    }
}

// ---------------------------------------------------------- adapters, part two

// Eight ranks (32 rc + 8 g ..) of u of the lane's row, summed over the splits.
__device__ __forceinline__ void load_u(const LinearArgs &a, int row, int rank, float (&u)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = 0.0f;
    if (row >= a.m || rank >= a.ad.rank) return;
    const float *p = a.ad.u + (int64_t)row * a.ad.rank + rank;
    for (int s = 0; s < a.ad.splits; ++s, p += (int64_t)a.m * a.ad.rank) {
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(p), hi = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] += lo[i], u[i + 4] += hi[i];
    }
}

// A power of two that brings the row's largest |u| (over all its ranks, held by
// the four lanes of the row) into [1, 2), and its inverse: u is rounded to 16
// bits after it, so the rounding is relative to the row and no f16 overflows.
__device__ __forceinline__ void row_factor(uint32_t m, float &down, float &up) {
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    const int e = min(max((int)(m >> 23), 1), 253);
    down = __builtin_bit_cast(float, (uint32_t)(254 - e) << 23);
    up = __builtin_bit_cast(float, (uint32_t)e << 23);
}

constexpr int kMaxRankSteps = 4;   // ranks up to 128, 32 a product

// Adds the adapters' second products for 16 rows (the wave's lanes' row is
// row0 + (lane & 15)) to FJ fragments of results in `d`: d[f] += alpha up
// (u B^T).  row_of(f) is the output channel of lane row r of fragment f.  Every
// `stride`-th adapter from `first` on that the rows name is taken.
template <class T, int FJ, class RowOf>
__device__ __forceinline__ void add_adapters(const LinearArgs &a, int row0, int lane, int first, int stride,
                                             RowOf row_of, f32x4 (&d)[FJ]) {
    const int r = lane & 15, g = lane >> 4, row = row0 + r;
    int id = row < a.m ? a.ad.row[row] : -1;
    if (id < 0 || id >= a.ad.count) id = -1;
    uint32_t left = (uint32_t)__ballot(id >= 0) & 0xffffu;
    if (!left) return;
    const int steps = (a.ad.rank + 31) / 32;
    float u[kMaxRankSteps][8];
    uint32_t m = 0;
#pragma unroll
    for (int s = 0; s < kMaxRankSteps; ++s)
        if (s < steps) {
            load_u(a, row, s * 32 + g * 8, u[s]);
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, u[s][i]) & 0x7fffffffu);
        }
    float down, up;
    row_factor(m, down, up);
    u32x4_t ub[kMaxRankSteps];
#pragma unroll
    for (int s = 0; s < kMaxRankSteps; ++s)
        if (s < steps) {
#pragma unroll
            for (int i = 0; i < 4; ++i) ub[s][i] = pack2<T>(u[s][2 * i] * down, u[s][2 * i + 1] * down);
        }
    const float scale = up * (row < a.m ? a.x.scale[row] : 0.0f);
    int n = 0;
    while (left) {
        const int ad = next_adapter(left, id);
        if (n++ % stride != first) continue;
        const typename T::elem *B = static_cast<const typename T::elem *>(a.ad.b) + (int64_t)ad * a.k * a.ad.rank;
        const float f = id == ad ? scale * a.ad.alpha[ad] : 0.0f;
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            const int ch = row_of(j);
            f32x4 t{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < kMaxRankSteps; ++s)
                if (s < steps) {
                    const int rank = s * 32 + g * 8;
                    u32x4_t w{0, 0, 0, 0};
                    if (ch < a.k && rank < a.ad.rank)
                        w = *reinterpret_cast<const u32x4_t *>(B + (int64_t)ch * a.ad.rank + rank);
                    t = T::mma(__builtin_bit_cast(typename T::v8, w), __builtin_bit_cast(typename T::v8, ub[s]), t);
                }
            if (id == ad)   // (not by a zero factor: another adapter's product may not be finite)
#pragma unroll
                for (int i = 0; i < 4; ++i) d[j][i] += f * t[i];
        }
    }
}

// --------------------------------------------------------------- few rows

// Up to 16 FI rows against 16 output channels a workgroup: eight waves take
// the 128-channel steps in turn, weights and rows straight from memory into
// registers (each weight is used once, so LDS would only be a detour), and
// their sums meet in LDS.  Bound by reading the weights.
template <class T, int WB, int FI, bool AD>
__global__ void __launch_bounds__(512) linear_few(LinearArgs a) {
    constexpr int kWaves = 8, kParts = kWaves / FI;
    __shared__ i32x4 part[kWaves][FI][64];
    __shared__ f32x4 extra[AD ? kParts : 1][FI][64];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = lane & 15, g = lane >> 4;
    const int ch0 = (int)blockIdx.x * 16;
    const __amdgpu_buffer_rsrc_t rx = range_of(a.x.codes, (int64_t)(a.m - 1) * a.x.pitch + a.x.used);
    const uint8_t *w0 = a.w.codes + (int64_t)ch0 * a.w.pitch;
    const __amdgpu_buffer_rsrc_t rw = range_of(w0, (int64_t)(a.k - 1 - ch0) * a.w.pitch + a.w.used);
    i32x4 acc[FI];
#pragma unroll
    for (int f = 0; f < FI; ++f) acc[f] = i32x4{0, 0, 0, 0};
    const uint32_t wrow = (uint32_t)r * (uint32_t)a.w.pitch;
    auto load_x = [&](int f, int at) {
        const int row = f * 16 + r;
        return __builtin_amdgcn_raw_buffer_load_b128(
            rx, (int)(at < a.x.used && row < a.m ? (uint32_t)row * (uint32_t)a.x.pitch + (uint32_t)at : kNowhere), 0, 0);
    };
    auto load_w = [&](int at) {
        return __builtin_amdgcn_raw_buffer_load_b128(rw, (int)(at < a.w.used ? wrow + (uint32_t)at : kNowhere), 0, 0);
    };
    for (int s = wave; s < a.steps; s += kWaves) {
        if constexpr (WB == 8) {
            // the depth's order is free as long as both operands share it
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = s * 128 + h * 64 + g * 16;
                const auto w = load_w(at);
#pragma unroll
                for (int f = 0; f < FI; ++f)
                    acc[f] = MmaI8::mma(__builtin_bit_cast(i32x4, w), __builtin_bit_cast(i32x4, load_x(f, at)), acc[f]);
            }
        } else {
            const auto w = load_w(s * 64 + g * 16);   // 32 channels
            i32x4 lo, hi;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint2 p = widen8(w[i]), q = widen8(w[i + 2]);
                lo[2 * i] = (int)p.x, lo[2 * i + 1] = (int)p.y;
                hi[2 * i] = (int)q.x, hi[2 * i + 1] = (int)q.y;
            }
            const int at = s * 128 + g * 32;
#pragma unroll
            for (int f = 0; f < FI; ++f) {
                acc[f] = MmaI8::mma(lo, __builtin_bit_cast(i32x4, load_x(f, at)), acc[f]);
                acc[f] = MmaI8::mma(hi, __builtin_bit_cast(i32x4, load_x(f, at + 16)), acc[f]);
            }
        }
    }
#pragma unroll
    for (int f = 0; f < FI; ++f) part[wave][f][lane] = acc[f];
    if constexpr (AD) {
        // wave = part * FI + fragment: the parts share the fragment's adapters
        f32x4 d[1] = {f32x4{0, 0, 0, 0}};
        add_adapters<T, 1>(a, wave % FI * 16, lane, wave / FI, kParts, [&](int) { return ch0 + r; }, d);
        extra[wave / FI][wave % FI][lane] = d[0];
    }
    __syncthreads();
    if (wave >= FI) return;
    const int row = wave * 16 + r, ch = ch0 + g * 4;   // results: channels ch .. ch + 3 of one row
    i32x4 t = part[0][wave][lane];
#pragma unroll
    for (int p = 1; p < kWaves; ++p) t += part[p][wave][lane];
    if (row >= a.m) return;
    const float xs = a.x.scale[row] * (WB == 4 ? 0.0625f : 1.0f);
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = ch + i < a.k ? (float)t[i] * xs * a.w.scale[ch + i] : 0.0f;
    if constexpr (AD) {
#pragma unroll
        for (int p = 0; p < kParts; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] += extra[p][wave][lane][i];
    }
    typename T::elem *out = static_cast<typename T::elem *>(a.y) + (int64_t)row * a.ldy + ch;
    if (a.vec && ch + 4 <= a.k) {
        *reinterpret_cast<uint2 *>(out) = uint2{pack2<T>(y[0], y[1]), pack2<T>(y[2], y[3])};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (ch + i < a.k) out[i] = (typename T::elem)y[i];
    }
}

// --------------------------------------------------------------- many rows

// TJ output channels by TI rows a workgroup of WJ x WI waves, each a tile of 64
// by 16 FI.  Steps of 128 channels are staged in one of two LDS buffers while
// the other is multiplied; rows and 8-bit weights go straight from memory to
// LDS, 4-bit ones through registers, where they are widened.
template <class T, int WB, int TJ, int TI, int WJ, int WI, bool AD>
__global__ void __launch_bounds__(WJ *WI * 64) linear_tile(LinearArgs a) {
    constexpr int FJ = 4, FI = TI / (16 * WI), kThreads = WJ * WI * 64, kBuffer = (TJ + TI) * kStepBytes;
    static_assert(TJ == WJ * 64);
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    int ti, tj;
    tile_at(xcd_run((int)blockIdx.x, a.tiles_i * a.tiles_j), a.tiles_i, a.tiles_j, ti, tj);
    const int i0 = ti * TI, j0 = tj * TJ;
    const u32x4_t rx = range_words(a.x.codes + (int64_t)i0 * a.x.pitch, (int64_t)(a.m - 1 - i0) * a.x.pitch + a.x.used);
    const uint8_t *wbase = a.w.codes + (int64_t)j0 * a.w.pitch;
    const int64_t wbytes = (int64_t)(a.k - 1 - j0) * a.w.pitch + a.w.used;
    const u32x4_t rw = range_words(wbase, wbytes);
    const __amdgpu_buffer_rsrc_t rw4 = range_of(wbase, wbytes);
    constexpr int kUnits = WB == 4 ? TJ * 4 / kThreads : 1;   // 16-byte vectors of 4-bit weights a thread
    u32x4_t held[kUnits];
    auto fetch = [&](int s, uint8_t *buf) {
        copy_rows<TI, kThreads>(buf + TJ * kStepBytes, rx, (uint32_t)a.x.pitch, s * 128, a.x.used, wave, lane);
        if constexpr (WB == 8) {
            copy_rows<TJ, kThreads>(buf, rw, (uint32_t)a.w.pitch, s * 128, a.w.used, wave, lane);
        } else {
#pragma unroll
            for (int n = 0; n < kUnits; ++n) {
                const int unit = n * kThreads + (int)threadIdx.x, row = unit >> 2, at = s * 64 + (unit & 3) * 16;
                held[n] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                    rw4, (int)(at < a.w.used ? (uint32_t)row * (uint32_t)a.w.pitch + (uint32_t)at : kNowhere), 0, 0));
            }
        }
    };
    auto settle = [&](uint8_t *buf) {
        if constexpr (WB == 4) {
#pragma unroll
            for (int n = 0; n < kUnits; ++n) {
                const int unit = n * kThreads + (int)threadIdx.x, row = unit >> 2, v = (unit & 3) * 2;
                const uint2 p = widen8(held[n][0]), q = widen8(held[n][1]);
                const uint2 s = widen8(held[n][2]), t = widen8(held[n][3]);
                *reinterpret_cast<uint4 *>(buf + row * kStepBytes + ((v ^ slot(row)) << 4)) = uint4{p.x, p.y, q.x, q.y};
                *reinterpret_cast<uint4 *>(buf + row * kStepBytes + (((v + 1) ^ slot(row)) << 4)) = uint4{s.x, s.y, t.x, t.y};
            }
        }
        copies_done();
    };
    const int jrow0 = (wave / WI) * 64, irow0 = (wave % WI) * FI * 16;
    i32x4 acc[FJ][FI];
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[j][i] = i32x4{0, 0, 0, 0};
    fetch(0, smem);
    settle(smem);
    __syncthreads();
    int buf = 0;
    for (int s = 0; s < a.steps; ++s) {
        uint8_t *cur = smem + buf * kBuffer, *next = smem + (buf ^ 1) * kBuffer;
        if (s + 1 < a.steps) fetch(s + 1, next);
        mma_step<MmaI8, FJ, FI>(cur, cur + TJ * kStepBytes, jrow0, irow0, lane, acc);
        if (s + 1 < a.steps) settle(next);
        __syncthreads();
        buf ^= 1;
    }
    // lane (r, g): channels ch .. ch + 15 of one row of each fragment i
    const int r = lane & 15, g = lane >> 4;
    const int ch = j0 + jrow0 + g * 16;
    float ws[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) ws[e] = a.w.scale[min(ch + e, a.k - 1)];
#pragma unroll
    for (int i = 0; i < FI; ++i) {
        const int row = i0 + irow0 + i * 16 + r;
        const float xs = row < a.m ? a.x.scale[row] * (WB == 4 ? 0.0625f : 1.0f) : 0.0f;
        f32x4 d[FJ];
#pragma unroll
        for (int j = 0; j < FJ; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[j][e] = (float)acc[j][i][e] * xs * ws[4 * j + e];
        if constexpr (AD)
            add_adapters<T, FJ>(a, i0 + irow0 + i * 16, lane, 0, 1,
                                [&](int j) { return j0 + jrow0 + j_row(j, r); }, d);
        if (row < a.m) {
            typename T::elem *out = static_cast<typename T::elem *>(a.y) + (int64_t)row * a.ldy + ch;
            if (a.vec && ch + 16 <= a.k) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<uint4 *>(out + 8 * h) =
                        uint4{pack2<T>(d[2 * h][0], d[2 * h][1]), pack2<T>(d[2 * h][2], d[2 * h][3]),
                              pack2<T>(d[2 * h + 1][0], d[2 * h + 1][1]), pack2<T>(d[2 * h + 1][2], d[2 * h + 1][3])};
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (ch + e < a.k) out[e] = (typename T::elem)d[e >> 2][e & 3];
            }
        }
    }
}

}  // namespace qconv

// Products of a 16-bit gradient with rows of codes and their scales:
//   out[i][j] = sum over t of p(i, t) scale[t] codes[t][j]
// The layer's input gradient (t: output channels, codes: the weights, p the
// output gradient) and its weight gradient (t: the batch's rows, codes: the
// 8-bit checkpoint of the input, p the output gradient transposed).
//
// A step stages 64 values of t in LDS as 16-bit floats, both operands with t
// innermost.  A thread takes 4 columns of 8 rows of codes (coalesced words),
// multiplies code by scale in 32 bits, rounds to the 16-bit type and writes four
// vectors of 8 t: the transposition is free, since every code is converted on
// its own anyway.  The rounding is exact for scales that are powers of two (as
// the quantiser gives them); for others it is one rounding of each operand to the
// gradient's own precision.  Sums are 32-bit.
#pragma once

#include "qlinear_device.h"

namespace qconv {

// Largest finite |scale| of a range, as a factor that brings it to 2^8: f16
// products of code and scale are then normal numbers over 22 binary orders of
// magnitude below the largest (bf16 has float's range and needs none).
template <class T, int THREADS>
__device__ __forceinline__ void scale_window(const float *scale, int begin, int end, uint32_t *lds, float &to,
                                             float &from) {
    if constexpr (sizeof(typename T::elem) != 2 || __is_same(T, BF16)) {
        to = from = 1.0f;
    } else {
        uint32_t m = 0;
        for (int t = begin + (int)threadIdx.x; t < end; t += THREADS) {
            const uint32_t b = __builtin_bit_cast(uint32_t, scale[t]) & 0x7fffffffu;
            if (b < 0x7f800000u) m = max(m, b);
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) m = max(m, lds[w]);
        __syncthreads();
        // exponents of to = 2^(8 - e) and its inverse, both normal
        const int e = min(max((int)(m >> 23) - 127, -118), 126);
        to = __builtin_bit_cast(float, (uint32_t)(127 + 8 - e) << 23);
        from = __builtin_bit_cast(float, (uint32_t)(127 - 8 + e) << 23);
    }
}

// How p reaches LDS: rows of t in whole vectors straight from memory (COPY),
// the same through registers with any alignment (ROWS), or p[t][i] transposed
// in registers (COLUMNS).
enum class PForm { COPY, ROWS, COLUMNS };

template <class T, int WB, PForm P, int TJ, int TI, int WJ, int WI>
__global__ void __launch_bounds__(WJ *WI * 64) grad_tile(GradArgs a) {
    constexpr int FJ = 4, FI = TI / (16 * WI), kThreads = WJ * WI * 64, kBuffer = (TJ + TI) * kStepBytes;
    static_assert(TJ == WJ * 64);
    using elem = typename T::elem;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int tid = (int)threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int tiles = a.tiles_i * a.tiles_j;
    const int split = (int)blockIdx.x / tiles;
    int ti, tj;
    tile_at(xcd_run((int)blockIdx.x - split * tiles, tiles), a.tiles_i, a.tiles_j, ti, tj);
    const int i0 = ti * TI, j0 = tj * TJ;
    const int s0 = split * a.steps_per_split, s1 = min(s0 + a.steps_per_split, a.steps);
    const elem *p = static_cast<const elem *>(a.p);
    float to, from;
    scale_window<T, kThreads>(a.b.scale, s0 * 64, min(s1 * 64, a.nt), reinterpret_cast<uint32_t *>(smem), to, from);

    // codes: a unit is 4 columns (one word, or half a word of 4-bit codes) of 8 rows
    constexpr int kGroups = TJ / 4, kUnits = (kGroups * 8 + kThreads - 1) / kThreads;
    // p transposed: a unit is 2 columns of 8 rows; in rows: one vector
    constexpr int kPUnits = P == PForm::COLUMNS ? TI / 2 * 8 / kThreads : P == PForm::ROWS ? TI * 8 / kThreads : 1;
    uint32_t cw[kUnits][8];
    float cs[kUnits][8];
    uint32_t pw[kPUnits][8];
    const u32x4_t rp_copy = P == PForm::COPY
                                ? range_words(p + (int64_t)i0 * a.ldp, ((int64_t)(a.ni - 1 - i0) * a.ldp + a.nt) * 2)
                                : u32x4_t{0, 0, 0, 0};

    auto fetch = [&](int s, uint8_t *buf) {
        const int t0 = s * 64;
        const __amdgpu_buffer_rsrc_t rc = range_of(a.b.codes + (int64_t)t0 * a.b.pitch,
                                                   (int64_t)(a.nt - 1 - t0) * a.b.pitch + a.b.used);
        const __amdgpu_buffer_rsrc_t rs = range_of(a.b.scale + t0, (int64_t)(a.nt - t0) * 4);
#pragma unroll
        for (int n = 0; n < kUnits; ++n) {
            const int unit = n * kThreads + tid, jg = unit % kGroups, tc = unit / kGroups;
            const int at = WB == 8 ? j0 + jg * 4 : (j0 + jg * 4) / 2;
            const bool in = tc < 8 && at < a.b.used;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int t = tc * 8 + e;
                const int off = (int)(in ? (uint32_t)t * (uint32_t)a.b.pitch + (uint32_t)at : kNowhere);
                if constexpr (WB == 8)
                    cw[n][e] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rc, off, 0, 0);
                else
                    cw[n][e] = (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rc, off, 0, 0);
                cs[n][e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, tc < 8 ? t * 4 : (int)kNowhere, 0, 0));
            }
        }
        if constexpr (P == PForm::COPY) {
            copy_rows<TI, kThreads>(buf + TJ * kStepBytes, rp_copy, (uint32_t)a.ldp * 2u, s * 128, a.nt * 2, wave, lane);
        } else if constexpr (P == PForm::ROWS) {
            const __amdgpu_buffer_rsrc_t rp = range_of(p + (int64_t)i0 * a.ldp, ((int64_t)(a.ni - 1 - i0) * a.ldp + a.nt) * 2);
#pragma unroll
            for (int n = 0; n < kPUnits; ++n) {
                const int unit = n * kThreads + tid, row = unit >> 3, t = t0 + (unit & 7) * 8;
                const uint32_t off = (uint32_t)row * (uint32_t)a.ldp * 2u + (uint32_t)t * 2u;
                if (a.vec_p && t0 + 64 <= a.nt) {
                    const auto v = __builtin_amdgcn_raw_buffer_load_b128(rp, (int)off, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) pw[n][e] = v[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(
                            rp, (int)(t + 2 * e < a.nt ? off + 4 * e : kNowhere), 0, 0);
                        const uint32_t hi = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(
                            rp, (int)(t + 2 * e + 1 < a.nt ? off + 4 * e + 2 : kNowhere), 0, 0);
                        pw[n][e] = lo | hi << 16;
                    }
                }
            }
        } else {
            const __amdgpu_buffer_rsrc_t rp = range_of(p + (int64_t)t0 * a.ldp + i0, ((int64_t)(a.nt - 1 - t0) * a.ldp + a.ni - i0) * 2);
#pragma unroll
            for (int n = 0; n < kPUnits; ++n) {
                const int unit = n * kThreads + tid, i = unit % (TI / 2) * 2, tc = unit / (TI / 2);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t off = (uint32_t)(tc * 8 + e) * (uint32_t)a.ldp * 2u + (uint32_t)i * 2u;
                    // rows past the last are past the range; columns past the last reach
                    // only results that are not stored
                    if (a.vec_p) {
                        pw[n][e] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rp, (int)(i0 + i < a.ni ? off : kNowhere), 0, 0);
                    } else {
                        const uint32_t lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(
                            rp, (int)(i0 + i < a.ni ? off : kNowhere), 0, 0);
                        const uint32_t hi = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(
                            rp, (int)(i0 + i + 1 < a.ni ? off + 2 : kNowhere), 0, 0);
                        pw[n][e] = lo | hi << 16;
                    }
                }
            }
        }
    };
    auto settle = [&](uint8_t *buf) {
#pragma unroll
        for (int n = 0; n < kUnits; ++n) {
            const int unit = n * kThreads + tid, jg = unit % kGroups, tc = unit / kGroups;
            if (kGroups * 8 % kThreads != 0 && tc >= 8) continue;
            u32x4_t v[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                float f[2][4];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t w = cw[n][2 * h + b];
                    const float sc = cs[n][2 * h + b] * to;
                    if constexpr (WB == 8) {
                        const uint32_t x = w ^ 0x80808080u;   // code + 128
                        const float off = -128.0f * sc;
                        f[b][0] = __builtin_fmaf((float)(x & 255u), sc, off);
                        f[b][1] = __builtin_fmaf((float)((x >> 8) & 255u), sc, off);
                        f[b][2] = __builtin_fmaf((float)((x >> 16) & 255u), sc, off);
                        f[b][3] = __builtin_fmaf((float)(x >> 24), sc, off);
                    } else {
                        const uint32_t x = w ^ 0x8888u;       // code + 8
                        const float off = -8.0f * sc;
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            f[b][c] = __builtin_fmaf((float)((x >> (4 * c)) & 15u), sc, off);
                    }
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c][h] = pack2<T>(f[0][c], f[1][c]);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int row = jg * 4 + c;
                *reinterpret_cast<u32x4_t *>(buf + row * kStepBytes + ((tc ^ slot(row)) << 4)) = v[c];
            }
        }
        uint8_t *pb = buf + TJ * kStepBytes;
        if constexpr (P == PForm::ROWS) {
#pragma unroll
            for (int n = 0; n < kPUnits; ++n) {
                const int unit = n * kThreads + tid, row = unit >> 3, tc = unit & 7;
                *reinterpret_cast<u32x4_t *>(pb + row * kStepBytes + ((tc ^ slot(row)) << 4)) =
                    u32x4_t{pw[n][0], pw[n][1], pw[n][2], pw[n][3]};
            }
        } else if constexpr (P == PForm::COLUMNS) {
#pragma unroll
            for (int n = 0; n < kPUnits; ++n) {
                const int unit = n * kThreads + tid, row = unit % (TI / 2) * 2, tc = unit / (TI / 2);
                u32x4_t even, odd;
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    even[h] = __builtin_amdgcn_perm(pw[n][2 * h + 1], pw[n][2 * h], 0x05040100u);
                    odd[h] = __builtin_amdgcn_perm(pw[n][2 * h + 1], pw[n][2 * h], 0x07060302u);
                }
                *reinterpret_cast<u32x4_t *>(pb + row * kStepBytes + ((tc ^ slot(row)) << 4)) = even;
                *reinterpret_cast<u32x4_t *>(pb + (row + 1) * kStepBytes + ((tc ^ slot(row + 1)) << 4)) = odd;
            }
        } else {
            copies_done();
        }
    };

    const int jrow0 = (wave / WI) * 64, irow0 = (wave % WI) * FI * 16;
    f32x4 acc[FJ][FI];
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[j][i] = f32x4{0, 0, 0, 0};
    fetch(s0, smem);
    settle(smem);
    __syncthreads();
    int buf = 0;
    for (int s = s0; s < s1; ++s) {
        uint8_t *cur = smem + buf * kBuffer, *next = smem + (buf ^ 1) * kBuffer;
        if (s + 1 < s1) fetch(s + 1, next);
        mma_step<MmaT<T>, FJ, FI>(cur, cur + TJ * kStepBytes, jrow0, irow0, lane, acc);
        if (s + 1 < s1) settle(next);
        __syncthreads();
        buf ^= 1;
    }
    const int r = lane & 15, g = lane >> 4;
    const int col = j0 + jrow0 + g * 16;
#pragma unroll
    for (int i = 0; i < FI; ++i) {
        const int row = i0 + irow0 + i * 16 + r;
        if (row >= a.ni || col >= a.nj) continue;
        f32x4 d[FJ];
#pragma unroll
        for (int j = 0; j < FJ; ++j) d[j] = acc[j][i] * from;
        if (a.splits > 1) {
            float *out = a.part + ((int64_t)split * a.ni + row) * a.ldpart + col;
#pragma unroll
            for (int j = 0; j < FJ; ++j)
                if (col + 4 * j < a.ldpart) *reinterpret_cast<f32x4 *>(out + 4 * j) = d[j];
        } else if constexpr (P == PForm::COLUMNS) {
            float *out = static_cast<float *>(a.out) + (int64_t)row * a.ldo + col;
#pragma unroll
            for (int j = 0; j < FJ; ++j) {
                if (a.vec_out && col + 4 * j + 4 <= a.nj) {
                    *reinterpret_cast<f32x4 *>(out + 4 * j) = d[j];
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (col + 4 * j + e < a.nj) out[4 * j + e] = d[j][e];
                }
            }
        } else {
            elem *out = static_cast<elem *>(a.out) + (int64_t)row * a.ldo + col;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 lo = d[2 * h], hi = d[2 * h + 1];
                if (a.vec_out && col + 8 * h + 8 <= a.nj) {
                    *reinterpret_cast<uint4 *>(out + 8 * h) = uint4{pack2<T>(lo[0], lo[1]), pack2<T>(lo[2], lo[3]),
                                                                    pack2<T>(hi[0], hi[1]), pack2<T>(hi[2], hi[3])};
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (col + 8 * h + e < a.nj) out[8 * h + e] = (elem)(e < 4 ? lo[e & 3] : hi[e & 3]);
                }
            }
        }
    }
}

// Adds the partial sums in the order of the splits and rounds once: four
// columns a thread.
template <class Out>
__global__ void __launch_bounds__(256) grad_sum(GradArgs a, int64_t first) {
    const int64_t at = (first + blockIdx.x) * 256 + threadIdx.x;
    const int64_t quads = a.ldpart / 4, row = at / quads;
    if (row >= a.ni) return;
    const int col = (int)(at - row * quads) * 4;
    const float *p = a.part + row * a.ldpart + col;
    f32x4 t = *reinterpret_cast<const f32x4 *>(p);
    for (int s = 1; s < a.splits; ++s) t += *reinterpret_cast<const f32x4 *>(p + (int64_t)s * a.ni * a.ldpart);
    Out *out = static_cast<Out *>(a.out) + row * a.ldo + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (col + e < a.nj) out[e] = (Out)t[e];
}

}  // namespace qconv

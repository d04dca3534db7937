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

// How p reaches LDS: rows of t in whole vectors straight from memory (ROWS_COPY),
// rows of i likewise, transposed when they are read (COLUMNS_COPY), or either
// through registers, with any alignment and width.
enum class PForm { ROWS_COPY, ROWS, COLUMNS_COPY, COLUMNS };
constexpr bool transposed(PForm p) { return p == PForm::COLUMNS_COPY || p == PForm::COLUMNS; }

// COLUMNS_COPY keeps p as it lies in memory, rows of TI values of one t, and a
// fragment is read by transposing loads: 16 lanes read 16 columns of four rows,
// and each gets its column of all four.  Row t's 32-byte unit u lies at unit
// u ^ unit_of(t): the rows of one load fall on different banks.
template <int TI>
__device__ __forceinline__ int unit_of(int t) {
    return TI == 256 ? (t & 3) | ((t >> 1) & 12) : TI == 128 ? (t & 3) | ((t >> 1) & 4) : ((t >> 1) & 1) | ((t >> 2) & 2);
}
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <class T>
__device__ __forceinline__ typename T::v8 read_transposed(const uint8_t *lds, int row_bytes) {
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds + 4 * row_bytes));
    return __builtin_bit_cast(typename T::v8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Up to four results from one row, `left` of them within it.
__device__ __forceinline__ void store4(float *out, f32x4 d, int left, bool vec) {
    if (vec && left >= 4) {
        *reinterpret_cast<f32x4 *>(out) = d;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) out[e] = d[e];
    }
}
template <class T>
__device__ __forceinline__ void store4(typename T::elem *out, f32x4 d, int left, bool vec) {
    if (vec && left >= 4) {
        *reinterpret_cast<uint2 *>(out) = uint2{pack2<T>(d[0], d[1]), pack2<T>(d[2], d[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) out[e] = (typename T::elem)d[e];
    }
}

// Codes through registers, converted on their way to LDS: 4-bit codes, and p of
// any alignment.  Each step multiplies one LDS buffer while the other is filled for
// the next: copies go out first, the codes that were loaded a step earlier are
// converted and stored in the shadow of the matrix instructions, and the codes
// after them are then loaded.
template <class T, int WB, PForm P, int TJ, int TI, int WJ, int WI>
__global__ void __launch_bounds__(WJ *WI * 64) grad_regs(GradArgs a) {
    constexpr int FJ = 4, FI = TI / (16 * WI), kThreads = WJ * WI * 64, kBuffer = (TJ + TI) * kStepBytes;
    constexpr int kWaves = kThreads / 64;
    static_assert(TJ == WJ * 64);
    using elem = typename T::elem;
    using v8 = typename T::v8;
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

    // codes: a unit is 4 columns (one word, or half a word of 4-bit codes) of 8
    // rows; a wave of the widest tile takes one group of 8 rows, whose scales are
    // then scalars
    constexpr int kGroups = TJ / 4, kUnits = (kGroups * 8 + kThreads - 1) / kThreads;
    constexpr bool kScalarScale = kGroups == 64 && kUnits == 1;
    // p in registers, transposed: a unit is 2 columns of 8 rows; in rows: one vector
    constexpr int kPUnits = P == PForm::COLUMNS ? TI / 2 * 8 / kThreads : P == PForm::ROWS ? TI * 8 / kThreads : 1;
    uint32_t cw[kUnits][8];
    float cs[kScalarScale ? 1 : kUnits][8];
    uint32_t pw[kPUnits][8];
    const u32x4_t rp_rows = P == PForm::ROWS_COPY
                                ? range_words(p + (int64_t)i0 * a.ldp, ((int64_t)(a.ni - 1 - i0) * a.ldp + a.nt) * 2)
                                : u32x4_t{0, 0, 0, 0};

    auto copy_p = [&](int s, uint8_t *buf) {
        uint8_t *pb = buf + TJ * kStepBytes;
        if constexpr (P == PForm::ROWS_COPY) {
            copy_rows<TI, kThreads>(pb, rp_rows, (uint32_t)a.ldp * 2u, s * 128, a.nt * 2, wave, lane);
        } else if constexpr (P == PForm::COLUMNS_COPY) {
            const int t0 = s * 64;
            const u32x4_t rp = range_words(p + (int64_t)t0 * a.ldp + i0, ((int64_t)(a.nt - 1 - t0) * a.ldp + a.ni - i0) * 2);
            constexpr int kRow = TI * 2;
#pragma unroll
            for (int n = 0; n < 64 * kRow / (1024 * kWaves); ++n) {
                const int at = (n * kWaves + wave) * 1024 + lane * 16, t = at / kRow, in = at % kRow;
                const int col = ((in >> 5) ^ unit_of<TI>(t)) * 32 + (in & 16);
                copy16(pb + (n * kWaves + wave) * 1024,
                       col < (a.ni - i0) * 2 ? (uint32_t)t * (uint32_t)a.ldp * 2u + (uint32_t)col : kNowhere, rp);
            }
        }
    };
    auto load = [&](int s) {
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
                if constexpr (!kScalarScale)
                    cs[n][e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, tc < 8 ? t * 4 : (int)kNowhere, 0, 0));
            }
        }
        if constexpr (P == PForm::ROWS) {
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
        } else if constexpr (P == PForm::COLUMNS) {
            const __amdgpu_buffer_rsrc_t rp = range_of(p + (int64_t)t0 * a.ldp + i0, ((int64_t)(a.nt - 1 - t0) * a.ldp + a.ni - i0) * 2);
#pragma unroll
            for (int n = 0; n < kPUnits; ++n) {
                const int unit = n * kThreads + tid, i = unit % (TI / 2) * 2, tc = unit / (TI / 2);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t off = (uint32_t)(tc * 8 + e) * (uint32_t)a.ldp * 2u + (uint32_t)i * 2u;
                    // rows past the last are past the range; columns past the last reach
                    // only results that are not stored
                    if (a.pair_p) {
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
    // What load() brought of step s, into a buffer.
    auto store = [&](int s, uint8_t *buf) {
        float ss[8];
        if constexpr (kScalarScale) {
            const int t = s * 64 + wave * 8;
            const __attribute__((address_space(4))) float *sc = (const __attribute__((address_space(4))) float *)(a.b.scale);
            if (t + 8 <= a.nt) {
#pragma unroll
                for (int e = 0; e < 8; ++e) ss[e] = sc[t + e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) ss[e] = t + e < a.nt ? sc[t + e] : 0.0f;
            }
        }
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
                    const float sc = (kScalarScale ? ss[2 * h + b] : cs[n][2 * h + b]) * to;
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
        }
    };

    const int jrow0 = (wave / WI) * 64, irow0 = (wave % WI) * FI * 16;
    const int r = lane & 15, g = lane >> 4;
    f32x4 acc[FJ][FI];
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[j][i] = f32x4{0, 0, 0, 0};
    // half a step: the 32 values of t of half ks
    auto multiply = [&](const uint8_t *buf, int ks) {
        const uint8_t *lj = buf, *li = buf + TJ * kStepBytes;
        v8 x[FJ], y[FI];
#pragma unroll
        for (int f = 0; f < FJ; ++f) {
            const int row = jrow0 + j_row(f, r);
            x[f] = *reinterpret_cast<const v8 *>(lj + row * kStepBytes + (((ks * 4 + g) ^ slot(row)) << 4));
        }
#pragma unroll
        for (int f = 0; f < FI; ++f) {
            if constexpr (P == PForm::COLUMNS_COPY) {
                const int t = ks * 32 + g * 8 + (r >> 2);
                y[f] = read_transposed<T>(li + t * (TI * 2) + ((((irow0 >> 4) + f) ^ unit_of<TI>(t)) << 5) + (r & 3) * 8, TI * 2);
            } else {
                const int row = irow0 + f * 16 + r;
                y[f] = *reinterpret_cast<const v8 *>(li + row * kStepBytes + (((ks * 4 + g) ^ slot(row)) << 4));
            }
        }
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) acc[j][i] = T::mma(x[j], y[i], acc[j][i]);
    };
    load(s0);
    copy_p(s0, smem);
    store(s0, smem);
    load(s0 + 1);
    copies_done();
    __syncthreads();
    int buf = 0;
    for (int s = s0; s < s1; ++s) {
        uint8_t *cur = smem + buf * kBuffer, *next = smem + (buf ^ 1) * kBuffer;
        // (past the last step these bring zeros, or another split's values, to a
        // buffer that is not read)
        copy_p(s + 1, next);
        multiply(cur, 0);
        store(s + 1, next);
        load(s + 2);
        multiply(cur, 1);
        copies_done();
        __syncthreads();
        buf ^= 1;
    }
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
        } else if constexpr (transposed(P)) {
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

// Everything by copies: 8-bit codes and p both lie in LDS as they lie in memory
// (three buffers of 64 rows of t: one multiplied, one landed, one on its way), and
// codes are read by transposing loads, 8 rows of one column a lane, and converted
// on their way to the matrix cores.  A matrix instruction of 16 cycles hides two
// vector instructions of a wave (measured: three cost a quarter more, four half),
// so a wave of the widest tile takes 32 columns of codes by all 256 of p and no
// code is converted twice; that reads p from LDS eight times over, which LDS can
// give.
template <int TJ>
__device__ __forceinline__ int code_unit_of(int t) {
    return TJ == 256 ? t & 15 : TJ == 128 ? (t >> 1) & 7 : (t >> 2) & 3;
}
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// Two codes (bytes 2 half, 2 half + 1 of w) times their scales.
template <class T>
__device__ __forceinline__ uint32_t scaled_pair(uint32_t w, int half, float s0, float s1) {
    return pack2<T>((float)(int8_t)(w >> (16 * half)) * s0, (float)(int8_t)(w >> (16 * half + 8)) * s1);
}

template <class T, PForm P, int TJ, int TI, int WJ, int WI>
__global__ void __launch_bounds__(WJ *WI * 64) grad_tile(GradArgs a) {
    static_assert(P == PForm::ROWS_COPY || P == PForm::COLUMNS_COPY);
    constexpr int FJ = TJ / (16 * WJ), FI = TI / (16 * WI), kThreads = WJ * WI * 64, kWaves = kThreads / 64;
    constexpr int kCodes = 64 * TJ, kP = TI * 128, kStage = kCodes + kP + 256;
    constexpr int kCodeCopies = kCodes / (1024 * kWaves), kPCopies = kP / (1024 * kWaves);
    constexpr int kCopies = kCodeCopies + kPCopies + 1;   // a wave's copies of a step
    using elem = typename T::elem;
    using v8 = typename T::v8;
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

    const u32x4_t rp_rows = range_words(p + (int64_t)i0 * a.ldp, ((int64_t)(a.ni - 1 - i0) * a.ldp + a.nt) * 2);
    // copy n of step s: the codes', p's, then the scales (every wave copies the same
    // ones to the same place, so that all have the same copies to wait for)
    struct Step {
        u32x4_t codes, p, scale;
    };
    auto step_of = [&](int s) {   // (a step's rows of t: 32-bit ranges from 64-bit bases)
        const int t0 = s * 64, rows = min(a.nt - t0, 64);
        Step q;
        q.codes = range_words(a.b.codes + (int64_t)t0 * a.b.pitch + j0,
                              rows > 0 ? (rows - 1) * (int)a.b.pitch + a.b.used - j0 : 0);
        q.p = P == PForm::ROWS_COPY ? rp_rows
                                    : range_words(p + (int64_t)t0 * a.ldp + i0,
                                                  rows > 0 ? ((rows - 1) * (int)a.ldp + a.ni - i0) * 2 : 0);
        q.scale = range_words(a.b.scale + t0, rows > 0 ? rows * 4 : 0);
        return q;
    };
    auto copy = [&](int n, int s, const Step &q, uint8_t *buf) {
        if (n < kCodeCopies) {
            const int at = (n * kWaves + wave) * 1024 + lane * 16, t = at / TJ, in = at % TJ;
            const int col = ((in >> 4) ^ code_unit_of<TJ>(t)) << 4;
            copy16(buf + (n * kWaves + wave) * 1024,
                   j0 + col < a.b.used ? (uint32_t)t * (uint32_t)a.b.pitch + (uint32_t)col : kNowhere, q.codes);
        } else if (n < kCodeCopies + kPCopies) {
            const int at0 = ((n - kCodeCopies) * kWaves + wave) * 1024;
            uint32_t off;
            if constexpr (P == PForm::ROWS_COPY) {
                const int row = (at0 >> 7) + (lane >> 3), at = s * 128 + (((lane & 7) ^ slot(row)) << 4);
                off = at < a.nt * 2 ? (uint32_t)row * (uint32_t)a.ldp * 2u + (uint32_t)at : kNowhere;
            } else {
                const int at = at0 + lane * 16, t = at / (TI * 2), in = at % (TI * 2);
                const int col = ((in >> 5) ^ unit_of<TI>(t)) * 32 + (in & 16);
                off = col < (a.ni - i0) * 2 ? (uint32_t)t * (uint32_t)a.ldp * 2u + (uint32_t)col : kNowhere;
            }
            copy16(buf + kCodes + at0, off, q.p);
        } else {
            copy4(buf + kCodes + kP, (uint32_t)lane * 4u, q.scale);
        }
    };

    const int jrow0 = (wave / WI) * 16 * FJ, irow0 = (wave % WI) * FI * 16;
    const int r = lane & 15, g = lane >> 4;
    f32x4 acc[FJ][FI];
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int i = 0; i < FI; ++i) acc[j][i] = f32x4{0, 0, 0, 0};
    // The 32 rows of t of half ks of a step: fragment f of p, and the codes and scales
    // as they lie in LDS.
    auto read_p = [&](const uint8_t *buf, int ks, int f) {
        const uint8_t *li = buf + kCodes;
        if constexpr (P == PForm::COLUMNS_COPY) {
            const int t = ks * 32 + g * 8 + (r >> 2);
            return read_transposed<T>(
                li + t * (TI * 2) + ((((irow0 >> 4) + f) ^ unit_of<TI>(t)) << 5) + (r & 3) * 8, TI * 2);
        } else {
            const int row = irow0 + f * 16 + r;
            return *reinterpret_cast<const v8 *>(li + row * kStepBytes + (((ks * 4 + g) ^ slot(row)) << 4));
        }
    };
    struct Codes {
        i32x2 q[FJ];
        f32x4 scale[2];
    };
    auto read_codes = [&](const uint8_t *buf, int ks) {
        Codes c;
        const float *sc = reinterpret_cast<const float *>(buf + kCodes + kP) + ks * 32 + g * 8;
        c.scale[0] = *reinterpret_cast<const f32x4 *>(sc);
        c.scale[1] = *reinterpret_cast<const f32x4 *>(sc + 4);
        const int t = ks * 32 + g * 8 + (r >> 1);
#pragma unroll
        for (int f = 0; f < FJ; ++f)
            c.q[f] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                (lds_i32x2 *)(buf + t * TJ + ((((jrow0 >> 4) + f) ^ code_unit_of<TJ>(t)) << 4) + (r & 1) * 8));
        return c;
    };
    // One half of a step from x (its codes, converted) and the first kAhead fragments
    // of p: each fragment of p is read kAhead groups of matrix instructions before its
    // own, and between the groups the next half's codes are converted and `spread`
    // does a part of other work.  The groups are fenced off from each other: a wave's
    // own vector instructions are the only ones sure to run in the matrix
    // instructions' shadow, and the scheduler gathers them.
    constexpr int kAhead = FI < 3 ? FI : 3;
    auto half = [&](const uint8_t *cur, int ks, const uint8_t *then, u32x4_t (&x)[FJ], v8 (&ahead)[kAhead], auto spread) {
        v8 y[FI + kAhead];
#pragma unroll
        for (int f = 0; f < kAhead; ++f) y[f] = ahead[f];
        const Codes c = read_codes(then, ks ^ 1);
        u32x4_t next[FJ];
#pragma unroll
        for (int i = 0; i < FI; ++i) {
            const int f = i + kAhead;
            y[f] = f < FI ? read_p(cur, ks, f) : read_p(then, ks ^ 1, f - FI);
            spread(i);
#pragma unroll
            for (int j = 0; j < FJ; ++j) acc[j][i] = T::mma(__builtin_bit_cast(v8, x[j]), y[i], acc[j][i]);
            // pairs of codes: 4 FJ of them over the groups after the first
            constexpr int kPairs = 4 * FJ, kGroups = FI > 1 ? FI - 1 : 1, kFirst = FI > 1 ? 1 : 0;
#pragma unroll
            for (int n = (i - kFirst) * kPairs / kGroups; n < (i - kFirst + 1) * kPairs / kGroups; ++n) {
                if (n < 0 || i < kFirst) continue;
                const int k = n >> 2, e = (n & 3) * 2;
                next[k][n & 3] = scaled_pair<T>((uint32_t)c.q[k][e >> 2], (e >> 1) & 1, c.scale[e >> 2][e & 3] * to,
                                                c.scale[e >> 2][(e & 3) + 1] * to);
                asm volatile("" : "+v"(next[k][n & 3]));   // here, not where the value is next used
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int f = 0; f < FJ; ++f) x[f] = next[f];
#pragma unroll
        for (int f = 0; f < kAhead; ++f) ahead[f] = y[FI + f];
    };
#pragma unroll
    for (int n = 0; n < kCopies; ++n) copy(n, s0, step_of(s0), smem);
#pragma unroll
    for (int n = 0; n < kCopies; ++n) copy(n, s0 + 1, step_of(s0 + 1), smem + kStage);
    copies_left<kCopies>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    u32x4_t x[FJ];
    v8 ahead[kAhead];
    {
        const Codes c = read_codes(smem, 0);
#pragma unroll
        for (int f = 0; f < FJ; ++f)
#pragma unroll
            for (int n = 0; n < 4; ++n)
                x[f][n] = scaled_pair<T>((uint32_t)c.q[f][n >> 1], n & 1, c.scale[n >> 1][(n & 1) * 2] * to,
                                         c.scale[n >> 1][(n & 1) * 2 + 1] * to);
#pragma unroll
        for (int f = 0; f < kAhead; ++f) ahead[f] = read_p(smem, 0, f);
    }
    int at = 0;
    for (int s = s0; s < s1; ++s) {
        const int after = at + 1 == 3 ? 0 : at + 1, fill = after + 1 == 3 ? 0 : after + 1;
        uint8_t *cur = smem + at * kStage, *then = smem + after * kStage, *third = smem + fill * kStage;
        half(cur, 0, cur, x, ahead, [](int) {});
        // the next step's copies have landed, and everyone is done with the step
        // before this one
        copies_left<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (past the last step these go to a buffer that is not multiplied)
        const Step q = step_of(s + 2);
        half(cur, 1, then, x, ahead, [&](int i) {
#pragma unroll
            for (int n = i * kCopies / FI; n < (i + 1) * kCopies / FI; ++n) copy(n, s + 2, q, third);
        });
        at = after;
    }
    copies_done();   // none may land in the LDS of a workgroup that comes after
#pragma unroll
    for (int i = 0; i < FI; ++i) {
        const int row = i0 + irow0 + i * 16 + r;
        if (row >= a.ni) continue;
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            const int col = j0 + jrow0 + 16 * j + 4 * g;
            const f32x4 d = acc[j][i] * from;
            if (a.splits > 1) {
                if (col < a.ldpart)
                    *reinterpret_cast<f32x4 *>(a.part + ((int64_t)split * a.ni + row) * a.ldpart + col) = d;
            } else if constexpr (transposed(P)) {
                store4(static_cast<float *>(a.out) + (int64_t)row * a.ldo + col, d, a.nj - col, a.vec_out);
            } else {
                store4<T>(static_cast<elem *>(a.out) + (int64_t)row * a.ldo + col, d, a.nj - col, a.vec_out);
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

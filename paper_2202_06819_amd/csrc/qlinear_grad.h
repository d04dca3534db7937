// Products of a 16-bit gradient with rows of codes and their scales:
//   out[i][j] = sum over t of p(i, t) scale[t] codes[t][j]
// The layer's input gradient (t: output channels, codes: the weights, p the
// output gradient) and its weight gradient (t: the batch's rows, codes: the
// 8-bit checkpoint of the input, p the output gradient transposed).
//
// A step stages 64 values of t in LDS, both operands as they lie in memory, and the
// operand that has t outermost is read by transposing loads.  A code times its scale
// is formed in 32 bits and rounded to the 16-bit type: exact for scales that are
// powers of two (as the quantiser gives them); for others it is one rounding of each
// operand to the gradient's own precision, which adds about as much error as the result's
// own rounding: relative to the results 0.0024 instead of 0.0017 in bf16 (4-bit weights,
// 4096 of them summed), 0.0003 instead of 0.0002 in f16.  Sums are 32-bit.
//
// Scales of groups (GS) are seldom powers of two, so there a scale enters as the sum of two
// parts: the first of as few bits as leave a 4-bit code times it exact in the 16-bit type,
// the second what is left, and each takes a product of its own.  Scales of the gradient's
// own type lose nothing; of longer ones the second product's rounding is 2^-12 of a product
// in bf16, 2^-18 in f16, at most (the rest is 2^-4 and 2^-7 of the scale).  So a gradient
// is as far from 64 bits as 32-bit products are, at twice the matrix instructions
// (4096 x 4096 x 4096 in bf16 191 us, 0.0017 off; with one rounded part 123 and 0.0024; 333
// rows of 2824 by 1001 in f16 25.4 and 24.1).  Experts' 4-bit weights with one scale a row are
// taken as one group.
#pragma once

#include "qlinear_device.h"
#include "qlinear_scales.h"

namespace qconv {

// LDS of a step's scales: one for each t, or the two parts of one for each t and 32 columns.
constexpr int grad_scale_bytes(int scale_bytes, int tile) { return scale_bytes ? tile / 32 * 512 : 256; }
constexpr int kGradStages = 3;
// Of a group of waves: its steps' codes, p and scales.
constexpr int grad_lds(int tile, int scale_bytes = 0) {
    return kGradStages * (tile * 64 + tile * 128 + grad_scale_bytes(scale_bytes, tile));
}

// A thread's scales of groups on their way (none without groups).
template <int N>
struct HeldScales {
    uint32_t q[N];
};
template <>
struct HeldScales<0> {};

// A power of two that brings the largest finite |scale| of a range to at most 65504 /
// 128, the largest f16 by the largest code, and above half of that: a code of -128 stays
// finite, and f16 products of code and scale are normal numbers for scales down to 2^-21
// of the largest (bf16 has float's range and needs none).
__device__ __forceinline__ uint32_t finite_size(float scale) {
    const uint32_t b = __builtin_bit_cast(uint32_t, scale) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}
// WAVES waves find it together, `which` of them being this one: m is the largest magnitude
// that the wave's lanes have seen, lds a place for all of theirs.
template <class T, int WAVES>
__device__ __forceinline__ void scale_window(uint32_t m, int which, uint32_t *lds, float &to, float &from) {
    if constexpr (__is_same(T, BF16)) {
        to = from = 1.0f;
    } else {
#pragma unroll
        for (int d = 32; d; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) lds[which] = m;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) m = max(m, lds[w]);
            __syncthreads();
        }
        // exponents of to = 2^(8 - e) and its inverse, both normal (-118 <= e <= 128); a
        // mantissa past 65504 / 32768 = 1 + 0x7fe000 / 2^23 takes the next e
        const int e = max((int)(m >> 23) - 127 + ((m & 0x7fffffu) > 0x7fe000u), -118);
        to = __builtin_bit_cast(float, (uint32_t)(127 + 8 - e) << 23);
        from = __builtin_bit_cast(float, (uint32_t)(127 - 8 + e) << 23);
    }
}

// Transposed, p lies in LDS as in memory, rows of TI values of one t, and a
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

// Three LDS buffers of 64 rows of t: one is multiplied, one has landed, one is on its
// way (five, in the smallest tile, made no step shorter: its steps are bound by their
// instructions).  8-bit codes, and p where its rows are whole aligned vectors (COPY), go
// straight from memory to LDS; 4-bit codes (widened to bytes) and any other p go through
// registers a step ahead.  Codes are read by transposing loads, 8 rows of one column a
// lane, and converted on their way to the matrix cores.  A matrix instruction of 16
// cycles hides two vector instructions of a wave (measured: three cost a quarter more,
// four half), so a wave of the widest tile takes 32 columns of codes by all 256 of p
// and no code is converted twice; that reads p from LDS eight times over, which LDS
// can give.  Where loads go through registers, the smaller tiles keep those of two steps
// on their way (777 rows, 1411 x 1003 in f16: 18.1 us, with one 19.8; the largest tile
// has no registers left for it).  The largest tile is bound by the matrix cores and the
// conversions beside them: 8192 x 4096 x 4096 takes 219 to 229 us, 1.2 PFLOP/s of the
// 1.53 that products of registers alone reach.
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

// A scale as two parts that add up to it: its first 5 (bf16) or 8 (f16) bits, which a 4-bit
// code leaves exact in the 16-bit type, and the rest.  Where the rest is nothing, or would
// vanish in 16 bits, the first part is taken one unit nearer to zero: the parts then have
// the same sign and neither is zero, so that an infinity in p meets no product of its own
// with zero, nor one of the other sign.  (A scale that is not finite is both parts for the
// same reason.)
template <class T>
__device__ __forceinline__ void split_scale(float s, float &first, float &rest) {
    constexpr uint32_t kUnit = __is_same(T, BF16) ? 0x80000u : 0x10000u;   // the first part's last bit
    const uint32_t b = __builtin_bit_cast(uint32_t, s), size = b & 0x7fffffffu, low = b & (kUnit - 1);
    const bool finite = size < 0x7f800000u, normal = finite && size >= 0x00800000u;
    first = normal ? __builtin_bit_cast(float, b - low - (low < kUnit / 64 ? kUnit : 0)) : s;
    rest = finite ? s - first : s;
}

//
// KS groups of waves deal a tile's steps out among them, each with buffers of its own,
// and their sums meet in LDS: with few tiles a CU's waves then still hide each other's
// waits, without partial sums in memory.
// GS: 0, or the bytes of a scale of a group of channels (4-bit codes); a wave's columns
// lie within 32 channels, so it reads one scale for each t as it does without groups.
template <class T, int WB, bool TRANSPOSED, bool COPY, int GS, int TJ, int TI, int WJ, int WI, int KS>
__device__ __forceinline__ void grad_product(GradArgs a, GroupArg groups, int split, int ti, int tj,
                                             uint8_t *all_smem) {
    constexpr int FJ = TJ / (16 * WJ), FI = TI / (16 * WI), kThreads = WJ * WI * 64, kWaves = kThreads / 64;
    constexpr int kCodes = 64 * TJ, kP = TI * 128, kStage = kCodes + kP + grad_scale_bytes(GS, TJ);
    constexpr int kCodeCopies = WB == 8 ? kCodes / (1024 * kWaves) : 0, kPCopies = COPY ? kP / (1024 * kWaves) : 0;
    constexpr int kCodeUnits = WB == 4 ? kCodes / (16 * kThreads) : 0, kPUnits = COPY ? 0 : kP / (16 * kThreads);
    constexpr int kCopies = kCodeCopies + kPCopies + (GS ? 0 : 1);   // a wave's copies of a step
    constexpr int kScaleUnits = GS ? 1 : 0;   // a thread's scales of a step: a row's, of its wave's columns
    static_assert(!GS || (WB == 4 && !TRANSPOSED && FJ == 2));
    constexpr int kParts = GS ? 2 : 1;   // of a scale: products of a fragment of codes
    using elem = typename T::elem;
    using v8 = typename T::v8;
    const int group = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kThreads);
    uint8_t *const smem = all_smem + group * (kGradStages * kStage);
    const int tid = (int)threadIdx.x % kThreads, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int i0 = ti * TI, j0 = tj * TJ;
    // the split's steps, dealt to the groups in runs; past them every operand is zero
    const int begin = split * a.steps_per_split, end = min(begin + a.steps_per_split, a.steps);
    const int run = (end - begin + KS - 1) / KS, s0 = begin + group * run, s1 = s0 + run;
    const int t_end = min(a.nt, end * 64);
    const elem *p = static_cast<const elem *>(a.p);
    float to, from;
    const u32x4_t rp_rows = range_words(p + (int64_t)i0 * a.ldp, ((int64_t)(a.ni - 1 - i0) * a.ldp + a.nt) * 2);
    // copy n of step s: the codes', p's, then the scales (every wave copies the same
    // ones to the same place, so that all have the same copies to wait for).  A Step
    // holds where its rows of t begin; it moves on by addition (the scalar instructions
    // of finding it anew were most of a small tile's step).
    struct Step {
        uint64_t codes, p, scale;
        int rows;   // of t, from here on
    };
    const int codes_step = 64 * (int)a.b.pitch, p_step = 64 * (int)a.ldp * 2;
    const int codes_last = a.b.used - j0, p_last = (a.ni - i0) * 2;   // bytes in reach of a step's last row
    Step place{(uint64_t)(a.b.codes + (int64_t)s0 * 64 * a.b.pitch + j0), (uint64_t)(p + (int64_t)s0 * 64 * a.ldp + i0),
               (uint64_t)(a.b.scale + s0 * 64), t_end - s0 * 64};
    const auto move_on = [&] {
        place.codes += codes_step;
        if (TRANSPOSED) place.p += p_step;
        place.scale += 256;
        place.rows -= 64;
    };
    struct Words {
        u32x4_t codes, p, scale;
    };
    const auto words_here = [&] {
        const int rows = min(place.rows, 64), before = rows - 1;
        Words q;
        q.codes = range_words((const void *)place.codes, rows > 0 ? before * (int)a.b.pitch + codes_last : 0);
        q.p = !TRANSPOSED ? rp_rows : range_words((const void *)place.p, rows > 0 ? before * (int)a.ldp * 2 + p_last : 0);
        q.scale = range_words((const void *)place.scale, rows > 0 ? rows * 4 : 0);
        return q;
    };
    auto copy = [&](int n, int s, const Words &q, uint8_t *buf) {
        if (n < kCodeCopies) {
            const int at = (n * kWaves + wave) * 1024 + lane * 16, t = at / TJ, in = at % TJ;
            const int col = ((in >> 4) ^ code_unit_of<TJ>(t)) << 4;
            copy16(buf + (n * kWaves + wave) * 1024,
                   j0 + col < a.b.used ? (uint32_t)t * (uint32_t)a.b.pitch + (uint32_t)col : kNowhere, q.codes);
        } else if (n < kCodeCopies + kPCopies) {
            const int at0 = ((n - kCodeCopies) * kWaves + wave) * 1024;
            uint32_t off;
            if constexpr (!TRANSPOSED) {
                const int row = (at0 >> 7) + (lane >> 3), at = s * 128 + (((lane & 7) ^ slot(row)) << 4);
                off = at < t_end * 2 ? (uint32_t)row * (uint32_t)a.ldp * 2u + (uint32_t)at : kNowhere;
            } else {
                const int at = at0 + lane * 16, t = at / (TI * 2), in = at % (TI * 2);
                const int col = ((in >> 5) ^ unit_of<TI>(t)) * 32 + (in & 16);
                off = col < (a.ni - i0) * 2 ? (uint32_t)t * (uint32_t)a.ldp * 2u + (uint32_t)col : kNowhere;
            }
            copy16(buf + kCodes + at0, off, q.p);
        } else if (n < kCopies) {
            copy4(buf + kCodes + kP, (uint32_t)lane * 4u, q.scale);
        }
    };

    // What goes through registers: units of 16 bytes of LDS, each from one load (p's of
    // any alignment).  A unit past the matrix is loaded from within it and put right
    // when it is stored, so that the loads of a step are always as many.
    constexpr int kFetches = kCodeUnits + kPUnits + kScaleUnits, kStages = kGradStages;
    constexpr int kFlight = TJ < 256 && kFetches > 0 ? 2 : 1;   // steps whose loads are on their way
    struct Units {
        uint2 code[kCodeUnits ? kCodeUnits : 1];
        u32x4_t p[kPUnits ? kPUnits : 1];
        [[no_unique_address]] HeldScales<kScaleUnits> scales;
    };
    // The scale of row t for the wave's 32 columns.
    const int jrow0 = (wave / WI) * 16 * FJ, irow0 = (wave % WI) * FI * 16;
    const auto group_scale = [&](int t) {
        const int64_t at = (int64_t)t * groups.pitch + group_of(groups, min((j0 + jrow0) / 32, (a.nj - 1) / 32));
        return load_scale<GS ? GS : 4>(groups, at);
    };
    const int p_rows = TRANSPOSED ? t_end : a.ni, p_count = TRANSPOSED ? a.ni : t_end;   // p as it lies in memory
    const bool narrow = !COPY && p_count < 8;   // rows shorter than a load: by elements
    auto p_place = [&](int s, int n, int &row, int &at) {
        const int unit = n * kThreads + tid;
        row = TRANSPOSED ? s * 64 + unit / (TI / 8) : i0 + unit / 8;
        at = TRANSPOSED ? i0 + unit % (TI / 8) * 8 : s * 64 + unit % 8 * 8;
    };
    auto fetch = [&](int s, Units &q) {
        if constexpr (WB == 4) {
#pragma unroll
            for (int n = 0; n < kCodeUnits; ++n) {
                const int unit = n * kThreads + tid, t = min(s * 64 + unit / (TJ / 16), a.nt - 1);
                const int at = min((j0 + unit % (TJ / 16) * 16) / 2, a.b.used - 8);
                q.code[n] = *reinterpret_cast<const uint2 *>(a.b.codes + (int64_t)t * a.b.pitch + at);
            }
        }
        // (waves of the same columns load the same scales, and write them to the same place)
        if constexpr (GS > 0) q.scales.q[0] = group_scale(min(s * 64 + lane, a.nt - 1));
        if constexpr (!COPY) {
#pragma unroll
            for (int n = 0; n < kPUnits; ++n) {
                int row, at;
                p_place(s, n, row, at);
                const elem *line = p + (int64_t)min(row, p_rows - 1) * a.ldp;
                if (narrow) {
                    u32x4_t v{0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (at == 0 && e < p_count)
                            v[e >> 1] |= (uint32_t)__builtin_bit_cast(uint16_t, line[e]) << (16 * (e & 1));
                    q.p[n] = v;
                } else {
                    __builtin_memcpy(&q.p[n], line + min(at, p_count - 8), 16);
                }
            }
        }
    };
    auto put = [&](int s, const Units &q, uint8_t *buf) {
        if constexpr (WB == 4) {
#pragma unroll
            for (int n = 0; n < kCodeUnits; ++n) {
                const int unit = n * kThreads + tid, t = unit / (TJ / 16), u = unit % (TJ / 16);
                const bool in = s * 64 + t < t_end && j0 + u * 16 < a.b.used * 2;
                const uint2 lo = widen8(in ? q.code[n].x : 0u), hi = widen8(in ? q.code[n].y : 0u);
                *reinterpret_cast<uint4 *>(buf + t * TJ + ((u ^ code_unit_of<TJ>(t)) << 4)) = uint4{lo.x, lo.y, hi.x, hi.y};
            }
        }
        if constexpr (GS > 0) {
            float *const at = reinterpret_cast<float *>(buf + kCodes + kP + (jrow0 >> 5) * 512) + lane;
            split_scale<T>(s * 64 + lane < t_end ? scale_value<GS ? GS : 4>(groups, q.scales.q[0]) * to : 0.0f, at[0], at[64]);
        }
        if constexpr (!COPY) {
#pragma unroll
            for (int n = 0; n < kPUnits; ++n) {
                const int unit = n * kThreads + tid;
                int row, at;
                p_place(s, n, row, at);
                u32x4_t v = q.p[n];
                if (row >= p_rows) {
                    v = u32x4_t{0, 0, 0, 0};
                } else if (!narrow && at + 8 > p_count) {
                    const int past = at + 8 - p_count;   // loaded so many elements too early
                    asm volatile("");   // a branch: few waves have such a unit (as choices: 777 rows 18.4 -> 19.5 us)
                    v = past < 8 ? __builtin_bit_cast(u32x4_t, __builtin_bit_cast(unsigned __int128, v) >> (16 * past))
                                 : u32x4_t{0, 0, 0, 0};
                }
                int to_lds;
                if constexpr (TRANSPOSED) {
                    const int t = unit / (TI / 8), u = unit % (TI / 8);
                    to_lds = t * (TI * 2) + (((u >> 1) ^ unit_of<TI>(t)) << 5) + (u & 1) * 16;
                } else {
                    to_lds = unit / 8 * kStepBytes + ((unit % 8 ^ slot(unit / 8)) << 4);
                }
                *reinterpret_cast<u32x4_t *>(buf + kCodes + to_lds) = v;
            }
        }
    };
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
        if constexpr (TRANSPOSED) {
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
        f32x4 scale[kParts][2];
    };
    // In tiles of 64 the scales' second parts are read and used after the first ones (14
    // registers of 128 spilled otherwise, in f16), in larger ones beside them.
    constexpr bool kLate = TJ == 64;
    auto read_scales = [&](const uint8_t *buf, int ks, int part, f32x4 (&s)[2]) {
        const float *sc = reinterpret_cast<const float *>(buf + kCodes + kP + (GS ? (jrow0 >> 5) * 512 : 0)) + part * 64 + ks * 32 + g * 8;
        s[0] = *reinterpret_cast<const f32x4 *>(sc);
        s[1] = *reinterpret_cast<const f32x4 *>(sc + 4);
    };
    auto read_codes = [&](const uint8_t *buf, int ks) {
        Codes c;
        read_scales(buf, ks, 0, c.scale[0]);
        const int t = ks * 32 + g * 8 + (r >> 1);
#pragma unroll
        for (int f = 0; f < FJ; ++f)
            c.q[f] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                (lds_i32x2 *)(buf + t * TJ + ((((jrow0 >> 4) + f) ^ code_unit_of<TJ>(t)) << 4) + (r & 1) * 8));
        return c;
    };
    // Pair n (0..3) of a fragment's eight codes, times part `part` of their scales.
    auto pair_of = [&](const Codes &c, int f, int n, int part) {
        const f32x4 s = c.scale[part][n >> 1];
        return scaled_pair<T>((uint32_t)c.q[f][n >> 1], n & 1, GS ? s[(n & 1) * 2] : s[(n & 1) * 2] * to,
                              GS ? s[(n & 1) * 2 + 1] : s[(n & 1) * 2 + 1] * to);
    };
    // One half of a step from x (its codes, converted) and the first kAhead fragments
    // of p: each fragment of p is read kAhead groups of matrix instructions before its
    // own, and between the groups the next half's codes are converted and `spread`
    // does a part of other work.  The groups are fenced off from each other: a wave's
    // own vector instructions are the only ones sure to run in the matrix
    // instructions' shadow, and the scheduler gathers them.
    constexpr int kAhead = FI < 3 ? FI : 3;
    auto half = [&](const uint8_t *cur, int ks, const uint8_t *then, u32x4_t (&x)[kParts * FJ], v8 (&ahead)[kAhead],
                    auto spread) {
        v8 y[FI + kAhead];
#pragma unroll
        for (int f = 0; f < kAhead; ++f) y[f] = ahead[f];
        Codes c = read_codes(then, ks ^ 1);
        u32x4_t next[kParts * FJ];
#pragma unroll
        for (int i = 0; i < FI; ++i) {
            const int f = i + kAhead;
            y[f] = f < FI ? read_p(cur, ks, f) : read_p(then, ks ^ 1, f - FI);
            spread(i);
            constexpr int kRest = kLate ? FI - 1 : 0;
            if (kParts > 1 && i == kRest) read_scales(then, ks ^ 1, kParts - 1, c.scale[kParts - 1]);
#pragma unroll
            for (int n = kParts * FJ - 1; n >= 0; --n) {   // (the small products first)
                const int j = FJ - 1 - n % FJ, part = n / FJ;
                acc[j][i] = T::mma(__builtin_bit_cast(v8, x[part * FJ + j]), y[i], acc[j][i]);
            }
            // pairs of codes: 4 FJ of each part over the groups after the first
            constexpr int kPairs = 4 * FJ * kParts, kGroups = FI > 1 ? FI - 1 : 1, kFirst = FI > 1 ? 1 : 0;
#pragma unroll
            for (int n = (i - kFirst) * kPairs / kGroups; n < (i - kFirst + 1) * kPairs / kGroups; ++n) {
                if (n < 0 || i < kFirst) continue;
                const int part = kLate ? n / (4 * FJ) : n % kParts, pair = kLate ? n % (4 * FJ) : n / kParts;
                const int k = part * FJ + (pair >> 2);
                next[k][pair & 3] = pair_of(c, pair >> 2, pair & 3, part);
                asm volatile("" : "+v"(next[k][pair & 3]));   // here, not where the value is next used
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int f = 0; f < kParts * FJ; ++f) x[f] = next[f];
#pragma unroll
        for (int f = 0; f < kAhead; ++f) ahead[f] = y[FI + f];
    };
#pragma unroll
    for (int m = 0; m < kStages - 1; ++m) {
        const Words q = words_here();
#pragma unroll
        for (int n = 0; n < kCopies; ++n) copy(n, s0 + m, q, smem + m * kStage);
        move_on();
    }
    Units units[kStages - 1];
    if constexpr (kFetches > 0)
#pragma unroll
        for (int m = 0; m < kStages - 1; ++m) fetch(s0 + m, units[m]);
    // (found while those are on their way; the last buffer is free until the first step)
    if constexpr (GS > 0) {
        // that of the wave's own 32 columns, which no other column's scale concerns: the waves
        // of the same columns take 64 rows of t each in turn
        constexpr int kSame = WI * KS, kDeep = 4;   // loads at once; past the end the last one again
        const int which = group * WI + wave % WI;
        uint32_t m = 0;
        if constexpr (!__is_same(T, BF16))
            for (int t0 = begin * 64 + which * 64; t0 < t_end; t0 += 64 * kSame * kDeep)
#pragma unroll
                for (int n = 0; n < kDeep; ++n)
                    m = max(m, finite_size(scale_value<GS>(groups, group_scale(min(t0 + n * 64 * kSame + lane, t_end - 1)))));
        scale_window<T, kSame>(m, which, reinterpret_cast<uint32_t *>(all_smem + (kStages - 1) * kStage) + wave / WI * kSame, to, from);
    } else {
        uint32_t m = 0;
        if constexpr (!__is_same(T, BF16))
            for (int t = begin * 64 + tid; t < t_end; t += kThreads) m = max(m, finite_size(a.b.scale[t]));
        scale_window<T, kWaves>(m, wave, reinterpret_cast<uint32_t *>(smem + (kStages - 1) * kStage), to, from);
    }
    if constexpr (WB == 4) to *= 0.0625f;
    if constexpr (kFetches > 0) {
#pragma unroll
        for (int m = 0; m < kStages - 1; ++m) put(s0 + m, units[m], smem + m * kStage);
        copies_left<0>();
#pragma unroll
        for (int m = 0; m < kFlight; ++m) fetch(s0 + kStages - 1 + m, units[m]);
    } else {
        copies_left<kCopies *(kStages - 2)>();
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    u32x4_t x[kParts * FJ];
    v8 ahead[kAhead];
    {
        Codes c = read_codes(smem, 0);
        if (kParts > 1) read_scales(smem, 0, kParts - 1, c.scale[kParts - 1]);
#pragma unroll
        for (int f = 0; f < kParts * FJ; ++f)
#pragma unroll
            for (int n = 0; n < 4; ++n) x[f][n] = pair_of(c, f % FJ, n, f / FJ);
#pragma unroll
        for (int f = 0; f < kAhead; ++f) ahead[f] = read_p(smem, 0, f);
    }
    int at = 0;
    auto step = [&](int s, Units &q_units) {
        const int after = at + 1 == kStages ? 0 : at + 1, fill = at == 0 ? kStages - 1 : at - 1;
        uint8_t *cur = smem + at * kStage, *then = smem + after * kStage, *last = smem + fill * kStage;
        half(cur, 0, cur, x, ahead, [](int) {});
        // The next step's copies have landed (each step issues its copies and then its
        // fetches: all that came later may be on the way), and everyone is done with
        // the step before this one.
        if (kFetches > 0 && narrow) copies_left<0>();
        else copies_left<kFetches + (kStages - 3) * (kCopies + kFetches)>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (past the last step these go to a buffer that is not multiplied)
        const int far = s + kStages - 1;
        const Words q = words_here();
        move_on();
        half(cur, 1, then, x, ahead, [&](int i) {
            if (i == 0) put(far, q_units, last);   // (before this step's copies: it waits for older loads only)
#pragma unroll
            for (int n = i * kCopies / FI; n < (i + 1) * kCopies / FI; ++n) copy(n, far, q, last);
            if (i == FI - 1) fetch(far + kFlight, q_units);
        });
        at = after;
    };
    for (int s = s0; s < s1; s += kFlight) {
        step(s, units[0]);
        if (kFlight == 2 && s + 1 < s1) step(s + 1, units[kFlight - 1]);
    }
    copies_done();   // none may land in the LDS of a workgroup that comes after
    if constexpr (KS > 1) {
        static_assert(FJ * FI * kThreads * 16 <= kGradStages * kStage);
        __syncthreads();   // nor where the groups' sums meet
        auto part = [&](int from, int f) {
            return reinterpret_cast<f32x4 *>(all_smem + from * (kGradStages * kStage)) + f * kThreads + tid;
        };
        if (group)
#pragma unroll
            for (int j = 0; j < FJ; ++j)
#pragma unroll
                for (int i = 0; i < FI; ++i) *part(group, j * FI + i) = acc[j][i];
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int from = 1; from < KS; ++from)
#pragma unroll
            for (int j = 0; j < FJ; ++j)
#pragma unroll
                for (int i = 0; i < FI; ++i) acc[j][i] += *part(from, j * FI + i);
    }
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
            } else if constexpr (TRANSPOSED) {
                store4(static_cast<float *>(a.out) + (int64_t)row * a.ldo + col, d, a.nj - col);
            } else {
                store4<T>(static_cast<elem *>(a.out) + (int64_t)row * a.ldo + col, d, a.nj - col);
            }
        }
    }
}

// Tile and split of a workgroup of tiles_i * tiles_j * splits.
struct GradPlace {
    int split, ti, tj;
};
__device__ __forceinline__ GradPlace grad_place(const GradArgs &a) {
    const int tiles = a.tiles_i * a.tiles_j;
    GradPlace p;
    p.split = (int)blockIdx.x / tiles;
    tile_at(xcd_run((int)blockIdx.x - p.split * tiles, tiles), a.tiles_i, a.tiles_j, p.ti, p.tj);
    return p;
}

template <class T, int WB, bool TRANSPOSED, bool COPY, int TJ, int TI, int WJ, int WI, int KS>
__global__ void __launch_bounds__(KS *WJ *WI * 64) grad_tile(GradArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t all_smem[];
    const GradPlace p = grad_place(a);
    grad_product<T, WB, TRANSPOSED, COPY, 0, TJ, TI, WJ, WI, KS>(a, GroupArg{}, p.split, p.ti, p.tj, all_smem);
}

// Adds the partial sums in the order of the splits and rounds once: four columns a
// thread.  Bound by reading them: 16 splits of 1024 x 1024, 64 MiB, take 12 us (15 with
// eight loads at once); 32 splits of 34 x 512, few enough for their waits to show, 4.2
// with eight loads at once, 10.4 one by one.  (Where there are splits, the plan keeps ni
// times nj below 2^28.)
template <class Out>
__global__ void __launch_bounds__(256) grad_sum(GradArgs a) {
    const uint32_t at = blockIdx.x * 256u + threadIdx.x, quads = (uint32_t)a.ldpart / 4, row = at / quads;
    if (row >= (uint32_t)a.ni) return;
    const int col = (int)(at - row * quads) * 4;
    const float *p = a.part + (int64_t)row * a.ldpart + col;
    const int64_t stride = (int64_t)a.ni * a.ldpart;
    f32x4 t = *reinterpret_cast<const f32x4 *>(p);
    int s = 1;
    if (a.splits > 16)   // few results
        for (; s + 8 <= a.splits; s += 8) {
            f32x4 v[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) v[n] = *reinterpret_cast<const f32x4 *>(p + (s + n) * stride);
#pragma unroll
            for (int n = 0; n < 8; ++n) t += v[n];
        }
    for (; s < a.splits; ++s) t += *reinterpret_cast<const f32x4 *>(p + s * stride);
    Out *out = static_cast<Out *>(a.out) + (int64_t)row * a.ldo + col;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (col + e < a.nj) out[e] = (Out)t[e];
}

}  // namespace qconv

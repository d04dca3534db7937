// Root-mean-square norm with the residual's addition, its output as 8-bit rows, and
// its gradient.
//   h = x + residual, rounded to their type;  r = (mean h^2 + eps)^(-1/2);  y = h r gain
//   codes and scale of y as of any quantised row (least e with max |y| <= 127 * 2^e)
//
// A code depends on which side of a half y / 2^e lies, so y's own rounding must not
// decide it: the sum of squares and r are formed in 64 bits, y in 32, and a y / 2^e
// within 2^-14 of a half (32 bits are off by 127 * 3 * 2^-24 = 2^-15.4 at most) is formed
// again in 64.  A row whose largest |y| lies that near to 127 * 2^e, or where 32 bits
// leave their normal range, is done in 64 bits as a whole.  What is still within 2^-30 of a
// half or a border is h gain, exact, divided by (mean h^2 + eps)^(1/2), a quotient, a root
// and a quotient again that are each rounded once: values that lie there in earnest are met
// exactly wherever the mean of squares is a number of 64 bits (products with the
// reciprocals of c and of the root missed half of those in rows of one magnitude).  So
// codes are those of the definition, whatever the order of the sums.
#include "qlinear_rows.h"

namespace qconv {

namespace {

// Eight gains from element `at`, of any of the three types (the branch is uniform).
struct RawGain {
    u32x4_t w[2];
};
__device__ __forceinline__ RawGain fetch_gain(const void *gain, int dtype, int at, int c) {
    RawGain g;
    if (dtype == QCONV_F32) {
        const Raw8<float> q = fetch8(static_cast<const float *>(gain), at, c);
        g.w[0] = __builtin_bit_cast(u32x4_t, q.w[0]), g.w[1] = __builtin_bit_cast(u32x4_t, q.w[1]);
    } else {
        g.w[0] = __builtin_bit_cast(u32x4_t, fetch8(static_cast<const _Float16 *>(gain), at, c).w[0]);
        g.w[1] = g.w[0];
    }
    return g;
}
__device__ __forceinline__ void unpack_gain(const RawGain &q, int dtype, int at, int c, float (&g)[8]) {
    if (dtype == QCONV_F32) unpack8(__builtin_bit_cast(Raw8<float>, q), at, c, g);
    else if (dtype == QCONV_BF16) unpack8(__builtin_bit_cast(Raw8<__bf16>, q.w[0]), at, c, g);
    else unpack8(__builtin_bit_cast(Raw8<_Float16>, q.w[0]), at, c, g);
}
__device__ __forceinline__ void load_gain(const void *gain, int dtype, int at, int c, float (&g)[8]) {
    unpack_gain(fetch_gain(gain, dtype, at, c), dtype, at, c, g);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// 1 / sqrt(x) to some 2^-52, for r: the instruction's 2^-26 or so, and two steps of Newton's
// method.
__device__ __forceinline__ double inverse_root(double x) {
    double y = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int n = 0; n < 2; ++n) y = __builtin_fma(0.5 * y, __builtin_fma(-x * y, y, 1.0), y);
    return y;
}

// x / 2^e to the nearest whole number, ties to even (|x| <= 127 * 2^e).
__device__ __forceinline__ int round_wide(double x, int e) { return (int)__builtin_rint(__builtin_ldexp(x, -e)); }

// Where 32 bits leave their normal range, or nearly: of a row's largest value.
__device__ __forceinline__ bool extreme(uint32_t m) { return m < 0x06000000u || m >= 0x7f000000u; }

// WAVES waves of a workgroup of four to each row (1: four rows a workgroup), KEEP vectors
// of eight values a lane in registers; longer rows read the rest again.  Between the row's
// loads and its codes lies one sum over its lanes: y's largest value is r times that of
// h gain.  Bound by memory: 8192 x 4096 bf16 with a residual take 47 us, 5.0 TB/s; of 16
// rows 4.7, a launch and one wait for memory.
template <class In, bool ADD, int WAVES, int KEEP>
__global__ void __launch_bounds__(256, WAVES == 1 && KEEP < 4 ? 6 : 1) norm_to_rows(NormArgs a) {
    constexpr int kLanes = WAVES * 64, kRows = 4 / WAVES, kNext = kLanes * 8;
    __shared__ double part[4];
    __shared__ uint32_t most[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? wave : 0);
    const bool mine = row < a.m;
    const int64_t at_row = mine ? row : 0;
    const In *x = static_cast<const In *>(a.x) + at_row * a.ldx;
    const In *residual = ADD ? static_cast<const In *>(a.residual) + at_row * a.ldr : nullptr;
    In *sum = ADD ? static_cast<In *>(a.sum) + at_row * a.lds : nullptr;
    const int at0 = (WAVES == 1 ? lane : (int)threadIdx.x) * 8;
    const int c = mine ? a.c : 0, whole = (c + 15) & ~15;

    // Eight values of h.  Their first visit writes them where there is a residual, any
    // other reads them there (the sum may lie in the residual's or x's own place).
    struct First {
        Raw8<In> x, residual;
        RawGain gain;
    };
    const auto fetch = [&](int at, First &q) {
        q.x = fetch8(x, at, a.c);
        if constexpr (ADD) q.residual = fetch8(residual, at, a.c);
        q.gain = fetch_gain(a.gain, a.gain_dtype, at, a.c);
    };
    const auto first = [&](int at, const First &q, float (&h)[8], float (&g)[8]) {
        unpack8(q.x, at, a.c, h);
        unpack_gain(q.gain, a.gain_dtype, at, a.c, g);
        if constexpr (ADD) {
            float s[8];
            unpack8(q.residual, at, a.c, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = (float)(In)(h[i] + s[i]);
            store8(sum, at, c, h);
        }
    };
    const auto again = [&](int at, float (&h)[8], float (&g)[8]) {
        load8(ADD ? (const In *)sum : x, at, c, h);
        load_gain(a.gain, a.gain_dtype, at, c, g);
    };

    float v[KEEP][8];   // h gain
    double squares = 0;
    uint32_t m = 0;
    const auto take = [&](float (&h)[8], const float (&g)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            squares = __builtin_fma((double)h[i], (double)h[i], squares);
            h[i] *= g[i];
            m = max(m, __builtin_bit_cast(uint32_t, h[i]) & 0x7fffffffu);
        }
    };
    First q[KEEP];
#pragma unroll
    for (int k = 0; k < KEEP; ++k) fetch(at0 + k * kNext, q[k]);
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        float g[8];
        first(at0 + k * kNext, q[k], v[k], g);
        if (!mine)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = 0.0f;
        take(v[k], g);
    }
    for (int at = at0 + KEEP * kNext; at < c; at += kNext) {
        First more;
        float h[8], g[8];
        fetch(at, more);
        first(at, more, h, g);
        take(h, g);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        squares += __shfl_xor(squares, d);
        m = max(m, (uint32_t)__shfl_xor((int)m, d));
    }
    if constexpr (WAVES > 1) {
        if (lane == 0) part[wave] = squares, most[wave] = m;
        __syncthreads();
        squares = (part[0] + part[1]) + (part[2] + part[3]);
        m = max(max(most[0], most[1]), max(most[2], most[3]));
    }
    const double r_wide = inverse_root(squares * a.inv_c + a.eps);
    const float r = (float)r_wide;
    const uint32_t top = __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, m) * r);

    uint8_t *out = a.codes + at_row * a.pitch;
    const auto put = [&](int at, const uint32_t (&q)[8]) {   // the low bytes
        *reinterpret_cast<uint2 *>(out + at) =
            uint2{__builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0c0c0400u), __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u), 0x05040100u),
                  __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[7], q[6], 0x0c0c0400u), __builtin_amdgcn_perm(q[5], q[4], 0x0c0c0400u), 0x05040100u)};
    };
    // top = 1.f * 2^p: e = p - 6 where 1.f <= 127 / 64, else p - 5
    const int from_border = (int)(top & 0x7fffffu) - 0x7e0000;
    const bool narrow = squares != 0 ? !extreme(m) && !extreme(top) && (from_border < -16 || from_border > 16) && r > 0x1p-120f && r < 0x1p120f
                                     : m == 0 && r < 0x1p120f;
    float scale;
    int e = -126;
    uint32_t any = 0;      // values that are not finite floats
    bool wide = !narrow;   // the lane's codes are to be quotients in 64 bits
    if (narrow) {
        e = max((int)(top >> 23) - 6 + (from_border > 0), 1) - 127;
        scale = m == 0 ? 0.0f : __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
        const float inv = m == 0 ? 0.0f : r * __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);   // r / 2^e
        // Adding 1.5 * 2^23 rounds to a whole number, ties to even, and leaves its two's
        // complement in the low bits.
        const auto round8 = [&](int at, const float (&p)[8]) {
            if (at >= whole) return;
            uint32_t q[8];
            float worst = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = p[i] * inv, b = t + 12582912.0f;
                worst = __builtin_fmaxf(worst, __builtin_fabsf(t - (b - 12582912.0f)));
                q[i] = __builtin_bit_cast(uint32_t, b);
            }
            if (worst > 0.5f - 0x1p-14f) {
                float h[8], g[8];
                again(at, h, g);
                // (products are off by 2^-42 at most; a quotient takes ten times as long)
                double near = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double t = __builtin_ldexp((double)h[i] * (double)g[i] * r_wide, -e), b = __builtin_rint(t);
                    near = __builtin_fmax(near, __builtin_fabs(t - b));
                    q[i] = (uint32_t)(int)b;
                }
                wide = wide || near > 0.5 - 0x1p-30;
            }
            put(at, q);
        };
#pragma unroll
        for (int k = 0; k < KEEP; ++k) round8(at0 + k * kNext, v[k]);
        for (int at = at0 + KEEP * kNext; at < whole; at += kNext) {
            float h[8], g[8];
            again(at, h, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] *= g[i];
            round8(at, h);
        }
    } else {
        const double root = __builtin_sqrt(squares / (double)a.c + a.eps);
        double most_wide = 0;
        bool bad = false;
        for (int at = at0; at < c; at += kNext) {
            float h[8], g[8];
            again(at, h, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double y = __builtin_fabs((double)h[i] * (double)g[i] / root);
                bad = bad || !(y <= (double)__FLT_MAX__);   // (a NaN too)
                most_wide = y > most_wide ? y : most_wide;
            }
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const double other = __shfl_xor(most_wide, d);
            most_wide = other > most_wide ? other : most_wide;
        }
        any = __any(bad) ? 1u : 0u;
        if constexpr (WAVES > 1) {
            __syncthreads();   // the sums before have been read
            if (lane == 0) part[wave] = most_wide, most[wave] = any;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                most_wide = part[w] > most_wide ? part[w] : most_wide;
                any |= most[w];
            }
        }
        if (most_wide > 0 && !any) {
            const int p = (int)(__builtin_bit_cast(uint64_t, most_wide) >> 52) - 1023;
            e = max(p - 6 + (most_wide > 127.0 * __builtin_ldexp(1.0, p - 6)), -126);
        }
        scale = any ? __builtin_nanf("") : most_wide == 0 ? 0.0f : __builtin_ldexpf(1.0f, e);
    }
    if (wide) {
        const double root = __builtin_sqrt(squares / (double)a.c + a.eps);
        for (int at = at0; at < whole; at += kNext) {
            float h[8], g[8];
            again(at, h, g);
            uint32_t q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = any ? 0u : (uint32_t)round_wide((double)h[i] * (double)g[i] / root, e);
            put(at, q);
        }
    }
    if (mine && at0 == 0) {
        a.scale[row] = scale;
        if (a.rstd) a.rstd[row] = r;
    }
}

template <class In, bool ADD, int WAVES, int KEEP>
hipError_t launch_norm(const NormArgs &a, hipStream_t stream) {
    constexpr int kRows = 4 / WAVES;
    NormArgs s = a;
    launch_slices(((int64_t)a.m + kRows - 1) / kRows, 256, [&](long long first, unsigned count) {
        const int64_t row = first * kRows;
        s.x = static_cast<const In *>(a.x) + row * a.ldx;
        if (ADD) s.residual = static_cast<const In *>(a.residual) + row * a.ldr;
        if (ADD) s.sum = static_cast<In *>(a.sum) + row * a.lds;
        s.codes = a.codes + row * a.pitch;
        s.scale = a.scale + row;
        s.rstd = a.rstd ? a.rstd + row : nullptr;
        s.m = (int32_t)(a.m - row);
        hipLaunchKernelGGL((norm_to_rows<In, ADD, WAVES, KEEP>), dim3(count), dim3(256), 0, stream, s);
    });
    return hipGetLastError();
}

template <class In, bool ADD>
hipError_t launch_norm(const NormArgs &a, hipStream_t stream) {
    // A wave holds rows of up to 2048 values, a workgroup of four longer ones.
    if (a.c <= 512) return launch_norm<In, ADD, 1, 1>(a, stream);
    if (a.c <= 1024) return launch_norm<In, ADD, 1, 2>(a, stream);
    if (a.c <= 2048) return launch_norm<In, ADD, 1, 4>(a, stream);
    if (a.c <= 4096) return launch_norm<In, ADD, 4, 2>(a, stream);
    return launch_norm<In, ADD, 4, 4>(a, stream);
}

// ---------------------------------------------------------------- gradient
//
// With t = dy gain, n = h r and z_m = sum_c t n / c:
//   dx = r (t - n z) (+ dsum),   dgain_c = sum_m dy n
// (rounding to codes is taken as the identity).  Sums are 32-bit; formed from n, they
// stay in range wherever the results do.

// WAVES waves take a row, ROWS rows side by side in a workgroup, which goes through the
// rows in steps of the whole grid, the next row's loads on their way.  A thread keeps its
// eight columns for all of them: the gain and dgain's sums stay in registers, and those go
// to the workspace once a workgroup.  Columns past the threads' own are read a second time,
// and their sums of dgain are added up in the workgroup's row of the workspace (LONG).
// Bound by memory: 8192 x 4096 bf16 with dsum take 55 us in all, 4.8 TB/s.
constexpr int backward_threads(int waves) { return waves == 16 ? 1024 : 512; }
template <class In, int WAVES, bool LONG>
__global__ void __launch_bounds__(backward_threads(WAVES)) norm_backward(NormGradArgs a) {
    constexpr int kNext = WAVES * 512, ROWS = backward_threads(WAVES) / 64 / WAVES;
    __shared__ float part[2][ROWS * WAVES];
    __shared__ float other[ROWS > 1 ? ROWS - 1 : 1][ROWS > 1 ? kNext : 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, which = wave / WAVES;
    const int at0 = ((int)threadIdx.x - which * WAVES * 64) * 8, c = a.c;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    // (a wave whose columns all lie past the row's end takes part in its barriers alone)
    const bool busy = __builtin_amdgcn_readfirstlane(at0) < c;
    float sums[8], gain[8];
    if (busy) load_gain(a.gain, a.gain_dtype, at0, c, gain);
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[i] = 0.0f;
    float *mine = a.part + (int64_t)blockIdx.x * a.ldpart;
    struct Row {
        Raw8<In> dy, h, dsum;
        float r;
    };
    const auto fetch = [&](int64_t row, Row &q) {
        q.r = a.rstd[row];
        q.dy = fetch8(static_cast<const In *>(a.dy) + row * a.lddy, at0, c);
        q.h = fetch8(static_cast<const In *>(a.h) + row * a.ldh, at0, c);
        if (a.dsum) q.dsum = fetch8(static_cast<const In *>(a.dsum) + row * a.ldds, at0, c);
    };
    bool fresh = true;
    int turn = 0;
    const int64_t first = (int64_t)blockIdx.x * ROWS;
    // (where none is left: the last row again, for nothing)
    const auto row_at = [&](int64_t row0) { return min(row0 + which, (int64_t)a.m - 1); };
    Row ahead;
    if (busy) fetch(row_at(first), ahead);
    for (int64_t row0 = first; row0 < a.m; row0 += stride, turn ^= 1) {
        const int64_t row = row_at(row0);
        const bool in = row0 + which < a.m;
        const Row now = ahead;
        const float r = now.r;
        float t[8], n[8], s = 0;   // dy gain and h r
        if (busy) {
            fetch(row_at(row0 + stride), ahead);
            unpack8(now.dy, at0, c, t);
            unpack8(now.h, at0, c, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[i] *= r;
                if (in) sums[i] = __builtin_fmaf(t[i], n[i], sums[i]);
                t[i] *= gain[i];
                s = __builtin_fmaf(t[i], n[i], s);
            }
        }
        const auto load = [&](int at, float (&dy)[8], float (&h)[8], float (&g)[8]) {
            load8(static_cast<const In *>(a.dy) + row * a.lddy, at, c, dy);
            load8(static_cast<const In *>(a.h) + row * a.ldh, at, c, h);
            load_gain(a.gain, a.gain_dtype, at, c, g);
        };
        if constexpr (LONG) {
            for (int at = at0 + kNext; at < c; at += kNext) {
                float p[8], q[8], g[8], old[8];
                load(at, p, q, g);
                load8((const float *)mine, at, c, old);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q[i] *= r;
                    old[i] = __builtin_fmaf(p[i], q[i], fresh ? 0.0f : old[i]);
                    s = __builtin_fmaf(p[i] * g[i], q[i], s);
                }
                store8(mine, at, c, old);
            }
            fresh = false;
        }
        if (busy) s = wave_sum(s);
        if constexpr (WAVES > 1) {
            if (lane == 0) part[turn][wave] = s;
            __syncthreads();   // (the other half of `part` is free: everyone has passed this barrier since it was read)
            s = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) s += part[turn][which * WAVES + w];
        }
        if (!in || !busy) continue;
        const float z = s / (float)c;
        const auto give = [&](int at, const float (&p)[8], const float (&q)[8], const Raw8<In> &add) {
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = r * __builtin_fmaf(-q[i], z, p[i]);
            if (a.dsum) {
                float more[8];
                unpack8(add, at, c, more);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] += more[i];
            }
            store8(static_cast<In *>(a.dx) + row * a.lddx, at, c, d);
        };
        give(at0, t, n, now.dsum);
        if constexpr (LONG)
            for (int at = at0 + kNext; at < c; at += kNext) {
                float p[8], q[8], g[8];
                load(at, p, q, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] *= g[i], q[i] *= r;
                Raw8<In> add{};
                if (a.dsum) add = fetch8(static_cast<const In *>(a.dsum) + row * a.ldds, at, c);
                give(at, p, q, add);
            }
    }
    if constexpr (ROWS > 1) {
        if (which)
#pragma unroll
            for (int i = 0; i < 8; ++i) other[which - 1][at0 + i] = sums[i];
        __syncthreads();
        if (which) return;
#pragma unroll
        for (int n = 0; n < ROWS - 1; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[i] += other[n][at0 + i];
    }
    store8(mine, at0, c, sums);
}

// dgain: the workgroups' sums, 32 columns a workgroup: 32 runs of them, added up in their
// order, meet by halves.
__global__ void __launch_bounds__(256) norm_gain_sum(NormGradArgs a) {
    __shared__ f32x4 part[4][8];
    const int quad = threadIdx.x & 7, run = threadIdx.x >> 3, wave = threadIdx.x >> 6;
    const int col = (int)blockIdx.x * 32 + quad * 4;
    const int per = (a.parts + 31) / 32, begin = run * per, end = min(begin + per, a.parts);
    f32x4 t{0, 0, 0, 0};
    if (col < a.c)
#pragma unroll 8
        for (int n = begin; n < end; ++n) t += *reinterpret_cast<const f32x4 *>(a.part + (int64_t)n * a.ldpart + col);
#pragma unroll
    for (int d = 8; d < 64; d <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] += __shfl_xor(t[i], d);
    if ((threadIdx.x & 63) < 8) part[wave][quad] = t;
    __syncthreads();
    if (threadIdx.x >= 8) return;
    t = (part[0][quad] + part[1][quad]) + (part[2][quad] + part[3][quad]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < a.c) a.dgain[col + i] = t[i];
}

template <class In, int WAVES, bool LONG = false>
hipError_t launch_backward(const NormGradArgs &a, hipStream_t stream) {
    if (a.parts) hipLaunchKernelGGL((norm_backward<In, WAVES, LONG>), dim3((unsigned)a.parts),
                                    dim3(backward_threads(WAVES)), 0, stream, a);
    hipLaunchKernelGGL(norm_gain_sum, dim3((unsigned)((a.c + 31) / 32)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

template <class In>
hipError_t launch_grad_of(const NormGradArgs &a, hipStream_t stream) {
    switch (norm_grad_waves(a.c)) {
        case 1: return launch_backward<In, 1>(a, stream);
        case 2: return launch_backward<In, 2>(a, stream);
        case 4: return launch_backward<In, 4>(a, stream);
        case 8: return launch_backward<In, 8>(a, stream);
        default: return a.c <= 8192 ? launch_backward<In, 16>(a, stream) : launch_backward<In, 16, true>(a, stream);
    }
}

}  // namespace

int norm_grad_waves(int64_t c) { return c <= 512 ? 1 : c <= 1024 ? 2 : c <= 2048 ? 4 : c <= 4096 ? 8 : 16; }
int norm_grad_parts(int64_t m, int64_t c) {
    // the workgroups that the CUs hold at once (their loads a row ahead fill the memory), of
    // four turns each at least, so that dgain's partial sums stay few beside the rows; of few
    // rows, one turn each
    const int64_t waves = norm_grad_waves(c), rows = waves == 16 ? 1 : 8 / waves, turns = (m + rows - 1) / rows;
    const int64_t most = waves == 16 ? 256 : 512, parts = turns / 4 > 64 ? turns / 4 : 64;
    return (int)(turns < parts ? turns : parts < most ? parts : most);
}

hipError_t launch_norm_rows(const NormArgs &a, int dtype, hipStream_t stream) {
    switch (dtype) {
        case QCONV_BF16: return a.residual ? launch_norm<__bf16, true>(a, stream) : launch_norm<__bf16, false>(a, stream);
        case QCONV_F16: return a.residual ? launch_norm<_Float16, true>(a, stream) : launch_norm<_Float16, false>(a, stream);
        default: return a.residual ? launch_norm<float, true>(a, stream) : launch_norm<float, false>(a, stream);
    }
}

hipError_t launch_norm_grad(const NormGradArgs &a, int dtype, hipStream_t stream) {
    switch (dtype) {
        case QCONV_BF16: return launch_grad_of<__bf16>(a, stream);
        case QCONV_F16: return launch_grad_of<_Float16>(a, stream);
        default: return launch_grad_of<float>(a, stream);
    }
}

}  // namespace qconv

// Root-mean-square norm with the residual's addition, its output as 8-bit rows, and
// its gradient.
//   h = x + residual, rounded to their type;  r = (mean h^2 + eps)^(-1/2);  y = h r gain
//   codes and scale of y as of any quantised row (least e with max |y| <= 127 * 2^e)
//
// A code depends on which side of a half y / 2^e lies, so y's own rounding must not
// decide it: the sum of squares and r are formed in 64 bits, y in 32, and a y / 2^e
// within 2^-14 of a half (32 bits are off by 127 * 3 * 2^-24 = 2^-15.4 at most) is formed
// again in 64.  A row whose largest |y| lies that near to 127 * 2^e, or where 32 bits
// leave their normal range, is done in 64 bits as a whole.  So codes are those of the
// definition, whatever the order of the sums.
#include "qlinear_rows.h"

namespace qconv {

namespace {

// Eight gains from element `at`, of any of the three types (the branch is uniform).
__device__ __forceinline__ void load_gain(const void *gain, int dtype, int at, int c, float (&g)[8]) {
    if (dtype == QCONV_F32) load8(static_cast<const float *>(gain), at, c, g);
    else if (dtype == QCONV_BF16) load8(static_cast<const __bf16 *>(gain), at, c, g);
    else load8(static_cast<const _Float16 *>(gain), at, c, g);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// x / 2^e to the nearest whole number, ties to even (|x| <= 127 * 2^e).
__device__ __forceinline__ int round_wide(double x, int e) { return (int)__builtin_rint(__builtin_ldexp(x, -e)); }

// WAVES waves of a workgroup of four to each row (1: four rows a workgroup), KEEP vectors
// of eight values a lane in registers; longer rows read the rest again.
template <class In, bool ADD, int WAVES, int KEEP>
__global__ void __launch_bounds__(256) norm_to_rows(NormArgs a) {
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

    // Eight values of h.  Their first visit writes them where there is a residual, the
    // second reads them there (the sum may lie in the residual's or x's own place).
    const auto first = [&](int at, float (&h)[8]) {
        load8(x, at, c, h);
        if constexpr (ADD) {
            float s[8];
            load8(residual, at, c, s);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = (float)(In)(h[i] + s[i]);
            store8(sum, at, c, h);
        }
    };
    const auto again = [&](int at, float (&h)[8]) { load8(ADD ? (const In *)sum : x, at, c, h); };

    float v[KEEP][8];
    double squares = 0;
    const auto add_squares = [&](const float (&h)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) squares = __builtin_fma((double)h[i], (double)h[i], squares);
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k) {
        if (at0 + k * kNext < c) first(at0 + k * kNext, v[k]);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < KEEP; ++k) add_squares(v[k]);
    for (int at = at0 + KEEP * kNext; at < c; at += kNext) {
        float h[8];
        first(at, h);
        add_squares(h);
    }
    squares = wave_sum(squares);
    if constexpr (WAVES > 1) {
        if (lane == 0) part[wave] = squares;
        __syncthreads();
        squares = (part[0] + part[1]) + (part[2] + part[3]);
    }
    const double r_wide = 1.0 / __builtin_sqrt(squares / (double)a.c + a.eps);
    const float r = (float)r_wide;

    // Every vector of the row: its place, its values.
    const auto each = [&](auto visit) {
#pragma unroll
        for (int k = 0; k < KEEP; ++k) visit(at0 + k * kNext, v[k]);
        for (int at = at0 + KEEP * kNext; at < whole; at += kNext) {
            float h[8];
            again(at, h);
            visit(at, h);
        }
    };
    uint32_t m = 0;
    each([&](int at, const float (&h)[8]) {
        if (at >= c) return;
        float g[8];
        load_gain(a.gain, a.gain_dtype, at, c, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, h[i] * r * g[i]) & 0x7fffffffu);
    });
#pragma unroll
    for (int d = 32; d; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    if constexpr (WAVES > 1) {
        if (lane == 0) most[wave] = m;
        __syncthreads();
        m = max(max(most[0], most[1]), max(most[2], most[3]));
    }
    uint8_t *out = a.codes + at_row * a.pitch;
    const auto put = [&](int at, const int (&q)[8]) {
        if (at >= whole) return;
        uint2 w{0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) w.x |= (uint32_t)(q[i] & 255) << (8 * i), w.y |= (uint32_t)(q[i + 4] & 255) << (8 * i);
        *reinterpret_cast<uint2 *>(out + at) = w;
    };
    // m = 1.f * 2^p: e = p - 6 where 1.f <= 127 / 64, else p - 5
    const int from_border = (int)(m & 0x7fffffu) - 0x7e0000;
    const bool doubtful = (from_border > -16 && from_border < 16) || (m < 0x06000000u && squares != 0) || m >= 0x7f000000u ||
                          !(r > 0x1p-120f && r < 0x1p120f);
    float scale;
    if (!doubtful) {
        const int e = max((int)(m >> 23) - 6 + (from_border > 0), 1) - 127;
        scale = m == 0 ? 0.0f : __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
        const float inv = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
        each([&](int at, const float (&h)[8]) {
            if (at >= whole) return;
            float g[8];
            load_gain(a.gain, a.gain_dtype, at, c, g);
            int q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float t = h[i] * r * g[i] * inv, n = __builtin_rintf(t);
                q[i] = (int)n;
                if (__builtin_fabsf(t - n) > 0.5f - 0x1p-14f) q[i] = round_wide((double)h[i] * r_wide * (double)g[i], e);
            }
            put(at, q);
        });
    } else {
        double top = 0;
        bool bad = false;
        each([&](int at, const float (&h)[8]) {
            if (at >= c) return;
            float g[8];
            load_gain(a.gain, a.gain_dtype, at, c, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double y = __builtin_fabs((double)h[i] * r_wide * (double)g[i]);
                bad = bad || !(y <= (double)__FLT_MAX__);   // (a NaN too)
                top = y > top ? y : top;
            }
        });
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const double other = __shfl_xor(top, d);
            top = other > top ? other : top;
        }
        uint32_t any = __any(bad) ? 1u : 0u;
        if constexpr (WAVES > 1) {
            __syncthreads();   // the sums before have been read
            if (lane == 0) part[wave] = top, most[wave] = any;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                top = part[w] > top ? part[w] : top;
                any |= most[w];
            }
        }
        int e = -126;
        if (top > 0 && !any) {
            const int p = (int)((uint64_t)__builtin_bit_cast(uint64_t, top) >> 52) - 1023;
            e = max(p - 6 + (top > 127.0 * __builtin_ldexp(1.0, p - 6)), -126);
        }
        scale = any ? __builtin_nanf("") : top == 0 ? 0.0f : __builtin_ldexpf(1.0f, e);
        each([&](int at, const float (&h)[8]) {
            if (at >= whole) return;
            float g[8];
            load_gain(a.gain, a.gain_dtype, at, c, g);
            int q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = any ? 0 : round_wide((double)h[i] * r_wide * (double)g[i], e);
            put(at, q);
        });
    }
    if (mine && at0 == 0) {
        a.scale[row] = scale;
        if (a.rstd) a.rstd[row] = r;
    }
}

template <class In, bool ADD>
hipError_t launch_norm(const NormArgs &a, hipStream_t stream) {
    // A wave holds rows of up to 2048 values, a workgroup of four longer ones.
    NormArgs s = a;
    const bool wide = a.c > 2048;
    const int64_t blocks = wide ? a.m : ((int64_t)a.m + 3) / 4;
    launch_slices(blocks, 256, [&](long long first, unsigned count) {
        const int64_t row = first * (wide ? 1 : 4);
        s.x = static_cast<const In *>(a.x) + row * a.ldx;
        if (ADD) s.residual = static_cast<const In *>(a.residual) + row * a.ldr;
        if (ADD) s.sum = static_cast<In *>(a.sum) + row * a.lds;
        s.codes = a.codes + row * a.pitch;
        s.scale = a.scale + row;
        s.rstd = a.rstd ? a.rstd + row : nullptr;
        s.m = (int32_t)(a.m - row);
        if (wide)
            hipLaunchKernelGGL((norm_to_rows<In, ADD, 4, 4>), dim3(count), dim3(256), 0, stream, s);
        else
            hipLaunchKernelGGL((norm_to_rows<In, ADD, 1, 4>), dim3(count), dim3(256), 0, stream, s);
    });
    return hipGetLastError();
}

// ---------------------------------------------------------------- gradient
//
// With t = dy gain, n = h r and z_m = sum_c t n / c:
//   dx = r (t - n z) (+ dsum),   dgain_c = sum_m dy n
// (rounding to codes is taken as the identity).  Sums are 32-bit; formed from n, they
// stay in range wherever the results do.

// A workgroup takes every gridDim.x-th row: its threads keep the same columns for all of
// them, KEEP vectors of eight each, so that dgain's sums stay in registers and go to the
// workspace once.  Columns past those are read a second time, and their sums of dgain
// are added up in the workgroup's own row of the workspace.
template <class In, int KEEP, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_backward(NormGradArgs a) {
    constexpr int kNext = THREADS * 8, kWaves = THREADS / 64;
    __shared__ float part[2][kWaves];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, at0 = (int)threadIdx.x * 8, c = a.c;
    float sums[KEEP][8];
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[k][i] = 0.0f;
    float *mine = a.part + (int64_t)blockIdx.x * a.ldpart;
    bool fresh = true;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x, turn ^= 1) {
        const In *dy = static_cast<const In *>(a.dy) + row * a.lddy, *h = static_cast<const In *>(a.h) + row * a.ldh;
        const In *dsum = a.dsum ? static_cast<const In *>(a.dsum) + row * a.ldds : nullptr;
        In *dx = static_cast<In *>(a.dx) + row * a.lddx;
        const float r = a.rstd[row];
        float t[KEEP][8], u[KEEP][8], s = 0;
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
            const int at = at0 + k * kNext;
            load8(dy, at, c, t[k]);
            load8(h, at, c, u[k]);
        }
#pragma unroll
        for (int k = 0; k < KEEP; ++k) {
            float g[8];
            load_gain(a.gain, a.gain_dtype, at0 + k * kNext, c, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[k][i] *= r;
                sums[k][i] = __builtin_fmaf(t[k][i], u[k][i], sums[k][i]);
                t[k][i] *= g[i];
                s = __builtin_fmaf(t[k][i], u[k][i], s);
            }
        }
        for (int at = at0 + KEEP * kNext; at < c; at += kNext) {
            float p[8], q[8], g[8], old[8];
            load8(dy, at, c, p);
            load8(h, at, c, q);
            load_gain(a.gain, a.gain_dtype, at, c, g);
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
        s = wave_sum(s);
        if (lane == 0) part[turn][wave] = s;
        __syncthreads();   // (the other half of `part` is free: everyone has passed this barrier since it was read)
        s = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += part[turn][w];
        const float z = s / (float)c;
        const auto give = [&](int at, const float (&p)[8], const float (&q)[8]) {
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = r * __builtin_fmaf(-q[i], z, p[i]);
            if (dsum) {
                float more[8];
                load8(dsum, at, c, more);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] += more[i];
            }
            store8(dx, at, c, d);
        };
#pragma unroll
        for (int k = 0; k < KEEP; ++k)
            if (at0 + k * kNext < c) give(at0 + k * kNext, t[k], u[k]);
        for (int at = at0 + KEEP * kNext; at < c; at += kNext) {
            float p[8], q[8], g[8];
            load8(dy, at, c, p);
            load8(h, at, c, q);
            load_gain(a.gain, a.gain_dtype, at, c, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] *= g[i], q[i] *= r;
            give(at, p, q);
        }
    }
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
        if (at0 + k * kNext < c) store8(mine, at0 + k * kNext, c, sums[k]);
}

// dgain: the workgroups' sums added in their order, 32 columns a workgroup.
__global__ void __launch_bounds__(256) norm_gain_sum(NormGradArgs a) {
    __shared__ f32x4 part[32][8];
    const int quad = threadIdx.x & 7, slice = threadIdx.x >> 3;
    const int col = (int)blockIdx.x * 32 + quad * 4;
    const int per = (a.parts + 31) / 32, begin = slice * per, end = min(begin + per, a.parts);
    f32x4 t{0, 0, 0, 0};
    if (col < a.c)
#pragma unroll 4
        for (int n = begin; n < end; ++n) t += *reinterpret_cast<const f32x4 *>(a.part + (int64_t)n * a.ldpart + col);
    part[slice][quad] = t;
    __syncthreads();
    if (slice) return;
    for (int n = 1; n < 32; ++n) t += part[n][quad];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < a.c) a.dgain[col + i] = t[i];
}

template <class In>
hipError_t launch_grad_of(const NormGradArgs &a, hipStream_t stream) {
    if (a.parts) {
        if (a.c <= 2048)
            hipLaunchKernelGGL((norm_backward<In, 1, 256>), dim3((unsigned)a.parts), dim3(256), 0, stream, a);
        else if (a.c <= 4096)
            hipLaunchKernelGGL((norm_backward<In, 2, 256>), dim3((unsigned)a.parts), dim3(256), 0, stream, a);
        else
            hipLaunchKernelGGL((norm_backward<In, 4, 256>), dim3((unsigned)a.parts), dim3(256), 0, stream, a);
    }
    hipLaunchKernelGGL(norm_gain_sum, dim3((unsigned)((a.c + 31) / 32)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

int norm_grad_parts(int64_t m) { return (int)(m < 512 ? m : 512); }

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

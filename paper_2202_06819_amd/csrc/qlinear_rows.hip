// Rows of floating values quantised to 8 bits, one power-of-two scale for each
// row:
//   e = the least integer with max |x| <= 127 * 2^e (at least -126),
//   scale = 2^e,  code = x / 2^e rounded to nearest, ties to even.
// A zero row has scale 0; a row that holds an infinity or a NaN has scale NaN
// and codes 0, so that every product with it is NaN.  With a power of two the
// quotient is exact, so codes do not depend on how it is formed, and code *
// scale has at most 7 significant bits: exact in either 16-bit type.
//
// One pass: a row's values stay in registers between its maximum and its
// codes.  Bound by memory (2 or 4 bytes read and 1 written a value): 8192 x 4096 bf16
// take 16.6 us, 6.05 TB/s.
#include "qlinear_rows.h"

namespace qconv {

namespace {

__device__ __forceinline__ uint32_t abs_max8(const float (&v)[8], uint32_t m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
    return m;
}

// Adding 1.5 * 2^23 rounds to a whole number, ties to even, and leaves its
// two's complement in the low bits; the product before it is exact.
__device__ __forceinline__ uint32_t code4(const float *v, float inv) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, __builtin_fmaf(v[i], inv, 12582912.0f));
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(w[3], w[2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), 0x05040100u);
}

// WAVES waves of a workgroup of four to each row, KEEP vectors of eight values
// a lane in registers; longer rows read the rest a second time.
template <class In, int WAVES, int KEEP>
__global__ void __launch_bounds__(256) quantize_rows(QuantizeArgs a) {
    constexpr int kLanes = WAVES * 64, kRows = 4 / WAVES;
    __shared__ uint32_t part[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? wave : 0);
    const bool mine = row < a.m;
    const In *x = static_cast<const In *>(a.x) + (mine ? row : 0) * a.ldx;
    const int at0 = (WAVES == 1 ? lane : (int)threadIdx.x) * 8;
    const int c = mine ? a.c : 0, whole = (c + 15) & ~15;
    float v[KEEP][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
        if (at0 + i * kLanes * 8 < c) load8(x, at0 + i * kLanes * 8, c, v[i]);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
#pragma unroll
    for (int i = 0; i < KEEP; ++i) m = abs_max8(v[i], m);
    for (int at = at0 + KEEP * kLanes * 8; at < c; at += kLanes * 8) {
        float w[8];
        load8(x, at, c, w);
        m = abs_max8(w, m);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    if constexpr (WAVES > 1) {
        if (lane == 0) part[wave] = m;
        __syncthreads();
        m = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    // m = 1.f * 2^p: e = p - 6 where 1.f <= 127 / 64, else p - 5
    const int e = max((int)(m >> 23) - 6 + ((m & 0x7fffffu) > 0x7e0000u), 1);
    const bool finite = m < 0x7f800000u;
    const float scale = !finite ? __builtin_nanf("") : m == 0 ? 0.0f : __builtin_bit_cast(float, (uint32_t)e << 23);
    const float inv = __builtin_bit_cast(float, (uint32_t)(254 - e) << 23);
    uint8_t *out = a.codes + (mine ? row : 0) * a.pitch;
    auto store = [&](int at, const float(&w)[8]) {
        if (at < whole)
            *reinterpret_cast<uint2 *>(out + at) = finite ? uint2{code4(w, inv), code4(w + 4, inv)} : uint2{0u, 0u};
    };
#pragma unroll
    for (int i = 0; i < KEEP; ++i) store(at0 + i * kLanes * 8, v[i]);
    for (int at = at0 + KEEP * kLanes * 8; at < whole; at += kLanes * 8) {
        float w[8];
        load8(x, at, c, w);
        store(at, w);
    }
    if (mine && at0 == 0) a.scale[row] = scale;
}

template <class In>
hipError_t launch(const QuantizeArgs &a, hipStream_t stream) {
    // A wave holds rows of up to 2048 values, a workgroup of four longer ones.
    QuantizeArgs s = a;
    const bool wide = a.c > 2048;
    const int64_t blocks = wide ? a.m : ((int64_t)a.m + 3) / 4;
    launch_slices(blocks, 256, [&](long long first, unsigned count) {
        const int64_t row = first * (wide ? 1 : 4);
        s.x = static_cast<const In *>(a.x) + row * a.ldx;
        s.codes = a.codes + row * a.pitch;
        s.scale = a.scale + row;
        s.m = (int32_t)(a.m - row);
        if (wide)
            hipLaunchKernelGGL((quantize_rows<In, 4, 4>), dim3(count), dim3(256), 0, stream, s);
        else
            hipLaunchKernelGGL((quantize_rows<In, 1, 4>), dim3(count), dim3(256), 0, stream, s);
    });
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const QuantizeArgs &a, int dtype, hipStream_t stream) {
    switch (dtype) {
        case QCONV_BF16: return launch<__bf16>(a, stream);
        case QCONV_F16: return launch<_Float16>(a, stream);
        default: return launch<float>(a, stream);
    }
}

}  // namespace qconv

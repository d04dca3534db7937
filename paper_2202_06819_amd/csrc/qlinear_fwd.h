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

// The adapter of a row; -1: none.
__device__ __forceinline__ int adapter_of(const LinearArgs &a, int row) {
    const int id = row < a.m ? a.ad.row[row] : -1;
    return id < a.ad.count ? max(id, -1) : -1;
}

// Partial sums of u over one of `splits` runs of channels, without the row
// scale: sum of codes times A for the row's own adapter.  A workgroup takes 16 NI
// rows (NI 2, above 512 rows: an A that is read serves twice the rows) and a run of
// 32-channel steps.  The adapters that the rows name are dealt to its waves, and where
// they are fewer than the waves, several waves share one, each with a run of its steps
// (so that a wave's loads lie side by side in A's rows), and all loads of A are in
// flight at once whether the rows agree or not; where there are few such workgroups,
// the adapters are dealt to several of them first (grid z).  A wave multiplies its
// adapter's A (RF fragments of 16 ranks) by all rows and keeps the rows that asked for
// it.  Bound by reading A, and for few rows by the waits of one load after another: 48
// rows, 4096 channels, 32 adapters of rank 16 take 9 us, 2003 rows, 2048 channels, 5 of
// rank 64 10.
constexpr int adapter_waves(int rf) { return rf == 8 ? 8 : 16; }
constexpr int adapter_lds(int rf, int ni) { return adapter_waves(rf) * rf * ni * 1024; }
template <class T, int RF, int NI>
__global__ void __launch_bounds__(adapter_waves(RF) * 64) adapter_rows(LinearArgs a, int steps_per_split) {
    constexpr int kWaves = adapter_waves(RF), kDeep = RF == 1 ? 8 / NI : RF == 2 ? 4 / NI : 2;   // steps loaded at once
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    auto part = reinterpret_cast<f32x4(*)[RF * NI][64]>(smem);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = lane & 15, g = lane >> 4;
    const int row0 = (int)blockIdx.x * 16 * NI;
    const int all = (a.c + 31) / 32;
    const int begin = (int)blockIdx.y * steps_per_split, end = min(begin + steps_per_split, all);
    int id[NI];
    uint32_t named = 0;   // 16 rows of each fragment
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        id[i] = adapter_of(a, row0 + i * 16 + r);
        named |= ((uint32_t)__ballot(id[i] >= 0) & 0xffffu) << (16 * i);
    }
    // the lowest row of `left` gives the next adapter; its rows leave the mask
    const auto next = [&](uint32_t &left) {
        const int at = __builtin_ctz(left);
        int ad = __builtin_amdgcn_readlane(id[0], at & 15);
        if (NI > 1 && at >= 16) ad = __builtin_amdgcn_readlane(id[NI - 1], at & 15);
#pragma unroll
        for (int i = 0; i < NI; ++i) left &= ~(((uint32_t)__ballot(id[i] == ad) & 0xffffu) << (16 * i));
        return ad;
    };
    // the n-th adapter that the rows name is for workgroup z = n mod Z of this place
    const int Z = (int)gridDim.z, z = (int)blockIdx.z;
    int distinct = 0, own[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) own[i] = -1;
    for (uint32_t left = named; left; ++distinct) {
        const int ad = next(left);
#pragma unroll
        for (int i = 0; i < NI; ++i) own[i] = id[i] == ad ? distinct : own[i];
    }
    const int here = (distinct - z + Z - 1) / Z;
    if (here <= 0) return;
    int classes = 1;
    while (classes < here && classes < kWaves) classes *= 2;
    const int mine = wave & (classes - 1), share = kWaves / classes;
    const int run = (end - begin + share - 1) / share, first = begin + wave / classes * run, last = min(first + run, end);
    const __amdgpu_buffer_rsrc_t rx = range_of(a.x.codes + (int64_t)row0 * a.x.pitch,
                                               (int64_t)(a.m - 1 - row0) * a.x.pitch + a.x.used);
    f32x4 sum[RF][NI];
#pragma unroll
    for (int f = 0; f < RF; ++f)
#pragma unroll
        for (int i = 0; i < NI; ++i) sum[f][i] = f32x4{0, 0, 0, 0};
    int n = 0;
    for (uint32_t left = named; left; ++n) {
        const int ad = next(left);
        if (n % Z != z || (n / Z & (classes - 1)) != mine) continue;
        // A's rows past the rank lie past the range, and load as zeros
        const __amdgpu_buffer_rsrc_t ra = range_of(
            static_cast<const typename T::elem *>(a.ad.a) + (int64_t)ad * a.ad.rank * a.c, (int64_t)a.ad.rank * a.c * 2);
        f32x4 d[RF][NI];
#pragma unroll
        for (int f = 0; f < RF; ++f)
#pragma unroll
            for (int i = 0; i < NI; ++i) d[f][i] = f32x4{0, 0, 0, 0};
        for (int s = first; s < last; s += kDeep) {
            u32x4_t w[kDeep][RF];
            uint2 q[kDeep][NI];
#pragma unroll
            for (int e = 0; e < kDeep; ++e) {
                const int at = (s + e) * 32 + g * 8;   // c is a multiple of 8: a vector is whole or absent
                const bool in = s + e < last && at < a.c;
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const auto v = __builtin_amdgcn_raw_buffer_load_b64(
                        rx, (int)(in ? (uint32_t)(i * 16 + r) * (uint32_t)a.x.pitch + (uint32_t)at : kNowhere), 0, 0);
                    q[e][i] = uint2{v[0], v[1]};
                }
#pragma unroll
                for (int f = 0; f < RF; ++f)
                    w[e][f] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                        ra, (int)(in ? (uint32_t)((f * 16 + r) * a.c + at) * 2u : kNowhere), 0, 0));
            }
#pragma unroll
            for (int e = 0; e < kDeep; ++e)
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const typename T::v8 b = codes_to_v8<T>(q[e][i]);
#pragma unroll
                    for (int f = 0; f < RF; ++f) d[f][i] = T::mma(__builtin_bit_cast(typename T::v8, w[e][f]), b, d[f][i]);
                }
        }
#pragma unroll
        for (int i = 0; i < NI; ++i)
            if (id[i] == ad)
#pragma unroll
                for (int f = 0; f < RF; ++f) sum[f][i] = d[f][i];
    }
#pragma unroll
    for (int f = 0; f < RF; ++f)
#pragma unroll
        for (int i = 0; i < NI; ++i) part[wave][f * NI + i][lane] = sum[f][i];
    __syncthreads();
    // lane (r, g) of fragment (f, i) holds ranks 16 f + 4 g + 0..3 of row 16 i + r
    for (int o = wave; o < RF * NI; o += kWaves) {
        const int f = o / NI, i = o % NI, row = row0 + i * 16 + r, rank = f * 16 + g * 4;
        f32x4 t = part[0][o][lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) t += part[w][o][lane];
        const int whose = NI > 1 && i ? own[NI - 1] : own[0];
        if (whose >= 0 && whose % Z == z && rank < a.ad.rank)   // (rows without an adapter have no u)
            *reinterpret_cast<f32x4 *>(a.ad.u + ((int64_t)blockIdx.y * a.m + row) * a.ad.rank + rank) = t;
    }
}

// ---------------------------------------------------------- adapters, part two

// Eight ranks of u of the lane's row, summed over the splits in their order, DEEP of
// them loaded at once.
template <int DEEP>
__device__ __forceinline__ void load_u(const LinearArgs &a, int row, int rank, float (&u)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = 0.0f;
    if (row >= a.m || rank >= a.ad.rank) return;
    const float *p = a.ad.u + (int64_t)row * a.ad.rank + rank;
#pragma unroll DEEP
    for (int s = 0; s < a.ad.splits; ++s, p += (int64_t)a.m * a.ad.rank) {
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(p), hi = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] += lo[i], u[i + 4] += hi[i];
    }
}

// A power of two that brings a row's largest |u| (its float bits) into [1, 2), and its
// inverse: u is split into 16-bit parts after it, so that their rounding is relative to
// the row and no f16 overflows.  Within 2^-40 .. 2^40: results scaled by it stay finite.
__device__ __forceinline__ void row_factor(uint32_t m, float &down, float &up) {
    const int e = min(max((int)(m >> 23), 127 - 40), 127 + 40);
    down = __builtin_bit_cast(float, (uint32_t)(254 - e) << 23);
    up = __builtin_bit_cast(float, (uint32_t)e << 23);
}

// Two values as a high and a low part in 16 bits, each rounded to nearest: what the two
// leave out is a rounding of a rounding (2^-16 of a bf16 value, 2^-22 of an f16 one), so
// that u's way through 16-bit products shows as little as the 32-bit sums' own order.
// One part alone costs a product less and as much error as the result's own rounding
// again (one row, 4096 channels: 0.0019 against 0.0017 of the result).
template <class T>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t &high, uint32_t &low) {
    high = pack2<T>(a, b);
    const typename T::v2 h = __builtin_bit_cast(typename T::v2, high);
    const float ha = (float)h[0], hb = (float)h[1];
    // (an infinity has no rest)
    low = pack2<T>(__builtin_isinf(ha) ? 0.0f : a - ha, __builtin_isinf(hb) ? 0.0f : b - hb);
}

// Adds the adapters' second products for 16 rows to FJ fragments of results: d[j] +=
// alpha xs (u B^T) for the row row0 + (lane & 15) and the output channels
// channel_of(j) of lane row r of fragment j.  Takes every `stride`-th adapter from
// `first` on that the rows name (`id`: the lane's row's), kBatch at a time, whose B
// are loaded together.  RS:
// products of 32 ranks at a time (2: ranks above 32, 64 at a time).
template <class T, int FJ, int RS, class ChannelOf>
__device__ __forceinline__ void add_adapters(const LinearArgs &a, int id, int row0, int lane, int first, int stride,
                                             ChannelOf channel_of, f32x4 (&d)[FJ]) {
    using v8 = typename T::v8;
    constexpr int kBatch = FJ * RS <= 2 ? 4 : 2;
    const int r = lane & 15, g = lane >> 4, row = row0 + r;
    const uint32_t named = (uint32_t)__ballot(id >= 0) & 0xffffu;
    if (!named) return;
    auto next_mine = [&](uint32_t &left, int &n) {
        int ad = -1;
        while (left) {
            ad = next_adapter(left, id);
            if (n++ % stride == first) return ad;
        }
        return -1;
    };
    for (int rank0 = 0; rank0 < a.ad.rank; rank0 += 32 * RS) {
        int ad[kBatch];
        float alpha[kBatch];
        u32x4_t w[kBatch][FJ][RS];
        uint32_t left = named;
        int n = 0;
        auto load_batch = [&] {
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                ad[b] = next_mine(left, n);
                alpha[b] = ad[b] >= 0 ? a.ad.alpha[ad[b]] : 0.0f;
                const typename T::elem *B =
                    static_cast<const typename T::elem *>(a.ad.b) + (int64_t)max(ad[b], 0) * a.k * a.ad.rank;
#pragma unroll
                for (int j = 0; j < FJ; ++j)
#pragma unroll
                    for (int s = 0; s < RS; ++s) {
                        const int ch = channel_of(j), rank = rank0 + s * 32 + g * 8;
                        w[b][j][s] = u32x4_t{0, 0, 0, 0};
                        if (ad[b] >= 0 && ch < a.k && rank < a.ad.rank)
                            w[b][j][s] = *reinterpret_cast<const u32x4_t *>(B + (int64_t)ch * a.ad.rank + rank);
                    }
            }
        };
        load_batch();
        if (ad[0] < 0) return;   // nothing for this wave
        u32x4_t high[RS], low[RS];
        float u[RS][8];
        uint32_t m = 0;
#pragma unroll
        for (int s = 0; s < RS; ++s) {
            load_u<8>(a, row, rank0 + s * 32 + g * 8, u[s]);
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max(m, __builtin_bit_cast(uint32_t, u[s][e]) & 0x7fffffffu);
        }
        m = max(m, (uint32_t)__shfl_xor((int)m, 16));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32));
        float down, up;
        row_factor(m, down, up);
#pragma unroll
        for (int s = 0; s < RS; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t h, l;
                split_pair<T>(u[s][2 * e] * down, u[s][2 * e + 1] * down, h, l);
                high[s][e] = h, low[s][e] = l;
            }
        const float scale = up * (row < a.m ? a.x.scale[row] : 0.0f);
        while (ad[0] >= 0) {
#pragma unroll
            for (int b = 0; b < kBatch; ++b)
#pragma unroll
                for (int j = 0; j < FJ; ++j) {
                    f32x4 t{0, 0, 0, 0};
#pragma unroll
                    for (int s = 0; s < RS; ++s) {
                        t = T::mma(__builtin_bit_cast(v8, w[b][j][s]), __builtin_bit_cast(v8, low[s]), t);
                        t = T::mma(__builtin_bit_cast(v8, w[b][j][s]), __builtin_bit_cast(v8, high[s]), t);
                    }
                    // (chosen, not by a zero factor: another adapter's product may not be finite)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        d[j][e] = id >= 0 && id == ad[b] ? __builtin_fmaf(scale * alpha[b], t[e], d[j][e]) : d[j][e];
                }
            load_batch();
        }
    }
}

// --------------------------------------------------------------- few rows

// 16 FI rows against 16 FJ output channels a workgroup: eight waves take the
// 128-channel steps in turn, several in flight, weights and rows straight from memory
// into registers (each weight is used once, so LDS would only be a detour), and
// their sums meet in LDS.  Bound by reading the weights, and with many rows by
// reading those from L2 once for each workgroup: hence wider ones where there are
// enough channels to fill the chip.  One row of 4096 channels against 4096 outputs of 4
// bits: 4.4 us without adapters (8.4 MB, 1.9 TB/s).
constexpr int few_lds(int fj, int fi, bool ad) { return 8 * 64 * 16 * (fj * fi + (ad ? fj : 0)); }
template <class T, int WB, int FJ, int FI, bool AD>
__global__ void __launch_bounds__(512) linear_few(LinearArgs a) {
    constexpr int kWaves = 8, kParts = kWaves / FI;
    constexpr int kWide = WB == 8 ? 2 : 1;   // 16-byte vectors of weights a lane and step
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    auto part = reinterpret_cast<i32x4(*)[FJ * FI][64]>(smem);                                // waves' sums
    auto extra = reinterpret_cast<f32x4(*)[FJ][64]>(smem + kWaves * FJ * FI * 64 * 16);   // the adapters' part
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = lane & 15, g = lane >> 4;
    const int ch0 = (int)blockIdx.x * 16 * FJ, row0 = (int)blockIdx.y * 16 * FI;
    const __amdgpu_buffer_rsrc_t rx = range_of(a.x.codes + (int64_t)row0 * a.x.pitch,
                                               (int64_t)(a.m - 1 - row0) * a.x.pitch + a.x.used);
    const __amdgpu_buffer_rsrc_t rw = range_of(a.w.codes + (int64_t)ch0 * a.w.pitch,
                                               (int64_t)(a.k - 1 - ch0) * a.w.pitch + a.w.used);
    i32x4 acc[FJ][FI];
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int f = 0; f < FI; ++f) acc[j][f] = i32x4{0, 0, 0, 0};
    struct Step {
        u32x4_t w[FJ][kWide], x[FI][2];
    };
    // lane (r, g) takes channels g * 32 .. + 31 of a step of 4-bit weights, g * 16 ..
    // + 15 of each half of one of 8-bit weights: the depth's order is free as long as
    // both operands share it
    auto load = [&](int s, Step &q) {
#pragma unroll
        for (int j = 0; j < FJ; ++j)
#pragma unroll
            for (int h = 0; h < kWide; ++h) {
                const int at = WB == 8 ? s * 128 + h * 64 + g * 16 : s * 64 + g * 16;
                q.w[j][h] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                    rw, (int)(at < a.w.used ? (uint32_t)(j * 16 + r) * (uint32_t)a.w.pitch + (uint32_t)at : kNowhere), 0, 0));
            }
#pragma unroll
        for (int f = 0; f < FI; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = WB == 8 ? s * 128 + h * 64 + g * 16 : s * 128 + g * 32 + h * 16;
                q.x[f][h] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                    rx, (int)(at < a.x.used ? (uint32_t)(f * 16 + r) * (uint32_t)a.x.pitch + (uint32_t)at : kNowhere), 0, 0));
            }
    };
    auto multiply = [&](const Step &q) {
#pragma unroll
        for (int j = 0; j < FJ; ++j) {
            i32x4 w[2];
            if constexpr (WB == 8) {
                w[0] = __builtin_bit_cast(i32x4, q.w[j][0]);
                w[1] = __builtin_bit_cast(i32x4, q.w[j][kWide - 1]);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint2 p = widen8(q.w[j][0][2 * h]), t = widen8(q.w[j][0][2 * h + 1]);
                    w[h] = i32x4{(int)p.x, (int)p.y, (int)t.x, (int)t.y};
                }
            }
#pragma unroll
            for (int f = 0; f < FI; ++f)
#pragma unroll
                for (int h = 0; h < 2; ++h) acc[j][f] = MmaI8::mma(w[h], __builtin_bit_cast(i32x4, q.x[f][h]), acc[j][f]);
        }
    };
    // wave = part * FI + fragment: the parts share the fragment's adapters.  Which ones
    // is asked first, their part computed while the first weights are on their way
    int id = -1;
    if constexpr (AD) id = adapter_of(a, row0 + wave % FI * 16 + r);
    asm volatile("" ::: "memory");
    // kFlight steps in flight (4 for 16 rows, where they are short; more made wider ones
    // slower)
    constexpr int kFlight = FI == 1 ? 4 : 2;
    Step q[kFlight];
#pragma unroll
    for (int e = 0; e < kFlight; ++e)
        if (wave + e * kWaves < a.steps) load(wave + e * kWaves, q[e]);
    if constexpr (AD) {
        f32x4 d[FJ];
#pragma unroll
        for (int j = 0; j < FJ; ++j) d[j] = f32x4{0, 0, 0, 0};
        const auto channel_of = [&](int j) { return ch0 + j * 16 + r; };
        if (a.ad.rank <= 32)
            add_adapters<T, FJ, 1>(a, id, row0 + wave % FI * 16, lane, wave / FI, kParts, channel_of, d);
        else
            add_adapters<T, FJ, 2>(a, id, row0 + wave % FI * 16, lane, wave / FI, kParts, channel_of, d);
#pragma unroll
        for (int j = 0; j < FJ; ++j) extra[wave][j][lane] = d[j];
    }
    for (int s = wave; s < a.steps; s += kFlight * kWaves) {
#pragma unroll
        for (int e = 0; e < kFlight; ++e) {
            if (s + e * kWaves < a.steps) multiply(q[e]);
            if (s + (kFlight + e) * kWaves < a.steps) load(s + (kFlight + e) * kWaves, q[e]);
        }
    }
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int f = 0; f < FI; ++f) part[wave][j * FI + f][lane] = acc[j][f];
    __syncthreads();
    // results: channels ch .. ch + 3 of one row
#pragma unroll
    for (int n = 0; n < (FJ * FI + kWaves - 1) / kWaves; ++n) {
        const int o = wave + n * kWaves, j = o / FI, f = o % FI;
        if (o >= FJ * FI) break;
        const int row = row0 + f * 16 + r, ch = ch0 + j * 16 + g * 4;
        i32x4 t = part[0][o][lane];
#pragma unroll
        for (int p = 1; p < kWaves; ++p) t += part[p][o][lane];
        if (row >= a.m || ch >= a.k) continue;
        const float xs = a.x.scale[row] * (WB == 4 ? 0.0625f : 1.0f);
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (float)t[e] * xs * a.w.scale[min(ch + e, a.k - 1)];
        if constexpr (AD)
#pragma unroll
            for (int p = 0; p < kParts; ++p) y += extra[p * FI + f][j][lane];
        store4<T>(static_cast<typename T::elem *>(a.y) + (int64_t)row * a.ldy + ch, y, a.k - ch);
    }
}

// --------------------------------------------------------------- many rows

// The adapters' second products of a workgroup's tile: further steps of the same tile
// product, in 16-bit floats.  u (64 ranks of it, scaled, as a high and a low part) stays in LDS;
// each adapter that the tile's rows name has its B copied to one of two buffers and
// takes a step, whose products go to the rows that named it.  So an adapter's B is
// read once for a tile, however its rows lie.  KS groups of THREADS threads deal the
// adapters out among them; a row's products are in the group that had its adapter.
// Bound by the wait for an adapter's B, one step ahead: 2003 rows, 2048 to 8192 channels,
// 5 adapters of rank 64 take 49 us, 42 without them.
template <class T, int TJ, int TI, int THREADS, int KS>
struct TileAdapters {
    const LinearArgs &a;
    uint8_t *smem;   // after the main loop: adapters of the rows | factors | adapters named | u, high and low | two B of each group
    int i0, j0;
    static constexpr int kU = TI * 12 + 16, kPart = TI * kStepBytes, kB = TJ * kStepBytes;
    static constexpr int kBytes = kU + 2 * kPart + KS * 2 * kB;
    static constexpr int kFill = THREADS * (KS < 2 ? KS : 2);   // threads that write u
    static constexpr bool kScaled = __is_same(T, F16);   // bf16 has float's range

    __device__ int *ids() const { return reinterpret_cast<int *>(smem); }
    __device__ float *factors() const { return reinterpret_cast<float *>(smem + TI * 4); }
    __device__ int *named() const { return reinterpret_cast<int *>(smem + TI * 8); }
    __device__ int *count() const { return reinterpret_cast<int *>(smem + TI * 12); }
    __device__ uint8_t *buffer(int group, int buf) const { return smem + kU + 2 * kPart + (group * 2 + buf) * kB; }
    __device__ float down(int row) const { return kScaled ? 1.0f / factors()[row] : 1.0f; }   // (a power of two: exact)
    __device__ float up(int row) const { return kScaled ? factors()[row] : 1.0f; }

    // alpha xs u of the tile's rows: 64 ranks from rank0, in two 16-bit parts in LDS.  The
    // row's factor comes from all of its ranks.
    __device__ void fill_u(int rank0) const {
        if ((int)threadIdx.x >= kFill) return;
#pragma unroll
        for (int n = 0; n < TI * 8 / kFill; ++n) {
            const int unit = n * kFill + (int)threadIdx.x, at = unit >> 3, v = unit & 7, row = i0 + at;
            const int id = adapter_of(a, row);
            const float s = id >= 0 ? a.ad.alpha[id] * a.x.scale[row] : 0.0f;
            float u[8];
            load_u<2>(a, id >= 0 ? row : a.m, rank0 + v * 8, u);
            float down = 1.0f, up = 1.0f;
            if constexpr (kScaled) {
                uint32_t m = 0;
                for (int c = 0; c < a.ad.rank; c += 64) {
                    float other[8];
                    load_u<2>(a, id >= 0 ? row : a.m, c + v * 8, other);
#pragma unroll
                    for (int e = 0; e < 8; ++e) m = max(m, __builtin_bit_cast(uint32_t, other[e] * s) & 0x7fffffffu);
                }
#pragma unroll
                for (int b = 1; b < 8; b <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, b));
                row_factor(m, down, up);
            }
            u32x4_t high, low;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t h, l;
                split_pair<T>(u[2 * e] * s * down, u[2 * e + 1] * s * down, h, l);
                high[e] = h, low[e] = l;
            }
            uint8_t *const to = smem + kU + at * kStepBytes + ((v ^ slot(at)) << 4);
            *reinterpret_cast<u32x4_t *>(to) = high;
            *reinterpret_cast<u32x4_t *>(to + kPart) = low;
            if (v == 0) ids()[at] = id, factors()[at] = up;
        }
    }
    // u of the first ranks, and the adapters that the rows name, each once.  (Their order
    // changes no result: a row has one.)
    __device__ void stage() const {
        if (threadIdx.x == 0) *count() = 0;
        fill_u(0);
        __syncthreads();
        const int rows64 = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
        if (rows64 < TI / 64) {   // those of its 64 rows that no row before them names
            int id[TI / 64];
#pragma unroll
            for (int n = 0; n < TI / 64; ++n) id[n] = n <= rows64 ? ids()[n * 64 + lane] : -1;
            const int own = ids()[rows64 * 64 + lane];
            int found = 0, mine = -1;
            for (uint64_t left = __ballot(own >= 0); left;) {
                const int ad = __builtin_amdgcn_readlane(own, __builtin_ctzll(left));
                left &= ~__ballot(own == ad);
                bool before = false;
#pragma unroll
                for (int n = 0; n < TI / 64 - 1; ++n) before = before || (n < rows64 && __ballot(id[n] == ad));
                if (before) continue;
                mine = lane == found ? ad : mine;
                ++found;
            }
            int base = 0;
            if (lane == 0) base = atomicAdd(count(), found);
            base = __builtin_amdgcn_readfirstlane(base);
            if (lane < found) named()[base + lane] = mine;
        }
        __syncthreads();
    }
    __device__ int named_at(int n, int total) const {
        return n < total ? __builtin_amdgcn_readfirstlane(named()[n]) : -1;
    }
    __device__ void copy_b(int ad, int rank0, uint8_t *to, int wave, int lane) const {
        const int64_t row_bytes = (int64_t)a.ad.rank * 2;
        const u32x4_t rb = range_words(static_cast<const uint8_t *>(a.ad.b) + ((int64_t)ad * a.k + j0) * row_bytes,
                                       (int64_t)(a.k - j0) * row_bytes);
        copy_rows<TJ, THREADS>(to, rb, (uint32_t)row_bytes, rank0 * 2, (int)row_bytes, wave, lane);
    }
    template <int FJ, int FI>
    __device__ void add(int jrow0, int irow0, int group, int wave, int lane, f32x4 (&d)[FJ][FI]) const {
        using v8 = typename T::v8;
        const int r = lane & 15, g = lane >> 4;
        const int total = __builtin_amdgcn_readfirstlane(*count());
        for (int rank0 = 0; rank0 < a.ad.rank; rank0 += 64) {
            if (rank0) {   // everyone is done with the ranks before
                __syncthreads();
                fill_u(rank0);
                __syncthreads();
            }
            int ad = named_at(group, total), buf = 0;
            if (ad >= 0) copy_b(ad, rank0, buffer(group, 0), wave, lane);
            for (int n = 0; n < total; n += KS) {
                const int after = named_at(n + KS + group, total);
                copies_done();
                __syncthreads();
                // (the other buffer: its step ended before this barrier)
                if (after >= 0) copy_b(after, rank0, buffer(group, buf ^ 1), wave, lane);
                const uint8_t *lj = buffer(group, buf);
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    if (ad < 0 || rank0 + ks * 32 >= a.ad.rank) break;
                    v8 w[FJ];
#pragma unroll
                    for (int j = 0; j < FJ; ++j) {
                        const int row = jrow0 + j_row(j, r);
                        w[j] = *reinterpret_cast<const v8 *>(lj + row * kStepBytes + (((ks * 4 + g) ^ slot(row)) << 4));
                    }
#pragma unroll
                    for (int i = 0; i < FI; ++i) {
                        const int row = irow0 + i * 16 + r;
                        const bool mine = ids()[row] == ad;
                        const uint64_t who = __ballot(mine);
                        if (!who) continue;
                        const uint8_t *const lu = smem + kU + row * kStepBytes + (((ks * 4 + g) ^ slot(row)) << 4);
                        const v8 high = *reinterpret_cast<const v8 *>(lu), low = *reinterpret_cast<const v8 *>(lu + kPart);
                        // (results are chosen, not made zero by u: another adapter's
                        // product may not be finite)
#pragma unroll
                        for (int j = 0; j < FJ; ++j) {
                            const f32x4 t = T::mma(w[j], high, T::mma(w[j], low, d[j][i]));
#pragma unroll
                            for (int e = 0; e < 4; ++e) d[j][i][e] = mine ? t[e] : d[j][i][e];
                        }
                    }
                }
                ad = after;
                buf ^= 1;
            }
        }
    }
};

// LDS of a workgroup: its groups' buffers, and in their place afterwards the adapters'.
template <class T, int TJ, int TI, int THREADS, int KS, bool AD>
constexpr int tile_lds() {
    const int steps = KS * 2 * (TJ + TI) * kStepBytes, adapters = AD ? TileAdapters<T, TJ, TI, THREADS, KS>::kBytes : 0;
    return steps > adapters ? steps : adapters;
}

// TJ output channels by TI rows a workgroup of WJ x WI waves, each a tile of 64
// by 16 FI.  Steps of 128 channels are staged in one of two LDS buffers while
// the other is multiplied; rows and 8-bit weights go straight from memory to
// LDS, 4-bit ones through registers, where they are widened.  KS such groups of
// waves deal the steps out among them, each with buffers of its own, and their sums
// meet in LDS: where there are too few tiles to fill the chip, a CU's waves then still
// hide each other's waits (256 rows of 8192 channels, 4096 outputs of 4 bits: 32 us with
// one group, 21.6 with two, 19.5 with four).  The largest tile is bound by the matrix
// cores, which its random operands hold to what power allows: 8192 x 4096 x 4096 takes
// 118 to 124 us, 2.2 to 2.3 POP/s of the 3.1 that products of registers alone reach.
template <class T, int WB, int TJ, int TI, int WJ, int WI, int KS, bool AD>
__global__ void __launch_bounds__(KS *WJ *WI * 64, TJ == 64 ? 4 : 2) linear_tile(LinearArgs a) {
    constexpr int FJ = 4, FI = TI / (16 * WI), kThreads = WJ * WI * 64, kBuffer = (TJ + TI) * kStepBytes;
    static_assert(TJ == WJ * 64);
    static_assert(KS == 1 || FI == 1);
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int group = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kThreads), thread = (int)threadIdx.x % kThreads;
    const int wave = __builtin_amdgcn_readfirstlane(thread >> 6), lane = threadIdx.x & 63;
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
                const int unit = n * kThreads + thread, row = unit >> 2, at = s * 64 + (unit & 3) * 16;
                held[n] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                    rw4, (int)(at < a.w.used ? (uint32_t)row * (uint32_t)a.w.pitch + (uint32_t)at : kNowhere), 0, 0));
            }
        }
    };
    auto settle = [&](uint8_t *buf) {
        if constexpr (WB == 4) {
#pragma unroll
            for (int n = 0; n < kUnits; ++n) {
                const int unit = n * kThreads + thread, row = unit >> 2, v = (unit & 3) * 2;
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
    // (a group's step past the last one is all zeros)
    uint8_t *const own = smem + group * 2 * kBuffer;
    fetch(group, own);
    settle(own);
    __syncthreads();
    int buf = 0;
    for (int s = 0; s < a.steps; s += KS) {
        uint8_t *cur = own + buf * kBuffer, *next = own + (buf ^ 1) * kBuffer;
        if (s + KS < a.steps) fetch(s + KS + group, next);
        mma_step<MmaI8, FJ, FI>(cur, cur + TJ * kStepBytes, jrow0, irow0, lane, acc);
        if (s + KS < a.steps) settle(next);
        __syncthreads();
        buf ^= 1;
    }
    // lane (r, g): channels ch .. ch + 15 of one row of each fragment i
    const int r = lane & 15, g = lane >> 4;
    const int ch = j0 + jrow0 + g * 16;
    if constexpr (KS > 1) {
        // (in a group's own buffers: not where the adapters' part begins)
        auto part = [&](int from, int j) {
            return reinterpret_cast<i32x4 *>(smem + from * 2 * kBuffer) + (wave * FJ + j) * 64 + lane;
        };
        if (group)
#pragma unroll
            for (int j = 0; j < FJ; ++j) *part(group, j) = acc[j][0], acc[j][0] = i32x4{0, 0, 0, 0};
        __syncthreads();
        if (!group)
#pragma unroll
            for (int from = 1; from < KS; ++from)
#pragma unroll
                for (int j = 0; j < FJ; ++j) acc[j][0] += *part(from, j);
    }
    TileAdapters<T, TJ, TI, kThreads, KS> ad{a, smem, i0, j0};
    if constexpr (AD) ad.stage();
    float ws[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) ws[e] = a.w.scale[min(ch + e, a.k - 1)];
    f32x4 d[FJ][FI];
#pragma unroll
    for (int i = 0; i < FI; ++i) {
        const int row = i0 + irow0 + i * 16 + r;
        float xs = row < a.m ? a.x.scale[row] * (WB == 4 ? 0.0625f : 1.0f) : 0.0f;
        if constexpr (AD) xs *= ad.down(irow0 + i * 16 + r);
#pragma unroll
        for (int j = 0; j < FJ; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[j][i][e] = (float)acc[j][i][e] * xs * ws[4 * j + e];
    }
    if constexpr (AD) {
        // (of a row whose scales are not finite, the groups past the first hold NaN too)
        if (KS > 1 && group)
#pragma unroll
            for (int j = 0; j < FJ; ++j) d[j][0] = f32x4{0, 0, 0, 0};
        ad.template add<FJ, FI>(jrow0, irow0, group, wave, lane, d);
        if constexpr (KS > 1) {
            __syncthreads();   // B's buffers are free
            auto part = [&](int from, int j) {
                return reinterpret_cast<f32x4 *>(ad.buffer(from, 0)) + (wave * FJ + j) * 64 + lane;
            };
            if (group)
#pragma unroll
                for (int j = 0; j < FJ; ++j) *part(group, j) = d[j][0];
            __syncthreads();
            if (!group)
#pragma unroll
                for (int from = 1; from < KS; ++from)
#pragma unroll
                    for (int j = 0; j < FJ; ++j) d[j][0] += *part(from, j);
        }
    }
    if (group) return;
#pragma unroll
    for (int i = 0; i < FI; ++i) {
        const int row = i0 + irow0 + i * 16 + r;
        if (row >= a.m) continue;
        const float up = AD ? ad.up(irow0 + i * 16 + r) : 1.0f;
        typename T::elem *out = static_cast<typename T::elem *>(a.y) + (int64_t)row * a.ldy + ch;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 lo = d[2 * h][i] * up, hi = d[2 * h + 1][i] * up;
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
}

}  // namespace qconv

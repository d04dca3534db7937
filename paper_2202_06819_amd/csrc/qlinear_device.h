// Device helpers of the linear layer's kernels: element types, the LDS tile
// that every matrix product here reads, and the copies that fill it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qlinear_internal.h"

namespace qconv {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_ptr_t;

// The two 16-bit floating types: 8-element vectors as the matrix cores take
// them, products of depth 32, rounding to nearest even.
struct BF16 {
    using elem = __bf16;
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x4 mma(v8 a, v8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};
struct F16 {
    using elem = _Float16;
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x4 mma(v8 a, v8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};

template <class T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), typename T::v2));
}

// Matrix products as the tile loop uses them: one 16-byte vector of a row for
// each operand.
struct MmaI8 {
    using frag = i32x4;
    using acc = i32x4;
    static __device__ __forceinline__ acc mma(frag a, frag b, acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
    }
};
template <class T>
struct MmaT {
    using frag = typename T::v8;
    using acc = f32x4;
    static __device__ __forceinline__ acc mma(frag a, frag b, acc c) { return T::mma(a, b, c); }
};

// ------------------------------------------------------------- the LDS tile
//
// A step of a product stages 128 bytes of each of its rows (128 int8 or 64
// 16-bit values of the sum's axis): row r's 16-byte vector v lies at
// r * 128 + 16 * (v ^ slot(r)).  A 16-byte LDS read serves 16 lanes at once, 0-3,
// 12-15, 20-23 and 24-27, then 4-11, 16-19 and 28-31, and so on (so the counters of
// bank conflicts say): parts of two neighbouring vectors of a fragment; a write
// serves lanes in a run.  slot() is linear over XOR, and keeps each such set that
// occurs here on banks of its own: rows in a run (fragments), the rows 16 g +
// (0..3) of a lane's 16 consecutive outputs, and, for transposing stores, every
// fourth row of 32 and every second of 16.
constexpr int kStepBytes = 128;
__host__ __device__ constexpr int slot(int row) {
    return (row & 7) ^ (row & 8 ? 5 : 0) ^ (row & 16 ? 6 : 0);
}

// Row of fragment f that lane row r (0..15) of the j operand reads, from the
// wave's first row: the four rows of the product that a lane receives from
// each of four fragments are then 16 consecutive ones.
__device__ __forceinline__ int j_row(int f, int r) { return (f >> 2) * 64 + (r >> 2) * 16 + (f & 3) * 4 + (r & 3); }

// One step: FJ x FI fragments of 16 x 16 from the rows at lj and li (the
// wave's first rows, 64- and 16-row aligned).  slot() is linear over XOR, so
// the fragment's part of a vector's place is a constant: eight lane addresses
// serve each operand.
template <class Mma, int FJ, int FI>
__device__ __forceinline__ void mma_step(const uint8_t *lj, const uint8_t *li, int jrow0, int irow0, int lane,
                                         typename Mma::acc (&acc)[FJ][FI]) {
    static_assert(FJ == 4, "a lane holds 16 consecutive rows of the product");
    using frag = typename Mma::frag;
    const int r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        frag a[FJ], b[FI];
#pragma unroll
        for (int f = 0; f < FJ; ++f) {
            const int row = jrow0 + j_row(f, r);
            a[f] = *reinterpret_cast<const frag *>(lj + row * kStepBytes + (((ks * 4 + g) ^ slot(row)) << 4));
        }
#pragma unroll
        for (int f = 0; f < FI; ++f) {
            const int row = irow0 + f * 16 + r;
            b[f] = *reinterpret_cast<const frag *>(li + row * kStepBytes + (((ks * 4 + g) ^ slot(row)) << 4));
        }
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) acc[j][i] = Mma::mma(a[j], b[i], acc[j][i]);
    }
}

// ------------------------------------------------------------ global memory

constexpr uint32_t kNowhere = 0x80000000u;     // an offset past every range: loads give zero
constexpr int64_t kMaxRange = 0x7ffffff0ll;

__device__ __forceinline__ int range_bytes(int64_t bytes) {
    return (int)(bytes < 0 ? 0 : bytes < kMaxRange ? bytes : kMaxRange);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t range_of(const void *base, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), (short)0, range_bytes(bytes), 0x00020000);
}
// The same as plain words, for copy16 (32-bit sizes: no clamp).
__device__ __forceinline__ u32x4_t range_words(const void *base, int bytes) {
    const uint64_t b = (uint64_t)base;
    return u32x4_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b),
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(b >> 32)),
                   (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}
__device__ __forceinline__ u32x4_t range_words(const void *base, int64_t bytes) {
    return range_words(base, range_bytes(bytes));
}

// Global memory straight into LDS: lane i's 16 bytes at buffer offset `off`
// land at lds + 16 i.  In assembly, so that the compiler does not make later
// LDS reads wait for it: copies_done() does, before the barrier.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16(uint8_t *lds, uint32_t off, u32x4_t rsrc) {
    const uint32_t m0v = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr_t *)lds);
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(m0v), "v"(off), "s"(rsrc)
                 : "memory", "m0");
}
// The same of 4 bytes a lane.
__device__ __forceinline__ void copy4(uint8_t *lds, uint32_t off, u32x4_t rsrc) {
    const uint32_t m0v = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr_t *)lds);
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :
                 : "s"(m0v), "v"(off), "s"(rsrc)
                 : "memory", "m0");
}
#pragma clang diagnostic pop
// Waits until at most N of the wave's copies are outstanding (they land in
// order), and for its LDS reads.
template <int N>
__device__ __forceinline__ void copies_left() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory"); }
__device__ __forceinline__ void copies_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// ROWS rows of a step by a workgroup of THREADS: row r's bytes
// col .. col + 127, zero past `used` and past the resource's range.
template <int ROWS, int THREADS>
__device__ __forceinline__ void copy_rows(uint8_t *lds, u32x4_t rsrc, uint32_t pitch, int col, int used, int wave,
                                          int lane) {
    constexpr int kWaves = THREADS / 64;
    static_assert(ROWS % (8 * kWaves) == 0);
#pragma unroll
    for (int n = 0; n < ROWS / (8 * kWaves); ++n) {
        const int row = (n * kWaves + wave) * 8 + (lane >> 3);
        const int at = col + (((lane & 7) ^ slot(row)) << 4);
        copy16(lds + (n * kWaves + wave) * 1024, at < used ? (uint32_t)row * pitch + (uint32_t)at : kNowhere, rsrc);
    }
}

// Eight 4-bit values (channel i in bits 4i..4i+3) as eight bytes in order, each
// 16 times its value.
__device__ __forceinline__ uint2 widen8(uint32_t v) {
    const uint32_t even = (v << 4) & 0xF0F0F0F0u, odd = v & 0xF0F0F0F0u;
    return uint2{__builtin_amdgcn_perm(odd, even, 0x05010400u), __builtin_amdgcn_perm(odd, even, 0x07030602u)};
}

// Up to `left` of four results from one row; whole ones in one store, of any alignment.
__device__ __forceinline__ void store4(float *out, f32x4 d, int left) {
    if (left >= 4) {
        __builtin_memcpy(out, &d, 16);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) out[e] = d[e];
    }
}
template <class T>
__device__ __forceinline__ void store4(typename T::elem *out, f32x4 d, int left) {
    if (left >= 4) {
        const uint2 w{pack2<T>(d[0], d[1]), pack2<T>(d[2], d[3])};
        __builtin_memcpy(out, &w, 8);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) out[e] = (typename T::elem)d[e];
    }
}

// Workgroups are dispatched to the eight XCDs in turn.  Tile `n` of `count`
// for workgroup `id`, such that each XCD (its own L2) gets a run of tiles.
__device__ __forceinline__ int xcd_run(int id, int count) {
    const int q = count >> 3, rem = count & 7, x = id & 7, at = id >> 3;
    return (x < rem ? x * (q + 1) : rem * (q + 1) + (x - rem) * q) + at;
}

// Tiles in strips of up to eight along i, j within a strip running slowest but
// for the strips: neighbours in a run share rows of both operands.
__device__ __forceinline__ void tile_at(int n, int tiles_i, int tiles_j, int &ti, int &tj) {
    const int strip = n / (8 * tiles_j), rest = n - strip * 8 * tiles_j;
    const int wide = min(8, tiles_i - strip * 8);
    tj = rest / wide;
    ti = strip * 8 + rest - tj * wide;
}

}  // namespace qconv

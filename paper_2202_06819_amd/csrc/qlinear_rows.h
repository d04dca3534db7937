// Rows of floating values, eight at a time.
#pragma once

#include "qlinear_device.h"

namespace qconv {

// Eight values of a row from element `at`, zero from c on, as they lie in memory and as
// floats.  They are loaded in 16-byte accesses whatever the row's alignment (1021 x 5003
// floats of rows that start on 8-byte boundaries: 12.6 us by single elements, 5.0 so, in a
// graph); the row's last ones with those before them, moved into place afterwards, so that
// every lane's loads are alike and a caller has many on their way.  (Rows of less than
// eight: by elements.)
template <class In>
struct Raw8 {
    typedef In whole __attribute__((ext_vector_type(16 / sizeof(In))));
    whole w[sizeof(In) / 2];
};
template <class In>
__device__ __forceinline__ Raw8<In> fetch8(const In *row, int at, int c) {
    Raw8<In> q;
    constexpr int kEach = 16 / sizeof(In);
    if (c >= 8) {
        const In *from = row + min(at, c - 8);
#pragma unroll
        for (int h = 0; h < (int)sizeof(In) / 2; ++h) __builtin_memcpy(&q.w[h], from + kEach * h, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) q.w[i / kEach][i % kEach] = at + i < c ? row[at + i] : (In)0.0f;
    }
    return q;
}
template <class In>
__device__ __forceinline__ void unpack8(const Raw8<In> &q, int at, int c, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)q.w[i * sizeof(In) / 16][i % (16 / sizeof(In))];
    const int past = c >= 8 ? at + 8 - c : 0;   // loaded so many elements too early
    if (past > 0) {
#pragma unroll
        for (int d = 4; d; d >>= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = past & d ? (i + d < 8 ? v[i + d < 8 ? i + d : 0] : 0.0f) : v[i];
        if (past >= 8)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
}
template <class In>
__device__ __forceinline__ void load8(const In *row, int at, int c, float (&v)[8]) {
    unpack8(fetch8(row, at, c), at, c, v);
}

// The same back: eight values rounded to the row's type, none from c on.
template <class Out>
__device__ __forceinline__ void store8(Out *row, int at, int c, const float (&v)[8]) {
    typedef Out whole __attribute__((ext_vector_type(16 / sizeof(Out))));
    if (at + 8 <= c) {
        whole w[sizeof(Out) / 2];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i * sizeof(Out) / 16][i % (16 / sizeof(Out))] = (Out)v[i];
#pragma unroll
        for (int h = 0; h < (int)sizeof(Out) / 2; ++h) __builtin_memcpy(row + at + 16 / sizeof(Out) * h, &w[h], 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i < c) row[at + i] = (Out)v[i];
    }
}

}  // namespace qconv

// Internal declarations of the linear layer on 8-bit rows, shared by its host
// code and its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qconv.h"
#include "qconv_internal.h"

namespace qconv {

// Rows of low-bit codes with one scale for each row, as the kernels read them.
struct RowsArg {
    const uint8_t *codes;
    const float *scale;
    int64_t pitch;       // bytes from row to row, a multiple of 16
    int32_t used;        // bytes of a row that are read: its channels, whole 16-byte vectors
    int32_t rows;
};

struct QuantizeArgs {
    const void *x;
    int64_t ldx;         // elements from row to row
    uint8_t *codes;
    int64_t pitch;
    float *scale;
    int32_t m, c;
};

struct AdapterArgs {
    const void *a;       // adapters x rank x c
    const void *b;       // adapters x k x rank
    const float *alpha;  // one factor for each adapter
    const int32_t *row;  // adapter of each row of x
    float *u;            // splits x m x rank partial sums of codes times a
    int32_t count, rank, splits;
};

struct LinearArgs {
    RowsArg x, w;
    void *y;
    int64_t ldy;         // elements from row to row
    int32_t m, c, k;
    int32_t steps;       // 128-channel steps
    int32_t tiles_j, tiles_i;
    AdapterArgs ad;
};

// out[i][j] = sum over t of p(i, t) scale[t] codes[t][j], with p(i, t) at
// p[i * ldp + t], or at p[t * ldp + i] for the transposed form.
struct GradArgs {
    const void *p;
    int64_t ldp;
    RowsArg b;           // rows: the sum's axis
    void *out;
    int64_t ldo;
    float *part;         // splits x ni x ldpart partial sums (splits > 1)
    int64_t ldpart;
    int32_t ni, nj, nt;
    int32_t vec_p;       // rows of p start on 16-byte boundaries
    int32_t tiles_i, tiles_j;
    int32_t splits, steps_per_split, steps;
};

hipError_t launch_quantize_rows(const QuantizeArgs &a, int dtype, hipStream_t stream);
hipError_t launch_linear(const LinearArgs &a, int w_bits, int dtype, hipStream_t stream);
hipError_t launch_grad(const GradArgs &a, bool transposed, int w_bits, int dtype, hipStream_t stream);

// Workgroup tiles (square), and how a product is cut: shared by the workspace
// sizes and the launches.
int linear_adapter_splits(int64_t m, int64_t c);
struct GradPlan {
    int tile, groups;    // 64, 128 or 256; groups of waves that deal its steps out
    int splits, steps_per_split, steps;
};
// Whether p's rows are whole 16-byte vectors, so that they can be copied to LDS.
inline bool whole_vectors(const GradArgs &a, bool transposed) {
    return a.vec_p && (transposed ? a.ni : a.nt) % 8 == 0;
}
GradPlan plan_grad(int64_t ni, int64_t nj, int64_t nt);

// Records a failure for qconv_last_error and returns `code`.
int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();

}  // namespace qconv

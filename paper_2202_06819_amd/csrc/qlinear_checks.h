// Argument checks that the linear layer's entry points share.
#pragma once

#include <stdint.h>

#include "qconv.h"
#include "qlinear_internal.h"

namespace qconv {

constexpr int64_t kMaxPitch = 1 << 22, kMaxStride = 1 << 21;
constexpr int32_t kMaxRows = 1 << 22, kMaxChannels = 131071;   // 128 * 128 * 131071 < 2^31

inline bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

inline int64_t round16(int64_t n) { return (n + 15) & ~(int64_t)15; }

struct Span {
    uintptr_t begin, end;
    Span(const void *p, int64_t bytes) : begin((uintptr_t)p), end((uintptr_t)p + (bytes > 0 ? bytes : 0)) {}
    bool meets(const Span &o) const { return begin < end && o.begin < o.end && begin < o.end && o.begin < end; }
};

// Bytes of rows x cols elements, `ld` from row to row.
inline int64_t strided_bytes(int64_t rows, int64_t cols, int64_t ld, int64_t size) {
    return rows <= 0 ? 0 : ((rows - 1) * ld + cols) * size;
}
inline int64_t rows_used(const qconv_rows *r) { return round16((int64_t)r->channels * r->bits / 8); }
inline Span rows_span(const qconv_rows *r) { return Span(r->codes, strided_bytes(r->rows, rows_used(r), r->pitch, 1)); }
inline Span scale_span(const qconv_rows *r) { return Span(r->scale, (int64_t)r->rows * 4); }

inline int check_rows(const qconv_rows *r, const char *name, bool four) {
    if (!r) return fail(QCONV_EINVAL, "%s is NULL", name);
    if (r->rows < 0 || r->channels < 1)
        return fail(QCONV_EINVAL, "%s: rows must be >= 0 and channels >= 1 (got %d, %d)", name, r->rows, r->channels);
    if (r->bits != 8 && !(four && r->bits == 4))
        return fail(QCONV_EUNSUPPORTED, "%s: bits must be 8%s (got %d)", name, four ? " or 4" : "", r->bits);
    if (r->channels > kMaxChannels)
        return fail(QCONV_EUNSUPPORTED, "%s: more than %d channels (got %d)", name, kMaxChannels, r->channels);
    if (r->bits == 4 && r->channels % 8)
        return fail(QCONV_EUNSUPPORTED, "%s: 4-bit rows need channels %% 8 == 0 (got %d)", name, r->channels);
    if (r->rows > kMaxRows) return fail(QCONV_EUNSUPPORTED, "%s: more than 2^22 rows (got %d)", name, r->rows);
    if (r->pitch % 16 || r->pitch < rows_used(r))
        return fail(QCONV_EINVAL, "%s: pitch must be a multiple of 16 of at least %lld bytes (got %lld)", name,
                    (long long)rows_used(r), (long long)r->pitch);
    if (r->pitch > kMaxPitch) return fail(QCONV_EUNSUPPORTED, "%s: pitch above 2^22 bytes", name);
    if (r->rows > 0 && (!r->codes || !r->scale)) return fail(QCONV_EINVAL, "%s: codes and scale must be non-NULL", name);
    if (!aligned(r->codes, 16) || !aligned(r->scale, 4))
        return fail(QCONV_EINVAL, "%s: codes must be 16-byte and scale 4-byte aligned", name);
    return QCONV_OK;
}

inline RowsArg rows_arg(const qconv_rows *r) {
    return {static_cast<const uint8_t *>(r->codes), r->scale, r->pitch, (int32_t)rows_used(r), r->rows};
}

inline int check_float16(int32_t dtype) {
    if (dtype != QCONV_BF16 && dtype != QCONV_F16)
        return fail(dtype == QCONV_F32 ? QCONV_EUNSUPPORTED : QCONV_EINVAL, "dtype must be QCONV_BF16 or QCONV_F16 (got %d)",
                    dtype);
    return QCONV_OK;
}

// A matrix of `size`-byte elements, `ld` of them from row to row.
inline int check_matrix(const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t size, const char *name) {
    if (ld < cols) return fail(QCONV_EINVAL, "%s: %lld elements from row to row, fewer than its %lld columns", name,
                               (long long)ld, (long long)cols);
    if (ld > kMaxStride) return fail(QCONV_EUNSUPPORTED, "%s: more than 2^21 elements from row to row", name);
    if (rows > 0 && cols > 0 && !p) return fail(QCONV_EINVAL, "%s must be non-NULL", name);
    if (!aligned(p, (uintptr_t)size)) return fail(QCONV_EINVAL, "%s must be aligned to its elements", name);
    return QCONV_OK;
}

inline bool wide_rows(const void *p, int64_t ld, int64_t size, uintptr_t align) {
    return aligned(p, align) && ld * size % (int64_t)align == 0;
}

inline int check_workspace(const void *ws, size_t given, size_t need) {
    if (need == 0) return QCONV_OK;
    if (!ws || given < need) return fail(QCONV_EWORKSPACE, "workspace holds %zu bytes, needs %zu", ws ? given : 0, need);
    if (!aligned(ws, 16)) return fail(QCONV_EINVAL, "workspace must be 16-byte aligned");
    return QCONV_OK;
}

inline int check_tiles(int64_t rows, int64_t cols) {
    // launches of fewer than 2^31 threads
    if (((rows + 63) / 64) * ((cols + 63) / 64) > (1ll << 22))
        return fail(QCONV_EUNSUPPORTED, "a result of %lld x %lld is too large for one launch", (long long)rows, (long long)cols);
    return QCONV_OK;
}

// Partial sums of a gradient whose sum is split.
inline size_t grad_workspace(int64_t ni, int64_t nj, int64_t nt) {
    const int splits = plan_grad(ni, nj, nt).splits;
    return splits > 1 ? (size_t)splits * (size_t)ni * (size_t)((nj + 3) / 4 * 4) * 4 : 0;
}

}  // namespace qconv

// Host side of the linear layer on 8-bit rows: argument validation, workspace
// sizes and launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qlinear_checks.h"

using namespace qconv;

namespace {

int check_adapters(const qconv_adapters *ad, const qconv_rows *x) {
    if (ad->count < 0) return fail(QCONV_EINVAL, "adapters: count must be >= 0");
    if (ad->count == 0) return QCONV_OK;
    if (ad->rank < 8 || ad->rank > 128 || ad->rank % 8)
        return fail(QCONV_EUNSUPPORTED, "adapters: rank must be a multiple of 8 up to 128 (got %d)", ad->rank);
    if (x->channels % 8) return fail(QCONV_EUNSUPPORTED, "adapters need channels %% 8 == 0 (got %d)", x->channels);
    if (!ad->a || !ad->b || !ad->alpha || (x->rows > 0 && !ad->row))
        return fail(QCONV_EINVAL, "adapters: a, b, alpha and row must be non-NULL");
    if (!aligned(ad->a, 16) || !aligned(ad->b, 16) || !aligned(ad->alpha, 4) || !aligned(ad->row, 4))
        return fail(QCONV_EINVAL, "adapters: a and b must be 16-byte, alpha and row 4-byte aligned");
    return QCONV_OK;
}

size_t adapter_workspace(int64_t m, int64_t c, const qconv_adapters *ad) {
    if (!ad || ad->count == 0 || m == 0) return 0;
    return (size_t)linear_adapter_splits(m, c) * (size_t)m * (size_t)ad->rank * 4;
}

int run_grad(GradArgs &a, bool transposed, int w_bits, int dtype, int64_t out_size, const qconv_rows *b, void *workspace,
             size_t workspace_bytes, void *stream) {
    int rc = check_tiles(a.ni, a.nj);
    if (rc != QCONV_OK) return rc;
    const size_t need = grad_workspace(a.ni, a.nj, a.nt);
    if ((rc = check_workspace(workspace, workspace_bytes, need)) != QCONV_OK) return rc;
    const Span out(a.out, strided_bytes(a.ni, a.nj, a.ldo, out_size)), ws(workspace, (int64_t)need);
    const Span in(a.p, transposed ? strided_bytes(a.nt, a.ni, a.ldp, 2) : strided_bytes(a.ni, a.nt, a.ldp, 2));
    for (const Span &s : {in, rows_span(b), scale_span(b)})
        if (out.meets(s) || ws.meets(s)) return fail(QCONV_EINVAL, "the output or the workspace overlaps an input");
    if (out.meets(ws)) return fail(QCONV_EINVAL, "the output overlaps the workspace");
    a.part = static_cast<float *>(workspace);
    a.ldpart = (a.nj + 3) / 4 * 4;
    const hipError_t e = launch_grad(a, transposed, w_bits, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(QCONV_EHIP, "gradient launch: %s", hipGetErrorString(e));
    return QCONV_OK;
}

}  // namespace

extern "C" {

int qconv_quantize_rows(const void *x, int32_t dtype, int64_t ldx, int32_t m, int32_t c, void *codes, int64_t pitch,
                        float *scale, void *stream) {
    clear_error();
    if (dtype != QCONV_BF16 && dtype != QCONV_F16 && dtype != QCONV_F32)
        return fail(QCONV_EINVAL, "dtype must be QCONV_BF16, QCONV_F16 or QCONV_F32 (got %d)", dtype);
    if (m < 0 || c < 1) return fail(QCONV_EINVAL, "m must be >= 0 and c >= 1 (got %d, %d)", m, c);
    if (c > kMaxChannels) return fail(QCONV_EUNSUPPORTED, "more than %d channels (got %d)", kMaxChannels, c);
    if (pitch % 16 || pitch < round16(c))
        return fail(QCONV_EINVAL, "pitch must be a multiple of 16 of at least %lld bytes (got %lld)", (long long)round16(c),
                    (long long)pitch);
    if (pitch > kMaxPitch) return fail(QCONV_EUNSUPPORTED, "pitch above 2^22 bytes");
    const int64_t size = dtype == QCONV_F32 ? 4 : 2;
    const int rc = check_matrix(x, m, c, ldx, size, "x");
    if (rc != QCONV_OK) return rc;
    if (m == 0) return QCONV_OK;
    if (!codes || !scale) return fail(QCONV_EINVAL, "codes and scale must be non-NULL");
    if (!aligned(codes, 16) || !aligned(scale, 4))
        return fail(QCONV_EINVAL, "codes must be 16-byte and scale 4-byte aligned");
    const Span in(x, strided_bytes(m, c, ldx, size)), out(codes, strided_bytes(m, round16(c), pitch, 1)),
        sc(scale, (int64_t)m * 4);
    if (in.meets(out) || in.meets(sc) || out.meets(sc)) return fail(QCONV_EINVAL, "x, codes and scale must not overlap");
    const QuantizeArgs a{x, ldx, static_cast<uint8_t *>(codes), pitch, scale, m, c};
    const hipError_t e = launch_quantize_rows(a, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(QCONV_EHIP, "quantiser launch: %s", hipGetErrorString(e));
    return QCONV_OK;
}

int qconv_linear_workspace_bytes(int32_t m, int32_t c, const qconv_adapters *adapters, size_t *bytes) {
    clear_error();
    if (!bytes) return fail(QCONV_EINVAL, "bytes is NULL");
    if (m < 0 || c < 1 || (adapters && (adapters->count < 0 || (adapters->count > 0 && adapters->rank < 1))))
        return fail(QCONV_EINVAL, "sizes must be positive");
    *bytes = adapter_workspace(m, c, adapters);
    return QCONV_OK;
}

int qconv_linear(const qconv_rows *x, const qconv_rows *w, const qconv_adapters *adapters, void *y, int32_t dtype,
                 int64_t ldy, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    int rc;
    if ((rc = check_rows(x, "x", false)) != QCONV_OK || (rc = check_rows(w, "w", true)) != QCONV_OK ||
        (rc = check_float16(dtype)) != QCONV_OK)
        return rc;
    if (x->channels != w->channels)
        return fail(QCONV_EINVAL, "x has %d channels, w %d", x->channels, w->channels);
    if (w->rows < 1) return fail(QCONV_EINVAL, "w has no rows");
    if (adapters && (rc = check_adapters(adapters, x)) != QCONV_OK) return rc;
    if ((rc = check_matrix(y, x->rows, w->rows, ldy, 2, "y")) != QCONV_OK ||
        (rc = check_tiles(x->rows, w->rows)) != QCONV_OK)
        return rc;
    if (x->rows == 0) return QCONV_OK;
    const size_t need = adapter_workspace(x->rows, x->channels, adapters);
    if ((rc = check_workspace(workspace, workspace_bytes, need)) != QCONV_OK) return rc;
    const Span out(y, strided_bytes(x->rows, w->rows, ldy, 2)), ws(workspace, (int64_t)need);
    for (const Span &s : {rows_span(x), scale_span(x), rows_span(w), scale_span(w)})
        if (out.meets(s) || ws.meets(s)) return fail(QCONV_EINVAL, "y or the workspace overlaps an input");
    if (out.meets(ws)) return fail(QCONV_EINVAL, "y overlaps the workspace");
    LinearArgs a{};
    a.x = rows_arg(x);
    a.w = rows_arg(w);
    a.y = y;
    a.ldy = ldy;
    a.m = x->rows;
    a.c = x->channels;
    a.k = w->rows;
    a.steps = (x->channels + 127) / 128;
    if (adapters && adapters->count) {
        const int64_t n = adapters->count, r = adapters->rank;
        for (const Span &s : {Span(adapters->a, n * r * a.c * 2), Span(adapters->b, n * r * a.k * 2),
                              Span(adapters->alpha, n * 4), Span(adapters->row, (int64_t)a.m * 4)})
            if (out.meets(s) || ws.meets(s)) return fail(QCONV_EINVAL, "y or the workspace overlaps an adapter");
        a.ad = {adapters->a, adapters->b, adapters->alpha, adapters->row, static_cast<float *>(workspace),
                adapters->count, adapters->rank, linear_adapter_splits(a.m, a.c)};
    }
    const hipError_t e = launch_linear(a, w->bits, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(QCONV_EHIP, "linear launch: %s", hipGetErrorString(e));
    return QCONV_OK;
}

int qconv_linear_grad_workspace_bytes(int32_t rows, int32_t cols, int32_t depth, size_t *bytes) {
    clear_error();
    if (!bytes) return fail(QCONV_EINVAL, "bytes is NULL");
    if (rows < 0 || cols < 1 || depth < 0) return fail(QCONV_EINVAL, "sizes must not be negative (cols: positive)");
    *bytes = rows == 0 ? 0 : grad_workspace(rows, cols, depth);
    return QCONV_OK;
}

int qconv_linear_grad_input(const void *dy, int32_t dtype, int64_t lddy, int32_t m, const qconv_rows *w, void *dx,
                            int64_t lddx, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    int rc;
    if ((rc = check_rows(w, "w", true)) != QCONV_OK || (rc = check_float16(dtype)) != QCONV_OK) return rc;
    if (w->rows < 1) return fail(QCONV_EINVAL, "w has no rows");
    if (m < 0) return fail(QCONV_EINVAL, "m must be >= 0 (got %d)", m);
    if (m > kMaxRows) return fail(QCONV_EUNSUPPORTED, "more than 2^22 rows (got %d)", m);
    if ((rc = check_matrix(dy, m, w->rows, lddy, 2, "dy")) != QCONV_OK ||
        (rc = check_matrix(dx, m, w->channels, lddx, 2, "dx")) != QCONV_OK)
        return rc;
    if (m == 0) return QCONV_OK;
    GradArgs a{};
    a.p = dy;
    a.ldp = lddy;
    a.b = rows_arg(w);
    a.out = dx;
    a.ldo = lddx;
    a.ni = m;
    a.nj = w->channels;
    a.nt = w->rows;
    a.vec_p = wide_rows(dy, lddy, 2, 16);
    return run_grad(a, false, w->bits, dtype, 2, w, workspace, workspace_bytes, stream);
}

int qconv_linear_grad_weight(const void *dy, int32_t dtype, int64_t lddy, int32_t k, const qconv_rows *x, float *dw,
                             int64_t lddw, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    int rc;
    if ((rc = check_rows(x, "x", false)) != QCONV_OK || (rc = check_float16(dtype)) != QCONV_OK) return rc;
    if (k < 1) return fail(QCONV_EINVAL, "k must be >= 1 (got %d)", k);
    if (k > kMaxRows) return fail(QCONV_EUNSUPPORTED, "more than 2^22 rows (got %d)", k);
    if ((rc = check_matrix(dy, x->rows, k, lddy, 2, "dy")) != QCONV_OK ||
        (rc = check_matrix(dw, k, x->channels, lddw, 4, "dw")) != QCONV_OK)
        return rc;
    GradArgs a{};
    a.p = dy;
    a.ldp = lddy;
    a.b = rows_arg(x);
    a.out = dw;
    a.ldo = lddw;
    a.ni = k;
    a.nj = x->channels;
    a.nt = x->rows;
    a.vec_p = wide_rows(dy, lddy, 2, 16);
    return run_grad(a, true, 8, dtype, 4, x, workspace, workspace_bytes, stream);
}

}  // extern "C"

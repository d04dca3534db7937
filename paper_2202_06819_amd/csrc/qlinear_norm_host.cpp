// Host side of the norm to 8-bit rows and its gradient: argument validation,
// workspace sizes and launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qlinear_checks.h"

using namespace qconv;

namespace {

int check_float(int32_t dtype, const char *name) {
    if (dtype != QCONV_BF16 && dtype != QCONV_F16 && dtype != QCONV_F32)
        return fail(QCONV_EINVAL, "%s must be QCONV_BF16, QCONV_F16 or QCONV_F32 (got %d)", name, dtype);
    return QCONV_OK;
}

int check_sizes(int32_t m, int32_t c) {
    if (m < 0 || c < 1) return fail(QCONV_EINVAL, "m must be >= 0 and c >= 1 (got %d, %d)", m, c);
    if (m > kMaxRows) return fail(QCONV_EUNSUPPORTED, "more than 2^22 rows (got %d)", m);
    if (c > kMaxChannels) return fail(QCONV_EUNSUPPORTED, "more than %d channels (got %d)", kMaxChannels, c);
    return QCONV_OK;
}

int64_t size_of(int32_t dtype) { return dtype == QCONV_F32 ? 4 : 2; }

size_t grad_bytes(int64_t m, int64_t c) { return (size_t)norm_grad_parts(m, c) * (size_t)((c + 3) / 4 * 4) * 4; }

}  // namespace

extern "C" {

int qconv_norm_rows(const void *x, int64_t ldx, const void *residual, int64_t ldr, void *sum, int64_t lds, int32_t dtype,
                    const void *gain, int32_t gain_dtype, double eps, int32_t m, int32_t c, void *codes, int64_t pitch,
                    float *scale, float *rstd, void *stream) {
    clear_error();
    int rc;
    if ((rc = check_float(dtype, "dtype")) != QCONV_OK || (rc = check_float(gain_dtype, "gain_dtype")) != QCONV_OK ||
        (rc = check_sizes(m, c)) != QCONV_OK)
        return rc;
    if (!(eps >= 0.0 && eps <= 1e30)) return fail(QCONV_EINVAL, "eps must be from 0 to 1e30 (got %g)", eps);
    if (pitch % 16 || pitch < round16(c))
        return fail(QCONV_EINVAL, "pitch must be a multiple of 16 of at least %lld bytes (got %lld)", (long long)round16(c),
                    (long long)pitch);
    if (pitch > kMaxPitch) return fail(QCONV_EUNSUPPORTED, "pitch above 2^22 bytes");
    const int64_t size = size_of(dtype);
    if ((rc = check_matrix(x, m, c, ldx, size, "x")) != QCONV_OK ||
        (rc = check_matrix(gain, 1, c, c, size_of(gain_dtype), "gain")) != QCONV_OK)
        return rc;
    if (m > 0 && !residual != !sum) return fail(QCONV_EINVAL, "residual and sum go together: both or neither");
    if ((residual || sum) && ((rc = check_matrix(residual, m, c, ldr, size, "residual")) != QCONV_OK ||
                              (rc = check_matrix(sum, m, c, lds, size, "sum")) != QCONV_OK))
        return rc;
    if (m == 0) return QCONV_OK;
    if (!codes || !scale) return fail(QCONV_EINVAL, "codes and scale must be non-NULL");
    if (!aligned(codes, 16) || !aligned(scale, 4) || !aligned(rstd, 4))
        return fail(QCONV_EINVAL, "codes must be 16-byte, scale and rstd 4-byte aligned");
    const int64_t one = (int64_t)m * 4;
    const Span in(x, strided_bytes(m, c, ldx, size)), add(residual, residual ? strided_bytes(m, c, ldr, size) : 0),
        g(gain, (int64_t)c * size_of(gain_dtype));
    const Span total(sum, sum ? strided_bytes(m, c, lds, size) : 0), out(codes, strided_bytes(m, round16(c), pitch, 1)),
        sc(scale, one), rs(rstd, rstd ? one : 0);
    for (const Span &o : {out, sc, rs})
        for (const Span &i : {in, add, g, total})
            if (o.meets(i)) return fail(QCONV_EINVAL, "codes, scale and rstd must not overlap another operand");
    if (out.meets(sc) || out.meets(rs) || sc.meets(rs)) return fail(QCONV_EINVAL, "codes, scale and rstd must not overlap");
    // every value of the sum is written by the lane that has read its summands
    const bool in_x = sum == x && (lds == ldx || m == 1), in_residual = sum == residual && (lds == ldr || m == 1);
    if (total.meets(g) || (total.meets(in) && !in_x) || (total.meets(add) && !in_residual))
        return fail(QCONV_EINVAL, "sum overlaps x, the residual or the gain (it may be the whole of x or of the residual)");
    const NormArgs a{x, residual, sum, ldx, ldr, lds, gain, static_cast<uint8_t *>(codes), pitch, scale, rstd, eps,
                     1.0 / c,
                     gain_dtype, m, c};
    const hipError_t e = launch_norm_rows(a, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(QCONV_EHIP, "norm launch: %s", hipGetErrorString(e));
    return QCONV_OK;
}

int qconv_norm_rows_grad_workspace_bytes(int32_t m, int32_t c, size_t *bytes) {
    clear_error();
    if (!bytes) return fail(QCONV_EINVAL, "bytes is NULL");
    const int rc = check_sizes(m, c);
    if (rc != QCONV_OK) return rc;
    *bytes = grad_bytes(m, c);
    return QCONV_OK;
}

int qconv_norm_rows_grad(const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *dsum, int64_t ldds,
                         int32_t dtype, const void *gain, int32_t gain_dtype, const float *rstd, int32_t m, int32_t c,
                         void *dx, int64_t lddx, float *dgain, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    int rc;
    if ((rc = check_float(dtype, "dtype")) != QCONV_OK || (rc = check_float(gain_dtype, "gain_dtype")) != QCONV_OK ||
        (rc = check_sizes(m, c)) != QCONV_OK)
        return rc;
    const int64_t size = size_of(dtype);
    if ((rc = check_matrix(dy, m, c, lddy, size, "dy")) != QCONV_OK || (rc = check_matrix(h, m, c, ldh, size, "h")) != QCONV_OK ||
        (dsum && (rc = check_matrix(dsum, m, c, ldds, size, "dsum")) != QCONV_OK) ||
        (rc = check_matrix(dx, m, c, lddx, size, "dx")) != QCONV_OK ||
        (rc = check_matrix(gain, 1, c, c, size_of(gain_dtype), "gain")) != QCONV_OK ||
        (rc = check_matrix(rstd, m, 1, 1, 4, "rstd")) != QCONV_OK || (rc = check_matrix(dgain, 1, c, c, 4, "dgain")) != QCONV_OK)
        return rc;
    const size_t need = grad_bytes(m, c);
    if ((rc = check_workspace(workspace, workspace_bytes, need)) != QCONV_OK) return rc;
    const Span add(dsum, dsum ? strided_bytes(m, c, ldds, size) : 0), out(dx, strided_bytes(m, c, lddx, size)),
        dg(dgain, (int64_t)c * 4), ws(workspace, (int64_t)need);
    for (const Span &i : {Span(dy, strided_bytes(m, c, lddy, size)), Span(h, strided_bytes(m, c, ldh, size)),
                          Span(gain, (int64_t)c * size_of(gain_dtype)), Span(rstd, (int64_t)m * 4), add}) {
        // every value of dx is written by the lane that has read dsum's
        const bool in_place = dsum && dx == dsum && (lddx == ldds || m == 1) && i.begin == add.begin && i.end == add.end;
        if ((out.meets(i) && !in_place) || dg.meets(i) || ws.meets(i))
            return fail(QCONV_EINVAL, "an output or the workspace overlaps an input (dx may be the whole of dsum)");
    }
    if (out.meets(dg) || out.meets(ws) || dg.meets(ws))
        return fail(QCONV_EINVAL, "the outputs and the workspace must not overlap");
    const NormGradArgs a{dy, h, dsum, dx, lddy, ldh, ldds, lddx, gain, rstd, dgain, static_cast<float *>(workspace),
                         (c + 3) / 4 * 4, gain_dtype, m, c, norm_grad_parts(m, c)};
    const hipError_t e = launch_norm_grad(a, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(QCONV_EHIP, "norm gradient launch: %s", hipGetErrorString(e));
    return QCONV_OK;
}

}  // extern "C"

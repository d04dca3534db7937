// Host side of the products with scales of groups of channels and of the experts'
// products: argument validation and launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "qlinear_checks.h"
#include "qlinear_plan.h"

using namespace qconv;

namespace {

constexpr int32_t kMaxGroup = 4096, kMaxExperts = 4096;
constexpr int64_t kMaxScalePitch = 1 << 17;

// The weights of a call, of either form.
struct Weights {
    RowsArg rows;
    GroupArg groups{};
    int32_t channels = 0, bits = 4, scale_bytes = 0, group = 0;   // scale_bytes 0: one scale a row
    Span codes{nullptr, 0}, scale{nullptr, 0};
};

int weights_of(const qconv_rows *w, Weights &to) {
    const int rc = check_rows(w, "w", true);
    if (rc != QCONV_OK) return rc;
    to.rows = rows_arg(w);
    to.channels = w->channels;
    to.bits = w->bits;
    to.codes = rows_span(w);
    to.scale = scale_span(w);
    return QCONV_OK;
}

int weights_of(const qconv_group_rows *w, Weights &to) {
    if (!w) return fail(QCONV_EINVAL, "w is NULL");
    if (w->scale_dtype != QCONV_BF16 && w->scale_dtype != QCONV_F16 && w->scale_dtype != QCONV_F32)
        return fail(QCONV_EINVAL, "w: scale_dtype must be QCONV_BF16, QCONV_F16 or QCONV_F32 (got %d)", w->scale_dtype);
    if (w->group < 32 || w->group % 32 || w->group > kMaxGroup)
        return fail(QCONV_EUNSUPPORTED, "w: group must be a multiple of 32 up to %d (got %d)", kMaxGroup, w->group);
    const int64_t size = w->scale_dtype == QCONV_F32 ? 4 : 2;
    // (the codes as those of 4-bit rows; their scales are another matter)
    static const float any = 0;
    const qconv_rows codes{w->codes, &any, w->pitch, w->rows, w->channels, 4};
    int rc = check_rows(&codes, "w", true);
    if (rc != QCONV_OK) return rc;
    const int64_t groups = (w->channels + w->group - 1) / w->group;
    if (w->scale_pitch < groups)
        return fail(QCONV_EINVAL, "w: %lld scales from row to row, fewer than its %lld groups", (long long)w->scale_pitch,
                    (long long)groups);
    if (w->scale_pitch > kMaxScalePitch) return fail(QCONV_EUNSUPPORTED, "w: more than 2^17 scales from row to row");
    if (w->rows > 0 && !w->scale) return fail(QCONV_EINVAL, "w: scale must be non-NULL");
    if (!aligned(w->scale, (uintptr_t)size)) return fail(QCONV_EINVAL, "w: scale must be aligned to its elements");
    to.rows = {static_cast<const uint8_t *>(w->codes), nullptr, w->pitch, (int32_t)rows_used(&codes), w->rows};
    const uint32_t per = (uint32_t)w->group / 32;
    to.groups = {w->scale, w->scale_pitch, ((1u << 20) + per - 1) / per, w->scale_dtype == QCONV_BF16};
    to.channels = w->channels;
    to.scale_bytes = (int32_t)size;
    to.group = w->group;
    to.codes = rows_span(&codes);
    to.scale = Span(w->scale, strided_bytes(w->rows, groups, w->scale_pitch, size));
    return QCONV_OK;
}

int check_experts(const int32_t *offsets, int32_t count) {
    if (count < 1) return fail(QCONV_EINVAL, "experts: count must be >= 1 (got %d)", count);
    if (count > kMaxExperts) return fail(QCONV_EUNSUPPORTED, "more than %d experts (got %d)", kMaxExperts, count);
    if (!offsets || !aligned(offsets, 4)) return fail(QCONV_EINVAL, "experts: offsets must be non-NULL and 4-byte aligned");
    return QCONV_OK;
}
Span offsets_span(const int32_t *offsets, int32_t count) { return Span(offsets, offsets ? ((int64_t)count + 1) * 4 : 0); }

// Tiles of experts' rows: one of each may be partly filled.
int check_expert_tiles(int64_t m, int64_t count, int64_t cols) { return check_tiles(m + 64 * std::min(m, count), cols); }

template <class W>
int forward(const qconv_rows *x, const W *w, const int32_t *offsets, int32_t count, void *y, int32_t dtype, int64_t ldy,
            void *stream) {
    clear_error();
    int rc;
    Weights ws;
    if ((rc = check_rows(x, "x", false)) != QCONV_OK || (rc = weights_of(w, ws)) != QCONV_OK ||
        (rc = check_float16(dtype)) != QCONV_OK || (count >= 0 && (rc = check_experts(offsets, count)) != QCONV_OK))
        return rc;
    const bool experts = count >= 0;
    if (x->channels != ws.channels) return fail(QCONV_EINVAL, "x has %d channels, w %d", x->channels, ws.channels);
    if (w->rows < 1) return fail(QCONV_EINVAL, "w has no rows");
    if (experts && w->rows % count) return fail(QCONV_EINVAL, "w: %d rows are not those of %d experts", w->rows, count);
    const int32_t k = experts ? w->rows / count : w->rows;
    if ((rc = check_matrix(y, x->rows, k, ldy, 2, "y")) != QCONV_OK ||
        (rc = experts ? check_expert_tiles(x->rows, count, k) : check_tiles(x->rows, k)) != QCONV_OK)
        return rc;
    if (x->rows == 0) return QCONV_OK;
    const Span out(y, strided_bytes(x->rows, k, ldy, 2));
    for (const Span &s : {rows_span(x), scale_span(x), ws.codes, ws.scale, offsets_span(offsets, count)})
        if (out.meets(s)) return fail(QCONV_EINVAL, "y overlaps an input");
    LinearArgs a{};
    a.x = rows_arg(x);
    a.w = ws.rows;
    a.y = y;
    a.ldy = ldy;
    a.m = x->rows;
    a.c = x->channels;
    a.k = k;
    a.steps = (x->channels + 127) / 128;
    const ExpertArg ex{offsets, count, x->rows};
    hipError_t e;
    if (!experts) e = launch_groups(a, ws.groups, ws.scale_bytes, ws.group, dtype, (hipStream_t)stream);
    else if (ws.scale_bytes) e = launch_expert_groups(a, ws.groups, ex, ws.scale_bytes, ws.group, dtype, (hipStream_t)stream);
    else e = launch_experts(a, ex, ws.bits, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(QCONV_EHIP, "product launch: %s", hipGetErrorString(e));
    return QCONV_OK;
}

// dx = dy w, of all rows (count < 0) or of experts' rows.
template <class W>
int grad_input(const void *dy, int32_t dtype, int64_t lddy, int32_t m, const W *w, const int32_t *offsets, int32_t count,
               void *dx, int64_t lddx, void *workspace, size_t workspace_bytes, void *stream) {
    clear_error();
    int rc;
    Weights ws;
    if ((rc = weights_of(w, ws)) != QCONV_OK || (rc = check_float16(dtype)) != QCONV_OK ||
        (count >= 0 && (rc = check_experts(offsets, count)) != QCONV_OK))
        return rc;
    const bool experts = count >= 0;
    if (w->rows < 1) return fail(QCONV_EINVAL, "w has no rows");
    if (experts && w->rows % count) return fail(QCONV_EINVAL, "w: %d rows are not those of %d experts", w->rows, count);
    if (m < 0) return fail(QCONV_EINVAL, "m must be >= 0 (got %d)", m);
    if (m > kMaxRows) return fail(QCONV_EUNSUPPORTED, "more than 2^22 rows (got %d)", m);
    const int32_t k = experts ? w->rows / count : w->rows;
    if ((rc = check_matrix(dy, m, k, lddy, 2, "dy")) != QCONV_OK ||
        (rc = check_matrix(dx, m, ws.channels, lddx, 2, "dx")) != QCONV_OK ||
        (rc = experts ? check_expert_tiles(m, count, ws.channels) : check_tiles(m, ws.channels)) != QCONV_OK)
        return rc;
    if (m == 0) return QCONV_OK;
    const size_t need = experts ? 0 : grad_workspace(m, ws.channels, k);
    if ((rc = check_workspace(workspace, workspace_bytes, need)) != QCONV_OK) return rc;
    const Span out(dx, strided_bytes(m, ws.channels, lddx, 2)), scratch(workspace, (int64_t)need);
    for (const Span &s : {Span(dy, strided_bytes(m, k, lddy, 2)), ws.codes, ws.scale, offsets_span(offsets, count)})
        if (out.meets(s) || scratch.meets(s)) return fail(QCONV_EINVAL, "the output or the workspace overlaps an input");
    if (out.meets(scratch)) return fail(QCONV_EINVAL, "the output overlaps the workspace");
    GradArgs a{};
    a.p = dy;
    a.ldp = lddy;
    a.b = ws.rows;
    a.out = dx;
    a.ldo = lddx;
    a.part = static_cast<float *>(workspace);
    a.ldpart = (ws.channels + 3) / 4 * 4;
    a.ni = m;
    a.nj = ws.channels;
    a.nt = k;
    a.vec_p = wide_rows(dy, lddy, 2, 16);
    const hipError_t e =
        experts ? launch_expert_grad_input(a, ws.groups, {offsets, count, m}, ws.bits, ws.scale_bytes, dtype, (hipStream_t)stream)
                : launch_group_grad(a, ws.groups, ws.scale_bytes, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(QCONV_EHIP, "gradient launch: %s", hipGetErrorString(e));
    return QCONV_OK;
}

}  // namespace

extern "C" {

int qconv_linear_groups(const qconv_rows *x, const qconv_group_rows *w, void *y, int32_t dtype, int64_t ldy, void *stream) {
    return forward(x, w, nullptr, -1, y, dtype, ldy, stream);
}

int qconv_linear_groups_grad_input(const void *dy, int32_t dtype, int64_t lddy, int32_t m, const qconv_group_rows *w, void *dx,
                                   int64_t lddx, void *workspace, size_t workspace_bytes, void *stream) {
    return grad_input(dy, dtype, lddy, m, w, nullptr, -1, dx, lddx, workspace, workspace_bytes, stream);
}

int qconv_linear_experts(const qconv_rows *x, const qconv_rows *w, const int32_t *offsets, int32_t experts, void *y,
                         int32_t dtype, int64_t ldy, void *stream) {
    return forward(x, w, offsets, std::max(experts, 0), y, dtype, ldy, stream);
}

int qconv_linear_experts_groups(const qconv_rows *x, const qconv_group_rows *w, const int32_t *offsets, int32_t experts,
                                void *y, int32_t dtype, int64_t ldy, void *stream) {
    return forward(x, w, offsets, std::max(experts, 0), y, dtype, ldy, stream);
}

int qconv_linear_experts_grad_input(const void *dy, int32_t dtype, int64_t lddy, int32_t m, const qconv_rows *w,
                                    const int32_t *offsets, int32_t experts, void *dx, int64_t lddx, void *stream) {
    return grad_input(dy, dtype, lddy, m, w, offsets, std::max(experts, 0), dx, lddx, nullptr, 0, stream);
}

int qconv_linear_experts_groups_grad_input(const void *dy, int32_t dtype, int64_t lddy, int32_t m, const qconv_group_rows *w,
                                           const int32_t *offsets, int32_t experts, void *dx, int64_t lddx, void *stream) {
    return grad_input(dy, dtype, lddy, m, w, offsets, std::max(experts, 0), dx, lddx, nullptr, 0, stream);
}

int qconv_linear_experts_grad_weight(const void *dy, int32_t dtype, int64_t lddy, int32_t k, const qconv_rows *x,
                                     const int32_t *offsets, int32_t experts, float *dw, int64_t lddw, void *stream) {
    clear_error();
    int rc;
    if ((rc = check_rows(x, "x", false)) != QCONV_OK || (rc = check_float16(dtype)) != QCONV_OK ||
        (rc = check_experts(offsets, experts)) != QCONV_OK)
        return rc;
    if (k < 1) return fail(QCONV_EINVAL, "k must be >= 1 (got %d)", k);
    const int64_t rows = (int64_t)experts * k;
    if (rows > kMaxRows) return fail(QCONV_EUNSUPPORTED, "more than 2^22 rows of weights (got %lld)", (long long)rows);
    if ((rc = check_matrix(dy, x->rows, k, lddy, 2, "dy")) != QCONV_OK ||
        (rc = check_matrix(dw, rows, x->channels, lddw, 4, "dw")) != QCONV_OK ||
        (rc = check_tiles((int64_t)experts * ((k + 63) / 64 * 64), x->channels)) != QCONV_OK)
        return rc;
    const Span out(dw, strided_bytes(rows, x->channels, lddw, 4));
    for (const Span &s : {Span(dy, strided_bytes(x->rows, k, lddy, 2)), rows_span(x), scale_span(x), offsets_span(offsets, experts)})
        if (out.meets(s)) return fail(QCONV_EINVAL, "the output overlaps an input");
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
    const hipError_t e = launch_expert_grad_weight(a, {offsets, experts, x->rows}, dtype, (hipStream_t)stream);
    if (e != hipSuccess) return fail(QCONV_EHIP, "gradient launch: %s", hipGetErrorString(e));
    return QCONV_OK;
}

}  // extern "C"

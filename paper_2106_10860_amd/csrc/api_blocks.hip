// extern "C" entry points of the exact 8-bit product and of layers of experts: argument checks, then the launchers.
#include "api_checks.h"
#include "block_common.h"

using namespace maddness;

namespace {

// 8-bit values and their exponents.
int check_blocks(const void *q, int64_t cols, int64_t ld, int64_t stride, const void *scale, int64_t lds, int64_t scale_stride, const char *name)
{
    if (!q || !scale) return fail(MADDNESS_E_INVAL, "%s: values or exponents are NULL", name);
    if (ld < cols) return fail(MADDNESS_E_INVAL, "%s: ld = %lld is smaller than its %lld columns", name, (long long)ld, (long long)cols);
    if (lds < ceil_div(cols, (int64_t)kBlock))
        return fail(MADDNESS_E_INVAL, "%s: lds = %lld is smaller than its %lld blocks", name, (long long)lds, (long long)ceil_div(cols, (int64_t)kBlock));
    if (!aligned(q, 16) || ld % 16 || stride % 16) return fail(MADDNESS_E_ALIGN, "%s: values not 16-byte aligned, or a stride that is no multiple of 16", name);
    if (!aligned(scale, 4) || lds % 4 || scale_stride % 4)
        return fail(MADDNESS_E_ALIGN, "%s: exponents not 4-byte aligned, or a stride that is no multiple of 4", name);
    return MADDNESS_OK;
}

int check_matrix(const maddness_block_matrix *m, bool may_float, const char *name)
{
    if (!m) return fail(MADDNESS_E_INVAL, "%s is NULL", name);
    int rc;
    if ((rc = check_size(m->rows, name)) != MADDNESS_OK || (rc = check_size(m->cols, name)) != MADDNESS_OK) return rc;
    if (m->dtype != kE4M3) {
        if (!may_float) return fail(MADDNESS_E_UNSUPPORTED, "%s: dtype = %d, only MADDNESS_E4M3 is supported here", name, m->dtype);
        return check_floats(m->data, m->dtype, m->rows, m->cols, m->ld, name);
    }
    if (m->tile != 1 && m->tile != kBlock) return fail(MADDNESS_E_INVAL, "%s: tile = %d, must be 1 or 128", name, m->tile);
    if (m->rows == 0 || m->cols == 0) return MADDNESS_OK;
    return check_blocks(m->data, m->cols, m->ld, m->stride, m->scale, m->lds, m->scale_stride, name);
}

int check_experts(int32_t E)
{
    if (E < 1 || E > MADDNESS_MAX_EXPERTS) return fail(MADDNESS_E_UNSUPPORTED, "E = %d, supported are 1..%d experts", E, MADDNESS_MAX_EXPERTS);
    return MADDNESS_OK;
}

// Rounded rows of a floating A: where they lie in the workspace.
struct Rounded {
    int64_t ld, lds, scale_at, bytes;
    Rounded(int64_t M, int64_t K)
    {
        ld = round_up(K, (int64_t)16);
        lds = round_up(ceil_div(K, (int64_t)kBlock), (int64_t)4);
        scale_at = M * ld;
        bytes = scale_at + M * lds;
    }
};

}  // namespace

extern "C" {

int maddness_quantise_blocks(const void *x, int32_t dtype, int64_t count, int64_t rows, int64_t cols, int64_t ldx, int64_t stride_x,
                             int32_t tile, const int32_t *source, int64_t source_rows, int32_t repeat, const float *factors, uint8_t *q,
                             int64_t ldq, uint8_t *scale, int64_t lds, uint8_t *qt, int64_t ldqt, uint8_t *scale_t, int64_t ldst,
                             void *stream)
{
    begin_call();
    int rc;
    if ((rc = check_size(rows, "rows")) != MADDNESS_OK || (rc = check_size(cols, "cols")) != MADDNESS_OK) return rc;
    if (count < 0) return fail(MADDNESS_E_INVAL, "count = %lld is negative", (long long)count);
    if (count > 65535) return fail(MADDNESS_E_UNSUPPORTED, "count = %lld, supported are up to 65535 matrices", (long long)count);
    if (tile != 1 && tile != kBlock) return fail(MADDNESS_E_INVAL, "tile = %d, must be 1 or 128", tile);
    if (!floating(dtype)) return fail(MADDNESS_E_INVAL, "x: dtype = %d is not F32, F16 or BF16", dtype);
    if (source) {
        if (count != 1) return fail(MADDNESS_E_INVAL, "source goes with one matrix, count = %lld", (long long)count);
        if (repeat < 1) return fail(MADDNESS_E_INVAL, "repeat = %d, must be >= 1", repeat);
        if ((rc = check_size(source_rows, "source_rows")) != MADDNESS_OK) return rc;
        if (source_rows * repeat > kMostRows) return fail(MADDNESS_E_UNSUPPORTED, "source_rows repeat = %lld, supported are up to 2^31 - 1", (long long)(source_rows * repeat));
        if (!aligned(source, 4) || !aligned(factors, 4)) return fail(MADDNESS_E_ALIGN, "source / factors not 4-byte aligned");
    }
    if (count == 0 || rows == 0 || cols == 0) return MADDNESS_OK;
    if (factors && !source) return fail(MADDNESS_E_INVAL, "factors without source");
    if ((rc = check_floats(x, dtype, source ? source_rows : rows, cols, ldx, "x")) != MADDNESS_OK) return rc;
    if (!q && !qt) return fail(MADDNESS_E_INVAL, "both q and qt are NULL");
    if (q && (rc = check_blocks(q, cols, ldq, 0, scale, lds, 0, "q")) != MADDNESS_OK) return rc;
    if (qt && (rc = check_blocks(qt, rows, ldqt, 0, scale_t, ldst, 0, "qt")) != MADDNESS_OK) return rc;
    if ((qt || tile != 1) && ceil_div(rows, (int64_t)kBlock) * ceil_div(cols, (int64_t)kBlock) > kMostRows)
        return fail(MADDNESS_E_UNSUPPORTED, "%lld x %lld values are too many", (long long)rows, (long long)cols);
    return launch_quantise_blocks(x, dtype, count, rows, cols, ldx, stride_x, tile, source, source ? source_rows : 0, source ? repeat : 1, factors, q,
                                  ldq, scale, lds, qt, ldqt, scale_t, ldst, static_cast<hipStream_t>(stream));
}

size_t maddness_block_product_workspace(int64_t a_rows, int64_t K, int32_t by, int32_t a_dtype)
{
    if (a_rows < 1 || K < 1 || a_dtype == kE4M3 || rounds_inside(a_rows, K, by)) return 0;
    return (size_t)Rounded(a_rows, K).bytes;
}

int maddness_block_product(const maddness_block_matrix *A, const maddness_block_matrix *B, int32_t by, int32_t groups, const int32_t *offsets,
                           const int32_t *source, int64_t slots, int32_t repeat, void *out, int32_t out_dtype, int64_t ldo, void *workspace,
                           size_t workspace_bytes, void *stream)
{
    begin_call();
    if (by != MADDNESS_DENSE && by != MADDNESS_BY_ROWS && by != MADDNESS_BY_DEPTH && by != MADDNESS_BY_CHOICE) return fail(MADDNESS_E_INVAL, "by = %d is not a maddness_product_groups", by);
    int rc;
    if ((rc = check_matrix(A, by != MADDNESS_BY_DEPTH, "A")) != MADDNESS_OK || (rc = check_matrix(B, false, "B")) != MADDNESS_OK) return rc;
    if (A->cols != B->cols) return fail(MADDNESS_E_INVAL, "A has %lld columns and B %lld", (long long)A->cols, (long long)B->cols);
    if (!floating(out_dtype)) return fail(MADDNESS_E_INVAL, "out: dtype = %d is not F32, F16 or BF16", out_dtype);
    if (by == MADDNESS_BY_CHOICE) {
        if ((rc = check_size(slots, "slots")) != MADDNESS_OK) return rc;
        if (slots > MADDNESS_MAX_CHOSEN) return fail(MADDNESS_E_UNSUPPORTED, "slots = %lld, supported are up to %d", (long long)slots, MADDNESS_MAX_CHOSEN);
        if (repeat < 1) return fail(MADDNESS_E_INVAL, "repeat = %d, must be >= 1", repeat);
        if (A->rows < ceil_div(slots, (int64_t)repeat))
            return fail(MADDNESS_E_INVAL, "A has %lld rows, %lld slots of %d to a row go with more", (long long)A->rows, (long long)slots, repeat);
        if (slots > 0 && !source) return fail(MADDNESS_E_INVAL, "source is NULL");
        if (!aligned(source, 4)) return fail(MADDNESS_E_ALIGN, "source not 4-byte aligned");
    } else if (source) {
        if (by != MADDNESS_BY_ROWS) return fail(MADDNESS_E_INVAL, "source goes with MADDNESS_BY_ROWS");
        if (repeat < 1) return fail(MADDNESS_E_INVAL, "repeat = %d, must be >= 1", repeat);
        if ((rc = check_size(slots, "slots")) != MADDNESS_OK) return rc;
        if (A->rows * repeat > kMostRows) return fail(MADDNESS_E_UNSUPPORTED, "A's rows times repeat = %lld, supported are up to 2^31 - 1", (long long)(A->rows * repeat));
        if (!aligned(source, 4)) return fail(MADDNESS_E_ALIGN, "source not 4-byte aligned");
    }
    const int64_t M = source || by == MADDNESS_BY_CHOICE ? slots : A->rows, N = B->rows, K = A->cols;
    if (by == MADDNESS_DENSE) {
        groups = 1;
    } else {
        if (groups < 1) return fail(MADDNESS_E_INVAL, "groups = %d, must be >= 1", groups);
        if (groups > 65535) return fail(MADDNESS_E_UNSUPPORTED, "groups = %d, supported are up to 65535", groups);
        if (!offsets && by != MADDNESS_BY_CHOICE) return fail(MADDNESS_E_INVAL, "offsets is NULL");
        if (!aligned(offsets, 4)) return fail(MADDNESS_E_ALIGN, "offsets not 4-byte aligned");
        if (by == MADDNESS_BY_DEPTH && K > 0 && (A->tile != 1 || B->tile != 1)) return fail(MADDNESS_E_INVAL, "A and B must have tile 1 to be cut by depth");
    }
    if (M == 0 || N == 0 || (source && A->rows == 0)) return MADDNESS_OK;
    if ((rc = check_floats(out, out_dtype, M, N, ldo, "out")) != MADDNESS_OK) return rc;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    ProductArgs p{};
    p.a = static_cast<const uint8_t *>(A->data); p.lda = A->ld;
    p.b = static_cast<const uint8_t *>(B->data); p.ldb = B->ld; p.stride_b = B->stride;
    p.scale_a = A->scale; p.lds_a = A->lds; p.shift_a = A->tile == kBlock ? 7 : 0;
    p.scale_b = B->scale; p.lds_b = B->lds; p.scale_stride_b = B->scale_stride; p.shift_b = B->tile == kBlock ? 7 : 0;
    p.M = M; p.N = N; p.K = K; p.a_rows = A->rows; p.by = by; p.groups = groups; p.offsets = offsets;
    p.source = source; p.source_limit = source ? A->rows * repeat : 0; p.repeat = source ? repeat : 1;
    p.out = out; p.ldo = ldo; p.out_stride = M * ldo;
    int a_dtype = A->dtype;
    if (a_dtype != kE4M3 && !rounds_inside(A->rows, K, by)) {
        if (K > 0) {
            const Rounded r(A->rows, K);
            if (!workspace || workspace_bytes < (size_t)r.bytes)
                return fail(MADDNESS_E_UNSUPPORTED, "workspace of %zu bytes given, %lld needed", workspace_bytes, (long long)r.bytes);
            if (!aligned(workspace, 16)) return fail(MADDNESS_E_ALIGN, "workspace not 16-byte aligned");
            uint8_t *q = static_cast<uint8_t *>(workspace), *scale = q + r.scale_at;
            rc = launch_quantise_blocks(A->data, a_dtype, 1, A->rows, K, A->ld, 0, 1, nullptr, 0, 1, nullptr, q, r.ld, scale, r.lds, nullptr, 0, nullptr, 0, s);
            if (rc != MADDNESS_OK) return rc;
            p.a = q; p.lda = r.ld; p.scale_a = scale; p.lds_a = r.lds; p.shift_a = 0;
        }
        a_dtype = kE4M3;
    }
    return launch_block_product(p, a_dtype, out_dtype, s);
}

static int check_route(const void *logits, int32_t dtype, int64_t T, int32_t E, int64_t ldl, int32_t scores, int32_t k)
{
    int rc;
    if ((rc = check_size(T, "T")) != MADDNESS_OK || (rc = check_experts(E)) != MADDNESS_OK) return rc;
    if (scores != MADDNESS_SOFTMAX && scores != MADDNESS_SIGMOID) return fail(MADDNESS_E_INVAL, "scores = %d is not a maddness_scores", scores);
    if (k < 1 || k > E) return fail(MADDNESS_E_INVAL, "k = %d, must be 1..E = %d", k, E);
    if (k > MADDNESS_MAX_CHOICE) return fail(MADDNESS_E_UNSUPPORTED, "k = %d, supported are up to %d", k, MADDNESS_MAX_CHOICE);
    return check_floats(logits, dtype, T, E, ldl, "logits");
}

int maddness_route(const void *logits, int32_t dtype, int64_t T, int32_t E, int64_t ldl, const float *bias, int32_t scores, int32_t groups,
                   int32_t kept_groups, int32_t k, int32_t renormalise, float factor, int32_t *ids, float *weights, void *stream)
{
    begin_call();
    int rc = check_route(logits, dtype, T, E, ldl, scores, k);
    if (rc != MADDNESS_OK) return rc;
    if (groups < 1 || E % groups) return fail(MADDNESS_E_INVAL, "groups = %d does not divide E = %d", groups, E);
    if (groups > 64) return fail(MADDNESS_E_UNSUPPORTED, "groups = %d, supported are up to 64", groups);
    if (kept_groups < 1 || kept_groups > groups) return fail(MADDNESS_E_INVAL, "kept_groups = %d, must be 1..groups = %d", kept_groups, groups);
    if (T == 0) return MADDNESS_OK;
    if (!ids || !weights) return fail(MADDNESS_E_INVAL, "ids / weights is NULL");
    if (!aligned(ids, 4) || !aligned(weights, 4) || !aligned(bias, 4)) return fail(MADDNESS_E_ALIGN, "ids / weights / bias not 4-byte aligned");
    return launch_route(logits, dtype, T, E, ldl, bias, scores, groups, kept_groups, k, renormalise != 0, factor, ids, weights,
                        static_cast<hipStream_t>(stream));
}

int maddness_route_gradient(const void *logits, int32_t dtype, int64_t T, int32_t E, int64_t ldl, int32_t scores, int32_t k, int32_t renormalise,
                            float factor, const int32_t *ids, const float *weights_gradient, void *gradient, int64_t ldd, void *stream)
{
    begin_call();
    int rc = check_route(logits, dtype, T, E, ldl, scores, k);
    if (rc != MADDNESS_OK) return rc;
    if (T == 0) return MADDNESS_OK;
    if (!ids || !weights_gradient) return fail(MADDNESS_E_INVAL, "ids / weights_gradient is NULL");
    if ((rc = check_floats(gradient, dtype, T, E, ldd, "gradient")) != MADDNESS_OK) return rc;
    if (!aligned(ids, 4) || !aligned(weights_gradient, 4)) return fail(MADDNESS_E_ALIGN, "ids / weights_gradient not 4-byte aligned");
    return launch_route_gradient(logits, dtype, T, E, ldl, scores, k, renormalise != 0, factor, ids, weights_gradient, gradient, ldd,
                                 static_cast<hipStream_t>(stream));
}

int64_t maddness_order_capacity(int64_t slots, int32_t E, int32_t align)
{
    if (slots < 0 || slots > kMostRows || E < 1 || E > MADDNESS_MAX_EXPERTS || align < 1 || align > 65536) return 0;
    return slots + std::min(slots, (int64_t)E) * (align - 1);
}

size_t maddness_order_workspace(int64_t slots, int32_t E)
{
    if (slots < 0 || slots > kMostRows || E < 1 || E > MADDNESS_MAX_EXPERTS) return 0;
    return order_workspace_bytes(slots, E);
}

int maddness_order(const int32_t *ids, int64_t slots, int32_t E, int32_t align, int32_t *offsets, int32_t *counts, int32_t *source, int64_t capacity,
                   int32_t *place, void *workspace, size_t workspace_bytes, void *stream)
{
    begin_call();
    int rc;
    if ((rc = check_size(slots, "slots")) != MADDNESS_OK || (rc = check_experts(E)) != MADDNESS_OK) return rc;
    if (align < 1 || align > 65536) return fail(MADDNESS_E_INVAL, "align = %d, must be 1..65536", align);
    if (capacity < maddness_order_capacity(slots, E, align))
        return fail(MADDNESS_E_INVAL, "capacity = %lld is smaller than the %lld places that may be needed", (long long)capacity,
                    (long long)maddness_order_capacity(slots, E, align));
    if ((rc = check_size(capacity, "capacity")) != MADDNESS_OK) return rc;
    if (!offsets) return fail(MADDNESS_E_INVAL, "offsets is NULL");
    if (slots > 0 && (!ids || !source || !place)) return fail(MADDNESS_E_INVAL, "ids / source / place is NULL");
    if (!aligned(ids, 4) || !aligned(offsets, 4) || !aligned(counts, 4) || !aligned(source, 4) || !aligned(place, 4) || !aligned(workspace, 4))
        return fail(MADDNESS_E_ALIGN, "ids / offsets / counts / source / place / workspace not 4-byte aligned");
    if (!source && capacity > 0) return fail(MADDNESS_E_INVAL, "source is NULL");
    const size_t need = order_workspace_bytes(slots, E);
    if (!workspace || workspace_bytes < need) return fail(MADDNESS_E_UNSUPPORTED, "workspace of %zu bytes given, %zu needed", workspace_bytes, need);
    return launch_order(ids, slots, E, align, offsets, counts, source, capacity, place, workspace, static_cast<hipStream_t>(stream));
}

static int check_combine(const void *y, int32_t y_dtype, int64_t rows, int64_t N, int64_t ldy, const int32_t *place, int64_t T, int32_t k)
{
    int rc;
    if ((rc = check_size(rows, "rows")) != MADDNESS_OK || (rc = check_size(N, "N")) != MADDNESS_OK || (rc = check_size(T, "T")) != MADDNESS_OK) return rc;
    if (k < 1) return fail(MADDNESS_E_INVAL, "k = %d, must be >= 1", k);
    if ((rc = check_floats(y, y_dtype, rows, N, ldy, "y")) != MADDNESS_OK) return rc;
    if (!place && T * k > rows) return fail(MADDNESS_E_INVAL, "place is NULL and y has %lld rows, fewer than T k = %lld", (long long)rows, (long long)(T * k));
    if (!aligned(place, 4)) return fail(MADDNESS_E_ALIGN, "place not 4-byte aligned");
    return MADDNESS_OK;
}

int maddness_combine(const void *y, int32_t y_dtype, int64_t rows, int64_t N, int64_t ldy, const int32_t *place, const float *weights, int64_t T,
                     int32_t k, void *out, int32_t out_dtype, int64_t ldo, void *stream)
{
    begin_call();
    int rc = check_combine(y, y_dtype, rows, N, ldy, place, T, k);
    if (rc != MADDNESS_OK) return rc;
    if ((rc = check_floats(out, out_dtype, T, N, ldo, "out")) != MADDNESS_OK) return rc;
    if (!aligned(weights, 4)) return fail(MADDNESS_E_ALIGN, "weights not 4-byte aligned");
    if (T == 0 || N == 0) return MADDNESS_OK;
    return launch_combine(y, y_dtype, rows, N, ldy, place, weights, T, k, out, out_dtype, ldo, static_cast<hipStream_t>(stream));
}

int maddness_combine_gradient(const void *gradient, int32_t dtype, int64_t ldg, const void *y, int32_t y_dtype, int64_t rows, int64_t N, int64_t ldy,
                              const int32_t *place, int64_t T, int32_t k, float *weights_gradient, void *stream)
{
    begin_call();
    int rc = check_combine(y, y_dtype, rows, N, ldy, place, T, k);
    if (rc != MADDNESS_OK) return rc;
    if ((rc = check_floats(gradient, dtype, T, N, ldg, "gradient")) != MADDNESS_OK) return rc;
    if (T == 0) return MADDNESS_OK;
    if (!weights_gradient) return fail(MADDNESS_E_INVAL, "weights_gradient is NULL");
    if (!aligned(weights_gradient, 4)) return fail(MADDNESS_E_ALIGN, "weights_gradient not 4-byte aligned");
    return launch_combine_gradient(gradient, dtype, ldg, y, y_dtype, rows, N, ldy, place, T, k, weights_gradient, static_cast<hipStream_t>(stream));
}

}  // extern "C"

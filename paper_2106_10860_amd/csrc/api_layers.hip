// extern "C" entry points of the integer product, the layer norm, the balance of experts and the gradients' norm: argument checks, then the launchers.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "api_checks.h"
#include "layers_common.h"

using namespace maddness;

namespace {

int check_integers(const void *q, int64_t cols, int64_t ld, const void *scale, const char *name)
{
    if (!scale) return fail(MADDNESS_E_INVAL, "%s: scale is NULL", name);
    if (!aligned(scale, 4)) return fail(MADDNESS_E_ALIGN, "%s: scale not 4-byte aligned", name);
    if (cols == 0) return MADDNESS_OK;
    if (!q) return fail(MADDNESS_E_INVAL, "%s: values are NULL", name);
    if (ld < cols) return fail(MADDNESS_E_INVAL, "%s: ld = %lld is smaller than its %lld columns", name, (long long)ld, (long long)cols);
    if (!aligned(q, 16) || ld % 16) return fail(MADDNESS_E_ALIGN, "%s: values not 16-byte aligned, or an ld that is no multiple of 16", name);
    return MADDNESS_OK;
}

int check_matrix(const maddness_integer_matrix *m, bool may_float, const char *name)
{
    if (!m) return fail(MADDNESS_E_INVAL, "%s is NULL", name);
    int rc;
    if ((rc = check_size(m->rows, name)) != MADDNESS_OK || (rc = check_size(m->cols, name)) != MADDNESS_OK) return rc;
    if (m->cols > MADDNESS_MAX_INTEGER_DEPTH)
        return fail(MADDNESS_E_UNSUPPORTED, "%s has %lld columns, sums of up to %d fit 32 bits", name, (long long)m->cols, MADDNESS_MAX_INTEGER_DEPTH);
    if (m->dtype != kI8) {
        if (!may_float) return fail(MADDNESS_E_UNSUPPORTED, "%s: dtype = %d, only MADDNESS_I8 is supported here", name, m->dtype);
        return check_floats(m->data, m->dtype, m->rows, m->cols, m->ld, name);
    }
    return m->rows == 0 ? MADDNESS_OK : check_integers(m->data, m->cols, m->ld, m->scale, name);
}

// Rounded rows of a floating A: where they lie in the workspace.
struct Rounded {
    int64_t ld, scale_at, bytes;
    Rounded(int64_t M, int64_t K)
    {
        ld = round_up(K, (int64_t)16);
        scale_at = M * ld;
        bytes = scale_at + M * 4;
    }
};

int check_workspace(const void *workspace, size_t given, size_t need, int64_t alignment)
{
    if (need == 0) return MADDNESS_OK;
    if (!workspace || given < need) return fail(MADDNESS_E_UNSUPPORTED, "workspace of %zu bytes given, %zu needed", workspace ? given : (size_t)0, need);
    if (!aligned(workspace, alignment)) return fail(MADDNESS_E_ALIGN, "workspace not %d-byte aligned", (int)alignment);
    return MADDNESS_OK;
}

// Parameters of a norm: a pair of vectors of one type, each of which may be missing.
int check_parameter(const void *p, int32_t dtype, const char *name)
{
    if (!p) return MADDNESS_OK;
    if (!floating(dtype)) return fail(MADDNESS_E_INVAL, "%s: dtype = %d is not F32, F16 or BF16", name, dtype);
    if (!aligned(p, bytes_of(dtype))) return fail(MADDNESS_E_ALIGN, "%s not aligned to its element size", name);
    return MADDNESS_OK;
}

constexpr int64_t kMostSummedColumns = (int64_t)1 << 26;    // 32 of them are a workgroup's of 1024

int check_norm(int64_t rows, int64_t cols)
{
    int rc;
    if ((rc = check_size(rows, "rows")) != MADDNESS_OK || (rc = check_size(cols, "cols")) != MADDNESS_OK) return rc;
    if (cols == 0) return fail(MADDNESS_E_INVAL, "cols = 0: a row without elements has no mean");
    return MADDNESS_OK;
}

int check_balance(const void *logits, int32_t dtype, int64_t T, int32_t E, int64_t ldl, int32_t scores)
{
    int rc;
    if ((rc = check_size(T, "T")) != MADDNESS_OK) return rc;
    if (E < 1 || E > MADDNESS_MAX_EXPERTS) return fail(MADDNESS_E_UNSUPPORTED, "E = %d, supported are 1..%d experts", E, MADDNESS_MAX_EXPERTS);
    if (scores != MADDNESS_SOFTMAX && scores != MADDNESS_SIGMOID) return fail(MADDNESS_E_INVAL, "scores = %d is not a maddness_scores", scores);
    return check_floats(logits, dtype, T, E, ldl, "logits");
}

constexpr int64_t kMostElements = (int64_t)1 << 40;

int check_tensors(const maddness_tensor *tensors, int64_t n, bool outs)
{
    if (n < 0) return fail(MADDNESS_E_INVAL, "n = %lld is negative", (long long)n);
    if (n > 0 && !tensors) return fail(MADDNESS_E_INVAL, "tensors is NULL");
    for (int64_t i = 0; i < n; ++i) {
        const maddness_tensor &t = tensors[i];
        if (t.count < 0) return fail(MADDNESS_E_INVAL, "tensor %lld: count = %lld is negative", (long long)i, (long long)t.count);
        if (t.count > kMostElements) return fail(MADDNESS_E_UNSUPPORTED, "tensor %lld: count = %lld, supported are up to 2^40", (long long)i, (long long)t.count);
        if (!floating(t.dtype) || (outs && !floating(t.out_dtype))) return fail(MADDNESS_E_INVAL, "tensor %lld: dtype is not F32, F16 or BF16", (long long)i);
        if (t.count == 0) continue;
        if (!t.data || (outs && !t.out)) return fail(MADDNESS_E_INVAL, "tensor %lld: data or out is NULL", (long long)i);
        if (!aligned(t.data, bytes_of(t.dtype)) || (outs && !aligned(t.out, bytes_of(t.out_dtype))))
            return fail(MADDNESS_E_ALIGN, "tensor %lld not aligned to its element size", (long long)i);
    }
    return MADDNESS_OK;
}

// What is written must not be read or written by another tensor's scaling: the workgroups go over the tensors in no order.
int check_apart(const maddness_tensor *tensors, int64_t n, const float *norm, bool norm_given)
{
    struct Range {
        uintptr_t begin, end;
        bool written;
        int64_t of;
    };
    std::vector<Range> ranges;
    ranges.reserve((size_t)(2 * n));
    for (int64_t i = 0; i < n; ++i) {
        const maddness_tensor &t = tensors[i];
        if (t.count == 0) continue;
        const uintptr_t data = reinterpret_cast<uintptr_t>(t.data), out = reinterpret_cast<uintptr_t>(t.out);
        ranges.push_back({out, out + (uintptr_t)(t.count * bytes_of(t.out_dtype)), true, i});
        if (data != out || t.dtype != t.out_dtype) ranges.push_back({data, data + (uintptr_t)(t.count * bytes_of(t.dtype)), false, i});
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
    // the range that reaches farthest of those before, and of the written ones among them
    const Range *far = nullptr, *far_written = nullptr;
    for (const Range &r : ranges) {
        const Range *meets = far_written && far_written->end > r.begin ? far_written : r.written && far && far->end > r.begin ? far : nullptr;
        if (meets) return fail(MADDNESS_E_INVAL, "tensors %lld and %lld overlap in what is written", (long long)meets->of, (long long)r.of);
        if (!far || r.end > far->end) far = &r;
        if (r.written && (!far_written || r.end > far_written->end)) far_written = &r;
    }
    const uintptr_t at = reinterpret_cast<uintptr_t>(norm);
    for (const Range &r : ranges)
        if ((r.written || !norm_given) && r.begin < at + 4 && r.end > at) return fail(MADDNESS_E_INVAL, "norm lies within tensor %lld", (long long)r.of);
    return MADDNESS_OK;
}

}  // namespace

extern "C" {

int maddness_quantise_rows(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ldx, int8_t *q, int64_t ldq, float *scale, void *stream)
{
    begin_call();
    int rc;
    if ((rc = check_size(rows, "rows")) != MADDNESS_OK || (rc = check_size(cols, "cols")) != MADDNESS_OK) return rc;
    if ((rc = check_floats(x, dtype, rows, cols, ldx, "x")) != MADDNESS_OK) return rc;
    if (rows == 0) return MADDNESS_OK;
    if ((rc = check_integers(q, cols, ldq, scale, "q")) != MADDNESS_OK) return rc;
    RowsArgs a{};
    a.x = x; a.rows = rows; a.n = cols; a.ldx = ldx; a.out = q; a.ldo = ldq; a.scale = scale;
    return launch_quantise_rows(a, dtype, static_cast<hipStream_t>(stream));
}

size_t maddness_integer_product_workspace(int64_t a_rows, int64_t K, int32_t a_dtype)
{
    if (a_rows < 1 || K < 1 || K > MADDNESS_MAX_INTEGER_DEPTH || a_dtype == kI8 || integer_rounds_inside(a_rows, K)) return 0;
    return (size_t)Rounded(a_rows, K).bytes;
}

int maddness_integer_product(const maddness_integer_matrix *A, const maddness_integer_matrix *B, const float *bias, void *out, int32_t out_dtype,
                             int64_t ldo, void *workspace, size_t workspace_bytes, void *stream)
{
    begin_call();
    int rc;
    if ((rc = check_matrix(A, true, "A")) != MADDNESS_OK || (rc = check_matrix(B, false, "B")) != MADDNESS_OK) return rc;
    if (A->cols != B->cols) return fail(MADDNESS_E_INVAL, "A has %lld columns and B %lld", (long long)A->cols, (long long)B->cols);
    const int64_t M = A->rows, N = B->rows, K = A->cols;
    if ((rc = check_floats(out, out_dtype, M, N, ldo, "out")) != MADDNESS_OK) return rc;
    if (!aligned(bias, 4)) return fail(MADDNESS_E_ALIGN, "bias not 4-byte aligned");
    if (M == 0 || N == 0) return MADDNESS_OK;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    IntegerArgs p{};
    p.a = A->data; p.lda = A->ld; p.scale_a = A->scale;
    p.b = static_cast<const int8_t *>(B->data); p.ldb = B->ld; p.scale_b = B->scale; p.bias = bias;
    p.M = M; p.N = N; p.K = K; p.out = out; p.ldo = ldo;
    int a_dtype = A->dtype;
    if (a_dtype != kI8 && !integer_rounds_inside(M, K)) {
        if (K > 0) {
            const Rounded r(M, K);
            if ((rc = check_workspace(workspace, workspace_bytes, (size_t)r.bytes, 16)) != MADDNESS_OK) return rc;
            RowsArgs a{};
            a.x = A->data; a.rows = M; a.n = K; a.ldx = A->ld; a.out = workspace; a.ldo = r.ld;
            a.scale = reinterpret_cast<float *>(static_cast<char *>(workspace) + r.scale_at);
            if ((rc = launch_quantise_rows(a, a_dtype, s)) != MADDNESS_OK) return rc;
            p.a = workspace; p.lda = r.ld; p.scale_a = a.scale;
        }
        a_dtype = kI8;
    }
    return launch_integer_product(p, a_dtype, out_dtype, s);
}

int maddness_layer_norm(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ldx, const void *weight, const void *bias, int32_t parameter_dtype,
                        float eps, void *out, int32_t out_dtype, int64_t ldo, float *scale, float *mean, float *rstd, void *stream)
{
    begin_call();
    int rc;
    if ((rc = check_norm(rows, cols)) != MADDNESS_OK || (rc = check_floats(x, dtype, rows, cols, ldx, "x")) != MADDNESS_OK) return rc;
    if ((rc = check_parameter(weight, parameter_dtype, "weight")) != MADDNESS_OK || (rc = check_parameter(bias, parameter_dtype, "bias")) != MADDNESS_OK) return rc;
    if (!(eps >= 0) || !std::isfinite(eps)) return fail(MADDNESS_E_INVAL, "eps = %g, must be finite and >= 0", (double)eps);
    if (!mean != !rstd) return fail(MADDNESS_E_INVAL, "mean and rstd go together");
    if (!aligned(mean, 4) || !aligned(rstd, 4)) return fail(MADDNESS_E_ALIGN, "mean / rstd not 4-byte aligned");
    if (out_dtype != kI8) {
        if (scale) return fail(MADDNESS_E_INVAL, "scale goes with an out of MADDNESS_I8");
        if ((rc = check_floats(out, out_dtype, rows, cols, ldo, "out")) != MADDNESS_OK) return rc;
    } else if (rows > 0 && (rc = check_integers(out, cols, ldo, scale, "out")) != MADDNESS_OK) {
        return rc;
    }
    if (rows == 0) return MADDNESS_OK;
    RowsArgs a{};
    a.x = x; a.rows = rows; a.n = cols; a.ldx = ldx; a.weight = weight; a.bias = bias; a.parameter_dtype = parameter_dtype; a.eps = eps;
    a.out = out; a.ldo = ldo; a.scale = scale; a.mean = mean; a.rstd = rstd;
    return launch_layer_norm(a, dtype, out_dtype, static_cast<hipStream_t>(stream));
}

size_t maddness_layer_norm_gradient_workspace(int64_t rows, int64_t cols)
{
    if (rows < 1 || cols < 1 || rows > kMostRows || cols > kMostRows) return 0;
    return layer_norm_gradient_workspace_bytes(rows, cols);
}

int maddness_layer_norm_gradient(const void *gradient, int32_t gradient_dtype, int64_t ldg, const void *x, int32_t dtype, int64_t rows, int64_t cols,
                                 int64_t ldx, const float *mean, const float *rstd, const void *weight, int32_t parameter_dtype, void *dx, int64_t ldd,
                                 float *dweight, float *dbias, void *workspace, size_t workspace_bytes, void *stream)
{
    begin_call();
    int rc;
    if ((rc = check_norm(rows, cols)) != MADDNESS_OK || (rc = check_floats(x, dtype, rows, cols, ldx, "x")) != MADDNESS_OK) return rc;
    if ((rc = check_floats(gradient, gradient_dtype, rows, cols, ldg, "gradient")) != MADDNESS_OK) return rc;
    if ((rc = check_parameter(weight, parameter_dtype, "weight")) != MADDNESS_OK) return rc;
    if (rows > 0 && (!mean || !rstd)) return fail(MADDNESS_E_INVAL, "mean / rstd is NULL");
    if (!aligned(mean, 4) || !aligned(rstd, 4)) return fail(MADDNESS_E_ALIGN, "mean / rstd not 4-byte aligned");
    if (dx && (rc = check_floats(dx, dtype, rows, cols, ldd, "dx")) != MADDNESS_OK) return rc;
    if (!dweight != !dbias) return fail(MADDNESS_E_INVAL, "dweight and dbias go together");
    if (!dx && !dweight) return fail(MADDNESS_E_INVAL, "dx and dweight are both NULL");
    if (dweight && cols > kMostSummedColumns) return fail(MADDNESS_E_UNSUPPORTED, "cols = %lld, dweight and dbias have up to 2^26", (long long)cols);
    if (!aligned(dweight, 4) || !aligned(dbias, 4)) return fail(MADDNESS_E_ALIGN, "dweight / dbias not 4-byte aligned");
    if (dweight && (rc = check_workspace(workspace, workspace_bytes, maddness_layer_norm_gradient_workspace(rows, cols), 16)) != MADDNESS_OK) return rc;
    NormGradientArgs a{};
    a.g = gradient; a.x = x; a.rows = rows; a.n = cols; a.ldg = ldg; a.ldx = ldx; a.mean = mean; a.rstd = rstd; a.weight = weight;
    a.parameter_dtype = parameter_dtype; a.dx = dx; a.ldd = ldd; a.dweight = dweight; a.dbias = dbias; a.partial = static_cast<float *>(workspace);
    return launch_layer_norm_gradient(a, gradient_dtype, dtype, static_cast<hipStream_t>(stream));
}

size_t maddness_balance_workspace(int64_t T, int32_t E)
{
    if (T < 0 || T > kMostRows || E < 1 || E > MADDNESS_MAX_EXPERTS) return 0;
    return balance_workspace_bytes(T, E);
}

int maddness_balance(const void *logits, int32_t dtype, int64_t T, int32_t E, int64_t ldl, int32_t scores, const int32_t *ids, int32_t k, float factor,
                     float *loss, int32_t *counts, float *push, void *workspace, size_t workspace_bytes, void *stream)
{
    begin_call();
    int rc = check_balance(logits, dtype, T, E, ldl, scores);
    if (rc != MADDNESS_OK) return rc;
    if (k < 1) return fail(MADDNESS_E_INVAL, "k = %d, must be >= 1", k);
    if (T * k > kMostRows) return fail(MADDNESS_E_UNSUPPORTED, "T k = %lld, supported are up to 2^31 - 1", (long long)(T * k));
    if ((T > 0 && !ids) || !loss || !counts || !push) return fail(MADDNESS_E_INVAL, "ids / loss / counts / push is NULL");
    if (!aligned(ids, 4) || !aligned(loss, 4) || !aligned(counts, 4) || !aligned(push, 4)) return fail(MADDNESS_E_ALIGN, "ids / loss / counts / push not 4-byte aligned");
    if ((rc = check_workspace(workspace, workspace_bytes, maddness_balance_workspace(T, E), 8)) != MADDNESS_OK) return rc;
    BalanceArgs a{};
    a.logits = logits; a.T = T; a.ldl = ldl; a.E = E; a.k = k; a.softmax = scores == MADDNESS_SOFTMAX; a.ids = ids; a.factor = factor;
    a.loss = loss; a.counts = counts; a.push = push;
    return launch_balance(a, dtype, workspace, static_cast<hipStream_t>(stream));
}

int maddness_balance_gradient(const void *logits, int32_t dtype, int64_t T, int32_t E, int64_t ldl, int32_t scores, const float *push,
                              const float *loss_gradient, const void *add, int64_t lda, void *gradient, int64_t ldd, void *stream)
{
    begin_call();
    int rc = check_balance(logits, dtype, T, E, ldl, scores);
    if (rc != MADDNESS_OK) return rc;
    if (T == 0) return MADDNESS_OK;
    if (!push) return fail(MADDNESS_E_INVAL, "push is NULL");
    if (!aligned(push, 4) || !aligned(loss_gradient, 4)) return fail(MADDNESS_E_ALIGN, "push / loss_gradient not 4-byte aligned");
    if (add && (rc = check_floats(add, dtype, T, E, lda, "add")) != MADDNESS_OK) return rc;
    if ((rc = check_floats(gradient, dtype, T, E, ldd, "gradient")) != MADDNESS_OK) return rc;
    BalanceArgs a{};
    a.logits = logits; a.T = T; a.ldl = ldl; a.E = E; a.softmax = scores == MADDNESS_SOFTMAX; a.push = const_cast<float *>(push);
    a.loss_gradient = loss_gradient; a.add = add; a.lda = lda; a.gradient = gradient; a.ldd = ldd;
    return launch_balance_gradient(a, dtype, static_cast<hipStream_t>(stream));
}

size_t maddness_gradient_norm_workspace(void) { return kNormPartials * sizeof(double); }

int maddness_gradient_norm(const maddness_tensor *tensors, int64_t n, float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    begin_call();
    int rc = check_tensors(tensors, n, false);
    if (rc != MADDNESS_OK) return rc;
    if (!norm) return fail(MADDNESS_E_INVAL, "norm is NULL");
    if (!aligned(norm, 4)) return fail(MADDNESS_E_ALIGN, "norm not 4-byte aligned");
    if ((rc = check_workspace(workspace, workspace_bytes, maddness_gradient_norm_workspace(), 8)) != MADDNESS_OK) return rc;
    return launch_gradient_norm(tensors, n, norm, static_cast<double *>(workspace), static_cast<hipStream_t>(stream));
}

int maddness_clip_gradients(const maddness_tensor *tensors, int64_t n, float max_norm, float *norm, int32_t norm_given, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    begin_call();
    int rc = check_tensors(tensors, n, true);
    if (rc != MADDNESS_OK) return rc;
    if (!(max_norm >= 0)) return fail(MADDNESS_E_INVAL, "max_norm = %g, must be >= 0", (double)max_norm);
    if (!norm) return fail(MADDNESS_E_INVAL, "norm is NULL");
    if (!aligned(norm, 4)) return fail(MADDNESS_E_ALIGN, "norm not 4-byte aligned");
    if (!norm_given && (rc = check_workspace(workspace, workspace_bytes, maddness_gradient_norm_workspace(), 8)) != MADDNESS_OK) return rc;
    try {
        if ((rc = check_apart(tensors, n, norm, norm_given != 0)) != MADDNESS_OK) return rc;
    } catch (const std::bad_alloc &) {
        return fail(MADDNESS_E_UNSUPPORTED, "no host memory to compare %lld tensors", (long long)n);
    }
    return launch_clip(tensors, n, max_norm, norm, norm_given != 0, static_cast<double *>(workspace), static_cast<hipStream_t>(stream));
}

}  // extern "C"

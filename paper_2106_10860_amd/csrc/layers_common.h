// What the kernels around exact layers share: integer products, layer norm, balance, gradients' norm.
#pragma once

#include "block_common.h"

namespace maddness {

constexpr int kI8 = MADDNESS_I8;

// Operands of an integer product as the launcher takes them.
struct IntegerArgs {
    const void *a;                      // 8-bit values, or elements of a_dtype
    const int8_t *b;
    const float *scale_a, *scale_b, *bias;
    int64_t lda, ldb, M, N, K;
    void *out;
    int64_t ldo;
};

// a_dtype: kI8, or a floating type that the kernel rounds by itself (integer_rounds_inside).
int launch_integer_product(const IntegerArgs &p, int a_dtype, int out_dtype, hipStream_t stream);
bool integer_rounds_inside(int64_t M, int64_t K);

// The rows of a matrix: to integers as they are, or normalised and to any type.
struct RowsArgs {
    const void *x;
    int64_t rows, n, ldx;
    const void *weight, *bias;
    int parameter_dtype;
    float eps;
    void *out;
    int64_t ldo;
    float *scale, *mean, *rstd;
};

int launch_quantise_rows(const RowsArgs &a, int dtype, hipStream_t stream);
int launch_layer_norm(const RowsArgs &a, int dtype, int out_dtype, hipStream_t stream);

struct NormGradientArgs {
    const void *g, *x;
    int64_t rows, n, ldg, ldx;
    const float *mean, *rstd;
    const void *weight;
    int parameter_dtype;
    void *dx;
    int64_t ldd;
    float *dweight, *dbias, *partial;
};

size_t layer_norm_gradient_workspace_bytes(int64_t rows, int64_t n);
int launch_layer_norm_gradient(const NormGradientArgs &a, int gradient_dtype, int dtype, hipStream_t stream);

struct BalanceArgs {
    const void *logits;
    int64_t T, ldl;
    int E, k;
    bool softmax;
    const int32_t *ids;
    float factor;
    float *loss;
    int32_t *counts;
    float *push;
    const float *loss_gradient;         // gradient only, from here
    const void *add;
    int64_t lda;
    void *gradient;
    int64_t ldd;
};

size_t balance_workspace_bytes(int64_t T, int E);
int launch_balance(const BalanceArgs &a, int dtype, void *workspace, hipStream_t stream);
int launch_balance_gradient(const BalanceArgs &a, int dtype, hipStream_t stream);

constexpr int kNormPartials = 2048;     // sums of squares, one for each workgroup
int launch_gradient_norm(const maddness_tensor *tensors, int64_t n, float *norm, double *partials, hipStream_t stream);
int launch_clip(const maddness_tensor *tensors, int64_t n, float max_norm, float *norm, bool given, double *partials, hipStream_t stream);

// ------------------------------------------------------------------------------------------------------------- 8-bit integers

// A row's scale from the bits of its largest magnitude (which order as the numbers do, infinities and NaN last).
__device__ __forceinline__ float integer_scale(uint32_t top)
{
    if (top >= 0x7f800000u) return __builtin_nanf("");
    return top == 0 ? 1.0f : fmaxf(__uint_as_float(top) / 127.0f, 1.17549435e-38f);
}

// x / s to the nearest integer, ties to even, in the low byte of the result; inv = 1 / s.  x inv is off by some 2^-16 at most, so the candidate is the
// nearest integer or one next to it, and the remainder x - q s, which an fma gives exactly (a multiple of half a step of s, or of x, of no more than 24 digits), decides.
__device__ __forceinline__ uint32_t nearest_integer(float x, float s, float inv)
{
    constexpr float kMagic = 12582912.0f;                     // 1.5 2^23: one more is one step
    const float t = __builtin_fmaf(x, inv, kMagic), q = t - kMagic;
    const float r = __builtin_fmaf(-q, s, x), twice = 2.0f * fabsf(r);        // (half of s need not be a number of fp32, where that is below 2^-125)
    uint32_t b = __float_as_uint(t);
    const bool other = twice > s || (twice == s && (b & 1));
    return b + (other ? (r > 0 ? 1u : 0xffffffffu) : 0u);
}

// Eight of them.  Where no x inv is within 2^-14 of a half the candidates are it, which costs a third of the operations (8192 bfloat16 rows of
// 4096 through a norm 31.8 us with each decided, 26.7 so); elsewhere each is decided.
__device__ __forceinline__ uint2 pack8_integers(const float (&v)[8], float s, float inv)
{
    constexpr float kMagic = 12582912.0f;
    if (!(s == s)) return make_uint2(0, 0);
    uint32_t b[8];
    float far = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = __builtin_fmaf(v[i], inv, kMagic);
        b[i] = __float_as_uint(t);
        far = fmaxf(far, fabsf(__builtin_fmaf(v[i], inv, kMagic - t)));
    }
    if (far > 0.49994f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = nearest_integer(v[i], s, inv);
    }
    auto four = [&](int i) INLINE_LAMBDA {
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[i + 3], b[i + 2], 0x0c0c0400), __builtin_amdgcn_perm(b[i + 1], b[i], 0x0c0c0400), 0x05040100);
    };
    return make_uint2(four(0), four(4));
}

}  // namespace maddness

// What the kernels on 8-bit block matrices share: the number format, its conversions and the search for an expert's rows.
#pragma once

#include <type_traits>

#include "common.h"
#include "device_common.h"

namespace maddness {

constexpr int kE4M3 = MADDNESS_E4M3;
constexpr int kBlock = MADDNESS_BLOCK;
constexpr int64_t kMostThreads = ((int64_t)1 << 32) - 1;        // that a dimension of a launch may have

using i32x4 = __attribute__((ext_vector_type(4))) int;
using i32x8 = __attribute__((ext_vector_type(8))) int;
using f32x4 = __attribute__((ext_vector_type(4))) float;

template <typename T>
__host__ __device__ constexpr T ceil_div(T a, T b) { return (a + b - 1) / b; }
template <typename T>
__host__ __device__ constexpr T round_up(T a, T b) { return ceil_div(a, b) * b; }

// Eight consecutive elements of a row of n >= 8, from column c on, as they are in memory (any alignment to the element).  A piece that would
// pass the row's end is read from n - 8 on instead: no branch, so that many can be on their way.
template <int DT>
struct __attribute__((packed, aligned(elem_size(DT)))) Raw {
    uint32_t w[2 * elem_size(DT)];
};

template <int DT>
__device__ __forceinline__ Raw<DT> load_raw(const void *x, int64_t row_at, int64_t c, int64_t n)
{
    return *reinterpret_cast<const Raw<DT> *>(static_cast<const char *>(x) + (row_at + min(c, n - 8)) * elem_size(DT));
}

template <int DT>
__device__ __forceinline__ void widen(const Raw<DT> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (DT == kF32) v[i] = __uint_as_float(r.w[i]);
        else if constexpr (DT == kBF16) v[i] = __uint_as_float(i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
        else v[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i / 2] >> (i & 1 ? 16 : 0)));
    }
}

// How many of the elements of a piece are before c.
__device__ __forceinline__ int before_column(int64_t c, int64_t n) { return (int)max(c - (n - 8), (int64_t)0); }

// Eight bytes of which the first `skip` are not wanted, those after them in their place, and zeros.
__device__ __forceinline__ uint2 in_place(uint2 b, int skip)
{
    const uint64_t m = skip < 8 ? (((uint64_t)b.y << 32) | b.x) >> (8 * skip) : 0;
    return make_uint2((uint32_t)m, (uint32_t)(m >> 32));
}

// A row of fewer than 8, from column c on, and zeros.
template <int DT>
__device__ __forceinline__ void load_short(const void *x, int64_t row_at, int64_t c, int64_t n, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < n ? widen_at<DT>(x, row_at + c + i) : 0.0f;
}

// |x| of a finite x as bits (they order as the numbers do), 0 for NaN and the infinities.
__device__ __forceinline__ uint32_t finite_magnitude(float x)
{
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// The exponent byte of a block whose largest magnitude has these bits.  A number m 2^E, 1 <= m < 2, is at most
// 448 2^e = 1.75 2^(8 + e) from e = E - 8 on where m <= 1.75, from E - 7 on where it is larger: the addition carries into the
// exponent just then.
__device__ __forceinline__ uint32_t exponent_byte(uint32_t top)
{
    if (top == 0) return 127;
    const int e = (int)((top + 0x1fffffu) >> 23) - 8;      // biased
    return (uint32_t)max(e, 1);
}

// Four values divided by 2^(byte - 127), to E4M3, nearest, ties to even; NaN for an infinity.
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d, uint32_t byte)
{
    using pair = __attribute__((ext_vector_type(2))) short;
    const float scale = __uint_as_float(byte << 23);
    const pair lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(pair{0, 0}, a, b, scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, c, d, scale, true));
}

// Largest value of the 16 lanes of a row of lanes, in all of them (rotations within the row).
__device__ __forceinline__ uint32_t row16_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x122, 0xf, 0xf, true));
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x121, 0xf, 0xf, true));
}

// fp32 to a result's type, nearest even.
template <int DT>
__device__ __forceinline__ void store_as(void *base, int64_t at, float x)
{
    if constexpr (DT == kF32) static_cast<float *>(base)[at] = x;
    else if constexpr (DT == kF16) static_cast<_Float16 *>(base)[at] = (_Float16)x;
    else static_cast<__bf16 *>(base)[at] = (__bf16)x;
}

// Two results as one word of a narrow type.
template <int DT>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    using pair16 = __attribute__((ext_vector_type(2))) _Float16;
    using pair_b = __attribute__((ext_vector_type(2))) __bf16;
    if constexpr (DT == kF16) return __builtin_bit_cast(uint32_t, (pair16){(_Float16)a, (_Float16)b});
    else return __builtin_bit_cast(uint32_t, (pair_b){(__bf16)a, (__bf16)b});
}

// N neighbouring results (any alignment to the element) in one store.
template <int DT, int N>
__device__ __forceinline__ void store_run(void *base, int64_t at, const float (&v)[N])
{
    struct __attribute__((packed, aligned(elem_size(DT)))) Words { uint32_t w[N * elem_size(DT) / 4]; };
    Words r;
#pragma unroll
    for (int i = 0; i < N * elem_size(DT) / 4; ++i) {
        if constexpr (DT == kF32) r.w[i] = __float_as_uint(v[i]);
        else r.w[i] = pack2<DT>(v[2 * i], v[2 * i + 1]);
    }
    *reinterpret_cast<Words *>(static_cast<char *>(base) + at * elem_size(DT)) = r;
}

// Entry e of an array of offsets, cut back to 0 .. limit.
__device__ __forceinline__ int64_t offset_at(const int32_t *offsets, int e, int64_t limit)
{
    return min(max((int64_t)offsets[e], (int64_t)0), limit);
}

// Every expert's rows are cut into pieces of their own, `rows` rows each, and the pieces are numbered through.  All lanes of a wavefront
// call count (how many there are; not needed before find) and find with the same arguments.
struct PieceSearch {
    int e0 = -1;                    // lane l holds expert e0 + l:
    int lo, hi, mine, upto;         // its rows' bounds, the number of its pieces, and of those from e0's up to and with them

    __device__ __forceinline__ void look(const int32_t *offsets, int groups, int64_t limit, int rows, int from)
    {
        if (e0 == from) return;
        e0 = from;
        const int lane = threadIdx.x & 63, e = e0 + lane;
        lo = e < groups ? (int)offset_at(offsets, e, limit) : 0;              // (limit < 2^31)
        hi = e < groups ? (int)offset_at(offsets, e + 1, limit) : 0;
        mine = hi > lo ? (int)ceil_div((uint32_t)(hi - lo), (uint32_t)rows) : 0;
        upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
    }

    __device__ __forceinline__ int64_t count(const int32_t *offsets, int groups, int64_t limit, int rows)
    {
        int64_t all = 0;
        for (int from = 0; from < groups; from += 64) {
            look(offsets, groups, limit, rows, from);
            all += __builtin_amdgcn_readlane(upto, 63);
        }
        return all;
    }

    // The expert of piece `piece`, or -1 where there are fewer; first and one-past-last row.
    __device__ __forceinline__ int find(const int32_t *offsets, int groups, int64_t limit, int rows, int64_t piece, int64_t &first, int64_t &last)
    {
        int64_t before = 0;
        for (int from = 0; from < groups; from += 64) {
            look(offsets, groups, limit, rows, from);
            const int64_t at = piece - before;
            const uint64_t has = __ballot(at < upto && at >= upto - mine);
            if (has) {
                const int l = __ffsll((unsigned long long)has) - 1;
                const int begin = __builtin_amdgcn_readlane(upto - mine, l);
                const int64_t low = __builtin_amdgcn_readlane(lo, l), high = __builtin_amdgcn_readlane(hi, l);
                first = low + (at - begin) * rows;
                last = min(first + rows, high);
                return from + l;
            }
            before += __builtin_amdgcn_readlane(upto, 63);
        }
        return -1;
    }
};

// Arguments of a product, as the launchers hand them on.
struct ProductArgs {
    const uint8_t *a, *b;              // 8-bit values (a: elements of a_dtype)
    const uint8_t *scale_a, *scale_b;
    int64_t lda, ldb, lds_a, lds_b;
    int64_t stride_b, scale_stride_b;  // between experts
    int shift_a, shift_b;              // row -> row of exponents: 0 or 7
    int64_t M, N, K, a_rows;           // (M: rows of out; of A where source is NULL)
    int by, groups;
    const int32_t *offsets;
    const int32_t *source;             // of each row of out: a slot, whose row of A is slot / repeat; NULL: rows as they are
    int64_t source_limit;              // a_rows * repeat
    int repeat;
    void *out;
    int64_t ldo, out_stride;
};

int launch_quantise_blocks(const void *x, int dtype, int64_t count, int64_t rows, int64_t cols, int64_t ldx, int64_t stride_x, int tile,
                           const int32_t *source, int64_t source_rows, int repeat, const float *factors, uint8_t *q, int64_t ldq,
                           uint8_t *scale, int64_t lds, uint8_t *qt, int64_t ldqt, uint8_t *scale_t, int64_t ldst, hipStream_t stream);

// a_dtype: kE4M3, or a floating type that the kernel rounds by itself (rounds_inside).
int launch_block_product(const ProductArgs &p, int a_dtype, int out_dtype, hipStream_t stream);
// Whether a product with a floating A of M rows rounds it inside its kernel; otherwise A is rounded into the workspace before.
bool rounds_inside(int64_t M, int64_t K, int by);

int launch_route(const void *logits, int dtype, int64_t T, int E, int64_t ldl, const float *bias, int scores, int groups, int kept, int k,
                 bool renormalise, float factor, int32_t *ids, float *weights, hipStream_t stream);
int launch_route_gradient(const void *logits, int dtype, int64_t T, int E, int64_t ldl, int scores, int k, bool renormalise, float factor,
                          const int32_t *ids, const float *dweights, void *gradient, int64_t ldd, hipStream_t stream);
size_t order_workspace_bytes(int64_t slots, int E);
int launch_order(const int32_t *ids, int64_t slots, int E, int align, int32_t *offsets, int32_t *counts, int32_t *source, int64_t capacity,
                 int32_t *place, void *workspace, hipStream_t stream);
int launch_combine(const void *y, int y_dtype, int64_t rows, int64_t N, int64_t ldy, const int32_t *place, const float *weights, int64_t T,
                   int k, void *out, int out_dtype, int64_t ldo, hipStream_t stream);
int launch_combine_gradient(const void *gradient, int dtype, int64_t ldg, const void *y, int y_dtype, int64_t rows, int64_t N, int64_t ldy,
                            const int32_t *place, int64_t T, int k, float *dweights, hipStream_t stream);

}  // namespace maddness

// Rounding to 8-bit block matrices: e = the least power of two that brings a block's largest magnitude to 448 or less,
// q = x 2^-e to the nearest E4M3 number.  The conversion instructions take the power of two in, so there is one rounding and the result does
// not depend on how the work is split; they make NaN of an infinity.  Bound by memory: b bytes read and 1 (both ways: 2) written per
// value.  binary16 and bfloat16 stay two to a register throughout, unless a factor has to be multiplied in.
#include "block_common.h"

namespace maddness {
namespace {

using u16x2 = __attribute__((ext_vector_type(2))) uint16_t;
using i16x2 = __attribute__((ext_vector_type(2))) short;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using f16x2 = __attribute__((ext_vector_type(2))) _Float16;

struct QuantiseArgs {
    const void *x;
    int64_t rows, cols, ldx, stride_x;
    int64_t readable;          // cols, or 0 where x has no rows (and source makes rows of zeros)
    const int32_t *source;
    int64_t slots;             // source_rows * repeat
    int repeat;
    const float *factors;
    uint8_t *q, *scale, *qt, *scale_t;
    int64_t ldq, lds, ldqt, ldst;
};

// Where row r's elements begin, and the factor of them; false for a row of zeros (whose place is that of another).
__device__ __forceinline__ bool find_row(const QuantiseArgs &a, int64_t r, int64_t &at, float &factor)
{
    factor = 1.0f;
    at = r * a.ldx;
    if (!a.source) return true;
    int s = a.source[r];
    const bool there = s >= 0 && s < a.slots;
    if (!there) s = 0;
    if (a.factors && a.slots > 0) factor = a.factors[s];
    at = (int64_t)(s / a.repeat) * a.ldx;
    return there;
}

// Eight neighbours of a row as they are computed with: two to a word (PAIRS) or widened to fp32.
template <int DT, bool FACTORS>
struct Eight {
    static constexpr bool PAIRS = DT != kF32 && !FACTORS;
    static constexpr int WORDS = PAIRS ? 4 : 8;
    static constexpr uint32_t INFINITE = !PAIRS ? 0x7f800000u : DT == kBF16 ? 0x7f80u : 0x7c00u;
    uint32_t w[WORDS];

    // From column c of a row of n on, where there are 8 to read from there; of a shorter row those that there are, and zeros.
    __device__ __forceinline__ void load(const void *x, int64_t row_at, int64_t c, int64_t n)
    {
        if (n >= 8) {
            const Raw<DT> r = load_raw<DT>(x, row_at, c, n);
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                if constexpr (PAIRS || DT == kF32) w[i] = r.w[i];
                else if constexpr (DT == kBF16) w[i] = i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16;
                else w[i] = __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i / 2] >> (i & 1 ? 16 : 0))));
            }
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                if constexpr (PAIRS) {
                    const uint16_t *at = static_cast<const uint16_t *>(x) + row_at;
                    w[i] = (c + 2 * i < n ? at[c + 2 * i] : 0u) | (c + 2 * i + 1 < n ? (uint32_t)at[c + 2 * i + 1] << 16 : 0u);
                } else {
                    w[i] = c + i < n ? __float_as_uint(widen_at<DT>(x, row_at + c + i)) : 0u;
                }
            }
        }
    }

    // Elements before `skip` (all, where the row is none) become 0.
    __device__ __forceinline__ void keep(int skip, bool there, float factor)
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            if constexpr (PAIRS) {
                const uint32_t lo = there && 2 * i >= skip ? 0xffffu : 0u, hi = there && 2 * i + 1 >= skip ? 0xffff0000u : 0u;
                w[i] &= lo | hi;
            } else {
                if constexpr (FACTORS) w[i] = __float_as_uint(__uint_as_float(w[i]) * factor);
                w[i] = there && i >= skip ? w[i] : 0u;
            }
        }
    }

    // Word i's magnitudes, as whole numbers in their order; FINITE: 0 for NaN and the infinities.
    template <bool FINITE>
    __device__ __forceinline__ uint32_t magnitude(int i) const
    {
        if constexpr (PAIRS) {
            const uint32_t m = w[i] & 0x7fff7fffu;
            if constexpr (!FINITE) return m;
            return ((m & 0xffffu) < INFINITE ? m & 0xffffu : 0u) | (m >> 16 < INFINITE ? m & 0xffff0000u : 0u);
        } else {
            const uint32_t m = w[i] & 0x7fffffffu;
            return !FINITE || m < INFINITE ? m : 0u;
        }
    }

    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        if constexpr (PAIRS) return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
        else return max(a, b);
    }

    // The larger of a word's magnitudes.
    static __device__ __forceinline__ uint32_t one(uint32_t a) { return PAIRS ? max(a & 0xffffu, a >> 16) : a; }

    // A magnitude as the bits of an fp32 number.
    static __device__ __forceinline__ uint32_t fp32_bits(uint32_t m)
    {
        if constexpr (!PAIRS) return m;
        else if constexpr (DT == kBF16) return m << 16;
        else return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)m));
    }
};

// Two values divided by 2^e, as the lower or upper half of a word of E4M3.
template <bool HIGH>
__device__ __forceinline__ i16x2 convert(i16x2 old, float a, float b, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, a, b, scale, HIGH); }

template <int DT, bool HIGH>
__device__ __forceinline__ i16x2 convert_pair(i16x2 old, uint32_t pair, float scale)
{
    if constexpr (DT == kBF16) return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, __builtin_bit_cast(bf16x2, pair), scale, HIGH);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(old, __builtin_bit_cast(f16x2, pair), scale, HIGH);
}

template <int DT, bool FACTORS>
__device__ __forceinline__ uint2 to_bytes(const Eight<DT, FACTORS> &v, float scale)
{
    i16x2 lo = {0, 0}, hi = {0, 0};
    if constexpr (Eight<DT, FACTORS>::PAIRS) {
        lo = convert_pair<DT, true>(convert_pair<DT, false>(lo, v.w[0], scale), v.w[1], scale);
        hi = convert_pair<DT, true>(convert_pair<DT, false>(hi, v.w[2], scale), v.w[3], scale);
    } else {
        auto f = [&](int i) INLINE_LAMBDA { return __uint_as_float(v.w[i]); };
        lo = convert<true>(convert<false>(lo, f(0), f(1), scale), f(2), f(3), scale);
        hi = convert<true>(convert<false>(hi, f(4), f(5), scale), f(6), f(7), scale);
    }
    return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

// The columns of a thread: 8 from c on, of which `skip` elements are before c where the row ends before c + 8 (skip >= 8: none is the row's).
struct Columns {
    int64_t c;
    int skip;
    __device__ __forceinline__ Columns(int64_t c_, int64_t n) : c(c_), skip(n >= 8 ? before_column(c_, n) : 0) {}
};

// Blocks of 1 x 128, rows only.  16 lanes take a block, 8 values each: the maximum stays within a row of lanes.  65536 x 1024 bfloat16 34.5 us,
// 5.8 TB/s read and written.
template <int DT, bool FACTORS>
__global__ __launch_bounds__(256) void quantise_rows_kernel(QuantiseArgs a, int64_t first_row, uint32_t blocks, uint32_t units)
{
    using V = Eight<DT, FACTORS>;
    const uint32_t unit = blockIdx.x * 16u + threadIdx.x / 16u;
    if (unit >= units) return;
    const int lane = threadIdx.x % 16;
    const int64_t r = first_row + unit / blocks, m = blockIdx.y;
    const uint32_t b = unit % blocks;
    const Columns col((int64_t)b * kBlock + lane * 8, a.cols);
    const char *x = static_cast<const char *>(a.x) + m * a.stride_x * elem_size(DT);
    V v;
    int64_t at;
    float factor;
    const bool there = find_row(a, r, at, factor);
    v.load(x, at, col.c, a.readable);
    v.keep(col.skip, there, factor);
    auto largest = [&](auto finite) INLINE_LAMBDA {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < V::WORDS; ++i) t = V::larger(t, v.template magnitude<decltype(finite)::value>(i));
        return V::one(t);
    };
    uint32_t top = largest(std::false_type{});
    if (__any(top >= V::INFINITE)) top = largest(std::true_type{});
    const uint32_t byte = exponent_byte(row16_max(V::fp32_bits(top)));
    const int64_t row = m * a.rows + r;
    if (col.c < round_up(a.cols, (int64_t)16)) *reinterpret_cast<uint2 *>(a.q + row * a.ldq + col.c) = in_place(to_bytes<DT, FACTORS>(v, __uint_as_float(byte << 23)), col.skip);
    uint8_t *s = a.scale + row * a.lds + b;
    if (lane == 0) *s = (uint8_t)byte;
    else if (b == blocks - 1 && b + lane < round_up(blocks, 4u)) s[lane] = 127;
}

// A tile of 128 x 128 to a workgroup, for transposes and common exponents: a thread holds 4 rows of 8 columns (with 8 rows and half the threads the
// kernel took 8 to 12 us for any small matrix, most of it the way through its instructions).  The transpose's bytes go through LDS in words of 4
// rows of one column, the words of a column exchanged by the writer's column group so that the lanes of a write fall on different banks.  8192 x 4096
// bfloat16 both ways 26 us, 5.1 TB/s.
constexpr int kTileThreads = 512, kRowsEach = 4;

template <int DT, bool FACTORS, int TILE>
__global__ __launch_bounds__(kTileThreads) void quantise_tiles_kernel(QuantiseArgs a, uint32_t blocks)
{
    using V = Eight<DT, FACTORS>;
    constexpr int WAVES = kTileThreads / 64;
    __shared__ uint32_t tops[WAVES][kBlock];
    __shared__ __attribute__((aligned(16))) uint32_t turned[kBlock][kBlock / kRowsEach];
    const int tid = threadIdx.x, cg = tid % 16, rg = tid / 16, wave = tid / 64;
    const uint32_t cb = blockIdx.x % blocks, rb = blockIdx.x / blocks, row_blocks = gridDim.x / blocks;
    const int64_t m = blockIdx.y, r0 = (int64_t)rb * kBlock + rg * kRowsEach;
    const Columns col((int64_t)cb * kBlock + cg * 8, a.cols);
    const char *x = static_cast<const char *>(a.x) + m * a.stride_x * elem_size(DT);
    V v[kRowsEach];
    float factor[kRowsEach];
    bool there[kRowsEach];
    // (rows beyond the end are read as the last: everything is asked for before anything is needed)
#pragma unroll
    for (int p = 0; p < kRowsEach; ++p) {
        int64_t at;
        there[p] = find_row(a, min(r0 + p, a.rows - 1), at, factor[p]) && r0 + p < a.rows;
        v[p].load(x, at, col.c, a.readable);
    }
#pragma unroll
    for (int p = 0; p < kRowsEach; ++p) v[p].keep(col.skip, there[p], factor[p]);
    uint32_t top_row[kRowsEach], top_col[V::WORDS];
    auto largest = [&](auto finite) INLINE_LAMBDA {
        uint32_t all = 0;
#pragma unroll
        for (int i = 0; i < V::WORDS; ++i) top_col[i] = 0;
#pragma unroll
        for (int p = 0; p < kRowsEach; ++p) {
            uint32_t t = 0;
#pragma unroll
            for (int i = 0; i < V::WORDS; ++i) {
                const uint32_t g = v[p].template magnitude<decltype(finite)::value>(i);
                t = V::larger(t, g);
                top_col[i] = V::larger(top_col[i], g);
            }
            top_row[p] = V::one(t);
            all = max(all, top_row[p]);
        }
        return all;
    };
    if (__any(largest(std::false_type{}) >= V::INFINITE)) largest(std::true_type{});
    float scale_col[8], scale_tile = 1.0f;
    auto store_rows = [&](int p, float scale) INLINE_LAMBDA {
        if (r0 + p < a.rows && col.c < round_up(a.cols, (int64_t)16))
            *reinterpret_cast<uint2 *>(a.q + (m * a.rows + r0 + p) * a.ldq + col.c) = in_place(to_bytes<DT, FACTORS>(v[p], scale), col.skip);
    };
    if constexpr (TILE == 1) {
        if (a.q) {
#pragma unroll
            for (int p = 0; p < kRowsEach; ++p) {
                const uint32_t byte = exponent_byte(row16_max(V::fp32_bits(top_row[p])));
                store_rows(p, __uint_as_float(byte << 23));
                if (r0 + p >= a.rows) continue;
                uint8_t *s = a.scale + (m * a.rows + r0 + p) * a.lds + cb;
                if (cg == 0) *s = (uint8_t)byte;
                else if (cb == blocks - 1 && cb + cg < round_up(blocks, 4u)) s[cg] = 127;
            }
        }
#pragma unroll
        for (int i = 0; i < V::WORDS; ++i) {
            const auto rows = __builtin_amdgcn_permlane16_swap(top_col[i], top_col[i], false, false);
            const uint32_t t = V::larger(rows[0], rows[1]);
            const auto halves = __builtin_amdgcn_permlane32_swap(t, t, false, false);
            top_col[i] = V::larger(halves[0], halves[1]);
        }
        if (rg % 4 == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i >= col.skip) tops[wave][cg * 8 + i - col.skip] = V::PAIRS ? top_col[i / (8 / V::WORDS)] >> (i % 2 * 16) & 0xffffu : top_col[i / (8 / V::WORDS)];
        }
        __syncthreads();
        // each column's exponent once, for all
        if (tid < kBlock) {
            uint32_t t = 0;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) t = max(t, tops[k][tid]);
            const uint32_t byte = exponent_byte(V::fp32_bits(t));
            tops[0][tid] = byte;
            const int64_t c = (int64_t)cb * kBlock + tid;
            if (c < a.cols) {
                uint8_t *s = a.scale_t + (m * a.cols + c) * a.ldst + rb;
                *s = (uint8_t)byte;
                if (rb == row_blocks - 1)
                    for (uint32_t pad = rb + 1; pad < round_up(row_blocks, 4u); ++pad) *++s = 127;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) scale_col[i] = __uint_as_float(tops[0][cg * 8 + max(i - col.skip, 0)] << 23);
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int p = 0; p < kRowsEach; ++p) top = max(top, top_row[p]);
        top = row16_max(top);
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        if (tid % 64 == 0) tops[wave][0] = top;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < WAVES; ++k) top = max(top, tops[k][0]);
        const uint32_t byte = exponent_byte(V::fp32_bits(top));
        scale_tile = __uint_as_float(byte << 23);
        if (a.q) {
#pragma unroll
            for (int p = 0; p < kRowsEach; ++p) store_rows(p, scale_tile);
            if (tid < 4) {
                uint8_t *s = a.scale + (m * row_blocks + rb) * a.lds + cb;
                if (tid == 0) *s = (uint8_t)byte;
                else if (cb == blocks - 1 && cb + tid < round_up(blocks, 4u)) s[tid] = 127;
            }
        }
        if (a.qt && tid < 4) {
            uint8_t *s = a.scale_t + (m * blocks + cb) * a.ldst + rb;
            if (tid == 0) *s = (uint8_t)byte;
            else if (rb == row_blocks - 1 && rb + tid < round_up(row_blocks, 4u)) s[tid] = 127;
        }
    }
    if (!a.qt) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float scale = TILE == 1 ? scale_col[i] : scale_tile;
        i16x2 bytes = {0, 0};
#pragma unroll
        for (int p = 0; p < kRowsEach; p += 2) {
            if constexpr (V::PAIRS) {
                const uint32_t a0 = v[p].w[i / 2], a1 = v[p + 1].w[i / 2];
                const uint32_t pair = i % 2 ? __builtin_amdgcn_perm(a1, a0, 0x07060302) : __builtin_amdgcn_perm(a1, a0, 0x05040100);
                bytes = p ? convert_pair<DT, true>(bytes, pair, scale) : convert_pair<DT, false>(bytes, pair, scale);
            } else {
                const float f0 = __uint_as_float(v[p].w[i]), f1 = __uint_as_float(v[p + 1].w[i]);
                bytes = p ? convert<true>(bytes, f0, f1, scale) : convert<false>(bytes, f0, f1, scale);
            }
        }
        if (i >= col.skip) turned[cg * 8 + i - col.skip][rg ^ (cg % 8 * 4)] = __builtin_bit_cast(uint32_t, bytes);
    }
    __syncthreads();
    const int64_t row_end = round_up(a.rows, (int64_t)16);
#pragma unroll
    for (int k = 0; k < kBlock * 8 / kTileThreads; ++k) {
        const int at = k * kTileThreads + tid, out_col = at / 8, piece = at % 8;
        const int64_t row = (int64_t)cb * kBlock + out_col, c = (int64_t)rb * kBlock + piece * 16;
        if (row >= a.cols || c >= row_end) continue;
        *reinterpret_cast<uint4 *>(a.qt + (m * a.cols + row) * a.ldqt + c) = *reinterpret_cast<const uint4 *>(&turned[out_col][(piece * 4) ^ (out_col / 8 % 8 * 4)]);
    }
}

template <int DT, bool FACTORS>
int launch_typed(const QuantiseArgs &a, int64_t count, int tile, hipStream_t stream)
{
    const int64_t blocks = ceil_div(a.cols, (int64_t)kBlock);
    if (tile == 1 && !a.qt) {
        // as many rows as 2^27 blocks make to a launch
        const int64_t most = std::max((int64_t)1, ((int64_t)1 << 27) / blocks);
        for (int64_t r = 0; r < a.rows; r += most) {
            const uint32_t units = (uint32_t)(std::min(most, a.rows - r) * blocks);
            note_kernel("quantise_rows_kernel", __PRETTY_FUNCTION__);
            hipLaunchKernelGGL((quantise_rows_kernel<DT, FACTORS>), dim3(ceil_div(units, 16u), (unsigned)count), dim3(256), 0, stream, a, r,
                               (uint32_t)blocks, units);
            const int rc = check_hip(hipGetLastError(), "launch quantise_rows_kernel");
            if (rc != MADDNESS_OK) return rc;
        }
        return MADDNESS_OK;
    }
    const dim3 grid((unsigned)(blocks * ceil_div(a.rows, (int64_t)kBlock)), (unsigned)count);
    if (grid.x * (int64_t)kTileThreads > kMostThreads) return fail(MADDNESS_E_UNSUPPORTED, "quantise: %lld x %lld values are too many", (long long)a.rows, (long long)a.cols);
    note_kernel("quantise_tiles_kernel", __PRETTY_FUNCTION__);
    if (tile == 1) hipLaunchKernelGGL((quantise_tiles_kernel<DT, FACTORS, 1>), grid, dim3(kTileThreads), 0, stream, a, (uint32_t)blocks);
    else hipLaunchKernelGGL((quantise_tiles_kernel<DT, FACTORS, kBlock>), grid, dim3(kTileThreads), 0, stream, a, (uint32_t)blocks);
    return check_hip(hipGetLastError(), "launch quantise_tiles_kernel");
}

template <int DT>
int launch_of(const QuantiseArgs &a, int64_t count, int tile, hipStream_t stream)
{
    return a.factors ? launch_typed<DT, true>(a, count, tile, stream) : launch_typed<DT, false>(a, count, tile, stream);
}

}  // namespace

int launch_quantise_blocks(const void *x, int dtype, int64_t count, int64_t rows, int64_t cols, int64_t ldx, int64_t stride_x, int tile,
                           const int32_t *source, int64_t source_rows, int repeat, const float *factors, uint8_t *q, int64_t ldq,
                           uint8_t *scale, int64_t lds, uint8_t *qt, int64_t ldqt, uint8_t *scale_t, int64_t ldst, hipStream_t stream)
{
    QuantiseArgs a{x, rows, cols, ldx, stride_x, source && source_rows == 0 ? 0 : cols, source, source_rows * repeat, repeat, factors, q, scale, qt, scale_t, ldq, lds, ldqt, ldst};
    if (dtype == MADDNESS_F32) return launch_of<kF32>(a, count, tile, stream);
    if (dtype == MADDNESS_F16) return launch_of<kF16>(a, count, tile, stream);
    return launch_of<kBF16>(a, count, tile, stream);
}

}  // namespace maddness

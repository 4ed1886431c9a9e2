// out[m][n] = sum_k A[m][k] B[n][k] of two 8-bit block matrices on the matrix cores.
//
// Two kinds of instruction multiply them.  The 8-bit one (v_mfma_scale_f32_16x16x128) takes the bytes and the powers of two as they
// are, but keeps its products to about 12 bits below the largest of them: measured, an error of up to 2^-11.1 of the largest product and of
// 1.5e-5 of the result for normal values, whatever the shape of the instruction.  The 16-bit one (v_mfma_f32_16x16x32_bf16) has half the
// rate, and its products and sums are those of fp32 (9e-9 of the result); an E4M3 number times a power of two is a bfloat16
// number, so the conversion to it takes the exponents in and is exact.  Results of 16 bits, which are rounded to 8 or 11 bits,
// come from the first, fp32 results from the second; few rows always from the second, as memory bounds them.
//
// B's rows (the columns of out) are the instruction's first operand and A's rows its second, so that a lane's four results are
// four neighbours in a row of out.  Lane l holds row l % 16, values 32 (l / 16) .. + 31 of an operand's block, and results
// n = 4 (l / 16) + i of row m = l % 16.
#include "block_common.h"

namespace maddness {
namespace {

using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;

// Eight E4M3 values times 2^(byte - 127), exactly; scale = byte << 23 (the conversion reads its exponent only, 255 gives NaN).
__device__ __forceinline__ bf16x8 widen8(int lo, int hi, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float as_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// A lane's 32 bytes of a row's block and the block's exponent.
struct Piece {
    i32x4 lo, hi;
    uint32_t byte;
};

// Reads them, 16 bytes that begin at or beyond column K from the row's last 16 that do not: in bounds, and cut off below.
__device__ __forceinline__ Piece load_piece(const uint8_t *row, const uint8_t *scale, int64_t kb, int group, int64_t K)
{
    const int64_t k = kb * kBlock + group * 32, last = (K - 1) & ~(int64_t)15;
    Piece p;
    p.lo = *reinterpret_cast<const i32x4 *>(row + min(k, last));
    p.hi = *reinterpret_cast<const i32x4 *>(row + min(k + 16, last));
    p.byte = scale[kb];
    return p;
}

// The first `keep` of 16 bytes, 0 for the others.
__device__ __forceinline__ i32x4 first_bytes(i32x4 v, int64_t keep)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int b = (int)min(max(keep - 4 * i, (int64_t)0), (int64_t)4);
        v[i] = b == 4 ? v[i] : v[i] & (int)((1u << (8 * b)) - 1);
    }
    return v;
}

__device__ __forceinline__ void cut(Piece &p, int64_t kb, int group, int64_t K)
{
    const int64_t k = kb * kBlock + group * 32;
    p.lo = first_bytes(p.lo, K - k);
    p.hi = first_bytes(p.hi, K - k - 16);
}

// The same of a floating A, rounded here: the block's maximum is that of the four lanes that hold the row.
template <int DT>
__device__ __forceinline__ Piece round_piece(const void *a, int64_t row_at, int64_t kb, int group, int64_t K)
{
    const int64_t k = kb * kBlock + group * 32;
    float v[4][8];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        load8<DT>(a, row_at + k + 8 * j, (int)max(min(K - k - 8 * j, (int64_t)8), (int64_t)0), v[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, finite_magnitude(v[j][i]));
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    Piece p;
    p.byte = exponent_byte(top);
    const float inv = inverse_scale(p.byte);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = scaled(v[j][i], inv);
        const int lo = (int)pack4(v[j][0], v[j][1], v[j][2], v[j][3]), hi = (int)pack4(v[j][4], v[j][5], v[j][6], v[j][7]);
        if (j < 2) { p.lo[2 * j] = lo; p.lo[2 * j + 1] = hi; }
        else { p.hi[2 * j - 4] = lo; p.hi[2 * j - 3] = hi; }
    }
    return p;
}

// What a workgroup computes: rows first .. last - 1 of A, with one expert's matrix, over the blocks kb0 .. kb1 - 1.
struct Part {
    int64_t first, last, kb0, kb1, K;
    const uint8_t *b, *scale_b;
    int64_t out_at;
};

__device__ __forceinline__ bool find_part(const ProductArgs &p, int rows, int64_t piece, int64_t group, Part &w)
{
    w.b = p.b;
    w.scale_b = p.scale_b;
    w.out_at = 0;
    w.K = p.K;
    w.kb0 = 0;
    if (p.by == MADDNESS_BY_ROWS) {
        const int e = find_piece(p.offsets, p.groups, p.M, rows, piece, w.first, w.last);
        if (e < 0) return false;
        w.b += e * p.stride_b;
        w.scale_b += e * p.scale_stride_b;
    } else {
        w.first = piece * rows;
        w.last = min(w.first + rows, p.M);
        if (p.by == MADDNESS_BY_DEPTH) {
            const int64_t lo = offset_at(p.offsets, (int)group, p.K), hi = offset_at(p.offsets, (int)group + 1, p.K);
            w.kb0 = lo / kBlock;
            w.K = hi / kBlock * kBlock;
            w.out_at = group * p.out_stride;
        }
    }
    w.kb1 = ceil_div(w.K, (int64_t)kBlock);
    return true;
}

// Few rows: 16 MT rows by 16 NT columns to a workgroup; its wavefronts take every WAVES-th block of the sum, DEPTH of them asked for
// at once, and add up in LDS, in their order.  Operands come straight from memory, in pieces of 32 bytes to a lane.
template <int AT, int MT, int NT, int WAVES, int DEPTH, int OUT>
__global__ __launch_bounds__(WAVES * 64) void product_few_kernel(ProductArgs p, uint32_t col_tiles)
{
    __shared__ f32x4 sums[WAVES][MT * NT][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r16 = lane % 16, g = lane / 16;
    const int64_t n0 = (int64_t)(blockIdx.x % col_tiles) * (16 * NT);
    Part w;
    if (!find_part(p, 16 * MT, blockIdx.x / col_tiles, blockIdx.y, w)) return;
    const uint8_t *row_b[NT], *row_a[MT], *scale_a[MT], *scale_b[NT];
    int64_t at_a[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t m = min(w.first + t * 16 + r16, w.last - 1);
        at_a[t] = m * p.lda;
        row_a[t] = p.a + (AT == kE4M3 ? at_a[t] : 0);
        scale_a[t] = AT == kE4M3 ? p.scale_a + (m >> p.shift_a) * p.lds_a : nullptr;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t n = min(n0 + t * 16 + r16, p.N - 1);
        row_b[t] = w.b + n * p.ldb;
        scale_b[t] = w.scale_b + (n >> p.shift_b) * p.lds_b;
    }
    f32x4 acc[MT][NT] = {};
    for (int64_t kb0 = w.kb0 + wave; kb0 < w.kb1; kb0 += DEPTH * WAVES) {
        Piece b[DEPTH][NT], a[DEPTH][MT];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int64_t kb = min(kb0 + d * WAVES, w.kb1 - 1);
#pragma unroll
            for (int t = 0; t < NT; ++t) b[d][t] = load_piece(row_b[t], scale_b[t], kb, g, w.K);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if constexpr (AT == kE4M3) a[d][t] = load_piece(row_a[t], scale_a[t], kb, g, w.K);
                else a[d][t] = round_piece<AT>(p.a, at_a[t], kb, g, w.K);
            }
        }
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int64_t kb = kb0 + d * WAVES;
            if (kb >= w.kb1) break;
            if ((kb + 1) * kBlock > w.K) {
#pragma unroll
                for (int t = 0; t < NT; ++t) cut(b[d][t], kb, g, w.K);
#pragma unroll
                for (int t = 0; t < MT; ++t) cut(a[d][t], kb, g, w.K);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                bf16x8 wb[NT], wa[MT];
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const i32x4 v = q < 2 ? b[d][t].lo : b[d][t].hi;
                    wb[t] = widen8(v[q % 2 * 2], v[q % 2 * 2 + 1], as_scale(b[d][t].byte));
                }
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const i32x4 v = q < 2 ? a[d][t].lo : a[d][t].hi;
                    wa[t] = widen8(v[q % 2 * 2], v[q % 2 * 2 + 1], as_scale(a[d][t].byte));
                }
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j], wa[i], acc[i][j], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < MT * NT * 256; o += WAVES * 64) {
        const int m = o / (16 * NT), n = o % (16 * NT);
        if (w.first + m >= w.last || n0 + n >= p.N) continue;
        const int tile = m / 16 * NT + n / 16, at = m % 16 + n % 16 / 4 * 16;
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) s += sums[k][tile][at][n % 4];
        store_as<OUT>(p.out, w.out_at + (w.first + m) * p.ldo + n0 + n, s);
    }
}

template <int AT, int OUT>
int launch_few(const ProductArgs &p, hipStream_t stream)
{
    constexpr int WAVES = 8;
    const bool small = p.by == MADDNESS_BY_ROWS ? p.M <= 16 * p.groups : p.M <= 16;
    const int rows = small ? 16 : 64, cols = small ? 16 : 32;
    const int64_t col_tiles = ceil_div(p.N, (int64_t)cols);
    const int64_t pieces = ceil_div(p.M, (int64_t)rows) + (p.by == MADDNESS_BY_ROWS ? p.groups : 0);
    if (col_tiles * pieces >= (int64_t)1 << 31) return fail(MADDNESS_E_UNSUPPORTED, "block product: %lld x %lld results are too many", (long long)p.M, (long long)p.N);
    const dim3 grid((unsigned)(col_tiles * pieces), p.by == MADDNESS_BY_DEPTH ? (unsigned)p.groups : 1u);
    note_kernel("product_few_kernel", __PRETTY_FUNCTION__);
    if (small) hipLaunchKernelGGL((product_few_kernel<AT, 1, 1, WAVES, AT == kF32 ? 2 : 4, OUT>), grid, dim3(WAVES * 64), 0, stream, p, (uint32_t)col_tiles);
    else if constexpr (AT == kE4M3)
        hipLaunchKernelGGL((product_few_kernel<AT, 4, 2, WAVES, 1, OUT>), grid, dim3(WAVES * 64), 0, stream, p, (uint32_t)col_tiles);
    return check_hip(hipGetLastError(), "launch product_few_kernel");
}

template <int OUT>
int launch_to(const ProductArgs &p, int a_dtype, hipStream_t stream)
{
    if (a_dtype == MADDNESS_F32) return launch_few<kF32, OUT>(p, stream);
    if (a_dtype == MADDNESS_F16) return launch_few<kF16, OUT>(p, stream);
    if (a_dtype == MADDNESS_BF16) return launch_few<kBF16, OUT>(p, stream);
    return launch_few<kE4M3, OUT>(p, stream);
}

}  // namespace

bool rounds_inside(int64_t M, int64_t N, int64_t K, int groups, int by) { return by == MADDNESS_DENSE && M <= 16; }

int launch_block_product(const ProductArgs &p, int a_dtype, int out_dtype, hipStream_t stream)
{
    if (out_dtype == MADDNESS_F32) return launch_to<kF32>(p, a_dtype, stream);
    if (out_dtype == MADDNESS_F16) return launch_to<kF16>(p, a_dtype, stream);
    return launch_to<kBF16>(p, a_dtype, stream);
}

}  // namespace maddness

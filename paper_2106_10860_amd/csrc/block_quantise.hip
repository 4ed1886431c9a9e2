// Rounding to 8-bit block matrices: e = the least power of two that brings a block's largest magnitude to 448 or less,
// q = x 2^-e to the nearest E4M3 number.  Multiplying by a power of two is exact, so there is one rounding and the result does not
// depend on how the work is split.  Bound by memory: b bytes read and 1 (both ways: 2) written per value.
#include "block_common.h"

namespace maddness {
namespace {

struct QuantiseArgs {
    const void *x;
    int64_t rows, cols, ldx, stride_x;
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
    if (a.factors) factor = a.factors[s];
    at = (int64_t)(s / a.repeat) * a.ldx;
    return there;
}

// Blocks of 1 x 128, rows only.  16 lanes take a block, 8 values each: the maximum stays within a row of lanes.
template <int DT>
__global__ __launch_bounds__(256) void quantise_rows_kernel(QuantiseArgs a, int64_t first_row, uint32_t blocks, uint32_t units)
{
    const uint32_t unit = blockIdx.x * 16u + threadIdx.x / 16u;
    if (unit >= units) return;
    const int lane = threadIdx.x % 16;
    const int64_t r = first_row + unit / blocks;
    const uint32_t b = unit % blocks;
    const int64_t c = (int64_t)b * kBlock + lane * 8, m = blockIdx.y;
    const char *x = static_cast<const char *>(a.x) + m * a.stride_x * elem_size(DT);
    float v[8];
    int64_t at = 0;
    float factor;
    const bool there = find_row(a, r, at, factor);
    if (a.cols >= 8) widen<DT>(load_raw<DT>(x, at, c, a.cols), c, a.cols, v);
    else load_short<DT>(x, at, c, a.cols, v);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (a.factors) v[i] *= factor;
        if (!there) v[i] = 0.0f;
        top = max(top, finite_magnitude(v[i]));
    }
    const uint32_t byte = exponent_byte(row16_max(top));
    const float inv = inverse_scale(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = scaled(v[i], inv);
    const int64_t row = m * a.rows + r;
    if (c < round_up(a.cols, (int64_t)16))
        *reinterpret_cast<uint2 *>(a.q + row * a.ldq + c) = make_uint2(pack4(v[0], v[1], v[2], v[3]), pack4(v[4], v[5], v[6], v[7]));
    uint8_t *s = a.scale + row * a.lds + b;
    if (lane == 0) *s = (uint8_t)byte;
    else if (b == blocks - 1 && b + lane < round_up(blocks, 4u)) s[lane] = 127;
}

// A tile of 128 x 128 to a workgroup, for transposes and common exponents: a thread holds 8 rows of 8 columns.  The transpose's
// bytes go through LDS in pieces of 8 (rows of one column), the pieces of a column exchanged by the writer's column group so that
// the lanes of a write fall on different banks.
template <int DT, int TILE>
__global__ __launch_bounds__(256) void quantise_tiles_kernel(QuantiseArgs a, uint32_t blocks)
{
    __shared__ uint32_t tops[4][kBlock];
    __shared__ uint2 turned[kBlock * 16];
    const int tid = threadIdx.x, cg = tid % 16, rg = tid / 16, wave = tid / 64;
    const uint32_t cb = blockIdx.x % blocks, rb = blockIdx.x / blocks, row_blocks = gridDim.x / blocks;
    const int64_t m = blockIdx.y, c = (int64_t)cb * kBlock + cg * 8, r0 = (int64_t)rb * kBlock + rg * 8;
    const char *x = static_cast<const char *>(a.x) + m * a.stride_x * elem_size(DT);
    float v[8][8], factor[8];
    uint32_t top_row[8], top_col[8] = {};
    Raw<DT> raw[8];
    int64_t at[8] = {};
    bool there[8];
    // (rows beyond the end are read as the last, and columns as widen says: everything is asked for before anything is needed)
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        there[p] = find_row(a, min(r0 + p, a.rows - 1), at[p], factor[p]) && r0 + p < a.rows;
        if (a.cols >= 8) raw[p] = load_raw<DT>(x, at[p], c, a.cols);
    }
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        if (a.cols >= 8) widen<DT>(raw[p], c, a.cols, v[p]);
        else load_short<DT>(x, at[p], c, a.cols, v[p]);
        top_row[p] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (a.factors) v[p][i] *= factor[p];
            if (!there[p]) v[p][i] = 0.0f;
            const uint32_t t = finite_magnitude(v[p][i]);
            top_row[p] = max(top_row[p], t);
            top_col[i] = max(top_col[i], t);
        }
    }
    float inv_col[8], inv_tile = 1.0f;
    uint32_t byte_tile = 0;
    if constexpr (TILE == 1) {
        if (a.q) {
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                const uint32_t byte = exponent_byte(row16_max(top_row[p]));
                const float inv = inverse_scale(byte);
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = scaled(v[p][i], inv);
                const int64_t row = m * a.rows + r0 + p;
                if (r0 + p >= a.rows) continue;
                if (c < round_up(a.cols, (int64_t)16))
                    *reinterpret_cast<uint2 *>(a.q + row * a.ldq + c) = make_uint2(pack4(w[0], w[1], w[2], w[3]), pack4(w[4], w[5], w[6], w[7]));
                uint8_t *s = a.scale + row * a.lds + cb;
                if (cg == 0) *s = (uint8_t)byte;
                else if (cb == blocks - 1 && cb + cg < round_up(blocks, 4u)) s[cg] = 127;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            top_col[i] = max(top_col[i], (uint32_t)__shfl_xor((int)top_col[i], 16));
            top_col[i] = max(top_col[i], (uint32_t)__shfl_xor((int)top_col[i], 32));
            if (rg % 4 == 0) tops[wave][cg * 8 + i] = top_col[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int col = cg * 8 + i;
            const uint32_t byte = exponent_byte(max(max(tops[0][col], tops[1][col]), max(tops[2][col], tops[3][col])));
            inv_col[i] = inverse_scale(byte);
            if (rg == 0 && c + i < a.cols) {
                uint8_t *s = a.scale_t + (m * a.cols + c + i) * a.ldst + rb;
                *s = (uint8_t)byte;
                if (rb == row_blocks - 1)
                    for (uint32_t k = rb + 1; k < round_up(row_blocks, 4u); ++k) *++s = 127;
            }
        }
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int p = 0; p < 8; ++p) top = max(top, top_row[p]);
        top = row16_max(top);
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        if (tid % 64 == 0) tops[wave][0] = top;
        __syncthreads();
        byte_tile = exponent_byte(max(max(tops[0][0], tops[1][0]), max(tops[2][0], tops[3][0])));
        inv_tile = inverse_scale(byte_tile);
        if (a.q) {
#pragma unroll
            for (int p = 0; p < 8; ++p) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] = scaled(v[p][i], inv_tile);
                if (r0 + p < a.rows && c < round_up(a.cols, (int64_t)16))
                    *reinterpret_cast<uint2 *>(a.q + (m * a.rows + r0 + p) * a.ldq + c) =
                        make_uint2(pack4(w[0], w[1], w[2], w[3]), pack4(w[4], w[5], w[6], w[7]));
            }
            if (tid < 4) {
                uint8_t *s = a.scale + (m * row_blocks + rb) * a.lds + cb;
                if (tid == 0) *s = (uint8_t)byte_tile;
                else if (cb == blocks - 1 && cb + tid < round_up(blocks, 4u)) s[tid] = 127;
            }
        }
        if (a.qt && tid < 4) {
            uint8_t *s = a.scale_t + (m * blocks + cb) * a.ldst + rb;
            if (tid == 0) *s = (uint8_t)byte_tile;
            else if (rb == row_blocks - 1 && rb + tid < round_up(row_blocks, 4u)) s[tid] = 127;
        }
    }
    if (!a.qt) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float inv = TILE == 1 ? inv_col[i] : inv_tile;
        float w[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) w[p] = scaled(v[p][i], inv);
        turned[(cg * 8 + i) * 16 + (rg ^ cg)] = make_uint2(pack4(w[0], w[1], w[2], w[3]), pack4(w[4], w[5], w[6], w[7]));
    }
    __syncthreads();
    const int64_t row_end = round_up(a.rows, (int64_t)16);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int at = k * 256 + tid, col = at / 8, piece = at % 8;
        const int64_t out_row = (int64_t)cb * kBlock + col, out_col = (int64_t)rb * kBlock + piece * 16;
        if (out_row >= a.cols || out_col >= row_end) continue;
        const uint2 lo = turned[col * 16 + ((piece * 2) ^ (col / 8))], hi = turned[col * 16 + ((piece * 2 + 1) ^ (col / 8))];
        *reinterpret_cast<uint4 *>(a.qt + (m * a.cols + out_row) * a.ldqt + out_col) = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
}

template <int DT>
int launch_typed(const QuantiseArgs &a, int64_t count, int tile, hipStream_t stream)
{
    const int64_t blocks = ceil_div(a.cols, (int64_t)kBlock);
    if (tile == 1 && !a.qt) {
        // as many rows as 2^30 blocks make to a launch
        const int64_t most = std::max((int64_t)1, ((int64_t)1 << 30) / blocks);
        for (int64_t r = 0; r < a.rows; r += most) {
            const uint32_t units = (uint32_t)(std::min(most, a.rows - r) * blocks);
            note_kernel("quantise_rows_kernel", __PRETTY_FUNCTION__);
            hipLaunchKernelGGL((quantise_rows_kernel<DT>), dim3(ceil_div(units, 16u), (unsigned)count), dim3(256), 0, stream, a, r,
                               (uint32_t)blocks, units);
            const int rc = check_hip(hipGetLastError(), "launch quantise_rows_kernel");
            if (rc != MADDNESS_OK) return rc;
        }
        return MADDNESS_OK;
    }
    const dim3 grid((unsigned)(blocks * ceil_div(a.rows, (int64_t)kBlock)), (unsigned)count);
    note_kernel("quantise_tiles_kernel", __PRETTY_FUNCTION__);
    if (tile == 1) hipLaunchKernelGGL((quantise_tiles_kernel<DT, 1>), grid, dim3(256), 0, stream, a, (uint32_t)blocks);
    else hipLaunchKernelGGL((quantise_tiles_kernel<DT, kBlock>), grid, dim3(256), 0, stream, a, (uint32_t)blocks);
    return check_hip(hipGetLastError(), "launch quantise_tiles_kernel");
}

}  // namespace

int launch_quantise_blocks(const void *x, int dtype, int64_t count, int64_t rows, int64_t cols, int64_t ldx, int64_t stride_x, int tile,
                           const int32_t *source, int64_t source_rows, int repeat, const float *factors, uint8_t *q, int64_t ldq,
                           uint8_t *scale, int64_t lds, uint8_t *qt, int64_t ldqt, uint8_t *scale_t, int64_t ldst, hipStream_t stream)
{
    QuantiseArgs a{x, rows, cols, ldx, stride_x, source, source_rows * repeat, repeat, factors, q, scale, qt, scale_t, ldq, lds, ldqt, ldst};
    if (dtype == MADDNESS_F32) return launch_typed<kF32>(a, count, tile, stream);
    if (dtype == MADDNESS_F16) return launch_typed<kF16>(a, count, tile, stream);
    return launch_typed<kBF16>(a, count, tile, stream);
}

}  // namespace maddness

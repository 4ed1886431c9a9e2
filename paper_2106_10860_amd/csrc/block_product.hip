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
#include <type_traits>

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

// A lane's 32 elements of a floating row's block as they are in memory, in pieces of 8.  Pieces that would pass column K are read from K - 8
// on instead (K >= 8), and moved into their place by round_piece.
template <int DT>
struct Raw {
    uint32_t w[4][2 * elem_size(DT)];
};

template <int DT>
__device__ __forceinline__ Raw<DT> load_raw(const void *a, int64_t row_at, int64_t kb, int group, int64_t K)
{
    struct __attribute__((packed, aligned(elem_size(DT)))) Words { uint32_t w[2 * elem_size(DT)]; };
    Raw<DT> r;
    const int64_t k = kb * kBlock + group * 32;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const Words p = *reinterpret_cast<const Words *>(static_cast<const char *>(a) + (row_at + min(k + 8 * j, K - 8)) * elem_size(DT));
#pragma unroll
        for (int i = 0; i < 2 * elem_size(DT); ++i) r.w[j][i] = p.w[i];
    }
    return r;
}

// Rounds them; the block's maximum is that of the four lanes that hold the row.
template <int DT>
__device__ __forceinline__ Piece round_piece(const Raw<DT> &r, int64_t kb, int group, int64_t K)
{
    float v[4][8];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (DT == kF32) v[j][i] = __uint_as_float(r.w[j][i]);
            else if constexpr (DT == kBF16) v[j][i] = __uint_as_float(i & 1 ? r.w[j][i / 2] & 0xffff0000u : r.w[j][i / 2] << 16);
            else v[j][i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[j][i / 2] >> (i & 1 ? 16 : 0)));
        }
    if ((kb + 1) * kBlock > K) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t moved = kb * kBlock + group * 32 + 8 * j - (K - 8);      // the piece's first element is at this place of the 8
            float in[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) in[i] = v[j][i];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (moved > 0) v[j][i] = 0.0f;
#pragma unroll
                for (int from = i + 1; from < 8; ++from)
                    if (from - i == moved) v[j][i] = in[from];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, finite_magnitude(v[j][i]));
    const auto rows = __builtin_amdgcn_permlane16_swap(top, top, false, false);
    top = max(rows[0], rows[1]);
    const auto halves = __builtin_amdgcn_permlane32_swap(top, top, false, false);
    top = max(halves[0], halves[1]);
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
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r16 = lane % 16, g = lane / 16;
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
        Raw<AT == kE4M3 ? kF32 : AT> raw[DEPTH][MT];
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int64_t kb = min(kb0 + d * WAVES, w.kb1 - 1);
#pragma unroll
            for (int t = 0; t < NT; ++t) b[d][t] = load_piece(row_b[t], scale_b[t], kb, g, w.K);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if constexpr (AT == kE4M3) a[d][t] = load_piece(row_a[t], scale_a[t], kb, g, w.K);
                else raw[d][t] = load_raw<AT>(p.a, at_a[t], kb, g, w.K);
            }
        }
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int64_t kb = kb0 + d * WAVES;
            if (kb >= w.kb1) break;
            if constexpr (AT != kE4M3)
#pragma unroll
                for (int t = 0; t < MT; ++t) a[d][t] = round_piece<AT>(raw[d][t], kb, g, w.K);
            if ((kb + 1) * kBlock > w.K) {
#pragma unroll
                for (int t = 0; t < NT; ++t) cut(b[d][t], kb, g, w.K);
                if constexpr (AT == kE4M3)
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

// Buffers of plain bytes, and the longest row of 8-bit values that 256 of stay below 2^32 bytes.
constexpr int kBufferFlags = 0x00027000;
constexpr int64_t kMostStride = (int64_t)1 << 23;
constexpr int kExpBlocks = 64;          // blocks whose exponents are in LDS at a time

// Four neighbours of a row of out.
template <int OUT>
__device__ __forceinline__ void store4(void *out, int64_t at, f32x4 v, int64_t n, int64_t N, bool wide)
{
    if (wide && n + 3 < N) {
        if constexpr (OUT == kF32) *reinterpret_cast<f32x4 *>(static_cast<float *>(out) + at) = v;
        else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(out) + at) = make_uint2(pack2<OUT>(v[0], v[1]), pack2<OUT>(v[2], v[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < N) store_as<OUT>(out, at + i, v[i]);
    }
}

// The index among a launch's workgroups that work, such that each of the 8 dies (workgroups go to them in turn) gets neighbours.
__device__ __forceinline__ uint32_t by_die(uint32_t id, uint32_t total)
{
    const uint32_t die = id % 8, each = total / 8, more = total % 8;
    return die * each + min(die, more) + id / 8;
}

// Many rows: BM x BN results to a workgroup of WM x WN wavefronts, each with (BM / WM) x (BN / WN) of them in registers.  Blocks of 128 values
// of the BM + BN rows go to LDS without passing registers, the next one while this one is multiplied.  A row's eight pieces of 16 bytes lie
// exchanged by half its index, so that the 16 rows that a read of the lanes goes to fall on all banks.  WIDE: the 16-bit instruction.
template <int BM, int BN, int WM, int WN, bool WIDE, int OUT>
__global__ __launch_bounds__(WM * WN * 64, 2) void product_tiles_kernel(ProductArgs p, uint32_t col_tiles)
{
    constexpr int WAVES = WM * WN, MT = BM / WM / 16, NT = BN / WN / 16, LOADS_A = BM / 8 / WAVES, LOADS_B = BN / 8 / WAVES;
    static_assert(WAVES % 2 == 0 && LOADS_A * 8 * WAVES == BM && LOADS_B * 8 * WAVES == BN, "a wavefront loads whole groups of 8 rows, all at even or all at odd places");
    __shared__ __attribute__((aligned(128))) uint8_t tiles[2][(BM + BN) * kBlock];
    __shared__ uint32_t exps[kExpBlocks / 4][BM + BN];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r16 = lane % 16, g = lane / 16;

    const uint32_t pieces = p.by == MADDNESS_BY_ROWS ? (uint32_t)count_pieces(p.offsets, p.groups, p.M, BM) : (uint32_t)ceil_div(p.M, (int64_t)BM);
    if (blockIdx.x >= pieces * col_tiles) return;
    // four pieces by all columns, then the next four: what a die works on at a time shares rows of both operands
    const uint32_t at = by_die(blockIdx.x, pieces * col_tiles), band = at / (4 * col_tiles), in_band = at % (4 * col_tiles);
    const uint32_t height = min(4u, pieces - band * 4);
    const int64_t n0 = (int64_t)(in_band / height) * BN;
    Part w;
    if (!find_part(p, BM, band * 4 + in_band % height, blockIdx.y, w)) return;

    // Rows are addressed by 32-bit offsets within the tile (the launcher keeps row strides to kMostStride).  What lies beyond the tile's last
    // row is out of the buffers' range; what lies beyond column K is cut off in LDS.
    const uint32_t lda = (uint32_t)p.lda, ldb = (uint32_t)p.ldb, blocks = (uint32_t)ceil_div(w.K, (int64_t)kBlock);
    const uint32_t rows = (uint32_t)(w.last - w.first), cols = (uint32_t)min((int64_t)BN, p.N - n0), width = round_up((uint32_t)w.K, 16u);
    const auto mem_a = __builtin_amdgcn_make_buffer_rsrc((void *)(p.a + w.first * p.lda), 0, (rows - 1) * lda + width, kBufferFlags);
    const auto mem_b = __builtin_amdgcn_make_buffer_rsrc((void *)(w.b + n0 * p.ldb), 0, (cols - 1) * ldb + width, kBufferFlags);
    const uint32_t chunk = (uint32_t)((lane % 8) ^ ((wave % 2) * 4 + lane / 16)) * 16, row0 = wave * 8 + lane / 8;
    const uint32_t at_a = row0 * lda + chunk, at_b = row0 * ldb + chunk;
    // (keeps the compiler from holding every sum of this and a multiple of a stride in a register of its own)
    auto again = [](uint32_t x) INLINE_LAMBDA { asm volatile("" : "+v"(x)); return x; };
    auto load = [&](uint8_t *tile, uint32_t kb) INLINE_LAMBDA {
        const uint32_t lane_a = again(at_a), lane_b = again(at_b);
#pragma unroll
        for (int i = 0; i < LOADS_A; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(mem_a, (__attribute__((address_space(3))) void *)(tile + (wave + i * WAVES) * 1024), 16,
                                                     lane_a + ((i * WAVES * 8) * lda + kb * kBlock), 0, 0, 0);
#pragma unroll
        for (int i = 0; i < LOADS_B; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(mem_b, (__attribute__((address_space(3))) void *)(tile + BM * kBlock + (wave + i * WAVES) * 1024), 16,
                                                     lane_b + ((i * WAVES * 8) * ldb + kb * kBlock), 0, 0, 0);
    };
    const int wm = wave / WN, wn = wave % WN;
    // The exponents of kExpBlocks blocks, four to a word, by rows.
    auto load_exps = [&](uint32_t kb) INLINE_LAMBDA {
        const uint32_t some = min((uint32_t)kExpBlocks, blocks - kb);
        for (int row = threadIdx.x; row < BM + BN; row += WAVES * 64) {
            const uint8_t *from = row < BM ? p.scale_a + (min(w.first + row, w.last - 1) >> p.shift_a) * p.lds_a
                                           : w.scale_b + (min(n0 + row - BM, p.N - 1) >> p.shift_b) * p.lds_b;
            for (uint32_t q = 0; q * 4 < some; ++q) exps[q][row] = *reinterpret_cast<const uint32_t *>(from + kb + q * 4);
        }
    };
    f32x4 acc[MT][NT] = {};
    const int half0 = r16 * kBlock + (((2 * g) ^ (r16 / 2)) * 16), half1 = r16 * kBlock + (((2 * g + 1) ^ (r16 / 2)) * 16);
    auto fragment = [&](const uint8_t *tile, int row) INLINE_LAMBDA {
        const i32x4 lo = *reinterpret_cast<const i32x4 *>(tile + row * kBlock + half0), hi = *reinterpret_cast<const i32x4 *>(tile + row * kBlock + half1);
        return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    // The columns from K on of the last block, in both operands, to zeros.
    auto cut_off = [&](uint8_t *tile) INLINE_LAMBDA {
        for (int row = threadIdx.x; row < BM + BN; row += WAVES * 64)
            for (int k = (int)(w.K % kBlock); k < kBlock; ++k) tile[row * kBlock + (((k / 16) ^ (row / 2 % 8)) * 16 + k % 16)] = 0;
        __syncthreads();
    };
    const uint32_t kb0 = (uint32_t)w.kb0, kb1 = (uint32_t)w.kb1;
    if (kb0 < kb1) {
        uint8_t *tile = tiles[0], *next = tiles[1];
        load(tile, kb0);
        load_exps(kb0 / kExpBlocks * kExpBlocks);
        uint32_t ea[MT], eb[NT];                             // this block's in the lowest byte
        __syncthreads();
        for (uint32_t kb = kb0;; ++kb) {
            if (kb + 1 == kb1 && w.K % kBlock) cut_off(tile);
            if (kb % 4 == 0 || kb == kb0) {
                const uint32_t *from = exps[kb % kExpBlocks / 4] + r16;
#pragma unroll
                for (int t = 0; t < MT; ++t) ea[t] = from[(wm * MT + t) * 16] >> (kb % 4 * 8);
#pragma unroll
                for (int t = 0; t < NT; ++t) eb[t] = from[BM + (wn * NT + t) * 16] >> (kb % 4 * 8);
            }
            // All fragments are asked for before the next block is: the compiler lets no read of LDS pass a load into it.
            i32x8 b[NT], a[MT];
#pragma unroll
            for (int j = 0; j < NT; ++j) b[j] = fragment(tile, BM + (wn * NT + j) * 16);
#pragma unroll
            for (int i = 0; i < MT; ++i) a[i] = fragment(tile, (wm * MT + i) * 16);
            __builtin_amdgcn_sched_barrier(0);
            if (kb + 1 < kb1) load(next, kb + 1);
            if constexpr (!WIDE) {
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a[i], acc[i][j], 0, 0, 0, (int)eb[j], 0, (int)ea[i]);
            } else {
                bf16x8 wb[NT][4];
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) wb[j][q] = widen8(b[j][2 * q], b[j][2 * q + 1], as_scale(eb[j] & 255));
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const bf16x8 wa = widen8(a[i][2 * q], a[i][2 * q + 1], as_scale(ea[i] & 255));
#pragma unroll
                        for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][q], wa, acc[i][j], 0, 0, 0);
                    }
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) ea[t] >>= 8;
#pragma unroll
            for (int t = 0; t < NT; ++t) eb[t] >>= 8;
            if (kb + 1 >= kb1) break;
            __syncthreads();
            if ((kb + 1) % kExpBlocks == 0) {
                load_exps(kb + 1);
                __syncthreads();
            }
            uint8_t *t = tile;
            tile = next;
            next = t;
        }
    }
    constexpr int64_t bytes = OUT == kF32 ? 4 : 2;
    const bool wide = (reinterpret_cast<uintptr_t>(p.out) | (uint64_t)(p.ldo * bytes) | (uint64_t)(w.out_at * bytes)) % (4 * bytes) == 0;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = w.first + (wm * MT + i) * 16 + r16;
        if (m >= w.last) continue;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t n = n0 + (wn * NT + j) * 16 + 4 * g;
            store4<OUT>(p.out, w.out_at + m * p.ldo + n, acc[i][j], n, p.N, wide);
        }
    }
}

template <int BM, int BN, int WM, int WN, int OUT>
int launch_tiles(const ProductArgs &p, hipStream_t stream)
{
    const int64_t col_tiles = ceil_div(p.N, (int64_t)BN), pieces = ceil_div(p.M, (int64_t)BM) + (p.by == MADDNESS_BY_ROWS ? p.groups : 0);
    if (col_tiles * pieces >= (int64_t)1 << 31) return fail(MADDNESS_E_UNSUPPORTED, "block product: %lld x %lld results are too many", (long long)p.M, (long long)p.N);
    const dim3 grid((unsigned)(col_tiles * pieces), p.by == MADDNESS_BY_DEPTH ? (unsigned)p.groups : 1u);
    note_kernel("product_tiles_kernel", __PRETTY_FUNCTION__);
    hipLaunchKernelGGL((product_tiles_kernel<BM, BN, WM, WN, OUT == kF32, OUT>), grid, dim3(WM * WN * 64), 0, stream, p, (uint32_t)col_tiles);
    return check_hip(hipGetLastError(), "launch product_tiles_kernel");
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
        hipLaunchKernelGGL((product_few_kernel<AT, 4, 2, WAVES, 2, OUT>), grid, dim3(WAVES * 64), 0, stream, p, (uint32_t)col_tiles);
    return check_hip(hipGetLastError(), "launch product_few_kernel");
}

template <int OUT>
int launch_to(const ProductArgs &p, int a_dtype, hipStream_t stream)
{
    if (a_dtype == MADDNESS_F32) return launch_few<kF32, OUT>(p, stream);
    if (a_dtype == MADDNESS_F16) return launch_few<kF16, OUT>(p, stream);
    if (a_dtype == MADDNESS_BF16) return launch_few<kBF16, OUT>(p, stream);
    const int64_t groups = p.by == MADDNESS_DENSE ? 1 : p.groups, rows = p.by == MADDNESS_BY_ROWS ? ceil_div(p.M, groups) : p.M;
    if (rows <= 64 || std::max(p.lda, p.ldb) > kMostStride) return launch_few<kE4M3, OUT>(p, stream);
    const int64_t large = ceil_div(rows, (int64_t)256) * ceil_div(p.N, (int64_t)256) * groups;
    if constexpr (OUT != kF32)
        if (large >= device_info().cus && rows >= 1024) return launch_tiles<256, 256, 2, 4, OUT>(p, stream);
    return launch_tiles<128, 128, 2, 2, OUT>(p, stream);
}

}  // namespace

bool rounds_inside(int64_t M, int64_t N, int64_t K, int groups, int by) { return by == MADDNESS_DENSE && M <= 16 && K >= 8; }

int launch_block_product(const ProductArgs &p, int a_dtype, int out_dtype, hipStream_t stream)
{
    if (out_dtype == MADDNESS_F32) return launch_to<kF32>(p, a_dtype, stream);
    if (out_dtype == MADDNESS_F16) return launch_to<kF16>(p, a_dtype, stream);
    return launch_to<kBF16>(p, a_dtype, stream);
}

}  // namespace maddness

// out[m][n] = sum_k A[m][k] B[n][k] of two 8-bit block matrices on the matrix cores.
//
// Two kinds of instruction multiply them.  The 16-bit one (v_mfma_f32_16x16x32_bf16) has products and sums of fp32 (9e-9 of the result).  The 8-bit one
// (v_mfma_scale_f32_16x16x128) takes the bytes and the powers of two as they are at twice the rate, but brings the products of eight neighbours k to a common
// exponent and cuts each off, towards 0, at 2^-13 of the power of two of the largest (of the sum of its factors' exponents, where a subnormal number's is that
// of the least normal one); the sums of eight are added up like fp32.  So an eight loses up to 7 2^-13 = 8.5e-4 of its largest product: measured 7.9e-4 of a
// sum of terms of one sign, 1.5e-5 of the result for normal values, 3e-4 with heavy tails.  That is below a quarter of what a result loses at most when it is rounded to
// bfloat16 (2^-8), but more than to binary16 (2^-11).  So bfloat16 results of many rows come from the 8-bit instruction, binary16 and fp32 results from the
// 16-bit one, and few rows always from that, as memory bounds them.
//
// B's rows (the columns of out) are the instruction's first operand and A's rows its second, so that a lane's four results are
// four neighbours in a row of out.  Lane l holds 32 values of row l % 16 of an operand's block (which 32 does not matter as long as they are
// the same ones of both operands), and results n = 4 (l / 16) + i of row m = l % 16.
#include "block_common.h"
#include "tile_loads.h"

namespace maddness {
namespace {

using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;

// Eight E4M3 values times 2^(byte - 127) as bfloat16 numbers: exactly for the bytes 3 to 246 (the values are multiples of 2^-9 of up to 448, bfloat16 has
// the multiples of 2^-133 with 8 digits below 2^128).  scale = byte << 23 (the conversion reads its exponent only, 255 gives NaN).
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

__device__ __forceinline__ void cut(Piece &p, int64_t kb, int group, int64_t K)
{
    const int64_t k = kb * kBlock + group * 32;
    p.lo = first_bytes(p.lo, K - k);
    p.hi = first_bytes(p.hi, K - k - 16);
}

// Whether A's rows are rounded within the few-rows kernel, by every workgroup for itself: while they fill 32 KiB of LDS at most, which costs a
// workgroup up to 64 values a thread (1.5 us), a launch of their own costs 5 us.
constexpr int64_t kInside = 32768, kInsideRows = 64;
constexpr int kMostChosen = MADDNESS_MAX_CHOSEN;

// What a workgroup computes: rows first .. last - 1 of A, with one expert's matrix, over the blocks kb0 .. kb1 - 1.
struct Part {
    int64_t first, last, kb0, kb1, K;
    const uint8_t *b, *scale_b;
    int64_t out_at;
};

__device__ __forceinline__ bool find_part(const ProductArgs &p, PieceSearch &search, int rows, int64_t piece, int64_t group, Part &w)
{
    w.b = p.b;
    w.scale_b = p.scale_b;
    w.out_at = 0;
    w.K = p.K;
    w.kb0 = 0;
    if (p.by == MADDNESS_BY_ROWS) {
        const int e = search.find(p.offsets, p.groups, p.M, rows, piece, w.first, w.last);
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

// Row m of the product's A: itself, or that of the slot's token; -1 where there is none.
__device__ __forceinline__ int64_t row_of_a(const ProductArgs &p, int64_t m)
{
    if (!p.source) return m;
    const int s = p.source[m];
    return s < 0 || s >= p.source_limit ? -1 : s / p.repeat;
}

// Few rows: 16 MT rows by 16 NT columns to a workgroup; its wavefronts take every WAVES-th block of the sum, DEPTH of them asked for
// at once, and add up in LDS, in their order.  B comes straight from memory, in pieces of 32 bytes to a lane, and so does an 8-bit A; a floating
// A is rounded into LDS while the first of B is on its way.  Bound by the way of one piece: 1 x 4096 x 4096 6.4 us (16.8 MB, 2.6 TB/s),
// 37 x 1000 x 510 7.9.
//
// CHOICE: of the slots, those whose id is the workgroup's expert, found by going through all ids, 16 MT at a time; no order of them is needed.  The rows of
// results are the slots themselves.  (24 slots of 64 experts of 1024 x 512: 8.4 us; the layer of it, with the choice and the sum, 16 us, 22 with an order.)
template <int AT, int MT, int NT, int WAVES, int DEPTH, int OUT, bool CHOICE>
__global__ __launch_bounds__(WAVES * 64) void product_few_kernel(ProductArgs p, uint32_t col_tiles)
{
    constexpr bool ROUND = AT != kE4M3;
    __shared__ int32_t slots[CHOICE ? kMostChosen : 1];
    __shared__ f32x4 sums[WAVES][MT * NT][64];
    __shared__ __attribute__((aligned(16))) uint8_t rounded[ROUND ? kInside + kInsideRows * 16 : 16], bytes[ROUND ? kInside / kBlock + kInsideRows : 16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t n0 = (int64_t)(blockIdx.x % col_tiles) * (16 * NT);
    Part w;
    PieceSearch search;
    int count = 0;
    if constexpr (CHOICE) {
        const int lane = threadIdx.x % 64;
        const int e = blockIdx.x / col_tiles;
        for (int base = 0; base < (int)p.M; base += 64) {
            const int slot = base + lane, id = slot < (int)p.M ? p.source[slot] : e + 1;
            const uint64_t here = __ballot(id == e);
            if (wave == 0 && id == e) slots[count + __popcll(here & (((uint64_t)1 << lane) - 1))] = slot;
            count += __popcll(here);
            if (e == 0 && wave == 0 && slot < (int)p.M && (id < 0 || id >= p.groups))
                for (int64_t n = n0; n < min(n0 + 16 * NT, p.N); ++n) store_as<OUT>(p.out, slot * p.ldo + n, 0.0f);
        }
        if (count == 0) return;
        w = Part{0, min(count, 16 * MT), 0, ceil_div(p.K, (int64_t)kBlock), p.K, p.b + e * p.stride_b, p.scale_b + e * p.scale_stride_b, 0};
        __syncthreads();
    } else {
        if (!find_part(p, search, 16 * MT, blockIdx.x / col_tiles, blockIdx.y, w)) return;
    }
    for (bool again = false;; again = true) {
        int lane = threadIdx.x % 64;
        if constexpr (CHOICE) asm volatile("" : "+v"(lane));  // (or all addresses that stay the same would be kept in registers, which then do for half the workgroups)
        const int r16 = lane % 16, g = lane / 16;
        const uint8_t *row_b[NT], *row_a[MT], *scale_a[MT], *scale_b[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int64_t n = min(n0 + t * 16 + r16, p.N - 1);
            row_b[t] = w.b + n * p.ldb;
            scale_b[t] = w.scale_b + (n >> p.shift_b) * p.lds_b;
        }
        Piece b[DEPTH][NT], a[DEPTH][MT];
        auto load = [&](int64_t kb0) INLINE_LAMBDA {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d)
#pragma unroll
                for (int t = 0; t < NT; ++t) b[d][t] = load_piece(row_b[t], scale_b[t], min(kb0 + d * WAVES, w.kb1 - 1), g, w.K);
        };
        const int64_t kb_first = w.kb0 + wave;
        if (kb_first < w.kb1) load(kb_first);

        const int blocks = ROUND ? (int)w.kb1 : 0, stride = blocks * kBlock + 16;
        if constexpr (ROUND) {
            const int units = again ? 0 : (int)p.a_rows * blocks;
            for (int unit = threadIdx.x / 16; unit < units; unit += WAVES * 4) {
                const int row = unit / blocks, kb = unit % blocks;
                const int64_t k = (int64_t)kb * kBlock + r16 * 8;
                float v[8];
                const int skip = before_column(k, p.K);
                widen<AT>(load_raw<AT>(p.a, row * p.lda, k, p.K), v);
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = i < skip ? top : max(top, finite_magnitude(v[i]));
                const uint32_t byte = exponent_byte(row16_max(top));
                *reinterpret_cast<uint2 *>(rounded + row * stride + kb * kBlock + r16 * 8) =
                    in_place(make_uint2(pack4(v[0], v[1], v[2], v[3], byte), pack4(v[4], v[5], v[6], v[7], byte)), skip);
                if (r16 == 0) bytes[unit] = (uint8_t)byte;
            }
            __syncthreads();
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const int64_t at = min(w.first + t * 16 + r16, w.last - 1), m = CHOICE ? slots[at] / p.repeat : max(row_of_a(p, at), (int64_t)0);
            row_a[t] = ROUND ? rounded + m * stride : p.a + m * p.lda;
            scale_a[t] = ROUND ? bytes + m * blocks : p.scale_a + (m >> p.shift_a) * p.lds_a;
        }
        f32x4 acc[MT][NT] = {};
        for (int64_t kb0 = kb_first; kb0 < w.kb1; kb0 += DEPTH * WAVES) {
            if (kb0 != kb_first) load(kb0);
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                const int64_t kb = min(kb0 + d * WAVES, w.kb1 - 1);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    if constexpr (ROUND) {
                        a[d][t].lo = *reinterpret_cast<const i32x4 *>(row_a[t] + kb * kBlock + g * 32);
                        a[d][t].hi = *reinterpret_cast<const i32x4 *>(row_a[t] + kb * kBlock + g * 32 + 16);
                        a[d][t].byte = scale_a[t][kb];
                    } else {
                        a[d][t] = load_piece(row_a[t], scale_a[t], kb, g, w.K);
                    }
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
            if (w.first + m >= w.last || n0 + n >= p.N || (!CHOICE && p.source && row_of_a(p, w.first + m) < 0)) continue;
            const int tile = m / 16 * NT + n / 16, at = m % 16 + n % 16 / 4 * 16;
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) s += sums[k][tile][at][n % 4];
            store_as<OUT>(p.out, w.out_at + (CHOICE ? slots[w.first + m] : w.first + m) * p.ldo + n0 + n, s);
        }
        w.first += 16 * MT;
        if (!CHOICE || w.first >= count) break;
        w.last = min(w.first + 16 * MT, (int64_t)count);
        __syncthreads();
    }
}

constexpr int kExpBlocks = 32;          // blocks whose exponents come to LDS at a time

template <int B, int A>
__device__ __forceinline__ f32x4 multiply(i32x8 b, i32x8 a, f32x4 c, int scale_b, int scale_a)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, 0, B, scale_b, A, scale_a);
}

// The same with the exponents' bytes as arguments, for calls that are written out.
__device__ __forceinline__ f32x4 multiply(i32x8 b, i32x8 a, f32x4 c, int scale_b, int byte_b, int scale_a, int byte_a)
{
    switch (byte_b * 4 + byte_a) {
    case 0: return multiply<0, 0>(b, a, c, scale_b, scale_a);
    case 1: return multiply<0, 1>(b, a, c, scale_b, scale_a);
    case 2: return multiply<0, 2>(b, a, c, scale_b, scale_a);
    case 3: return multiply<0, 3>(b, a, c, scale_b, scale_a);
    case 4: return multiply<1, 0>(b, a, c, scale_b, scale_a);
    case 5: return multiply<1, 1>(b, a, c, scale_b, scale_a);
    case 6: return multiply<1, 2>(b, a, c, scale_b, scale_a);
    case 7: return multiply<1, 3>(b, a, c, scale_b, scale_a);
    case 8: return multiply<2, 0>(b, a, c, scale_b, scale_a);
    case 9: return multiply<2, 1>(b, a, c, scale_b, scale_a);
    case 10: return multiply<2, 2>(b, a, c, scale_b, scale_a);
    case 11: return multiply<2, 3>(b, a, c, scale_b, scale_a);
    case 12: return multiply<3, 0>(b, a, c, scale_b, scale_a);
    case 13: return multiply<3, 1>(b, a, c, scale_b, scale_a);
    case 14: return multiply<3, 2>(b, a, c, scale_b, scale_a);
    default: return multiply<3, 3>(b, a, c, scale_b, scale_a);
    }
}

// Many rows: BM x BN results to a workgroup of WM x WN wavefronts, each with (BM / WM) x (BN / WN) of them in registers.  Blocks of 128 values
// of the BM + BN rows go to LDS without passing registers, the next ones while this one is multiplied.  A row's eight pieces of 16 bytes lie
// exchanged by its index, so that the rows that a read of the lanes goes to fall on all banks.  WIDE: the 16-bit instruction.
//
// Eight wavefronts are two to a SIMD, and take turns: while one half of them reads its fragments of a block from LDS, the other half multiplies the ones
// that it has read before.  16384 x 4096 x 4096 to bfloat16: 268 us with all eight reading and then all multiplying, 229 to 250 in turns (the more the more
// the operands change from call to call), 2200 to 2400 TFLOP/s, 0.9 of what the library's product of 8-bit matrices without exponents reaches; to binary16, by the
// 16-bit instruction, 453.  The matrix cores are busy half of the time in either, by their counter; of a block's 1.8 us the rest goes to the way of 64 KiB from
// L2 to LDS, of which one block is under way at a time.  (The first twenty calls after a pause take up to a quarter longer each, until the clocks are up.)
template <int BM, int BN, int WM, int WN, bool WIDE, bool GATHER, int OUT>
__global__ __launch_bounds__(WM * WN * 64, 2) void product_tiles_kernel(ProductArgs p, uint32_t col_tiles)
{
    constexpr int WAVES = WM * WN, MT = BM / WM / 16, NT = BN / WN / 16, LOADS_A = BM / 8 / WAVES, LOADS_B = BN / 8 / WAVES;
    static_assert(MT % 4 == 0 && NT % 4 == 0, "a lane's exponents are whole words");
    static_assert(WAVES % 2 == 0 && LOADS_A * 8 * WAVES == BM && LOADS_B * 8 * WAVES == BN, "a wavefront loads whole groups of 8 rows, all at even or all at odd places");
    __shared__ __attribute__((aligned(128))) uint8_t tiles[2][(BM + BN) * kBlock];
    __shared__ uint32_t exps[2][kExpBlocks][(BM + BN) / 4];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r16 = lane % 16, g = lane / 16;

    PieceSearch search;
    const uint32_t pieces = p.by == MADDNESS_BY_ROWS ? (uint32_t)search.count(p.offsets, p.groups, p.M, BM) : (uint32_t)ceil_div(p.M, (int64_t)BM);
    if (blockIdx.x >= pieces * col_tiles) return;
    // four pieces by all columns, then the next four: what a die works on at a time shares rows of both operands
    const uint32_t at = by_die(blockIdx.x, pieces * col_tiles), band = at / (4 * col_tiles), in_band = at % (4 * col_tiles);
    const uint32_t height = min(4u, pieces - band * 4);
    const int64_t n0 = (int64_t)(in_band / height) * BN;
    Part w;
    if (!find_part(p, search, BM, band * 4 + in_band % height, blockIdx.y, w)) return;

    // Rows are addressed by 32-bit offsets within the tile (the launcher keeps row strides to kMostStride).  What lies beyond the tile's last
    // row is out of the buffers' range; what lies beyond column K is cut off from the fragments.
    const uint32_t lda = (uint32_t)p.lda, ldb = (uint32_t)p.ldb, blocks = (uint32_t)ceil_div(w.K, (int64_t)kBlock);
    const uint32_t rows = (uint32_t)(w.last - w.first), cols = (uint32_t)min((int64_t)BN, p.N - n0), width = round_up((uint32_t)w.K, 16u);
    const i32x4 mem_a = buffer_of(p.a + (GATHER ? 0 : w.first * p.lda), ((GATHER ? (uint32_t)p.a_rows : rows) - 1) * lda + width);
    const i32x4 mem_b = buffer_of(w.b + n0 * p.ldb, (cols - 1) * ldb + width);
    const uint32_t chunk = (uint32_t)((lane % 8) ^ (lane / 8)) * 16, row0 = wave * 8 + lane / 8;
    const uint32_t at_a = row0 * lda + chunk, at_b = row0 * ldb + chunk;
    uint32_t from_a[LOADS_A];
    if constexpr (GATHER) {
#pragma unroll
        for (int i = 0; i < LOADS_A; ++i)
            from_a[i] = (uint32_t)max(row_of_a(p, min(w.first + row0 + i * WAVES * 8, w.last - 1)), (int64_t)0) * lda + chunk;
    }
    // (keeps the compiler from holding every sum of this and a multiple of a stride in a register of its own)
    auto again = [](uint32_t x) INLINE_LAMBDA { asm volatile("" : "+v"(x)); return x; };
    const uint32_t tiles_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)tiles[0] + wave * 1024;
    auto load_one = [&](int i, uint32_t stage, uint32_t kb, uint32_t wanted, auto always) INLINE_LAMBDA {
        const uint32_t to = tiles_at + stage * ((BM + BN) * kBlock) + (i < LOADS_A ? i * WAVES * 1024 : BM * kBlock + (i - LOADS_A) * WAVES * 1024);
        uint32_t at = i < LOADS_A ? again(at_a) + ((i * WAVES * 8) * lda + kb * kBlock) : again(at_b) + (((i - LOADS_A) * WAVES * 8) * ldb + kb * kBlock);
        if constexpr (GATHER)
            if (i < LOADS_A) at = from_a[i < LOADS_A ? i : 0] + kb * kBlock;
        if constexpr (decltype(always)::value) load_to_lds(i < LOADS_A ? mem_a : mem_b, at, to);
        else load_to_lds_if(wanted, i < LOADS_A ? mem_a : mem_b, at, to);
    };
    auto load = [&](uint32_t stage, uint32_t kb) INLINE_LAMBDA {
#pragma unroll
        for (int i = 0; i < LOADS_A + LOADS_B; ++i) load_one(i, stage, kb, 1, std::true_type{});
    };
    const int wm = wave / WN, wn = wave % WN;
    // The exponents of kExpBlocks blocks: of each block the rows' bytes, those of rows r, r + 16, r + 32 and r + 48 of every 64 in a word.  So a lane gets
    // those of four fragments at once, and the instruction takes the byte that it needs.
    auto load_exps = [&](uint32_t chunk_of) INLINE_LAMBDA {
        const uint32_t last_word = (blocks - 1) / 4 * 4;
        for (int row = threadIdx.x; row < BM + BN; row += WAVES * 64) {
            const int64_t m = min(w.first + row, w.last - 1);
            const uint8_t *from = row < BM ? p.scale_a + ((GATHER ? max(row_of_a(p, m), (int64_t)0) : m) >> p.shift_a) * p.lds_a
                                           : w.scale_b + (min(n0 + row - BM, p.N - 1) >> p.shift_b) * p.lds_b;
            uint32_t words[kExpBlocks / 4];                  // (all on their way before the first is needed; beyond the last block that again)
#pragma unroll
            for (int q = 0; q < kExpBlocks / 4; ++q) words[q] = *reinterpret_cast<const uint32_t *>(from + min(chunk_of * kExpBlocks + q * 4, last_word));
            uint8_t *to = reinterpret_cast<uint8_t *>(exps[chunk_of % 2][0]) + row / 64 * 64 + row % 16 * 4 + row % 64 / 16;
#pragma unroll
            for (int k = 0; k < kExpBlocks; ++k) to[k * (BM + BN)] = (uint8_t)(words[k / 4] >> (k % 4 * 8));
        }
    };
    f32x4 acc[MT][NT] = {};
    // A lane's 32 values of a row are pieces g and g + 4: the same ones of both operands, and then a read of the 64 lanes takes 4 clocks (of pieces
    // 2 g and 2 g + 1 it takes 7).
    const int half0 = r16 * kBlock + ((g ^ (r16 % 8)) * 16), half1 = half0 ^ 64;
    auto fragment = [&](const uint8_t *tile, int row) INLINE_LAMBDA {
        const i32x4 lo = *reinterpret_cast<const i32x4 *>(tile + row * kBlock + half0), hi = *reinterpret_cast<const i32x4 *>(tile + row * kBlock + half1);
        return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    const uint32_t kb0 = (uint32_t)w.kb0, kb1 = (uint32_t)w.kb1;
    if (kb0 < kb1) {
        constexpr int LOADS = LOADS_A + LOADS_B;
        constexpr bool TURNS = WAVES == 8;
        const bool second = TURNS && wave >= WAVES / 2;      // the half that reads while the first multiplies
        load(0, kb0);
        // Later chunks are fetched when the one before is a quarter done: its place was the one's before that, which nobody reads any more.
        const uint32_t chunk0 = kb0 / kExpBlocks;
        load_exps(chunk0);
        if (kb0 % kExpBlocks >= kExpBlocks / 4) load_exps(chunk0 + 1);
        wait_for_loads();
        meet();
        uint32_t stage = 0;
        if (second) {
            if (kb0 + 1 < kb1) load(1, kb0 + 1);
            meet();
        }
        for (uint32_t kb = kb0;; ++kb) {
            if (!second && kb + 1 < kb1) load(stage ^ 1, kb + 1);
            if (kb % kExpBlocks == kExpBlocks / 4 && kb != kb0 && kb / kExpBlocks * kExpBlocks + kExpBlocks < kb1) load_exps(kb / kExpBlocks + 1);
            const uint8_t *tile = tiles[stage];
            const uint32_t *from = exps[kb / kExpBlocks % 2][kb % kExpBlocks] + r16;
            uint32_t ea[ceil_div(MT, 4)], eb[ceil_div(NT, 4)];
#pragma unroll
            for (int t = 0; t < MT; t += 4) ea[t / 4] = from[(wm * MT + t) * 4];
#pragma unroll
            for (int t = 0; t < NT; t += 4) eb[t / 4] = from[BM / 4 + (wn * NT + t) * 4];
            i32x8 b[NT], a[MT];
#pragma unroll
            for (int j = 0; j < NT; ++j) b[j] = fragment(tile, BM + (wn * NT + j) * 16);
#pragma unroll
            for (int i = 0; i < MT; ++i) a[i] = fragment(tile, (wm * MT + i) * 16);
            if (kb + 1 == kb1 && w.K % kBlock) {
                const int keep = (int)(w.K % kBlock) - g * 16;
                i32x8 mask;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int n = min(max(keep - i % 4 * 4 - i / 4 * 64, 0), 4);
                    mask[i] = n == 4 ? -1 : (int)((1u << (8 * n)) - 1);
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) b[j] &= mask;
#pragma unroll
                for (int i = 0; i < MT; ++i) a[i] &= mask;
            }
            bf16x8 wb[WIDE ? NT : 1][4], wa[WIDE && TURNS ? MT : 1][4];
            auto widen_fragment = [&](const i32x8 &v, uint32_t byte, bf16x8 (&to)[4]) INLINE_LAMBDA {
#pragma unroll
                for (int q = 0; q < 4; ++q) to[q] = widen8(v[2 * q], v[2 * q + 1], as_scale(byte & 255));
            };
            if constexpr (WIDE) {
#pragma unroll
                for (int j = 0; j < NT; ++j) widen_fragment(b[j], eb[j / 4] >> (j % 4 * 8), wb[j]);
                if constexpr (TURNS) {
#pragma unroll
                    for (int i = 0; i < MT; ++i) widen_fragment(a[i], ea[i / 4] >> (i % 4 * 8), wa[i]);
                }
            }
            if constexpr (TURNS) {
                // (the next block has to have come when the first half reads it, which is when the second half has done so with this one)
                if (second) wait_for_loads();
                else wait_for_reads();
                meet();
                __builtin_amdgcn_s_setprio(1);               // (the half that multiplies before the one that reads)
            }
            if constexpr (!WIDE) {
                const uint32_t more = __builtin_amdgcn_readfirstlane(TURNS && second && kb + 2 < kb1);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
#pragma unroll
                    for (int j = 0; j < NT; ++j)
                        acc[i][j] = multiply(b[j], a[i], acc[i][j], (int)eb[j / 4], j % 4, (int)ea[i / 4], i % 4);
                    // the second half's loads among its products, as each takes some time to get away
                    if constexpr (TURNS) {
#pragma unroll
                        for (int l = i * LOADS / MT; l < (i + 1) * LOADS / MT; ++l) load_one(l, stage, kb + 2, more, std::false_type{});
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                if constexpr (!TURNS) {
                    // B's fragments and two of A's, then two more of A's before the products of the last two
                    __builtin_amdgcn_sched_group_barrier(kReads, 2 * NT + 4, 0);
#pragma unroll
                    for (int i = 0; i < MT / 2; ++i) {
                        if (i + 1 < MT / 2) __builtin_amdgcn_sched_group_barrier(kReads, 4, 0);
                        __builtin_amdgcn_sched_group_barrier(kProducts, 2 * NT, 0);
                    }
                }
            } else {
                const uint32_t more = __builtin_amdgcn_readfirstlane(TURNS && second && kb + 2 < kb1);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if constexpr (!TURNS) widen_fragment(a[i], ea[i / 4] >> (i % 4 * 8), wa[0]);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
#pragma unroll
                        for (int j = 0; j < NT; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][q], wa[TURNS ? i : 0][q], acc[i][j], 0, 0, 0);
                    if constexpr (TURNS) {
#pragma unroll
                        for (int l = i * LOADS / MT; l < (i + 1) * LOADS / MT; ++l) load_one(l, stage, kb + 2, more, std::false_type{});
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            if constexpr (TURNS) __builtin_amdgcn_s_setprio(0);
            if (kb + 1 >= kb1) break;
            if (!second) wait_for_loads();
            meet();
            stage ^= 1;
        }
        if (TURNS && !second) meet();                        // (the second half is one behind)
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = w.first + (wm * MT + i) * 16 + r16;
        if (m >= w.last || (GATHER && row_of_a(p, m) < 0)) continue;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t n = n0 + (wn * NT + j) * 16 + 4 * g, at = w.out_at + m * p.ldo + n;
            const float four[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (n + 4 <= p.N) {
                store_run<OUT>(p.out, at, four);
            } else {
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (n + k < p.N) store_as<OUT>(p.out, at + k, four[k]);
            }
        }
    }
}

// Whether results of a type need the products of the 16-bit instruction.
template <int OUT>
constexpr bool kWide = OUT != kBF16;

template <int BM, int BN, int WM, int WN, bool GATHER, int OUT>
int launch_tiles(const ProductArgs &p, hipStream_t stream)
{
    const int64_t col_tiles = ceil_div(p.N, (int64_t)BN), pieces = ceil_div(p.M, (int64_t)BM) + (p.by == MADDNESS_BY_ROWS ? p.groups : 0);
    if (col_tiles * pieces * WM * WN * 64 > kMostThreads) return fail(MADDNESS_E_UNSUPPORTED, "block product: %lld x %lld results are too many", (long long)p.M, (long long)p.N);
    const dim3 grid((unsigned)(col_tiles * pieces), p.by == MADDNESS_BY_DEPTH ? (unsigned)p.groups : 1u);
    note_kernel("product_tiles_kernel", __PRETTY_FUNCTION__);
    hipLaunchKernelGGL((product_tiles_kernel<BM, BN, WM, WN, kWide<OUT>, GATHER, OUT>), grid, dim3(WM * WN * 64), 0, stream, p, (uint32_t)col_tiles);
    return check_hip(hipGetLastError(), "launch product_tiles_kernel");
}

template <int AT, int OUT, int MT, int NT, int DEPTH, bool CHOICE>
int launch_few_as(const ProductArgs &p, hipStream_t stream)
{
    constexpr int WAVES = 8;
    const int64_t col_tiles = ceil_div(p.N, (int64_t)(16 * NT));
    const int64_t pieces = CHOICE ? p.groups : ceil_div(p.M, (int64_t)(16 * MT)) + (p.by == MADDNESS_BY_ROWS ? p.groups : 0);
    if (col_tiles * pieces * WAVES * 64 > kMostThreads) return fail(MADDNESS_E_UNSUPPORTED, "block product: %lld x %lld results are too many", (long long)p.M, (long long)p.N);
    const dim3 grid((unsigned)(col_tiles * pieces), p.by == MADDNESS_BY_DEPTH ? (unsigned)p.groups : 1u);
    note_kernel("product_few_kernel", __PRETTY_FUNCTION__);
    hipLaunchKernelGGL((product_few_kernel<AT, MT, NT, WAVES, DEPTH, OUT, CHOICE>), grid, dim3(WAVES * 64), 0, stream, p, (uint32_t)col_tiles);
    return check_hip(hipGetLastError(), "launch product_few_kernel");
}

// Rows of A that one matrix of B goes with, about.
int64_t rows_each(const ProductArgs &p) { return p.by == MADDNESS_BY_ROWS ? ceil_div(p.M, (int64_t)p.groups) : p.M; }

template <int AT, int OUT>
int launch_few(const ProductArgs &p, hipStream_t stream)
{
    // a wavefront's share of the sum is one block: more columns to a workgroup instead
    const bool shallow = p.K <= 8 * kBlock;
    if (p.by == MADDNESS_BY_CHOICE) return shallow ? launch_few_as<AT, OUT, 1, 4, 1, true>(p, stream) : launch_few_as<AT, OUT, 1, 1, 4, true>(p, stream);
    if (rows_each(p) > 16) return launch_few_as<AT, OUT, 4, 2, 2, false>(p, stream);
    return shallow ? launch_few_as<AT, OUT, 1, 4, 1, false>(p, stream) : launch_few_as<AT, OUT, 1, 1, 4, false>(p, stream);
}

template <bool GATHER, int OUT>
int launch_shape(const ProductArgs &p, int64_t rows, int64_t groups, hipStream_t stream)
{
    // Larger tiles have less to read for each product, but need enough of them for every compute unit: 256 x 256 one each (8192 x 4096 x 4096 to
    // bfloat16 127 us, 143 by 128 x 128; 2048 x 4096 x 4096 57 and 38), of 256 x 128 with the 16-bit instruction two (to fp32 225 and 241 us; 62 and 66).  Rows that
    // are gathered come in short pieces, which larger tiles leave half empty.
    if constexpr (!GATHER) {
        constexpr int64_t BN = kWide<OUT> ? 128 : 256;
        const int64_t large = ceil_div(rows, (int64_t)256) * ceil_div(p.N, BN) * groups;
        if (rows >= 1024 && large >= (kWide<OUT> ? 2 : 1) * device_info().cus) {
            if constexpr (kWide<OUT>) return launch_tiles<256, 128, 4, 2, false, OUT>(p, stream);
            else return launch_tiles<256, 256, 2, 4, false, OUT>(p, stream);
        }
    }
    return launch_tiles<128, 128, 2, 2, GATHER, OUT>(p, stream);
}

template <int OUT>
int launch_to(const ProductArgs &p, int a_dtype, hipStream_t stream)
{
    if (a_dtype == MADDNESS_F32) return launch_few<kF32, OUT>(p, stream);
    if (a_dtype == MADDNESS_F16) return launch_few<kF16, OUT>(p, stream);
    if (a_dtype == MADDNESS_BF16) return launch_few<kBF16, OUT>(p, stream);
    if (p.by == MADDNESS_BY_CHOICE) return launch_few<kE4M3, OUT>(p, stream);
    const int64_t rows = rows_each(p), groups = p.by == MADDNESS_DENSE ? 1 : p.groups;
    const bool far = std::max(p.lda, p.ldb) > kMostStride || (p.source && p.a_rows * p.lda >= (int64_t)1 << 32);
    // Between the two by what they take, in microseconds, fitted to sizes from 300 x 300 x 300 to 1024 x 4096 x 4096: the few-rows kernel makes more workgroups of
    // a product, and so wins where the other leaves compute units without work (1024 x 512 x 512: 7.0 against 9.0, 128 x 4096 x 4096: 20 against 25,
    // 256 x 4096 x 4096: 38 against 25).  Experts' rows count as their average, as only the device knows the rest: where one expert has all, the few-rows kernel
    // takes no longer than with even shares (64 experts of 1024 x 1024, 2048 rows: 43 us and 60; 14 as a dense product), the other neither (12800 rows 38 and 40).
    const double blocks = (double)ceil_div(p.by == MADDNESS_BY_DEPTH ? ceil_div(p.K, groups) : p.K, (int64_t)kBlock);
    const double small = (double)(ceil_div(rows, (int64_t)64) * ceil_div(p.N, (int64_t)32) * groups), tiles = (double)(ceil_div(rows, (int64_t)128) * ceil_div(p.N, (int64_t)128) * groups);
    const double cus = device_info().cus, step = kWide<OUT> ? 0.85 : 0.6;
    const double few_us = 5.0 + std::max(1.0, small / cus) * (1.0 + 0.45 * blocks);
    const double tiles_us = 7.5 + std::max(1.0, tiles / cus) * (tiles > cus ? 0.8 : 1.0) * (1.0 + step * blocks);
    if (far || (rows <= 64 && p.by != MADDNESS_BY_DEPTH) || few_us <= tiles_us) return launch_few<kE4M3, OUT>(p, stream);
    if (p.source) return launch_shape<true, OUT>(p, rows, groups, stream);
    return launch_shape<false, OUT>(p, rows, groups, stream);
}

}  // namespace

bool rounds_inside(int64_t M, int64_t K, int by)
{
    return by != MADDNESS_BY_DEPTH && M <= kInsideRows && K >= 8 && M * round_up(K, (int64_t)kBlock) <= kInside;
}

int launch_block_product(const ProductArgs &p, int a_dtype, int out_dtype, hipStream_t stream)
{
    if (out_dtype == MADDNESS_F32) return launch_to<kF32>(p, a_dtype, stream);
    if (out_dtype == MADDNESS_F16) return launch_to<kF16>(p, a_dtype, stream);
    return launch_to<kBF16>(p, a_dtype, stream);
}

}  // namespace maddness

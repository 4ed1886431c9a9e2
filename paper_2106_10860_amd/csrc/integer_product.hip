// out[m][n] = A.scale[m] B.scale[n] sum_k A[m][k] B[n][k] + bias[n] of two matrices of 8-bit integers, on the integer matrix cores.
//
// The instruction (v_mfma_i32_16x16x64_i8) adds exactly in 32 bits, so results depend on no split of the sum; the scales come in once, at the end.
// B's rows (the columns of out) are its first operand and A's rows its second, so that a lane's four results are four neighbours in a row of out.
// Lane l holds 16 values of row l % 16 of an operand (which 16 of the 64 does not matter as long as they are the same ones of both operands), and results
// n = 4 (l / 16) + i of row m = l % 16.
#include "layers_common.h"
#include "tile_loads.h"

namespace maddness {
namespace {

// A lane's 32 bytes of a row's 128, at group * 32.
struct Piece {
    i32x4 lo, hi;
};

// Reads them, 16 bytes that begin at or beyond column K from the row's last 16 that do not: in bounds, and cut off of one operand.
__device__ __forceinline__ Piece load_piece(const int8_t *row, int64_t kb, int group, int64_t K)
{
    const int64_t k = kb * kBlock + group * 32, last = (K - 1) & ~(int64_t)15;
    return Piece{*reinterpret_cast<const i32x4 *>(row + min(k, last)), *reinterpret_cast<const i32x4 *>(row + min(k + 16, last))};
}

__device__ __forceinline__ i32x4 multiply(i32x4 b, i32x4 a, i32x4 c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(b, a, c, 0, 0, 0); }

// A result: every step rounded on its own, so that all kernels give the same.
__device__ __forceinline__ float scaled(int32_t sum, float scale_a, float scale_b, const float *bias, int64_t n)
{
#pragma clang fp contract(off)
    const float v = (float)sum * scale_a * scale_b;
    return bias ? v + bias[n] : v;
}

// Whether A's rows are rounded within the few-rows kernel, by every workgroup for its own 32 at most: while they fill 16 KiB of LDS, which costs 1 us (one row of
// 4096) to 3.7 (16 of 1024); a launch of its own costs 3.9 (8 rows of 4096: 6.5 within the kernel).
constexpr int64_t kInside = 16384, kInsideRows = 32, kMostInside = 64;

// Few rows: 16 MT rows by 16 NT columns to a workgroup; its wavefronts take every WAVES-th block of 128 of the sum, up to DEPTH of them asked for
// at once, and add up in LDS.  B comes straight from memory, in pieces of 32 bytes to a lane, and so does an 8-bit A; a floating A is rounded into
// LDS while the first of B is on its way.  (One row through 4096 x 4096, other matrices from call to call: 6.2 us with four blocks at once, 6.7 with one.)
template <int AT, int MT, int NT, int WAVES, int DEPTH, int OUT>
__global__ __launch_bounds__(WAVES * 64) void integer_few_kernel(IntegerArgs p, uint32_t col_tiles)
{
    constexpr bool ROUND = AT != kI8;
    __shared__ i32x4 sums[WAVES][MT * NT][64];
    __shared__ __attribute__((aligned(16))) int8_t rounded[ROUND ? kInside + kInsideRows * 16 : 16];
    __shared__ uint32_t tops[MT * 16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, r16 = lane % 16, g = lane / 16;
    const int64_t n0 = (int64_t)(blockIdx.x % col_tiles) * (16 * NT), first = (int64_t)(blockIdx.x / col_tiles) * (16 * MT), last = min(first + 16 * MT, p.M);
    const int64_t blocks = ceil_div(p.K, (int64_t)kBlock);
    const int8_t *row_b[NT], *row_a[MT];
#pragma unroll
    for (int t = 0; t < NT; ++t) row_b[t] = p.b + min(n0 + t * 16 + r16, p.N - 1) * p.ldb;
    Piece b[DEPTH][NT];
    auto load = [&](int64_t kb0) INLINE_LAMBDA {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            if (kb0 + d * WAVES >= blocks) break;
#pragma unroll
            for (int t = 0; t < NT; ++t) b[d][t] = load_piece(row_b[t], kb0 + d * WAVES, g, p.K);
        }
    };

    const int stride = (int)blocks * kBlock + 16;
    if constexpr (ROUND) {
        // Sixteen lanes to 128 values of a row.  All of A is asked for at once, before B, which then comes while A is rounded.
        constexpr int ONCE = kInside / kBlock / (WAVES * 4);          // turns of the workgroup, of which few rows need few
        const int units = (int)((last - first) * blocks);
        auto read = [&](int unit, int &row, int &k) INLINE_LAMBDA {
            row = unit / (int)blocks;
            k = unit % (int)blocks * kBlock + r16 * 8;
            return load_raw<AT>(p.a, (first + row) * p.lda, k, p.K);
        };
        Raw<AT> kept[ONCE];
        int rows[ONCE], ks[ONCE];
#pragma unroll
        for (int u = 0; u < ONCE; ++u)
            if (u * WAVES * 4 < units) kept[u] = read(min((int)threadIdx.x / 16 + u * WAVES * 4, units - 1), rows[u], ks[u]);
        if ((int)threadIdx.x < MT * 16) tops[threadIdx.x] = 0;
        if (wave < blocks) load(wave);
        __syncthreads();
        auto largest = [&](const Raw<AT> &raw, int row) INLINE_LAMBDA {
            float v[8];
            widen<AT>(raw, v);
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);      // (those of a neighbour's piece do no harm)
            top = row16_max(top);
            if (r16 == 0) atomicMax(&tops[row], top);
        };
        auto round = [&](const Raw<AT> &raw, int row, int k) INLINE_LAMBDA {
            const float s = integer_scale(tops[row]), inv = 1.0f / s;
            float v[8];
            widen<AT>(raw, v);
            *reinterpret_cast<uint2 *>(rounded + row * stride + k) = in_place(pack8_integers(v, s, inv), before_column(k, p.K));
        };
#pragma unroll
        for (int u = 0; u < ONCE; ++u)
            if (u * WAVES * 4 < units && (int)threadIdx.x / 16 + u * WAVES * 4 < units) largest(kept[u], rows[u]);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < ONCE; ++u)
            if (u * WAVES * 4 < units && (int)threadIdx.x / 16 + u * WAVES * 4 < units) round(kept[u], rows[u], ks[u]);
        __syncthreads();
    } else {
        if (wave < blocks) load(wave);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t m = min(t * 16 + r16, (int)(last - first) - 1);
        row_a[t] = ROUND ? rounded + m * stride : static_cast<const int8_t *>(p.a) + (first + m) * p.lda;
    }
    i32x4 acc[MT][NT] = {};
    for (int64_t kb0 = wave; kb0 < blocks; kb0 += DEPTH * WAVES) {
        if (kb0 != wave) load(kb0);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int64_t kb = kb0 + d * WAVES;
            if (kb >= blocks) break;
            Piece a[MT];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                if constexpr (ROUND) {
                    a[t].lo = *reinterpret_cast<const i32x4 *>(row_a[t] + kb * kBlock + g * 32);
                    a[t].hi = *reinterpret_cast<const i32x4 *>(row_a[t] + kb * kBlock + g * 32 + 16);
                } else {
                    a[t] = load_piece(row_a[t], kb, g, p.K);
                }
            }
            if (!ROUND && (kb + 1) * kBlock > p.K) {          // (rounded rows end in zeros)
                const int64_t k = kb * kBlock + g * 32;
#pragma unroll
                for (int t = 0; t < MT; ++t) a[t] = Piece{first_bytes(a[t].lo, p.K - k), first_bytes(a[t].hi, p.K - k - 16)};
            }
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = multiply(b[d][j].lo, a[i].lo, acc[i][j]);
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = multiply(b[d][j].hi, a[i].hi, acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < MT * NT * 256; o += WAVES * 64) {
        const int m = o / (16 * NT), n = o % (16 * NT);
        if (first + m >= last || n0 + n >= p.N) continue;
        const int tile = m / 16 * NT + n / 16, at = m % 16 + n % 16 / 4 * 16;
        int32_t s = 0;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) s += sums[k][tile][at][n % 4];
        const float scale_a = ROUND ? integer_scale(tops[m]) : p.K ? p.scale_a[first + m] : 1.0f;
        store_as<OUT>(p.out, (first + m) * p.ldo + n0 + n, scaled(s, scale_a, p.scale_b[n0 + n], p.bias, n0 + n));
    }
}

// 16 bytes of results from LDS to row m of out, from column n on, as far as they are there.
template <int OUT>
__device__ __forceinline__ void store_line(const uint8_t *from, const IntegerArgs &p, int64_t m, int64_t n)
{
    constexpr int RUN = 16 / elem_size(OUT);
    const i32x4 run = *reinterpret_cast<const i32x4 *>(from);
    if (m >= p.M) return;
    const int64_t to = m * p.ldo + n;
    if (n + RUN <= p.N) {
        struct __attribute__((packed, aligned(elem_size(OUT)))) Words { i32x4 w; };
        reinterpret_cast<Words *>(static_cast<char *>(p.out) + to * elem_size(OUT))->w = run;
    } else {
#pragma unroll
        for (int k = 0; k < RUN - 1; ++k)
            if (n + k < p.N) {
                if constexpr (OUT == kF32) static_cast<int32_t *>(p.out)[to + k] = run[k];
                else static_cast<uint16_t *>(p.out)[to + k] = (uint16_t)((uint32_t)run[k / 2] >> (k % 2 * 16));
            }
    }
}

// Many rows: BM x BN results to a workgroup of WM x WN wavefronts, each with (BM / WM) x (BN / WN) of them in registers.  Blocks of 128 values
// of the BM + BN rows go to LDS without passing registers: whole lines of memory, as the way from L2 takes one at a time (of half lines it brings half the bytes).  There two blocks
// of A and three of B have a place, and a block is multiplied in two halves: the fragments of one are read while those of the other are multiplied.  So the wavefronts meet
// once in a block, when the last of it is in registers and the next has come; then A's place is free for the block after that one.
//
// A row's eight pieces of 16 bytes lie exchanged by its index, so that the rows that a read of the lanes goes to fall on all banks.
//
// 8192 x 4096 x 4096 119 us, 2300 TOP/s (the library's product of the same matrices 132, with neither scales nor bfloat16).  Of that some 14 us go to the two turns' first
// blocks and results; a block of 256 x 256 takes 1.36 us, 0.85 of them the matrix cores' at full clocks: with zeros in place of the values a block takes 0.97, so what bounds
// it now is power.
template <int BM, int BN, int WM, int WN, int OUT>
__global__ __launch_bounds__(WM * WN * 64, 2) void integer_tiles_kernel(IntegerArgs p, uint32_t col_tiles)
{
    constexpr int WAVES = WM * WN, MT = BM / WM / 16, NT = BN / WN / 16, LOADS_A = BM / 8 / WAVES, LOADS_B = BN / 8 / WAVES;
    constexpr uint32_t PLACE_A = BM * kBlock, PLACE_B = BN * kBlock;
    static_assert(WAVES % 2 == 0 && LOADS_A * 8 * WAVES == BM && LOADS_B * 8 * WAVES == BN, "a wavefront loads whole groups of 8 rows, all at even or all at odd places");
    static_assert(MT >= LOADS_A && MT >= LOADS_B, "a load to each row of products at most");
    __shared__ __attribute__((aligned(128))) uint8_t tile[2 * PLACE_A + 3 * PLACE_B];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r16 = lane % 16, g = lane / 16;

    // four pieces by all columns, then the next four: what a die works on at a time shares rows of both operands
    const uint32_t pieces = (uint32_t)ceil_div(p.M, (int64_t)BM), at = by_die(blockIdx.x, pieces * col_tiles);
    const uint32_t band = at / (4 * col_tiles), in_band = at % (4 * col_tiles), height = min(4u, pieces - band * 4);
    const int64_t n0 = (int64_t)(in_band / height) * BN, m0 = (int64_t)(band * 4 + in_band % height) * BM;

    // Rows are addressed by 32-bit offsets within the tile (the launcher keeps row strides to kMostStride, so these are below 2^31).  What lies beyond the tile's last
    // row, and beyond the last block, is out of the buffers' range; what lies beyond column K is cut off from A's fragments.
    const uint32_t lda = (uint32_t)p.lda, ldb = (uint32_t)p.ldb, blocks = (uint32_t)ceil_div(p.K, (int64_t)kBlock);
    const uint32_t rows = (uint32_t)min((int64_t)BM, p.M - m0), cols = (uint32_t)min((int64_t)BN, p.N - n0), width = round_up((uint32_t)p.K, 16u);
    const i32x4 mem_a = buffer_of(static_cast<const uint8_t *>(p.a) + m0 * p.lda, (rows - 1) * lda + width);
    const i32x4 mem_b = buffer_of(reinterpret_cast<const uint8_t *>(p.b) + n0 * p.ldb, (cols - 1) * ldb + width);
    const uint32_t chunk = (uint32_t)((lane % 8) ^ (lane / 8)) * 16, row0 = wave * 8 + lane / 8;
    const uint32_t at_a = row0 * lda + chunk, at_b = row0 * ldb + chunk;
    // (keeps the compiler from holding every sum of this and a multiple of a stride in a register of its own)
    auto again = [](uint32_t x) INLINE_LAMBDA { asm volatile("" : "+v"(x)); return x; };
    const uint32_t tile_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)tile + wave * 1024;
    auto column = [&](uint32_t kb) INLINE_LAMBDA { return kb < blocks ? kb * kBlock : 0x80000000u; };
    auto load_a = [&](int i, uint32_t place, uint32_t kb) INLINE_LAMBDA {
        load_to_lds(mem_a, again(at_a) + ((i * WAVES * 8) * lda + column(kb)), tile_at + place + i * WAVES * 1024);
    };
    auto load_b = [&](int i, uint32_t place, uint32_t kb) INLINE_LAMBDA {
        load_to_lds(mem_b, again(at_b) + ((i * WAVES * 8) * ldb + column(kb)), tile_at + 2 * PLACE_A + place + i * WAVES * 1024);
    };
    const int wm = wave / WN, wn = wave % WN, tail = (int)(p.K % kBlock);
    const uint32_t from = r16 * kBlock + ((g ^ (r16 % 8)) * 16), from_a = from + wm * MT * 16 * kBlock, from_b = from + 2 * PLACE_A + wn * NT * 16 * kBlock;
    i32x4 acc[MT][NT] = {};
    struct Fragments {
        i32x4 a[MT], b[NT];
    } first, second;
    // The r-th of a half's fragments, B's first; the halves of a row's pieces differ in one bit of their place.
    auto read_one = [&](int r, int half, uint32_t place_a, uint32_t place_b, Fragments &f) INLINE_LAMBDA {
        if (r < NT) f.b[r] = *reinterpret_cast<const i32x4 *>(tile + place_b + (from_b ^ (half * 64)) + r * 16 * kBlock);
        else f.a[r - NT] = *reinterpret_cast<const i32x4 *>(tile + place_a + (from_a ^ (half * 64)) + (r - NT) * 16 * kBlock);
    };
    auto cut = [&](Fragments &f, int keep) INLINE_LAMBDA {
        i32x4 mask;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int bytes = min(max(keep - g * 16 - k * 4, 0), 4);
            mask[k] = bytes == 4 ? -1 : (int)((1u << (8 * bytes)) - 1);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) f.a[i] &= mask;
    };
    auto multiply_and = [&](const Fragments &f, auto beside) INLINE_LAMBDA {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            beside(i);
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = multiply(f.b[j], f.a[i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (blocks) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int i = 0; i < LOADS_A; ++i) load_a(i, s * PLACE_A, s);
#pragma unroll
            for (int i = 0; i < LOADS_B; ++i) load_b(i, s * PLACE_B, s);
        }
        wait_for_loads_but<LOADS_A + LOADS_B>();
        meet();
#pragma unroll
        for (int r = 0; r < MT + NT; ++r) read_one(r, 0, 0, 0, first);
        uint32_t place_a = 0, place_b = 0, far_b = 2 * PLACE_B;           // of this block, and of B's block after the next
        for (uint32_t kb = 0; kb < blocks; ++kb) {
            const bool last = kb + 1 == blocks && tail;
            if (last) cut(first, tail);
            multiply_and(first, [&](int i) INLINE_LAMBDA {
#pragma unroll
                for (int r = i * (MT + NT) / MT; r < (i + 1) * (MT + NT) / MT; ++r) read_one(r, 1, place_a, place_b, second);
                if (i < LOADS_B) load_b(i, far_b, kb + 2);
            });
            wait_for_loads_but<LOADS_B>();
            meet();
            if (last) cut(second, tail - 64);
            const uint32_t free_a = place_a;
            place_a ^= PLACE_A;
            far_b = place_b;
            place_b = place_b == 2 * PLACE_B ? 0 : place_b + PLACE_B;
            multiply_and(second, [&](int i) INLINE_LAMBDA {
#pragma unroll
                for (int r = i * (MT + NT) / MT; r < (i + 1) * (MT + NT) / MT; ++r) read_one(r, 0, place_a, place_b, first);
                if (i < LOADS_A) load_a(i, free_a, kb + 2);
            });
        }
        wait_for_loads();                                    // (its place in LDS is another's from here on)
        meet();
    }
    // A wavefront's results go through its part of LDS, half of its rows at a time, so that they are stored in whole lines: lanes hold four neighbours
    // of sixteen rows each, pieces of 8 or 16 bytes (8192 x 4096 x 128 to bfloat16: 34 us with those, 29 in lines).
    constexpr int ROWS = MT * 8, COLS = NT * 16, RUN = 16 / elem_size(OUT), LINE = COLS * elem_size(OUT) + 16;
    static_assert(ROWS * LINE * WAVES <= (int)sizeof(tile), "the wavefronts' results fit LDS");
    uint8_t *const mine = tile + wave * ROWS * LINE;
    const int64_t col0 = n0 + wn * COLS + lane % (COLS / RUN) * RUN;
    float scale_b[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) scale_b[j][k] = p.scale_b[min(n0 + (wn * NT + j) * 16 + 4 * g + k, p.N - 1)];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int64_t row0 = m0 + wm * MT * 16 + half * ROWS;
#pragma unroll
        for (int i = 0; i < MT / 2; ++i) {
            const float scale_a = p.scale_a[min(row0 + i * 16 + r16, p.M - 1)];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const i32x4 sum = acc[half * (MT / 2) + i][j];
                float four[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) four[k] = scaled(sum[k], scale_a, scale_b[j][k], p.bias, min(n0 + (wn * NT + j) * 16 + 4 * g + k, p.N - 1));
                store_run<OUT>(mine + (i * 16 + r16) * LINE, j * 16 + 4 * g, four);
            }
        }
        wave_lds_fence();
#pragma unroll
        for (int q = 0; q < ROWS * COLS / RUN / 64; ++q) {
            const int row = q * (64 * RUN / COLS) + lane / (COLS / RUN);
            store_line<OUT>(mine + row * LINE + lane % (COLS / RUN) * 16, p, row0 + row, col0);
        }
        wave_lds_fence();
    }
}

template <int BM, int BN, int WM, int WN, int OUT>
int launch_tiles(const IntegerArgs &p, hipStream_t stream)
{
    const int64_t col_tiles = ceil_div(p.N, (int64_t)BN), pieces = ceil_div(p.M, (int64_t)BM);
    if (col_tiles * pieces * WM * WN * 64 > kMostThreads) return fail(MADDNESS_E_UNSUPPORTED, "integer product: %lld x %lld results are too many", (long long)p.M, (long long)p.N);
    note_kernel("integer_tiles_kernel", __PRETTY_FUNCTION__);
    hipLaunchKernelGGL((integer_tiles_kernel<BM, BN, WM, WN, OUT>), dim3((unsigned)(col_tiles * pieces)), dim3(WM * WN * 64), 0, stream, p, (uint32_t)col_tiles);
    return check_hip(hipGetLastError(), "launch integer_tiles_kernel");
}

template <int AT, int OUT, int MT, int NT, int DEPTH>
int launch_few_as(const IntegerArgs &p, hipStream_t stream)
{
    constexpr int WAVES = 8;
    const int64_t col_tiles = ceil_div(p.N, (int64_t)(16 * NT)), pieces = ceil_div(p.M, (int64_t)(16 * MT));
    if (col_tiles * pieces * WAVES * 64 > kMostThreads) return fail(MADDNESS_E_UNSUPPORTED, "integer product: %lld x %lld results are too many", (long long)p.M, (long long)p.N);
    note_kernel("integer_few_kernel", __PRETTY_FUNCTION__);
    hipLaunchKernelGGL((integer_few_kernel<AT, MT, NT, WAVES, DEPTH, OUT>), dim3((unsigned)(col_tiles * pieces)), dim3(WAVES * 64), 0, stream, p, (uint32_t)col_tiles);
    return check_hip(hipGetLastError(), "launch integer_few_kernel");
}

int64_t tiles_of(const IntegerArgs &p, int64_t rows, int64_t cols) { return ceil_div(p.M, rows) * ceil_div(p.N, cols); }

// The smallest pieces that one workgroup to a compute unit is enough for: 32 x 4096 x 4096 by 16 x 16, 32 x 16 and 32 x 32 results 9.5, 8.1 and 10.0 us, 32 x 1024 x 4096 5.7, 7.4 and
// 9.7, 64 x 4096 x 4096 16.6, 13.0 and 10.1.
template <int AT, int OUT>
int launch_few(const IntegerArgs &p, hipStream_t stream)
{
    const int64_t cus = device_info().cus;
    if (tiles_of(p, 16, 16) <= cus || p.M <= 16) return launch_few_as<AT, OUT, 1, 1, 4>(p, stream);
    if (tiles_of(p, 32, 16) <= cus) return launch_few_as<AT, OUT, 2, 1, 4>(p, stream);
    return launch_few_as<AT, OUT, 2, 2, 2>(p, stream);
}

template <int OUT>
int launch_to(const IntegerArgs &p, int a_dtype, hipStream_t stream)
{
    if (a_dtype == MADDNESS_F32) return launch_few<kF32, OUT>(p, stream);
    if (a_dtype == MADDNESS_F16) return launch_few<kF16, OUT>(p, stream);
    if (a_dtype == MADDNESS_BF16) return launch_few<kBF16, OUT>(p, stream);
    const int64_t cus = device_info().cus;
    const bool far = std::max(p.lda, p.ldb) > kMostStride;
    if (far || p.K == 0 || p.M <= 16 || tiles_of(p, 32, 32) <= cus) return launch_few<kI8, OUT>(p, stream);
    // Larger tiles have less to read for each product, but need enough of them for every compute unit, and depth for their beginning and end.  By 64 x 128, 128 x 128, 128 x 256
    // and 256 x 256 results 512 x 4096 x 4096 takes 17.0, 19.6, - and 41.6 us, 2048 x 4096 x 4096 45.9, 36.0, 33.0 and 49.2, 4096 x 4096 x 4096 94, 68, - and 64,
    // 8192 x 4096 x 4096 - , 130, 125 and 118; 1024 x 4096 x 4096 24.0, 23.0, 26.2 and 43.5, 1024 x 4096 x 512 7.0, 7.5, - and 14.0, 1024 x 4096 x 1024 13.3, 9.2, - and 17.9, 4096 x 2048 x 1024 - , 14.2, 13.7 and 20.7,
    // 32768 x 1024 x 512 - , 32.3, 34.5 and 37.5.  (128 x 128 results by four wavefronts, two workgroups to a compute unit, take as long to read their fragments from LDS as to multiply them.)
    if (tiles_of(p, 64, 128) <= (p.K <= 512 ? 2 : 1) * cus) return launch_tiles<64, 128, 1, 4, OUT>(p, stream);
    if (p.K >= 1024 && tiles_of(p, 256, 256) * 4 >= 3 * cus) return launch_tiles<256, 256, 2, 4, OUT>(p, stream);
    if (p.K >= 1024 && tiles_of(p, 128, 256) <= cus && tiles_of(p, 128, 128) > cus) return launch_tiles<128, 256, 2, 4, OUT>(p, stream);
    return launch_tiles<128, 128, 2, 2, OUT>(p, stream);
}

}  // namespace

bool integer_rounds_inside(int64_t M, int64_t K)
{
    return M <= kMostInside && K >= 8 && std::min(M, kInsideRows) * round_up(K, (int64_t)kBlock) <= kInside;
}

int launch_integer_product(const IntegerArgs &p, int a_dtype, int out_dtype, hipStream_t stream)
{
    if (out_dtype == MADDNESS_F32) return launch_to<kF32>(p, a_dtype, stream);
    if (out_dtype == MADDNESS_F16) return launch_to<kF16>(p, a_dtype, stream);
    return launch_to<kBF16>(p, a_dtype, stream);
}

}  // namespace maddness

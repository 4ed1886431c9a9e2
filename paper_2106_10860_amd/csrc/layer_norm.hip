// Rows that stay in registers from their load to their store: to 8-bit integers, through a layer norm, and back through its gradient.
//
//   mu = mean(x), v = mean((x - mu)^2), r = 1 / sqrt(v + eps), h = (x - mu) r, y = h weight + bias
//   u = g weight, dx = r (u - mean(u) - h mean(u h)), dweight = sum over rows of g h, dbias = sum over rows of g
//
// All of it moves bytes: a row is read once, its sums go around the lanes that hold it (a wavefront for up to 1024 elements, else as many of a workgroup as
// have it in pieces of 8 and 16 bytes or more), and it is written once.  What the norm's parameters need of the lanes stays in their registers, so a workgroup takes rows in turn, and
// asks for the next one before it works on this one.  32768 rows of 4096 bfloat16: forward 96 us (5.6 TB/s of what is read and written, the copy of 1 GiB 5.0), gradient 155 (5.2).
#include "lanes.h"
#include "layers_common.h"

namespace maddness {
namespace {

constexpr int64_t kLongestRow = 16 * 64 * 2 * 8;       // that a workgroup holds: 16 wavefronts with 2 pieces of 8 to a lane, or 8 with 4
constexpr auto larger_bits = [](uint32_t a, uint32_t b) INLINE_LAMBDA { return max(a, b); };

// A value over the WAVES wavefronts that share a row, in all their lanes, added in the wavefronts' order.  Calls of a kernel take turns with two
// arrays in LDS: who writes to one again has met the others at the call between.
template <int WAVES, typename T, typename F>
__device__ __forceinline__ T over_row(T x, T (&slots)[WAVES], F f)
{
    x = over_lanes<64>(x, f);
    if constexpr (WAVES > 1) {
        if (threadIdx.x % 64 == 0) slots[threadIdx.x / 64] = x;
        __syncthreads();
        x = slots[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) x = f(x, slots[w]);
    }
    return x;
}

__device__ __forceinline__ float fused(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ __forceinline__ double fused(double a, double b, double c) { return __builtin_fma(a, b, c); }

// Which of a row's n elements (n >= 8) a lane holds as its piece: the eight from column `at` on, of which the first `skip` are its neighbour's too.
struct Place {
    int at, skip;
};

template <int WAVES>
__device__ __forceinline__ Place place_of(int piece, int n)
{
    const int c = (piece * WAVES * 64 + (WAVES == 1 ? threadIdx.x % 64 : threadIdx.x)) * 8;
    return Place{min(c, n - 8), min(max(c - (n - 8), 0), 8)};
}

// Eight parameters of either type, or `otherwise` where there are none.
__device__ __forceinline__ void load_parameters(const void *p, int dtype, int at, int n, float otherwise, float (&v)[8])
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = otherwise;
    } else if (dtype == kF32) {
        widen<kF32>(load_raw<kF32>(p, 0, at, n), v);
    } else if (dtype == kF16) {
        widen<kF16>(load_raw<kF16>(p, 0, at, n), v);
    } else {
        widen<kBF16>(load_raw<kBF16>(p, 0, at, n), v);
    }
}

constexpr int rows_at_once(int waves) { return waves == 1 ? 4 : 1; }      // rows to a workgroup
constexpr int threads_of(int waves) { return waves == 1 ? 256 : waves * 64; }

// Whether a piece, and element i of it, are counted here and not by a neighbour.  WHOLE: rows are whole pieces, of which all or none is.
template <bool WHOLE>
__device__ __forceinline__ bool counts(const Place &p) { return !WHOLE || p.skip == 0; }
template <bool WHOLE>
__device__ __forceinline__ bool counts(const Place &p, int i) { return WHOLE || i >= p.skip; }

// 1 / sqrt(x) to a step of fp32 (the instruction takes numbers below 2^-126 for 0).
__device__ __forceinline__ float inverse_root(float x) { return x < 1e-30f ? 1.0f / sqrtf(x) : __builtin_amdgcn_rsqf(x); }

// NORM: normalised; else as they are (to integers).  8192 rows of 4096 bfloat16 through a norm to integers 24 us, 4.2 TB/s: the vector units are
// busy for 60 % of it.  Rows of 8 to WAVES * PER * 512 elements.
template <int XT, int OT, bool NORM, int WAVES, int PER, bool WHOLE>
__global__ __launch_bounds__(threads_of(WAVES)) void rows_kernel(RowsArgs a)
{
    __shared__ float sums[2][WAVES];
    __shared__ uint32_t tops[WAVES];
    const int n = (int)a.n;
    const float each = 1.0f / (float)n;
    const int64_t first = (int64_t)blockIdx.x * rows_at_once(WAVES) + (WAVES == 1 ? threadIdx.x / 64 : 0), step = (int64_t)gridDim.x * rows_at_once(WAVES);
    Place place[PER];
    float weight[NORM ? PER : 1][8], bias[NORM ? PER : 1][8];
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        place[p] = place_of<WAVES>(p, n);
        if constexpr (NORM) {
            load_parameters(a.weight, a.parameter_dtype, place[p].at, n, 1.0f, weight[p]);
            load_parameters(a.bias, a.parameter_dtype, place[p].at, n, 0.0f, bias[p]);
        }
    }
    Raw<XT> raw[PER];
    auto load = [&](int64_t row) INLINE_LAMBDA {
#pragma unroll
        for (int p = 0; p < PER; ++p) raw[p] = load_raw<XT>(a.x, row * a.ldx, place[p].at, n);
    };
    if (first < a.rows) load(first);
    for (int64_t row = first; row < a.rows; row += step) {
        float v[PER][8];
#pragma unroll
        for (int p = 0; p < PER; ++p) widen<XT>(raw[p], v[p]);
        if (row + step < a.rows) load(row + step);
        if constexpr (NORM) {
            float sum = 0.0f;
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                if (!counts<WHOLE>(place[p])) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += counts<WHOLE>(place[p], i) ? v[p][i] : 0.0f;
            }
            const float mean = over_row<WAVES>(sum, sums[0], plus) / (float)n;      // (a rounded 1 / n would leave a row of one number uncentred)
            float squares = 0.0f;
#pragma unroll
            for (int p = 0; p < PER; ++p) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[p][i] -= mean;
                if (!counts<WHOLE>(place[p])) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) squares = counts<WHOLE>(place[p], i) ? __builtin_fmaf(v[p][i], v[p][i], squares) : squares;
            }
            const float rstd = inverse_root(over_row<WAVES>(squares, sums[1], plus) * each + a.eps);
            if (a.mean && threadIdx.x % (WAVES * 64) == 0) {
                a.mean[row] = mean;
                a.rstd[row] = rstd;
            }
#pragma unroll
            for (int p = 0; p < PER; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[p][i] = __builtin_fmaf(v[p][i] * rstd, weight[p][i], bias[p][i]);      // (written out, so that all of this kernel's forms round alike)
        }
        if constexpr (OT == kI8) {
            uint32_t top = 0;
#pragma unroll
            for (int p = 0; p < PER; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[p][i]) & 0x7fffffffu);   // (a neighbour's do no harm)
            top = over_row<WAVES>(top, tops, larger_bits);
            if constexpr (WAVES > 1 && !NORM) __syncthreads();                                          // (one array, and no other call between)
            const float s = integer_scale(top), inv = 1.0f / s;
            if (threadIdx.x % (WAVES * 64) == 0) a.scale[row] = s;
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                const int c = place[p].at + place[p].skip;       // (a column of the row, or the first behind it)
                const int own = (p * WAVES * 64 + (WAVES == 1 ? threadIdx.x % 64 : threadIdx.x)) * 8;
                if (own >= round_up(n, 16)) continue;
                const uint2 q = c == own ? in_place(pack8_integers(v[p], s, inv), place[p].skip) : make_uint2(0, 0);
                *reinterpret_cast<uint2 *>(static_cast<int8_t *>(a.out) + row * a.ldo + own) = q;
            }
        } else {
#pragma unroll
            for (int p = 0; p < PER; ++p)
                if (place[p].skip < 8) store_run<OT>(a.out, row * a.ldo + place[p].at, v[p]);
        }
    }
}

// Rows of any length, a workgroup to each, read again for every sum.  A thread adds every 1024th element, one after the other: for long rows in fp64 (SUM), as there is no end to how
// many (4096 rows of 20000 223 us, 214 in fp32; 512 of 300000 562 and 552); the one element that a thread has of a row below 8 needs none of it (2^19 rows of 7 1.55 ms, 2.31 with
// fp64 between the lanes).
template <int XT, int OT, bool NORM, typename SUM>
__global__ __launch_bounds__(1024) void rows_any_kernel(RowsArgs a)
{
    __shared__ SUM sums[2][16];
    __shared__ uint32_t tops[16];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int64_t from = row * a.ldx;
        float mean = 0.0f, rstd = 1.0f;
        if constexpr (NORM) {
            SUM sum = 0, squares = 0;
            for (int64_t c = threadIdx.x; c < a.n; c += 1024) sum += (SUM)widen_at<XT>(a.x, from + c);
            mean = (float)(over_row<16>(sum, sums[0], plus) / (SUM)a.n);
            for (int64_t c = threadIdx.x; c < a.n; c += 1024) {
                const SUM d = (SUM)(widen_at<XT>(a.x, from + c) - mean);
                squares = fused(d, d, squares);
            }
            rstd = 1.0f / sqrtf((float)(over_row<16>(squares, sums[1], plus) / (SUM)a.n) + a.eps);
            if (a.mean && threadIdx.x == 0) {
                a.mean[row] = mean;
                a.rstd[row] = rstd;
            }
        }
        auto value = [&](int64_t c) INLINE_LAMBDA {
            const float x = widen_at<XT>(a.x, from + c);
            if constexpr (!NORM) return x;
            return __builtin_fmaf((x - mean) * rstd, a.weight ? widen_at(a.weight, a.parameter_dtype, c) : 1.0f, a.bias ? widen_at(a.bias, a.parameter_dtype, c) : 0.0f);
        };
        if constexpr (OT == kI8) {
            uint32_t top = 0;
            for (int64_t c = threadIdx.x; c < a.n; c += 1024) top = max(top, __float_as_uint(value(c)) & 0x7fffffffu);
            top = over_row<16>(top, tops, larger_bits);
            __syncthreads();
            const float s = integer_scale(top), inv = 1.0f / s;
            if (threadIdx.x == 0) a.scale[row] = s;
            int8_t *out = static_cast<int8_t *>(a.out) + row * a.ldo;
            for (int64_t c = threadIdx.x; c < round_up(a.n, (int64_t)16); c += 1024) out[c] = c < a.n && s == s ? (int8_t)nearest_integer(value(c), s, inv) : (int8_t)0;
        } else {
            for (int64_t c = threadIdx.x; c < a.n; c += 1024) store_as<OT>(a.out, row * a.ldo + c, value(c));
            if constexpr (!NORM) __syncthreads();
        }
    }
}

template <int XT, int OT, bool NORM, int WAVES, int PER>
int launch_rows_as(const RowsArgs &a, hipStream_t stream)
{
    const bool whole = NORM && a.n % 8 == 0;
    const int64_t groups = ceil_div(a.rows, (int64_t)rows_at_once(WAVES)), most = (int64_t)device_info().cus * (WAVES == 1 ? 8 : 32 / WAVES);
    note_kernel("rows_kernel", __PRETTY_FUNCTION__);
    const dim3 grid((unsigned)std::min(groups, most)), block(threads_of(WAVES));
    if (whole) hipLaunchKernelGGL((rows_kernel<XT, OT, NORM, WAVES, PER, NORM>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((rows_kernel<XT, OT, NORM, WAVES, PER, false>), grid, block, 0, stream, a);
    return check_hip(hipGetLastError(), "launch rows_kernel");
}

template <int XT, int OT, bool NORM>
int launch_rows(const RowsArgs &a, hipStream_t stream)
{
    if (a.n < 8 || a.n > kLongestRow) {
        note_kernel("rows_any_kernel", __PRETTY_FUNCTION__);
        const dim3 grid((unsigned)std::min(a.rows, (int64_t)device_info().cus * 2));
        if (NORM && a.n >= 8) hipLaunchKernelGGL((rows_any_kernel<XT, OT, NORM, std::conditional_t<NORM, double, float>>), grid, dim3(1024), 0, stream, a);
        else hipLaunchKernelGGL((rows_any_kernel<XT, OT, NORM, float>), grid, dim3(1024), 0, stream, a);
        return check_hip(hipGetLastError(), "launch rows_any_kernel");
    }
    if (a.n <= 512) return launch_rows_as<XT, OT, NORM, 1, 1>(a, stream);
    if (a.n <= 1024) return launch_rows_as<XT, OT, NORM, 1, 2>(a, stream);
    if (a.n <= 2048) return launch_rows_as<XT, OT, NORM, 4, 1>(a, stream);
    if (a.n <= 4096) return launch_rows_as<XT, OT, NORM, 4, 2>(a, stream);
    if (a.n <= 8192) return launch_rows_as<XT, OT, NORM, 8, 2>(a, stream);
    return launch_rows_as<XT, OT, NORM, 16, 2>(a, stream);
}

// --------------------------------------------------------------------------------------------------------------- the gradient

// dx row by row, and of all rows that a workgroup takes the sums of g h and g for its lanes' columns; partial is [2][gridDim.x][n].  Two workgroups to a compute unit at most: more would leave more
// partial sums (of 4096 columns 16.8 MB as it is, 5 us of the 160 that 32768 rows take) and are no faster, as a row ahead keeps memory busy.
template <int GT, int XT, int WAVES, int PER, bool SUMS, bool WHOLE>
__global__ __launch_bounds__(threads_of(WAVES)) void norm_gradient_kernel(NormGradientArgs a)
{
    constexpr int ROWS = rows_at_once(WAVES);
    __shared__ float sums[2][2][WAVES];
    __shared__ float gathered[WAVES == 1 && SUMS ? ROWS : 1][WAVES == 1 && SUMS ? PER * 512 : 1];
    const int n = (int)a.n;
    const float each = 1.0f / (float)n;
    const int64_t first = (int64_t)blockIdx.x * ROWS + (WAVES == 1 ? threadIdx.x / 64 : 0), step = (int64_t)gridDim.x * ROWS;
    Place place[PER];
    float weight[PER][8], dweight[SUMS ? PER : 1][8] = {}, dbias[SUMS ? PER : 1][8] = {};
#pragma unroll
    for (int p = 0; p < PER; ++p) {
        place[p] = place_of<WAVES>(p, n);
        load_parameters(a.weight, a.parameter_dtype, place[p].at, n, 1.0f, weight[p]);
    }
    Raw<XT> raw_x[PER];
    Raw<GT> raw_g[PER];
    float mean = 0.0f, rstd = 0.0f;
    auto load = [&](int64_t row) INLINE_LAMBDA {
        mean = a.mean[row];
        rstd = a.rstd[row];
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            raw_x[p] = load_raw<XT>(a.x, row * a.ldx, place[p].at, n);
            raw_g[p] = load_raw<GT>(a.g, row * a.ldg, place[p].at, n);
        }
    };
    // (4 pieces to a lane leave no registers for the next row beside them)
    constexpr bool AHEAD = PER < 4;
    if (AHEAD && first < a.rows) load(first);
    int turn = 0;
    for (int64_t row = first; row < a.rows; row += step, turn ^= 1) {
        if constexpr (!AHEAD) load(row);
        float h[PER][8], g[PER][8];
        const float r = rstd;
        float su = 0.0f, suh = 0.0f;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
            widen<XT>(raw_x[p], h[p]);
            widen<GT>(raw_g[p], g[p]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[p][i] = (h[p][i] - mean) * r;
                if constexpr (SUMS) {
                    dweight[p][i] = __builtin_fmaf(g[p][i], h[p][i], dweight[p][i]);
                    dbias[p][i] += g[p][i];
                }
                g[p][i] *= weight[p][i];
            }
            if (!counts<WHOLE>(place[p])) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                su += counts<WHOLE>(place[p], i) ? g[p][i] : 0.0f;
                suh = counts<WHOLE>(place[p], i) ? __builtin_fmaf(g[p][i], h[p][i], suh) : suh;
            }
        }
        if (AHEAD && row + step < a.rows) load(row + step);
        if (!a.dx) continue;
        su = over_lanes<64>(su, plus);
        suh = over_lanes<64>(suh, plus);
        if constexpr (WAVES > 1) {
            if (threadIdx.x % 64 == 0) {
                sums[turn][0][threadIdx.x / 64] = su;
                sums[turn][1][threadIdx.x / 64] = suh;
            }
            __syncthreads();
            su = suh = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                su += sums[turn][0][w];
                suh += sums[turn][1][w];
            }
        }
        su /= (float)n;                                       // (as the mean: a gradient of one number is centred to 0)
        suh *= each;
#pragma unroll
        for (int p = 0; p < PER; ++p) {
#pragma unroll
            for (int i = 0; i < 8; ++i) g[p][i] = r * __builtin_fmaf(-h[p][i], suh, g[p][i] - su);
            if (place[p].skip < 8) store_run<XT>(a.dx, row * a.ldd + place[p].at, g[p]);
        }
    }
    if constexpr (SUMS) {
        float *to_weight = a.partial + (int64_t)blockIdx.x * n, *to_bias = to_weight + (int64_t)gridDim.x * n;
        if constexpr (WAVES == 1) {
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                float (&mine)[PER][8] = which ? dbias : dweight;
                __syncthreads();
#pragma unroll
                for (int p = 0; p < PER; ++p)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i >= place[p].skip) gathered[threadIdx.x / 64][place[p].at + i] = mine[p][i];
                __syncthreads();
                for (int c = threadIdx.x; c < n; c += 256) {
                    float s = gathered[0][c];
#pragma unroll
                    for (int w = 1; w < ROWS; ++w) s += gathered[w][c];
                    (which ? to_bias : to_weight)[c] = s;
                }
            }
        } else {
#pragma unroll
            for (int p = 0; p < PER; ++p) {
                if (place[p].skip == 8) continue;
                store_run<kF32>(to_weight, place[p].at, dweight[p]);
                store_run<kF32>(to_bias, place[p].at, dbias[p]);
            }
        }
    }
}

// Rows of any length: dx, read twice; SUM as in rows_any_kernel.
template <int GT, int XT, typename SUM>
__global__ __launch_bounds__(1024) void norm_gradient_any_kernel(NormGradientArgs a)
{
    __shared__ SUM sums[2][16];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float mean = a.mean[row], r = a.rstd[row];
        SUM all_u = 0, all_uh = 0;
        for (int64_t c = threadIdx.x; c < a.n; c += 1024) {
            const float u = widen_at<GT>(a.g, row * a.ldg + c) * (a.weight ? widen_at(a.weight, a.parameter_dtype, c) : 1.0f);
            all_u += (SUM)u;
            all_uh = fused((SUM)u, (SUM)((widen_at<XT>(a.x, row * a.ldx + c) - mean) * r), all_uh);
        }
        const float su = (float)(over_row<16>(all_u, sums[0], plus) / (SUM)a.n), suh = (float)(over_row<16>(all_uh, sums[1], plus) / (SUM)a.n);
        for (int64_t c = threadIdx.x; c < a.n; c += 1024) {
            const float u = widen_at<GT>(a.g, row * a.ldg + c) * (a.weight ? widen_at(a.weight, a.parameter_dtype, c) : 1.0f);
            const float h = (widen_at<XT>(a.x, row * a.ldx + c) - mean) * r;
            store_as<XT>(a.dx, row * a.ldd + c, r * __builtin_fmaf(-h, suh, u - su));
        }
    }
}

// Their sums over the rows that a workgroup takes, a thread to a column: of long rows few workgroups share the rows, so a thread adds many, in fp64.
template <int GT, int XT>
__global__ __launch_bounds__(256) void norm_sums_any_kernel(NormGradientArgs a)
{
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.n) return;
    double dweight = 0.0, dbias = 0.0;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const double g = (double)widen_at<GT>(a.g, row * a.ldg + c);
        dweight = __builtin_fma(g, (double)((widen_at<XT>(a.x, row * a.ldx + c) - a.mean[row]) * a.rstd[row]), dweight);
        dbias += g;
    }
    a.partial[blockIdx.y * a.n + c] = (float)dweight;
    a.partial[(gridDim.y + blockIdx.y) * a.n + c] = (float)dbias;
}

// Sums of `parts` rows of partial sums (none: 0): 32 columns to a workgroup, its 32 runs of 32 lanes take every 32nd row, whole
// lines of them.  blockIdx.y: weight or bias.  (512 rows of 4096 5 us, by 16 columns 7; of 510 3.2, by 64 columns 4.7.)
__global__ __launch_bounds__(1024) void column_sums_kernel(const float *partial, int64_t parts, int64_t n, float *dweight, float *dbias)
{
    __shared__ float sums[16][32];
    const int column = threadIdx.x % 32, run = threadIdx.x / 32;
    const int64_t c = (int64_t)blockIdx.x * 32 + column;
    const float *from = partial + blockIdx.y * parts * n + min(c, n - 1);
    float s = 0.0f;
#pragma unroll 8
    for (int64_t p = run; p < parts; p += 32) s += from[p * n];
    s += from_lane<32>(s);
    if (threadIdx.x % 64 < 32) sums[threadIdx.x / 64][column] = s;
    __syncthreads();
    if (threadIdx.x < 32 && c < n) {
        s = sums[0][column];
#pragma unroll
        for (int w = 1; w < 16; ++w) s += sums[w][column];
        (blockIdx.y ? dbias : dweight)[c] = s;
    }
}

// How the gradient of rows of n is split: wavefronts to a row, workgroups that take rows in turn.
int waves_of(int64_t n) { return n <= 1024 ? 1 : n <= 4096 ? 4 : 8; }

int64_t parts_of(int64_t rows, int64_t n)
{
    const int64_t cus = device_info().cus;
    if (n < 8 || n > kLongestRow) return std::min(ceil_div(rows, (int64_t)16), std::max((int64_t)1, 8 * cus / ceil_div(n, (int64_t)256)));
    const int waves = waves_of(n);
    return std::min(ceil_div(rows, (int64_t)rows_at_once(waves)), cus * (n > 8192 ? 1 : 2));
}

template <int GT, int XT, int WAVES, int PER>
int launch_gradient_as(const NormGradientArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)parts_of(a.rows, a.n)), block(threads_of(WAVES));
    note_kernel("norm_gradient_kernel", __PRETTY_FUNCTION__);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    if (a.n % 8) a.dweight ? launch(norm_gradient_kernel<GT, XT, WAVES, PER, true, false>) : launch(norm_gradient_kernel<GT, XT, WAVES, PER, false, false>);
    else a.dweight ? launch(norm_gradient_kernel<GT, XT, WAVES, PER, true, true>) : launch(norm_gradient_kernel<GT, XT, WAVES, PER, false, true>);
    return check_hip(hipGetLastError(), "launch norm_gradient_kernel");
}

template <int GT, int XT>
int launch_gradient(const NormGradientArgs &a, hipStream_t stream)
{
    if (a.n < 8 || a.n > kLongestRow) {
        if (a.dx) {
            note_kernel("norm_gradient_any_kernel", __PRETTY_FUNCTION__);
            const dim3 grid((unsigned)std::min(a.rows, (int64_t)device_info().cus * 2));
            if (a.n < 8) hipLaunchKernelGGL((norm_gradient_any_kernel<GT, XT, float>), grid, dim3(1024), 0, stream, a);
            else hipLaunchKernelGGL((norm_gradient_any_kernel<GT, XT, double>), grid, dim3(1024), 0, stream, a);
        }
        if (a.dweight) {
            note_kernel("norm_sums_any_kernel", __PRETTY_FUNCTION__);
            hipLaunchKernelGGL((norm_sums_any_kernel<GT, XT>), dim3((unsigned)ceil_div(a.n, (int64_t)256), (unsigned)parts_of(a.rows, a.n)), dim3(256), 0, stream, a);
        }
        return check_hip(hipGetLastError(), "launch norm_gradient_any_kernel");
    }
    if (a.n <= 512) return launch_gradient_as<GT, XT, 1, 1>(a, stream);
    if (a.n <= 1024) return launch_gradient_as<GT, XT, 1, 2>(a, stream);
    if (a.n <= 2048) return launch_gradient_as<GT, XT, 4, 1>(a, stream);
    if (a.n <= 4096) return launch_gradient_as<GT, XT, 4, 2>(a, stream);
    if (a.n <= 8192) return launch_gradient_as<GT, XT, 8, 2>(a, stream);
    return launch_gradient_as<GT, XT, 8, 4>(a, stream);
}

template <int GT>
int launch_gradient_of(const NormGradientArgs &a, int dtype, hipStream_t stream)
{
    if (dtype == MADDNESS_F32) return launch_gradient<GT, kF32>(a, stream);
    if (dtype == MADDNESS_F16) return launch_gradient<GT, kF16>(a, stream);
    return launch_gradient<GT, kBF16>(a, stream);
}

template <int XT>
int launch_norm(const RowsArgs &a, int out_dtype, hipStream_t stream)
{
    if (out_dtype == kI8) return launch_rows<XT, kI8, true>(a, stream);
    if (out_dtype == MADDNESS_F32) return launch_rows<XT, kF32, true>(a, stream);
    if (out_dtype == MADDNESS_F16) return launch_rows<XT, kF16, true>(a, stream);
    return launch_rows<XT, kBF16, true>(a, stream);
}

}  // namespace

int launch_quantise_rows(const RowsArgs &a, int dtype, hipStream_t stream)
{
    if (dtype == MADDNESS_F32) return launch_rows<kF32, kI8, false>(a, stream);
    if (dtype == MADDNESS_F16) return launch_rows<kF16, kI8, false>(a, stream);
    return launch_rows<kBF16, kI8, false>(a, stream);
}

int launch_layer_norm(const RowsArgs &a, int dtype, int out_dtype, hipStream_t stream)
{
    if (dtype == MADDNESS_F32) return launch_norm<kF32>(a, out_dtype, stream);
    if (dtype == MADDNESS_F16) return launch_norm<kF16>(a, out_dtype, stream);
    return launch_norm<kBF16>(a, out_dtype, stream);
}

size_t layer_norm_gradient_workspace_bytes(int64_t rows, int64_t n) { return (size_t)(2 * parts_of(rows, n) * n) * sizeof(float); }

int launch_layer_norm_gradient(const NormGradientArgs &a, int gradient_dtype, int dtype, hipStream_t stream)
{
    int rc = MADDNESS_OK;
    if (a.rows > 0) {
        if (gradient_dtype == MADDNESS_F32) rc = launch_gradient_of<kF32>(a, dtype, stream);
        else if (gradient_dtype == MADDNESS_F16) rc = launch_gradient_of<kF16>(a, dtype, stream);
        else rc = launch_gradient_of<kBF16>(a, dtype, stream);
    }
    if (rc != MADDNESS_OK || !a.dweight) return rc;
    const int64_t parts = a.rows > 0 ? parts_of(a.rows, a.n) : 0;
    note_kernel("column_sums_kernel", nullptr);
    hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)ceil_div(a.n, (int64_t)32), 2), dim3(1024), 0, stream, a.partial, parts, a.n, a.dweight, a.dbias);
    return check_hip(hipGetLastError(), "launch column_sums_kernel");
}

}  // namespace maddness

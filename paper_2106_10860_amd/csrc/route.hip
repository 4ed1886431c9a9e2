// The choice of experts, the slots in the order of their experts, and the weighted sum of what the experts gave; with the
// gradients of the scores and of the weights.  All of it is memory-bound next to the experts' products.
#include "block_common.h"

namespace maddness {
namespace {

constexpr int kWaves = 4;               // tokens to a workgroup where a wavefront takes one
constexpr float kNone = -__builtin_inff();

template <typename T>
__device__ __forceinline__ T wave_sum(T x)
{
#pragma unroll
    for (int d = 32; d; d /= 2) x += __shfl_xor(x, d);
    return x;
}

// The value that lane (l + D) mod 16 of the row of 16 lanes has (D = 8, 4, 2, 1), lane l ^ 16, lane l ^ 32.
template <int D>
__device__ __forceinline__ uint32_t from_lane(uint32_t x)
{
    if constexpr (D < 16) {
        return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x120 + D, 0xf, 0xf, true);
    } else if constexpr (D == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}

template <int D>
__device__ __forceinline__ float from_lane(float x) { return __uint_as_float(from_lane<D>(__float_as_uint(x))); }

template <int D>
__device__ __forceinline__ double from_lane(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    return __builtin_bit_cast(double, from_lane<D>((uint32_t)b) | ((uint64_t)from_lane<D>((uint32_t)(b >> 32)) << 32));
}

// f over the LANES (16 or 64) lanes that share a token, in all of them.
template <int LANES, typename T, typename F>
__device__ __forceinline__ T over_lanes(T x, F f)
{
    x = f(x, from_lane<8>(x));
    x = f(x, from_lane<4>(x));
    x = f(x, from_lane<2>(x));
    x = f(x, from_lane<1>(x));
    if constexpr (LANES == 64) {
        x = f(x, from_lane<16>(x));
        x = f(x, from_lane<32>(x));
    }
    return x;
}

constexpr auto larger = [](auto a, auto b) INLINE_LAMBDA {
    if constexpr (sizeof(a) == 8) return fmax(a, b);
    else return fmaxf(a, b);
};
// One of two values (of two variables the language's own choice is a place, which the compiler then finds by their number).
template <typename T>
__device__ __forceinline__ T either(bool first, T a, T b) { return first ? a : b; }

constexpr auto plus = [](auto a, auto b) INLINE_LAMBDA { return a + b; };

struct RouteArgs {
    const void *logits;
    int64_t T, ldl;
    int E;
    const float *bias;
    int groups, kept, k;
    bool softmax, renormalise;
    float factor;
    int32_t *ids;
    float *weights;
    const int32_t *chosen;      // gradient: the ids of before,
    const float *dweights;      // what comes in
    void *gradient;             // and what goes out
    int64_t ldd;
    bool pieces;                // rows can be read and written in whole runs
};

constexpr float kTop = 3.402823466e38f;

// R neighbouring elements.
template <int DT, int R>
struct alignas(R *elem_size(DT) < 16 ? R * elem_size(DT) : 16) Run {
    char bytes[R * elem_size(DT)];
};

// How a token's logits become scores: the largest and the sum of a softmax.
struct Scale {
    float top, sum;
};

__device__ __forceinline__ float score_of(float x, bool softmax, Scale c)
{
    if (!(x > kNone)) return 0.0f;
    x = fminf(x, kTop);
    return softmax ? expf(x - c.top) / c.sum : 1.0f / (1.0f + expf(-x));
}

// The i-th of a lane's R experts.  In runs of RUN neighbours, which the lanes have in turn: all R in one where a choice by groups asks for it, else in
// runs of 16 bytes, so that what the lanes read and write at a time is without gaps (32768 tokens, 256 experts, fp32: the gradient 25.3 us with
// runs of 64 bytes, 18.4 now).
template <int LANES, int RUN>
__device__ __forceinline__ int expert_at(int lane, int i) { return i / RUN * RUN * LANES + lane * RUN + i % RUN; }

template <int DT, int R>
constexpr int kRun = R * elem_size(DT) < 16 ? R : 16 / elem_size(DT);

// The scores of a lane's experts into s; returns which of them are in the choice at all (bit i).
template <int DT, int LANES, int R, int RUN>
__device__ __forceinline__ uint32_t load_scores(const RouteArgs &a, int64_t t, int lane, float (&s)[R], Scale &c)
{
    if (a.pieces) {
        Run<DT, RUN> run[R / RUN] = {};
#pragma unroll
        for (int q = 0; q < R / RUN; ++q) {
            const int e = expert_at<LANES, RUN>(lane, q * RUN);
            if (e < a.E) run[q] = *reinterpret_cast<const Run<DT, RUN> *>(static_cast<const char *>(a.logits) + (t * a.ldl + e) * elem_size(DT));
        }
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = expert_at<LANES, RUN>(lane, i) < a.E ? widen_at<DT>(run[i / RUN].bytes, i % RUN) : kNone;
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int e = expert_at<LANES, RUN>(lane, i);
            s[i] = widen_at<DT>(a.logits, t * a.ldl + min(e, a.E - 1));
            if (e >= a.E) s[i] = kNone;
        }
    }
    uint32_t seen = 0;
    c = Scale{-kTop, 1.0f};
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const bool in = s[i] > kNone;                          // (not for a NaN)
        seen |= (uint32_t)in << i;
        s[i] = fminf(s[i], kTop);
        c.top = in ? fmaxf(c.top, s[i]) : c.top;
    }
    if (a.softmax) {
        c.top = over_lanes<LANES>(c.top, larger);
        double total = 0.0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i] = seen >> i & 1 ? expf(s[i] - c.top) : 0.0f;
            total += (double)s[i];
        }
        c.sum = (float)over_lanes<LANES>(total, plus);
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = seen >> i & 1 ? s[i] / c.sum : 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = seen >> i & 1 ? 1.0f / (1.0f + expf(-s[i])) : 0.0f;
    }
    return seen;
}

// A key and its expert as one number of 64 bits: a double of 1 to 2, in whose fraction the key's bits (turned so that they order as the keys
// do) come first and the expert after them, the lower the larger.  So a maximum is one instruction, and no two are equal.  1 is no key.
__device__ __forceinline__ double ordered(float key, int e)
{
    const uint32_t b = __float_as_uint(key + 0.0f);            // (-0 becomes 0)
    const uint32_t o = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return __builtin_bit_cast(double, 0x3ff0000000000000ull | ((uint64_t)o << 20) | (uint32_t)(1024 - e));
}

__device__ __forceinline__ int expert_of(double x) { return 1024 - (int)(__builtin_bit_cast(uint64_t, x) & 0xfffff); }

// Largest first: odd-even merge sort.
template <int R>
__device__ __forceinline__ void sort_down(double (&x)[R])
{
#pragma unroll
    for (int p = 1; p < R; p *= 2)
#pragma unroll
        for (int q = p; q; q /= 2)
#pragma unroll
            for (int j = q % p; j + q < R; j += 2 * q)
#pragma unroll
                for (int i = 0; i < q; ++i) {
                    const int lo = i + j, hi = i + j + q;
                    if (hi >= R || lo / (2 * p) != hi / (2 * p)) continue;
                    const double a = x[lo], b = x[hi];
                    x[lo] = fmax(a, b);
                    x[hi] = fmin(a, b);
                }
}

// LANES lanes to a token, R experts to a lane.  The lane sorts its experts; then k times the first of all lanes is the next choice, and leaves its
// lane's list.  Bound by the vector units: E / LANES exponentials, divisions and a sort for each lane (32768 tokens, 8 of 256 experts out of 4 of 8 groups
// 32 us, 33.6 MB read; the vector units busy for 61 % of the cycles by their counter).  KEEP: how much of a lane's list is needed for k (with all 16 of it 37.6).
template <int DT, int LANES, int R, int KEEP>
__global__ __launch_bounds__(256) void route_kernel(RouteArgs a)
{
    constexpr int TOKENS = 256 / LANES;
    __shared__ __attribute__((aligned(16))) float all_keys[TOKENS][LANES * (R < 2 ? 2 : R)], all_values[TOKENS][64];
    const int lane = threadIdx.x % LANES, mine = threadIdx.x / LANES;
    const int64_t t_any = (int64_t)blockIdx.x * TOKENS + mine, t = min(t_any, a.T - 1);      // (no lane leaves: the others exchange with it)
    float key[R];
    Scale c;
    const uint32_t seen = load_scores<DT, LANES, R, R>(a, t, lane, key, c);
    const int e0 = lane * R;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (a.bias) key[i] += a.bias[min(e0 + i, a.E - 1)];
        if (!(seen >> i & 1) || !(key[i] > kNone)) key[i] = kNone;
    }
    if (a.groups > 1) {
        const int size = a.E / a.groups;
        const bool whole = size % R == 0;                      // a lane's experts are all of one group: its two largest stand for them
        float best = kNone, second = kNone;
        auto rank = [&](float x) INLINE_LAMBDA {
            second = fmaxf(second, fminf(best, x));
            best = fmaxf(best, x);
        };
        if (whole) {
#pragma unroll
            for (int i = 0; i < R; ++i) rank(key[i]);
            all_keys[mine][2 * lane] = best;
            all_keys[mine][2 * lane + 1] = second;
            best = second = kNone;
        } else {
#pragma unroll
            for (int i = 0; i < R; ++i) all_keys[mine][e0 + i] = key[i];
        }
        wave_lds_fence();
        if (lane < a.groups) {
            const int n = whole ? size / R * 2 : size;
            for (int i = 0; i < n; ++i) rank(all_keys[mine][lane * n + i]);
        }
        // (a sum of two keys may be minus infinity where both are near the lowest number; a group without an expert has none: NaN is before nothing)
        const bool any = best > kNone;
        const float value = any ? (second > kNone ? best + second : best) : __builtin_nanf("");
        if (lane < a.groups) all_values[mine][lane] = value;
        wave_lds_fence();
        int before = 0;
        for (int g = 0; g < a.groups; ++g) {
            const float other = all_values[mine][g];
            before += other > value || (other == value && g < lane);
        }
        uint64_t kept = __ballot(lane < a.groups && any && before < a.kept);
        if constexpr (LANES == 16) kept = kept >> (threadIdx.x & 48) & 0xffff;
        int g = e0 / size, end = (g + 1) * size;
        if (whole) {
            const bool mine_kept = kept >> min(g, 63) & 1;
#pragma unroll
            for (int i = 0; i < R; ++i) key[i] = mine_kept ? key[i] : kNone;
        } else {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                if (e0 + i == end) {
                    ++g;
                    end += size;
                }
                if (!(kept >> min(g, 63) & 1)) key[i] = kNone;
            }
        }
    }
    double list[R];
#pragma unroll
    for (int i = 0; i < R; ++i) list[i] = key[i] > kNone ? ordered(key[i], e0 + i) : 1.0;
    sort_down<R>(list);
    int id = -1, id_high = -1;                                 // of choice `lane`, and 16 + lane
    for (int j = 0; j < a.k; ++j) {
        const double first = over_lanes<LANES>(list[0], larger);
        const int e = first > 1.0 ? expert_of(first) : -1;
        if (j == lane) id = e;
        if (LANES == 16 && j == 16 + lane) id_high = e;
        const bool won = list[0] == first;
#pragma unroll
        for (int i = 0; i + 1 < KEEP; ++i) list[i] = either(won, list[i + 1], list[i]);
        list[KEEP - 1] = either(won, 1.0, list[KEEP - 1]);
    }
    auto weight = [&](int e) INLINE_LAMBDA { return e < 0 ? 0.0f : score_of(widen_at<DT>(a.logits, t * a.ldl + e), a.softmax, c); };
    float w = weight(id), w_high = LANES == 16 && a.k > 16 ? weight(id_high) : 0.0f;
    if (a.renormalise) {
        float total = 0.0f;                                    // in the choice's order
        for (int j = 0; j < a.k; ++j) total += __shfl(either(j < 16 || LANES == 64, w, w_high), (threadIdx.x & 63 & -LANES) + (LANES == 64 ? j : j % 16));
        w = total > 0.0f ? w / total : 0.0f;
        w_high = total > 0.0f ? w_high / total : 0.0f;
    }
    if (t_any >= a.T) return;
    if (lane < a.k) {
        a.ids[t * a.k + lane] = id;
        a.weights[t * a.k + lane] = w * a.factor;
    }
    if (LANES == 16 && 16 + lane < a.k) {
        a.ids[t * a.k + 16 + lane] = id_high;
        a.weights[t * a.k + 16 + lane] = w_high * a.factor;
    }
}

// w_j = factor s_j (/ sum of the chosen s): with g_j the gradient of s_j, dx = s (g - sum g s) for the softmax and g s (1 - s) for
// the sigmoid.  The few g_j are spread over the row in LDS.  Bound by memory where there are many tokens (32768 of 256 experts 18.4 us, 67 MB).
template <int DT, int LANES, int R>
__global__ __launch_bounds__(256) void route_gradient_kernel(RouteArgs a)
{
    constexpr int TOKENS = 256 / LANES, HALVES = LANES == 16 ? 2 : 1, RUN = kRun<DT, R>;
    __shared__ __attribute__((aligned(16))) float spread[TOKENS][LANES * R];
    const int lane = threadIdx.x % LANES, row = threadIdx.x / LANES, first_lane = threadIdx.x & 63 & -LANES;
    const int64_t t_any = (int64_t)blockIdx.x * TOKENS + row, t = min(t_any, a.T - 1);
    float s[R];
    Scale c;
    int id[HALVES];
    float mine[HALVES], g[HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        const int j = h * 16 + lane, at = min(j, a.k - 1);
        id[h] = a.chosen[t * a.k + at];
        g[h] = a.dweights[t * a.k + at] * a.factor;
        if (j >= a.k || id[h] < 0 || id[h] >= a.E) id[h] = -1;
    }
    const uint32_t seen = load_scores<DT, LANES, R, RUN>(a, t, lane, s, c);
#pragma unroll
    for (int i = 0; i < R; ++i) spread[row][expert_at<LANES, RUN>(lane, i)] = 0.0f;
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        mine[h] = id[h] < 0 ? 0.0f : score_of(widen_at<DT>(a.logits, t * a.ldl + max(id[h], 0)), a.softmax, c);
        if (id[h] < 0) g[h] = 0.0f;
    }
    float all = 0.0f;
    if (a.renormalise || a.softmax) {
        float total = 0.0f;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) total += mine[h], all += g[h] * mine[h];
        total = over_lanes<LANES>(total, plus);
        all = over_lanes<LANES>(all, plus);
        if (a.renormalise) {
#pragma unroll
            for (int h = 0; h < HALVES; ++h) g[h] = total > 0.0f && id[h] >= 0 ? (g[h] - all / total) / total : 0.0f;
            all = 0.0f;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) all += g[h] * mine[h];
            all = over_lanes<LANES>(all, plus);
        }
    }
    // An expert that is there more than once gets the sum, in the order of the choices, from the first of them.
    float sum[HALVES];
    bool first[HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) sum[h] = 0.0f, first[h] = id[h] >= 0;
    for (int j = 0; j < a.k; ++j) {
        const int from = first_lane + (LANES == 16 ? j % 16 : j);
        const int other = __shfl(either(j < 16, id[0], id[HALVES - 1]), from);
        const float gj = __shfl(either(j < 16, g[0], g[HALVES - 1]), from);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            if (other == id[h]) {
                sum[h] += gj;
                if (j < h * 16 + lane) first[h] = false;
            }
        }
    }
    wave_lds_fence();
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
        if (first[h]) spread[row][id[h]] = sum[h];
    wave_lds_fence();
    if (t_any >= a.T) return;
    Run<DT, RUN> run[R / RUN];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const float d = spread[row][expert_at<LANES, RUN>(lane, i)];
        const float dx = a.softmax ? s[i] * (d - all) : d * s[i] * (1.0f - s[i]);
        store_as<DT>(run[i / RUN].bytes, i % RUN, seen >> i & 1 ? dx : 0.0f);
    }
    if (a.pieces) {
#pragma unroll
        for (int q = 0; q < R / RUN; ++q) {
            const int e = expert_at<LANES, RUN>(lane, q * RUN);
            if (e < a.E) *reinterpret_cast<Run<DT, RUN> *>(static_cast<char *>(a.gradient) + (t * a.ldd + e) * elem_size(DT)) = run[q];
        }
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int e = expert_at<LANES, RUN>(lane, i);
            if (e < a.E) store_as<DT>(a.gradient, t * a.ldd + e, widen_at<DT>(run[i / RUN].bytes, i % RUN));
        }
    }
}

template <int DT, int LANES, int R>
int launch_route_as(RouteArgs a, hipStream_t stream)
{
    constexpr int TOKENS = 256 / LANES;
    const int64_t blocks = ceil_div(a.T, (int64_t)TOKENS), bytes = std::min(R * elem_size(DT), 16);
    const int run = a.gradient ? kRun<DT, R> : R;
    const uintptr_t places = reinterpret_cast<uintptr_t>(a.logits) | reinterpret_cast<uintptr_t>(a.gradient) | (uintptr_t)((a.ldl | a.ldd) * elem_size(DT));
    a.pieces = a.E % run == 0 && places % bytes == 0;
    if (a.gradient) {
        note_kernel("route_gradient_kernel", __PRETTY_FUNCTION__);
        hipLaunchKernelGGL((route_gradient_kernel<DT, LANES, R>), dim3((unsigned)blocks), dim3(256), 0, stream, a);
        return check_hip(hipGetLastError(), "launch route_gradient_kernel");
    }
    note_kernel("route_kernel", __PRETTY_FUNCTION__);
    if constexpr (R > 8) {
        if (a.k <= 8) {
            hipLaunchKernelGGL((route_kernel<DT, LANES, R, 8>), dim3((unsigned)blocks), dim3(256), 0, stream, a);
            return check_hip(hipGetLastError(), "launch route_kernel");
        }
    }
    hipLaunchKernelGGL((route_kernel<DT, LANES, R, R>), dim3((unsigned)blocks), dim3(256), 0, stream, a);
    return check_hip(hipGetLastError(), "launch route_kernel");
}

template <int DT>
int launch_route_some(const RouteArgs &a, hipStream_t stream)
{
    // 16 lanes to a token while a lane then has at most 16 experts, and a group its lane; but not for so few tokens that each has a SIMD to itself and
    // the shorter way of fewer experts to a lane counts
    if (a.groups <= 16 && (a.E <= 64 || a.T > 4 * device_info().cus)) {
        if (a.E <= 16) return launch_route_as<DT, 16, 1>(a, stream);
        if (a.E <= 32) return launch_route_as<DT, 16, 2>(a, stream);
        if (a.E <= 64) return launch_route_as<DT, 16, 4>(a, stream);
        if (a.E <= 128) return launch_route_as<DT, 16, 8>(a, stream);
        if (a.E <= 256) return launch_route_as<DT, 16, 16>(a, stream);
    }
    if (a.E <= 256) return launch_route_as<DT, 64, 4>(a, stream);
    if (a.E <= 512) return launch_route_as<DT, 64, 8>(a, stream);
    return launch_route_as<DT, 64, 16>(a, stream);
}

constexpr int64_t kMostTokens = (int64_t)1 << 25;               // of a launch, so that its threads can be counted in 32 bits

template <int DT>
int launch_route_typed(const RouteArgs &a, hipStream_t stream)
{
    int rc = MADDNESS_OK;
    for (int64_t t = 0; t < a.T && rc == MADDNESS_OK; t += kMostTokens) {
        RouteArgs part = a;
        part.T = std::min(kMostTokens, a.T - t);
        part.logits = static_cast<const char *>(a.logits) + t * a.ldl * elem_size(DT);
        if (a.gradient) {
            part.chosen += t * a.k;
            part.dweights += t * a.k;
            part.gradient = static_cast<char *>(a.gradient) + t * a.ldd * elem_size(DT);
        } else {
            part.ids += t * a.k;
            part.weights += t * a.k;
        }
        rc = launch_route_some<DT>(part, stream);
    }
    return rc;
}

int launch_route_any(const RouteArgs &a, int dtype, hipStream_t stream)
{
    if (dtype == MADDNESS_F32) return launch_route_typed<kF32>(a, stream);
    if (dtype == MADDNESS_F16) return launch_route_typed<kF16>(a, stream);
    return launch_route_typed<kBF16>(a, stream);
}

// ------------------------------------------------------------------------------------------------ slots by their experts

// A counting sort by chunks of slots: how many of a chunk go to each expert, where the first of each begins, the places.  Counts
// are sums of ones and places follow the slots' order, so the result does not depend on timing.
__host__ __device__ inline int64_t chunk_slots(int64_t slots) { return std::max((int64_t)256, round_up(ceil_div(slots, (int64_t)1024), (int64_t)64)); }

__global__ __launch_bounds__(256) void order_count_kernel(const int32_t *ids, int64_t slots, int E, int64_t chunk, int32_t *counts, int32_t *source,
                                                          int64_t capacity)
{
    __shared__ int32_t n[MADDNESS_MAX_EXPERTS];
    for (int e = threadIdx.x; e < E; e += 256) n[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * chunk, last = min(first + chunk, slots);
    for (int64_t i = first + threadIdx.x; i < last; i += 256) {
        const int e = ids[i];
        if (e >= 0 && e < E) atomicAdd(&n[e], 1);
    }
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < capacity; i += (int64_t)gridDim.x * 256) source[i] = -1;
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += 256) counts[(int64_t)blockIdx.x * E + e] = n[e];
}

// Sum over the threads before this one, of 1024 threads.
__device__ __forceinline__ int64_t sum_before(int64_t mine, int64_t (&waves)[16])
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t o = __shfl_up((long long)upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += waves[w];
    return upto - mine;
}

// In each of (a power of two of) parts of the chunks a thread for each expert: the sums of the parts, then the chunks' beginnings.
__global__ __launch_bounds__(1024) void order_offsets_kernel(int32_t *begin, int64_t chunks, int E, int align, int32_t *offsets, int32_t *counts)
{
    __shared__ int32_t sums[1024];
    __shared__ int64_t waves[16];
    int width = 1;
    while (width < E) width *= 2;
    width = max(width, 16);                                  // (at most 64 parts)
    const int e = threadIdx.x % width, part = threadIdx.x / width, parts = 1024 / width;
    const int64_t each = ceil_div(chunks, (int64_t)parts), c0 = part * each, c1 = min(c0 + each, chunks);
    int total = 0;
    if (e < E)
        for (int64_t c = c0; c < c1; c += 8) {
            int n[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) n[i] = c + i < c1 ? begin[(c + i) * E + e] : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) total += n[i];
        }
    sums[threadIdx.x] = total;
    __syncthreads();
    int at = 0, all = 0;                                     // of this expert: before this part, and in all
    for (int p = 0; p < parts; ++p) {
        const int n = sums[p * width + e];
        at += p < part ? n : 0;
        all += n;
    }
    if (e < E)
        for (int64_t c = c0; c < c1; c += 8) {
            int n[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) n[i] = c + i < c1 ? begin[(c + i) * E + e] : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (c + i < c1) begin[(c + i) * E + e] = at;
                at += n[i];
            }
        }
    const bool first = part == 0 && e < E;
    const int64_t room = first ? ceil_div((int64_t)all, (int64_t)align) * align : 0, before = sum_before(room, waves);
    if (first) {
        offsets[e] = (int32_t)before;
        if (e == E - 1) offsets[E] = (int32_t)(before + room);
        if (counts) counts[e] = all;
    }
}

// The lanes whose e is this lane's (none for a negative one).
__device__ __forceinline__ uint64_t same_expert(int e, int E)
{
    uint64_t same = __ballot(e >= 0);
    for (int b = 0; 1 << b < E; ++b) {
        const bool bit = e >> b & 1;
        const uint64_t m = __ballot(bit);
        same &= bit ? m : ~m;
    }
    return same;
}

// Up to kOrderAtOnce slots: all of it by one workgroup, each wavefront with a stretch of the slots, in a launch instead of three (8198 slots 8.4 us;
// the three, for 49152, 5 each).
constexpr int64_t kOrderAtOnce = 16384;

__global__ __launch_bounds__(1024) void order_kernel(const int32_t *ids, int slots, int E, int align, int32_t *offsets, int32_t *counts, int32_t *source,
                                                     int64_t capacity, int32_t *place)
{
    __shared__ int32_t next[16][MADDNESS_MAX_EXPERTS];       // how many of a stretch go to an expert; then, where its next one goes
    __shared__ int32_t first[MADDNESS_MAX_EXPERTS], taken[MADDNESS_MAX_EXPERTS];
    __shared__ int64_t waves[16];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, e_mine = threadIdx.x;
    const int stretch = round_up(ceil_div(slots, 16), 64), begin = wave * stretch, end = min(begin + stretch, slots);
    constexpr int TURNS = kOrderAtOnce / 1024;
    int mine[TURNS];                                         // the stretch's experts
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        const int i = begin + u * 64 + lane;
        mine[u] = i < end ? ids[i] : -1;
    }
    for (int e = lane; e < E; e += 64) next[wave][e] = 0;
    wave_lds_fence();
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        if (mine[u] >= E) mine[u] = -1;
        if (mine[u] >= 0) atomicAdd(&next[wave][mine[u]], 1);
    }
    __syncthreads();
    int total = 0;
    if (e_mine < E)
        for (int w = 0; w < 16; ++w) total += next[w][e_mine];
    const int64_t room = ceil_div((int64_t)total, (int64_t)align) * align, before = sum_before(room, waves);
    if (e_mine < E) {
        int at = (int)before;
        for (int w = 0; w < 16; ++w) {
            const int n = next[w][e_mine];
            next[w][e_mine] = at;
            at += n;
        }
        first[e_mine] = (int)before;
        taken[e_mine] = total;
        offsets[e_mine] = (int32_t)before;
        if (e_mine == E - 1) offsets[E] = (int32_t)(before + room);
        if (counts) counts[e_mine] = total;
    }
    __syncthreads();
    // the places without a slot
    for (int e = wave; e < E; e += 16) {
        const int to = e + 1 < E ? first[e + 1] : (int)capacity;
        for (int i = first[e] + taken[e] + lane; i < to; i += 64) source[i] = -1;
    }
#pragma unroll
    for (int u = 0; u < TURNS; ++u) {
        const int i = begin + u * 64 + lane, e = mine[u];
        if (begin + u * 64 >= end) break;
        const uint64_t same = same_expert(e, E);
        int at = -1;
        if (e >= 0) {
            at = next[wave][e] + __popcll(same & (((uint64_t)1 << lane) - 1));
            source[at] = i;
        }
        if (i < end) place[i] = at;
        wave_lds_fence();
        if (e >= 0 && (same >> lane) == 1) next[wave][e] = at + 1;      // the last of them
        wave_lds_fence();
    }
}

__global__ __launch_bounds__(64) void order_place_kernel(const int32_t *ids, int64_t slots, int E, int64_t chunk, const int32_t *begin,
                                                         const int32_t *offsets, int32_t *source, int32_t *place)
{
    __shared__ int32_t next[MADDNESS_MAX_EXPERTS];
    const int lane = threadIdx.x;
    for (int e = lane; e < E; e += 64) next[e] = offsets[e] + begin[(int64_t)blockIdx.x * E + e];
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * chunk, last = min(first + chunk, slots);
    for (int64_t i0 = first; i0 < last; i0 += 64) {
        const int64_t i = i0 + lane;
        int e = i < last ? ids[i] : -1;
        if (e >= E) e = -1;
        const uint64_t same = same_expert(e, E);
        int at = -1;
        if (e >= 0) {
            at = next[e] + __popcll(same & (((uint64_t)1 << lane) - 1));
            source[at] = (int32_t)i;
        }
        if (i < last) place[i] = at;
        __syncthreads();
        if (e >= 0 && (same >> lane) == 1) next[e] = at + 1; // the last of them
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------------- the weighted sum

struct CombineArgs {
    const void *y;
    int64_t rows, N, ldy;
    const int32_t *place;
    const float *weights;
    int64_t T;
    int k;
    void *out;
    int64_t ldo;
    const void *gradient;
    int64_t ldg;
    float *dweights;
};

// A wavefront to a token (several where the rows are long); up to 8 of the token's rows are on their way at once.  Bound by memory: 8192 tokens, 6
// rows of 1024 each, to bfloat16: from bfloat16 19 us, 6.1 TB/s, from fp32 33 us, 6.5 TB/s.
template <int YT, int OT>
__global__ __launch_bounds__(kWaves * 64) void combine_kernel(CombineArgs a)
{
    constexpr int AT_ONCE = YT == kF32 ? 4 : 8;
    const int lane = threadIdx.x % 64;
    const int64_t t = (int64_t)blockIdx.x * kWaves + threadIdx.x / 64, c0 = ((int64_t)blockIdx.y * 64 + lane) * 8;
    if (t >= a.T || c0 >= a.N) return;
    const bool shorter = a.N < 8;
    const int64_t c = shorter ? 0 : min(c0, a.N - 8);        // (the last piece computes some of the one before again, to the same values)
    float sum[8] = {};
    for (int j0 = 0; j0 < a.k; j0 += AT_ONCE) {
        int p[AT_ONCE];
        float w[AT_ONCE];
        Raw<YT> raw[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int64_t at = t * a.k + min(j0 + j, a.k - 1);
            p[j] = a.place ? a.place[at] : (int)at;
            w[j] = a.weights ? a.weights[at] : 1.0f;
            if (j0 + j >= a.k || p[j] >= a.rows) p[j] = -1;
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
            if (j0 + j < a.k && !shorter && a.rows > 0) raw[j] = load_raw<YT>(a.y, (int64_t)max(p[j], 0) * a.ldy, c, a.N);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            if (j0 + j >= a.k || a.rows == 0) break;
            float v[8];
            if (shorter) load_short<YT>(a.y, (int64_t)max(p[j], 0) * a.ldy, c, a.N, v);
            else widen<YT>(raw[j], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = p[j] < 0 ? sum[i] : sum[i] + w[j] * v[i];
        }
    }
    const int64_t at = t * a.ldo + c;
    if (!shorter) {
        store_run<OT>(a.out, at, sum);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < a.N) store_as<OT>(a.out, at + i, sum[i]);
    }
}

template <int GT, int YT>
__global__ __launch_bounds__(kWaves * 64) void combine_gradient_kernel(CombineArgs a)
{
    const int lane = threadIdx.x % 64;
    const int64_t t = (int64_t)blockIdx.x * kWaves + threadIdx.x / 64;
    if (t >= a.T) return;
    for (int j = 0; j < a.k; ++j) {
        const int64_t p = a.place ? a.place[t * a.k + j] : t * a.k + j;
        float sum = 0.0f;
        if (p >= 0 && p < a.rows) {
            const int64_t at_g = t * a.ldg, at_y = p * a.ldy;
            for (int64_t c = lane * 8; c < a.N; c += 512) {
                float g[8], v[8];
                if (a.N >= 8) {
                    const Raw<GT> raw_g = load_raw<GT>(a.gradient, at_g, c, a.N);
                    const Raw<YT> raw_y = load_raw<YT>(a.y, at_y, c, a.N);
                    widen<GT>(raw_g, g);
                    widen<YT>(raw_y, v);
                    const int skip = before_column(c, a.N);
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[i] = i < skip ? 0.0f : g[i], v[i] = i < skip ? 0.0f : v[i];
                } else {
                    load_short<GT>(a.gradient, at_g, c, a.N, g);
                    load_short<YT>(a.y, at_y, c, a.N, v);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += g[i] * v[i];
            }
        }
        sum = wave_sum(sum);
        if (lane == 0) a.dweights[t * a.k + j] = sum;
    }
}

template <int YT, int OT>
int launch_combine_some(const CombineArgs &a, hipStream_t stream)
{
    const int64_t blocks = ceil_div(a.T, (int64_t)kWaves);
    if (a.dweights) {
        note_kernel("combine_gradient_kernel", __PRETTY_FUNCTION__);
        hipLaunchKernelGGL((combine_gradient_kernel<OT, YT>), dim3((unsigned)blocks), dim3(kWaves * 64), 0, stream, a);
        return check_hip(hipGetLastError(), "launch combine_gradient_kernel");
    }
    const int64_t across = ceil_div(a.N, (int64_t)512);
    if (across > 65535) return fail(MADDNESS_E_UNSUPPORTED, "combine: rows of %lld are too long", (long long)a.N);
    note_kernel("combine_kernel", __PRETTY_FUNCTION__);
    hipLaunchKernelGGL((combine_kernel<YT, OT>), dim3((unsigned)blocks, (unsigned)across), dim3(kWaves * 64), 0, stream, a);
    return check_hip(hipGetLastError(), "launch combine_kernel");
}

template <int YT, int OT>
int launch_combine_as(const CombineArgs &a, hipStream_t stream)
{
    int rc = MADDNESS_OK;
    for (int64_t t = 0; t < a.T && rc == MADDNESS_OK; t += kMostTokens) {
        CombineArgs part = a;
        part.T = std::min(kMostTokens, a.T - t);
        if (a.place) part.place += t * a.k;
        else part.y = static_cast<const char *>(a.y) + t * a.k * a.ldy * elem_size(YT), part.rows -= t * a.k;
        if (a.weights) part.weights += t * a.k;
        if (a.dweights) {
            part.gradient = static_cast<const char *>(a.gradient) + t * a.ldg * elem_size(OT);
            part.dweights += t * a.k;
        } else {
            part.out = static_cast<char *>(a.out) + t * a.ldo * elem_size(OT);
        }
        rc = launch_combine_some<YT, OT>(part, stream);
    }
    return rc;
}

template <int YT>
int launch_combine_to(const CombineArgs &a, int dtype, hipStream_t stream)
{
    if (dtype == MADDNESS_F32) return launch_combine_as<YT, kF32>(a, stream);
    if (dtype == MADDNESS_F16) return launch_combine_as<YT, kF16>(a, stream);
    return launch_combine_as<YT, kBF16>(a, stream);
}

int launch_combine_any(const CombineArgs &a, int y_dtype, int dtype, hipStream_t stream)
{
    if (y_dtype == MADDNESS_F32) return launch_combine_to<kF32>(a, dtype, stream);
    if (y_dtype == MADDNESS_F16) return launch_combine_to<kF16>(a, dtype, stream);
    return launch_combine_to<kBF16>(a, dtype, stream);
}

}  // namespace

int launch_route(const void *logits, int dtype, int64_t T, int E, int64_t ldl, const float *bias, int scores, int groups, int kept, int k,
                 bool renormalise, float factor, int32_t *ids, float *weights, hipStream_t stream)
{
    RouteArgs a{};
    a.logits = logits; a.T = T; a.ldl = ldl; a.E = E; a.bias = bias; a.groups = groups; a.kept = kept; a.k = k;
    a.softmax = scores == MADDNESS_SOFTMAX; a.renormalise = renormalise; a.factor = factor; a.ids = ids; a.weights = weights;
    return launch_route_any(a, dtype, stream);
}

int launch_route_gradient(const void *logits, int dtype, int64_t T, int E, int64_t ldl, int scores, int k, bool renormalise, float factor,
                          const int32_t *ids, const float *dweights, void *gradient, int64_t ldd, hipStream_t stream)
{
    RouteArgs a{};
    a.logits = logits; a.T = T; a.ldl = ldl; a.E = E; a.k = k; a.softmax = scores == MADDNESS_SOFTMAX; a.renormalise = renormalise;
    a.factor = factor; a.chosen = ids; a.dweights = dweights; a.gradient = gradient; a.ldd = ldd;
    return launch_route_any(a, dtype, stream);
}

size_t order_workspace_bytes(int64_t slots, int E)
{
    return (size_t)std::max((int64_t)1, ceil_div(slots, chunk_slots(slots))) * E * sizeof(int32_t);
}

int launch_order(const int32_t *ids, int64_t slots, int E, int align, int32_t *offsets, int32_t *counts, int32_t *source, int64_t capacity,
                 int32_t *place, void *workspace, hipStream_t stream)
{
    if (slots <= kOrderAtOnce) {
        note_kernel("order_kernel", nullptr);
        hipLaunchKernelGGL(order_kernel, dim3(1), dim3(1024), 0, stream, ids, (int)slots, E, align, offsets, counts, source, capacity, place);
        return check_hip(hipGetLastError(), "launch order_kernel");
    }
    const int64_t chunk = chunk_slots(slots), chunks = std::max((int64_t)1, ceil_div(slots, chunk));
    int32_t *begin = static_cast<int32_t *>(workspace);
    note_kernel("order_count_kernel", nullptr);
    hipLaunchKernelGGL(order_count_kernel, dim3((unsigned)chunks), dim3(256), 0, stream, ids, slots, E, chunk, begin, source, capacity);
    hipLaunchKernelGGL(order_offsets_kernel, dim3(1), dim3(1024), 0, stream, begin, chunks, E, align, offsets, counts);
    hipLaunchKernelGGL(order_place_kernel, dim3((unsigned)chunks), dim3(64), 0, stream, ids, slots, E, chunk, begin, offsets, source, place);
    return check_hip(hipGetLastError(), "launch order_place_kernel");
}

int launch_combine(const void *y, int y_dtype, int64_t rows, int64_t N, int64_t ldy, const int32_t *place, const float *weights, int64_t T,
                   int k, void *out, int out_dtype, int64_t ldo, hipStream_t stream)
{
    CombineArgs a{};
    a.y = y; a.rows = rows; a.N = N; a.ldy = ldy; a.place = place; a.weights = weights; a.T = T; a.k = k; a.out = out; a.ldo = ldo;
    return launch_combine_any(a, y_dtype, out_dtype, stream);
}

int launch_combine_gradient(const void *gradient, int dtype, int64_t ldg, const void *y, int y_dtype, int64_t rows, int64_t N, int64_t ldy,
                            const int32_t *place, int64_t T, int k, float *dweights, hipStream_t stream)
{
    CombineArgs a{};
    a.gradient = gradient; a.ldg = ldg; a.y = y; a.rows = rows; a.N = N; a.ldy = ldy; a.place = place; a.T = T; a.k = k; a.dweights = dweights;
    return launch_combine_any(a, y_dtype, dtype, stream);
}

}  // namespace maddness

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

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int d = 32; d; d /= 2) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

// The scores of a lane's R logits (expert 64 i + lane) into s; returns which of them are in the choice at all (bit i).
template <int DT, int R>
__device__ __forceinline__ uint32_t load_scores(const void *logits, int64_t at, int E, int lane, bool softmax, float (&s)[R])
{
    uint32_t seen = 0;
    float top = -3.402823466e38f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int e = 64 * i + lane;
        const float x = e < E ? widen_at<DT>(logits, at + e) : kNone;
        s[i] = fminf(x, 3.402823466e38f);
        if (x > kNone) {
            seen |= 1u << i;
            top = fmaxf(top, s[i]);
        }
    }
    if (softmax) {
        top = wave_max(top);
        double total = 0.0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i] = seen >> i & 1 ? expf(s[i] - top) : 0.0f;
            total += (double)s[i];
        }
        const float sum = (float)wave_sum(total);
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = seen >> i & 1 ? s[i] / sum : 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = seen >> i & 1 ? 1.0f / (1.0f + expf(-s[i])) : 0.0f;
    }
    return seen;
}

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
};

// Keys as whole numbers in the same order, the lower expert the larger among equals.
__device__ __forceinline__ uint64_t ordered(float key, int e)
{
    const uint32_t b = __float_as_uint(key + 0.0f);      // (-0 becomes 0)
    return ((uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32) | (0xffffffffu - (uint32_t)e);
}

template <int DT, int R>
__global__ __launch_bounds__(kWaves * 64) void route_kernel(RouteArgs a)
{
    __shared__ float all_keys[kWaves][R * 64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t t = (int64_t)blockIdx.x * kWaves + wave;
    if (t >= a.T) return;
    float s[R], key[R];
    const uint32_t seen = load_scores<DT, R>(a.logits, t * a.ldl, a.E, lane, a.softmax, s);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        key[i] = seen >> i & 1 ? (a.bias ? s[i] + a.bias[64 * i + lane] : s[i]) : kNone;
        if (!(key[i] > kNone)) key[i] = kNone;                // (a NaN)
    }
    if (a.groups > 1) {
        float *keys = all_keys[wave];
        const int size = a.E / a.groups;
#pragma unroll
        for (int i = 0; i < R; ++i) keys[64 * i + lane] = key[i];
        wave_lds_fence();
        float best = kNone, second = kNone;
        if (lane < a.groups)
            for (int i = 0; i < size; ++i) {
                const float x = keys[lane * size + i];
                second = fmaxf(second, fminf(best, x));
                best = fmaxf(best, x);
            }
        const float value = best > kNone ? (second > kNone ? best + second : best) : kNone;
        int before = 0;
        for (int g = 0; g < a.groups; ++g) {
            const float other = __shfl(value, g);
            before += other > value || (other == value && g < lane);
        }
        const uint64_t kept = __ballot(value > kNone && before < a.kept);
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (!(kept >> min((64 * i + lane) / size, 63) & 1)) key[i] = kNone;
    }
    int id = -1;
    float w = 0.0f;
    for (int j = 0; j < a.k; ++j) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint64_t o = ordered(key[i], 64 * i + lane);
            if (key[i] > kNone && o > best) best = o;
        }
#pragma unroll
        for (int d = 32; d; d /= 2) {
            const uint64_t o = (uint64_t)__shfl_xor((unsigned long long)best, d);
            best = o > best ? o : best;
        }
        if (!best) break;
        const int e = (int)(0xffffffffu - (uint32_t)best);
        float mine = 0.0f;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (64 * i + lane == e) {
                mine = s[i];
                key[i] = kNone;
            }
        mine = __shfl(mine, e % 64);
        if (lane == j) {
            id = e;
            w = mine;
        }
    }
    if (a.renormalise) {
        float total = 0.0f;
        for (int j = 0; j < a.k; ++j) total += __shfl(w, j);
        w = total > 0.0f ? w / total : 0.0f;
    }
    if (lane < a.k) {
        a.ids[t * a.k + lane] = id;
        a.weights[t * a.k + lane] = w * a.factor;
    }
}

// w_j = factor s_j (/ sum of the chosen s): with g_j the gradient of s_j, dx = s (g - sum g s) for the softmax and g s (1 - s) for
// the sigmoid.
template <int DT, int R>
__global__ __launch_bounds__(kWaves * 64) void route_gradient_kernel(RouteArgs a)
{
    __shared__ float all_scores[kWaves][R * 64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t t = (int64_t)blockIdx.x * kWaves + wave;
    if (t >= a.T) return;
    float s[R], ds[R];
    const uint32_t seen = load_scores<DT, R>(a.logits, t * a.ldl, a.E, lane, a.softmax, s);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        all_scores[wave][64 * i + lane] = s[i];
        ds[i] = 0.0f;
    }
    wave_lds_fence();
    int id = -1;
    float mine = 0.0f, g = 0.0f;
    if (lane < a.k) {
        id = a.chosen[t * a.k + lane];
        if (id < 0 || id >= a.E) id = -1;
        else {
            mine = all_scores[wave][id];
            g = a.dweights[t * a.k + lane] * a.factor;
        }
    }
    if (a.renormalise) {
        const float total = wave_sum(mine), both = wave_sum(g * mine);
        g = total > 0.0f && id >= 0 ? (g - both / total) / total : 0.0f;
    }
    for (int j = 0; j < a.k; ++j) {
        const int e = __shfl(id, j);
        const float gj = __shfl(g, j);
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (64 * i + lane == e) ds[i] += gj;
    }
    float all = 0.0f;
    if (a.softmax) all = wave_sum(g * mine);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int e = 64 * i + lane;
        if (e >= a.E) continue;
        const float dx = a.softmax ? s[i] * (ds[i] - all) : ds[i] * s[i] * (1.0f - s[i]);
        store_as<DT>(a.gradient, t * a.ldd + e, seen >> i & 1 ? dx : 0.0f);
    }
}

template <int DT, int R>
int launch_route_as(const RouteArgs &a, hipStream_t stream)
{
    const int64_t blocks = ceil_div(a.T, (int64_t)kWaves);
    if (blocks >= (int64_t)1 << 31) return fail(MADDNESS_E_UNSUPPORTED, "route: %lld tokens are too many", (long long)a.T);
    if (a.gradient) {
        note_kernel("route_gradient_kernel", __PRETTY_FUNCTION__);
        hipLaunchKernelGGL((route_gradient_kernel<DT, R>), dim3((unsigned)blocks), dim3(kWaves * 64), 0, stream, a);
        return check_hip(hipGetLastError(), "launch route_gradient_kernel");
    }
    note_kernel("route_kernel", __PRETTY_FUNCTION__);
    hipLaunchKernelGGL((route_kernel<DT, R>), dim3((unsigned)blocks), dim3(kWaves * 64), 0, stream, a);
    return check_hip(hipGetLastError(), "launch route_kernel");
}

template <int DT>
int launch_route_typed(const RouteArgs &a, hipStream_t stream)
{
    if (a.E <= 64) return launch_route_as<DT, 1>(a, stream);
    if (a.E <= 128) return launch_route_as<DT, 2>(a, stream);
    if (a.E <= 256) return launch_route_as<DT, 4>(a, stream);
    if (a.E <= 512) return launch_route_as<DT, 8>(a, stream);
    return launch_route_as<DT, 16>(a, stream);
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
__host__ __device__ inline int64_t chunk_slots(int64_t slots) { return std::max((int64_t)1024, round_up(ceil_div(slots, (int64_t)1024), (int64_t)64)); }

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

__global__ __launch_bounds__(MADDNESS_MAX_EXPERTS) void order_offsets_kernel(int32_t *begin, int64_t chunks, int E, int align, int32_t *offsets, int32_t *counts)
{
    __shared__ int64_t upto[MADDNESS_MAX_EXPERTS];
    const int e = threadIdx.x;
    int64_t total = 0;
    if (e < E)
        for (int64_t c = 0; c < chunks; ++c) {
            const int32_t n = begin[c * E + e];
            begin[c * E + e] = (int32_t)total;
            total += n;
        }
    const int64_t room = ceil_div(total, (int64_t)align) * align;
    upto[e] = room;
    __syncthreads();
    for (int d = 1; d < MADDNESS_MAX_EXPERTS; d *= 2) {
        const int64_t before = e >= d ? upto[e - d] : 0;
        __syncthreads();
        upto[e] += before;
        __syncthreads();
    }
    if (e < E) {
        offsets[e] = (int32_t)(upto[e] - room);
        if (e == E - 1) offsets[E] = (int32_t)upto[e];
        if (counts) counts[e] = (int32_t)total;
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
        uint64_t same = __ballot(e >= 0);                    // the lanes with this lane's expert
#pragma unroll
        for (int b = 0; b < 10; ++b) {
            const bool bit = e >> b & 1;
            const uint64_t m = __ballot(bit);
            same &= bit ? m : ~m;
        }
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

template <int YT, int OT>
__global__ __launch_bounds__(kWaves * 64) void combine_kernel(CombineArgs a)
{
    const int lane = threadIdx.x % 64;
    const int64_t t = (int64_t)blockIdx.x * kWaves + threadIdx.x / 64;
    if (t >= a.T) return;
    for (int64_t c = lane * 8; c < a.N; c += 512) {
        const int n = (int)min(a.N - c, (int64_t)8);
        float sum[8] = {};
        for (int j = 0; j < a.k; ++j) {
            const int p = a.place[t * a.k + j];
            if (p < 0 || p >= a.rows) continue;
            const float w = a.weights ? a.weights[t * a.k + j] : 1.0f;
            float v[8];
            load8<YT>(a.y, p * a.ldy + c, n, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += w * v[i];
        }
        for (int i = 0; i < n; ++i) store_as<OT>(a.out, t * a.ldo + c + i, sum[i]);
    }
}

template <int GT, int YT>
__global__ __launch_bounds__(kWaves * 64) void combine_gradient_kernel(CombineArgs a)
{
    const int lane = threadIdx.x % 64;
    const int64_t t = (int64_t)blockIdx.x * kWaves + threadIdx.x / 64;
    if (t >= a.T) return;
    for (int j = 0; j < a.k; ++j) {
        const int p = a.place[t * a.k + j];
        float sum = 0.0f;
        if (p >= 0 && p < a.rows)
            for (int64_t c = lane * 8; c < a.N; c += 512) {
                const int n = (int)min(a.N - c, (int64_t)8);
                float g[8], v[8];
                load8<GT>(a.gradient, t * a.ldg + c, n, g);
                load8<YT>(a.y, p * a.ldy + c, n, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += g[i] * v[i];
            }
        sum = wave_sum(sum);
        if (lane == 0) a.dweights[t * a.k + j] = sum;
    }
}

template <int YT, int OT>
int launch_combine_as(const CombineArgs &a, hipStream_t stream)
{
    const int64_t blocks = ceil_div(a.T, (int64_t)kWaves);
    if (blocks >= (int64_t)1 << 31) return fail(MADDNESS_E_UNSUPPORTED, "combine: %lld tokens are too many", (long long)a.T);
    if (a.gradient) {
        note_kernel("combine_gradient_kernel", __PRETTY_FUNCTION__);
        hipLaunchKernelGGL((combine_gradient_kernel<OT, YT>), dim3((unsigned)blocks), dim3(kWaves * 64), 0, stream, a);
        return check_hip(hipGetLastError(), "launch combine_gradient_kernel");
    }
    note_kernel("combine_kernel", __PRETTY_FUNCTION__);
    hipLaunchKernelGGL((combine_kernel<YT, OT>), dim3((unsigned)blocks), dim3(kWaves * 64), 0, stream, a);
    return check_hip(hipGetLastError(), "launch combine_kernel");
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
    const int64_t chunk = chunk_slots(slots), chunks = std::max((int64_t)1, ceil_div(slots, chunk));
    int32_t *begin = static_cast<int32_t *>(workspace);
    note_kernel("order_count_kernel", nullptr);
    hipLaunchKernelGGL(order_count_kernel, dim3((unsigned)chunks), dim3(256), 0, stream, ids, slots, E, chunk, begin, source, capacity);
    hipLaunchKernelGGL(order_offsets_kernel, dim3(1), dim3(MADDNESS_MAX_EXPERTS), 0, stream, begin, chunks, E, align, offsets, counts);
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

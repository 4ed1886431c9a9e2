// How evenly the tokens fall on the experts: counts, the loss that keeps them alike, and its gradient.  Bound by reading the logits.
#include "lanes.h"
#include "layers_common.h"

namespace maddness {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr float kTop = 3.402823466e38f;

constexpr auto larger = [](float a, float b) INLINE_LAMBDA { return fmaxf(a, b); };

// The four neighbours of every 4 LANES experts that a lane has: i of its R.
template <int LANES>
__device__ __forceinline__ int expert_at(int lane, int i) { return i / 4 * 4 * LANES + lane * 4 + i % 4; }

template <int DT>
struct alignas(4 * elem_size(DT)) Four {
    char bytes[4 * elem_size(DT)];
};

// A token's scores over LANES lanes, R to a lane, and their sum; 0 for masked ones and beyond E.
template <int DT, int LANES, int R>
__device__ __forceinline__ float load_scores(const BalanceArgs &a, bool pieces, int64_t t, int lane, float (&s)[R], uint32_t &seen)
{
    float x[R];
#pragma unroll
    for (int q = 0; q < R / 4; ++q) {
        const int e = expert_at<LANES>(lane, 4 * q);
        if (pieces) {
            Four<DT> four = {};
            if (e < a.E) four = *reinterpret_cast<const Four<DT> *>(static_cast<const char *>(a.logits) + (t * a.ldl + e) * elem_size(DT));
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * q + i] = widen_at<DT>(four.bytes, i);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[4 * q + i] = widen_at<DT>(a.logits, t * a.ldl + min(e + i, a.E - 1));
        }
    }
    seen = 0;
    float top = -kTop;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const bool in = x[i] > -__builtin_inff() && expert_at<LANES>(lane, i) < a.E;       // (not for a NaN)
        seen |= (uint32_t)in << i;
        x[i] = in ? fminf(x[i], kTop) : -kTop;
        top = fmaxf(top, x[i]);
    }
    float sum = 0.0f;
    if (a.softmax) top = over_lanes<LANES>(top, larger);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const float v = a.softmax ? expf(x[i] - top) : 1.0f / (1.0f + expf(-x[i]));
        s[i] = seen >> i & 1 ? v : 0.0f;
        sum += s[i];
    }
    return over_lanes<LANES>(sum, plus);
}

// Where the workgroups leave their sums.
struct Workspace {
    double *losses;                     // [kMostSlices]
    uint32_t *ticket;
    int32_t *live, *chosen;             // [groups]: tokens that count, ids that are experts
    float *mass;                        // [groups][E]
    int32_t *counts;                    // [groups][E]
};

constexpr int kSlice = 16, kMostSlices = MADDNESS_MAX_EXPERTS / kSlice;     // experts to a workgroup of the second kernel

__host__ __device__ inline Workspace workspace_of(void *base, int64_t groups, int E)
{
    Workspace w;
    w.losses = static_cast<double *>(base);
    w.ticket = reinterpret_cast<uint32_t *>(w.losses + kMostSlices);
    w.live = reinterpret_cast<int32_t *>(w.ticket + 2);
    w.chosen = w.live + groups;
    w.mass = reinterpret_cast<float *>(w.chosen + groups);
    w.counts = reinterpret_cast<int32_t *>(w.mass + groups * E);
    return w;
}

// Every workgroup's share: its tokens' p added up for each expert, and its part of the ids counted.
template <int DT, int LANES, int R>
__global__ __launch_bounds__(kThreads) void balance_kernel(BalanceArgs a, void *base, bool pieces)
{
    constexpr int TOKENS = 64 / LANES;                         // of a wavefront at a time
    __shared__ int32_t counts[R * LANES];
    __shared__ float mass[kWaves][R * LANES];
    __shared__ int32_t lives[kWaves];
    const Workspace w = workspace_of(base, gridDim.x, a.E);
    const int wave = threadIdx.x / 64, lane = threadIdx.x % LANES, part = threadIdx.x % 64 / LANES;
    if (blockIdx.x == 0 && threadIdx.x == 0) *w.ticket = 0;
    for (int e = threadIdx.x; e < a.E; e += kThreads) counts[e] = 0;
    __syncthreads();
    const int64_t ids = a.T * a.k;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < ids; i += (int64_t)gridDim.x * kThreads) {
        const int id = a.ids[i];
        if (id >= 0 && id < a.E) atomicAdd(&counts[id], 1);
    }
    float sum[R] = {};
    int live = 0;
    for (int64_t t = ((int64_t)blockIdx.x * kWaves + wave) * TOKENS + part; t < a.T; t += (int64_t)gridDim.x * kWaves * TOKENS) {
        float s[R];
        uint32_t seen;
        const float all = load_scores<DT, LANES, R>(a, pieces, t, lane, s, seen);
        if (all > 0.0f) {
            ++live;
            const float scale = 1.0f / all;
#pragma unroll
            for (int i = 0; i < R; ++i) sum[i] += s[i] * scale;
        }
    }
    if constexpr (LANES == 16) {
        live += (int)from_lane<16>((uint32_t)live);
        live += (int)from_lane<32>((uint32_t)live);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            sum[i] += from_lane<16>(sum[i]);
            sum[i] += from_lane<32>(sum[i]);
        }
    }
    if (part == 0) {
#pragma unroll
        for (int i = 0; i < R; ++i) mass[wave][expert_at<LANES>(lane, i)] = sum[i];
        if (lane == 0) lives[wave] = live;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kThreads) {
        float m = mass[0][e];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) m += mass[v][e];
        w.mass[(int64_t)blockIdx.x * a.E + e] = m;
        w.counts[(int64_t)blockIdx.x * a.E + e] = counts[e];
    }
    if (threadIdx.x < 64) {
        uint32_t chosen = 0;
        for (int e = threadIdx.x; e < a.E; e += 64) chosen += (uint32_t)counts[e];
        chosen = over_lanes<64>(chosen, plus);
        if (threadIdx.x == 0) {
            int all = 0;
            for (int v = 0; v < kWaves; ++v) all += lives[v];
            w.live[blockIdx.x] = all;
            w.chosen[blockIdx.x] = (int32_t)chosen;
        }
    }
}

// The workgroups' shares together: 16 experts to a workgroup, its 64 runs of 16 lanes take every 64th share.  The workgroup that is done last adds the
// experts' parts of the loss up, in their order.
__global__ __launch_bounds__(1024) void balance_sum_kernel(BalanceArgs a, void *base, int groups)
{
    __shared__ double masses[64][kSlice];
    __shared__ int32_t counts[64][kSlice];
    __shared__ int64_t lives[16], chosens[16];
    const Workspace w = workspace_of(base, groups, a.E);
    const int column = threadIdx.x % kSlice, run = threadIdx.x / kSlice, e = blockIdx.x * kSlice + column;
    int64_t live = 0, chosen = 0;
    for (int g = threadIdx.x; g < groups; g += 1024) {
        live += w.live[g];
        chosen += w.chosen[g];
    }
    double mass = 0.0;
    int32_t count = 0;
    for (int g = run; g < groups; g += 64) {
        mass += (double)w.mass[(int64_t)g * a.E + min(e, a.E - 1)];
        count += w.counts[(int64_t)g * a.E + min(e, a.E - 1)];
    }
    masses[run][column] = mass;
    counts[run][column] = count;
#pragma unroll
    for (int d = 32; d; d /= 2) {
        live += __shfl_xor(live, d);
        chosen += __shfl_xor(chosen, d);
    }
    if (threadIdx.x % 64 == 0) {
        lives[threadIdx.x / 64] = live;
        chosens[threadIdx.x / 64] = chosen;
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    double part = 0.0;
    live = chosen = 0;
    for (int v = 0; v < 16; ++v) {
        live += lives[v];
        chosen += chosens[v];
    }
    if (threadIdx.x < kSlice && e < a.E) {
        mass = 0.0;
        count = 0;
#pragma unroll 8
        for (int r = 0; r < 64; ++r) {
            mass += masses[r][column];
            count += counts[r][column];
        }
        const float push = live && chosen ? (float)((double)a.factor * a.E * count / ((double)chosen * (double)live)) : 0.0f;
        a.counts[e] = count;
        a.push[e] = push;
        part = push * mass;
    }
    part = over_lanes<16>(part, plus);
    if (threadIdx.x != 0) return;
    if (gridDim.x == 1) {
        *a.loss = (float)part;
        return;
    }
    __hip_atomic_store(&w.losses[blockIdx.x], part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint32_t before = __hip_atomic_fetch_add(w.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    if (before + 1 != gridDim.x) return;
    part = 0.0;
#pragma unroll 1
    for (uint32_t i = 0; i < gridDim.x; ++i) part += __hip_atomic_load(&w.losses[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *a.loss = (float)part;
}

template <int DT, int LANES, int R>
__global__ __launch_bounds__(kThreads) void balance_gradient_kernel(BalanceArgs a, bool pieces, bool add_pieces)
{
    constexpr int TOKENS = 64 / LANES;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % LANES, part = threadIdx.x % 64 / LANES;
    const float times = a.loss_gradient ? *a.loss_gradient : 1.0f;
    float push[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int e = expert_at<LANES>(lane, i);
        push[i] = e < a.E ? a.push[e] : 0.0f;
    }
    for (int64_t t = ((int64_t)blockIdx.x * kWaves + wave) * TOKENS + part; t < a.T; t += (int64_t)gridDim.x * kWaves * TOKENS) {
        float s[R];
        uint32_t seen;
        const float all = load_scores<DT, LANES, R>(a, pieces, t, lane, s, seen), scale = all > 0.0f ? 1.0f / all : 0.0f;
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < R; ++i) dot += s[i] * scale * push[i];
        dot = over_lanes<LANES>(dot, plus);
#pragma unroll
        for (int q = 0; q < R / 4; ++q) {
            const int e = expert_at<LANES>(lane, 4 * q);
            float d[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 4 * q + i;
                d[i] = seen >> j & 1 ? times * (s[j] * scale * (push[j] - dot) * (a.softmax ? 1.0f : 1.0f - s[j])) : 0.0f;
            }
            if (add_pieces) {
                if (e >= a.E) continue;
                if (a.add) {
                    const Four<DT> four = *reinterpret_cast<const Four<DT> *>(static_cast<const char *>(a.add) + (t * a.lda + e) * elem_size(DT));
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[i] += widen_at<DT>(four.bytes, i);
                }
                store_run<DT>(a.gradient, t * a.ldd + e, d);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (e + i < a.E) store_as<DT>(a.gradient, t * a.ldd + e + i, a.add ? d[i] + widen_at<DT>(a.add, t * a.lda + e + i) : d[i]);
            }
        }
    }
}

int64_t groups_of(int64_t T, int E)
{
    const int64_t tokens = kWaves * (E <= 64 ? 4 : 1);
    return std::min(std::max(ceil_div(T, tokens), (int64_t)1), (int64_t)device_info().cus);
}

// Rows that can be read and written four at a time.
bool fours(const void *p, int64_t ld, int E, int dtype)
{
    return E % 4 == 0 && ld % 4 == 0 && reinterpret_cast<uintptr_t>(p) % (4 * elem_size(dtype)) == 0;
}

template <int DT, int LANES, int R>
int launch_as(const BalanceArgs &a, void *workspace, hipStream_t stream)
{
    const bool pieces = fours(a.logits, a.ldl, a.E, DT);
    if (a.gradient) {
        const int64_t groups = std::min(ceil_div(a.T, (int64_t)(kWaves * (64 / LANES))), (int64_t)device_info().cus * 4);
        note_kernel("balance_gradient_kernel", __PRETTY_FUNCTION__);
        hipLaunchKernelGGL((balance_gradient_kernel<DT, LANES, R>), dim3((unsigned)groups), dim3(kThreads), 0, stream, a, pieces,
                           a.E % 4 == 0 && (!a.add || fours(a.add, a.lda, a.E, DT)));
        return check_hip(hipGetLastError(), "launch balance_gradient_kernel");
    }
    const int64_t groups = groups_of(a.T, a.E);
    note_kernel("balance_kernel", __PRETTY_FUNCTION__);
    hipLaunchKernelGGL((balance_kernel<DT, LANES, R>), dim3((unsigned)groups), dim3(kThreads), 0, stream, a, workspace, pieces);
    hipLaunchKernelGGL(balance_sum_kernel, dim3((unsigned)ceil_div(a.E, kSlice)), dim3(1024), 0, stream, a, workspace, (int)groups);
    return check_hip(hipGetLastError(), "launch balance_kernel");
}

template <int DT>
int launch_of(const BalanceArgs &a, void *workspace, hipStream_t stream)
{
    if (a.E <= 64) return launch_as<DT, 16, 4>(a, workspace, stream);
    if (a.E <= 256) return launch_as<DT, 64, 4>(a, workspace, stream);
    return launch_as<DT, 64, 16>(a, workspace, stream);
}

int launch(const BalanceArgs &a, int dtype, void *workspace, hipStream_t stream)
{
    if (dtype == MADDNESS_F32) return launch_of<kF32>(a, workspace, stream);
    if (dtype == MADDNESS_F16) return launch_of<kF16>(a, workspace, stream);
    return launch_of<kBF16>(a, workspace, stream);
}

}  // namespace

size_t balance_workspace_bytes(int64_t T, int E)
{
    const int64_t groups = groups_of(T, E);
    return (size_t)(kMostSlices * 8 + 8 + groups * 8 + groups * E * 8);
}

int launch_balance(const BalanceArgs &a, int dtype, void *workspace, hipStream_t stream) { return launch(a, dtype, workspace, stream); }

int launch_balance_gradient(const BalanceArgs &a, int dtype, hipStream_t stream) { return launch(a, dtype, nullptr, stream); }

}  // namespace maddness

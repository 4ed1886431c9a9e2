// How evenly the tokens fall on the experts: counts, the loss that keeps them alike, and its gradient.
//
//   p = s / sum s, push[e] = factor E counts[e] / (n L), loss = sum_e push[e] sum_t p[t][e], dlogits = p (push - sum p push) (1 - s for a sigmoid)
//
// A token's experts lie on 4, 16 or 64 lanes, four neighbours to a lane, so its sums go around lanes without memory; what it adds to the experts' shares stays in registers until a workgroup is done.
// 32768 tokens, 256 experts, fp32: 12.7 us for counts and shares (2.7 TB/s) and 4.5 for their sums, both bound by latency (a wavefront has 8 tokens, which it asks for in two turns behind
// the counting; vector units busy for 38 % and 1 %), 16.1 for the gradient (4.2 TB/s).
#include "lanes.h"
#include "layers_common.h"

namespace maddness {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kGradientWaves = 4;
constexpr float kTop = 3.402823466e38f;

constexpr auto larger = [](float a, float b) INLINE_LAMBDA { return fmaxf(a, b); };

// f over the LANES lanes that share a token, in all of them.
template <int LANES, typename T, typename F>
__device__ __forceinline__ T over_token(T x, F f)
{
    if constexpr (LANES == 4) {
        x = f(x, __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0xb1, 0xf, 0xf, true)));       // lane l ^ 1
        return f(x, __builtin_bit_cast(T, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x4e, 0xf, 0xf, true)));    // lane l ^ 2
    } else {
        return over_lanes<LANES>(x, f);
    }
}

// The sum over the lanes of the wavefront's tokens that have the same experts, in all of them.
template <int LANES, typename T>
__device__ __forceinline__ T over_tokens(T x)
{
    if constexpr (LANES == 4) {
        x += from_lane<8>(x);
        x += from_lane<4>(x);
    }
    if constexpr (LANES <= 16) {
        x += from_lane<16>(x);
        x += from_lane<32>(x);
    }
    return x;
}

// e^x by the 2^x instruction, whose argument's rounding is put back: to 2 steps of fp32 (results below 2^-126 are 0).  The library's function takes twice the operations.  x is kept to
// -128 .. 88: from 88.73 on the result would be infinite, and what is put back, an infinity of either sign, could make it no number.
__device__ __forceinline__ float exponential(float x)
{
    constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596303e-8f, kLn2 = 0.693147182f;
    x = __builtin_amdgcn_fmed3f(x, -128.0f, 88.0f);
    const float t = x * kLog2e, e = __builtin_amdgcn_exp2f(t);
    return __builtin_fmaf(e, kLn2 * __builtin_fmaf(x, kLog2eRest, __builtin_fmaf(x, kLog2e, -t)), e);
}

// 1 / (1 + e^-x); 0 where that is below 2^-126, as the instruction gives no such numbers (so it is for all x below -88 too, which have e^88 here: a comparison of its own
// takes 1.2 us of the 31 that 32768 tokens of 256 experts take).
// `other` is 1 minus that, as e^-x s: the difference itself has fewer digits the nearer s is to 1, and none from a logit of 18 on.  (Where s is 0 here so is this, and nothing that it is
// a factor of beside s.)
__device__ __forceinline__ float sigmoid(float x, float &other)
{
    const float e = exponential(-x), s = __builtin_amdgcn_rcpf(1.0f + e);
    other = e * s;
    return s;
}

// The four neighbours of every 4 LANES experts that a lane has: i of its R.
template <int LANES>
__device__ __forceinline__ int expert_at(int lane, int i) { return i / 4 * 4 * LANES + lane * 4 + i % 4; }

template <int DT>
struct alignas(4 * elem_size(DT)) Four {
    char bytes[4 * elem_size(DT)];
};

// A lane's logits of a token.
template <int DT, int LANES, int R>
__device__ __forceinline__ void load_logits(const BalanceArgs &a, bool pieces, int64_t t, int lane, float (&x)[R])
{
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
}

// A token's scores over LANES lanes, R to a lane, and their sum; 0 for masked ones and beyond E.  slope: 1, or of a sigmoid 1 - s.
template <int LANES, int R>
__device__ __forceinline__ float scores_of(const BalanceArgs &a, int lane, float (&x)[R], float (&s)[R], float (&slope)[R], uint32_t &seen)
{
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
    if (a.softmax) top = over_token<LANES>(top, larger);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        slope[i] = 1.0f;
        const float v = a.softmax ? exponential(x[i] - top) : sigmoid(x[i], slope[i]);
        s[i] = seen >> i & 1 ? v : 0.0f;
        sum += s[i];
    }
    return over_token<LANES>(sum, plus);
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

__device__ __forceinline__ float push_of(const BalanceArgs &a, int64_t count, int64_t chosen, int64_t live)
{
    return live && chosen ? (float)((double)a.factor * a.E * (double)count / ((double)chosen * (double)live)) : 0.0f;
}

// Every workgroup's share: its tokens' p added up for each expert, and its part of the ids counted.  Four tokens of a lane are asked for at a time, and their sums over the lanes go on
// beside each other.  ALL: the only workgroup, which gives the results (few tokens: a launch less).
template <int DT, int LANES, int R, bool ALL>
__global__ __launch_bounds__(kThreads) void balance_kernel(BalanceArgs a, void *base, bool pieces)
{
    constexpr int TOKENS = 64 / LANES, ONCE = R <= 4 ? 4 : 1;  // of a wavefront side by side, and in turn
    __shared__ int32_t counts[R * LANES];
    __shared__ float mass[kWaves][R * LANES];
    __shared__ int32_t lives[kWaves];
    __shared__ double parts[kWaves];
    const Workspace w = workspace_of(base, gridDim.x, a.E);
    const int wave = threadIdx.x / 64, lane = threadIdx.x % LANES, part = threadIdx.x % 64 / LANES;
    if (!ALL && blockIdx.x == 0 && threadIdx.x == 0) *w.ticket = 0;
    for (int e = threadIdx.x; e < a.E; e += kThreads) counts[e] = 0;
    __syncthreads();
    const int64_t ids = a.T * a.k;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < ids; i += (int64_t)gridDim.x * kThreads) {
        const int id = a.ids[i];
        if (id >= 0 && id < a.E) atomicAdd(&counts[id], 1);
    }
    float sum[R] = {};
    int live = 0;
    const int64_t step = (int64_t)gridDim.x * kWaves * TOKENS;
    for (int64_t t = ((int64_t)blockIdx.x * kWaves + wave) * TOKENS + part; t < a.T; t += ONCE * step) {
        float x[ONCE][R], s[R], slope[R];
#pragma unroll
        for (int u = 0; u < ONCE; ++u) load_logits<DT, LANES, R>(a, pieces, min(t + u * step, a.T - 1), lane, x[u]);
#pragma unroll
        for (int u = 0; u < ONCE; ++u) {
            uint32_t seen;
            const float all = scores_of<LANES, R>(a, lane, x[u], s, slope, seen);
            const bool here = all > 0.0f && t + u * step < a.T;
            live += here;
            const float scale = here ? 1.0f / all : 0.0f;
#pragma unroll
            for (int i = 0; i < R; ++i) sum[i] += s[i] * scale;
        }
    }
    live = (int)over_tokens<LANES>((uint32_t)live);
#pragma unroll
    for (int i = 0; i < R; ++i) sum[i] = over_tokens<LANES>(sum[i]);
    if (part == 0) {
#pragma unroll
        for (int i = 0; i < R; ++i) mass[wave][expert_at<LANES>(lane, i)] = sum[i];
        if (lane == 0) lives[wave] = live;
    }
    __syncthreads();
    uint32_t chosen = 0;
    int all = 0;
    if (ALL || threadIdx.x < 64) {
        for (int e = threadIdx.x % 64; e < a.E; e += 64) chosen += (uint32_t)counts[e];
        chosen = over_lanes<64>(chosen, plus);
        for (int v = 0; v < kWaves; ++v) all += lives[v];
    }
    const int e = threadIdx.x;                                 // (E <= kThreads)
    float m = 0.0f;
    if (e < a.E) {
        m = mass[0][e];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) m += mass[v][e];
    }
    if constexpr (ALL) {
        double loss = 0.0;
        if (e < a.E) {
            const float push = push_of(a, counts[e], chosen, all);
            a.counts[e] = counts[e];
            a.push[e] = push;
            loss = (double)push * m;
        }
        loss = over_lanes<64>(loss, plus);
        if (threadIdx.x % 64 == 0) parts[wave] = loss;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int v = 1; v < kWaves; ++v) loss += parts[v];
            *a.loss = (float)loss;
        }
    } else {
        if (e < a.E) {
            w.mass[(int64_t)blockIdx.x * a.E + e] = m;
            w.counts[(int64_t)blockIdx.x * a.E + e] = counts[e];
        }
        if (threadIdx.x == 0) {
            w.live[blockIdx.x] = all;
            w.chosen[blockIdx.x] = (int32_t)chosen;
        }
    }
}

// The workgroups' shares together: 16 experts to a workgroup, its 64 runs of 16 lanes take every 64th share.  The workgroup that is done last adds the
// experts' parts of the loss up, a lane to each.
__global__ __launch_bounds__(1024) void balance_sum_kernel(BalanceArgs a, void *base, int groups)
{
    __shared__ double masses[16][kSlice];
    __shared__ uint32_t counts[16][kSlice];
    __shared__ uint32_t lives[16], chosens[16];
    const Workspace w = workspace_of(base, groups, a.E);
    const int column = threadIdx.x % kSlice, run = threadIdx.x / kSlice, wave = threadIdx.x / 64, e = blockIdx.x * kSlice + column;
    uint32_t live = 0, chosen = 0, count = 0;                  // (all below 2^31)
    double mass = 0.0;
    for (int g = threadIdx.x; g < groups; g += 1024) {
        live += (uint32_t)w.live[g];
        chosen += (uint32_t)w.chosen[g];
    }
#pragma unroll 4
    for (int g = run; g < groups; g += 64) {
        mass += (double)w.mass[(int64_t)g * a.E + min(e, a.E - 1)];
        count += (uint32_t)w.counts[(int64_t)g * a.E + min(e, a.E - 1)];
    }
    live = over_lanes<64>(live, plus);
    chosen = over_lanes<64>(chosen, plus);
    mass += from_lane<16>(mass);
    mass += from_lane<32>(mass);
    count += from_lane<16>(count);
    count += from_lane<32>(count);
    if (threadIdx.x % 64 < kSlice) {
        masses[wave][column] = mass;
        counts[wave][column] = count;
        lives[wave] = live;
        chosens[wave] = chosen;
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    mass = 0.0;
    live = chosen = count = 0;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        mass += masses[v][column];
        count += counts[v][column];
        live += lives[v];
        chosen += chosens[v];
    }
    double part = 0.0;
    if (threadIdx.x < kSlice && e < a.E) {
        const float push = push_of(a, count, chosen, live);
        a.counts[e] = (int32_t)count;
        a.push[e] = push;
        part = push * mass;
    }
    part = over_lanes<16>(part, plus);
    if (gridDim.x == 1) {
        if (threadIdx.x == 0) *a.loss = (float)part;
        return;
    }
    uint32_t before = 0;
    if (threadIdx.x == 0) {
        __hip_atomic_store(&w.losses[blockIdx.x], part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        before = __hip_atomic_fetch_add(w.ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
    }
    if ((uint32_t)__builtin_amdgcn_readfirstlane((int)before) + 1 != gridDim.x) return;
    static_assert(kMostSlices <= 64, "a lane to each part");
    part = threadIdx.x < gridDim.x ? __hip_atomic_load(&w.losses[threadIdx.x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
    part = over_lanes<64>(part, plus);
    if (threadIdx.x == 0) *a.loss = (float)part;
}

template <int DT, int LANES, int R>
__global__ __launch_bounds__(kGradientWaves * 64) void balance_gradient_kernel(BalanceArgs a, bool pieces, bool add_pieces)
{
    constexpr int TOKENS = 64 / LANES, ONCE = R <= 4 ? 2 : 1;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % LANES, part = threadIdx.x % 64 / LANES;
    const float times = a.loss_gradient ? *a.loss_gradient : 1.0f;
    float push[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int e = expert_at<LANES>(lane, i);
        push[i] = e < a.E ? a.push[e] : 0.0f;
    }
    const int64_t step = (int64_t)gridDim.x * kGradientWaves * TOKENS;
    for (int64_t t0 = ((int64_t)blockIdx.x * kGradientWaves + wave) * TOKENS + part; t0 < a.T; t0 += ONCE * step) {
        float x[ONCE][R];
#pragma unroll
        for (int u = 0; u < ONCE; ++u) load_logits<DT, LANES, R>(a, pieces, min(t0 + u * step, a.T - 1), lane, x[u]);
#pragma unroll
        for (int u = 0; u < ONCE; ++u) {
            const int64_t t = t0 + u * step;
            float s[R], slope[R];
            uint32_t seen;
            const float all = scores_of<LANES, R>(a, lane, x[u], s, slope, seen), scale = all > 0.0f ? 1.0f / all : 0.0f;
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < R; ++i) dot += s[i] * scale * push[i];
            dot = over_token<LANES>(dot, plus);
            if (t >= a.T) continue;
#pragma unroll
            for (int q = 0; q < R / 4; ++q) {
                const int e = expert_at<LANES>(lane, 4 * q);
                float d[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = 4 * q + i;
                    d[i] = seen >> j & 1 ? times * (s[j] * scale * (push[j] - dot) * slope[j]) : 0.0f;
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
}

// Lanes that share a token, and how many experts they have room for.
constexpr int lanes_of(int E) { return E <= 16 ? 4 : E <= 64 ? 16 : 64; }
constexpr int slots_of(int E) { return E <= 16 ? 16 : E <= 64 ? 64 : E <= 256 ? 256 : 1024; }

// One workgroup while that has 32 experts' places to a thread or fewer (512 tokens of 8 experts: 5.8 us, by two launches 3.7 and 3.5).
int64_t groups_of(int64_t T, int E)
{
    if (T * slots_of(E) <= 32 * kThreads) return 1;
    return std::min(ceil_div(T, (int64_t)(kWaves * (64 / lanes_of(E)))), (int64_t)device_info().cus);
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
        const int64_t groups = std::min(ceil_div(a.T, (int64_t)(kGradientWaves * (64 / LANES))), (int64_t)device_info().cus * 8);
        note_kernel("balance_gradient_kernel", __PRETTY_FUNCTION__);
        hipLaunchKernelGGL((balance_gradient_kernel<DT, LANES, R>), dim3((unsigned)groups), dim3(kGradientWaves * 64), 0, stream, a, pieces,
                           a.E % 4 == 0 && (!a.add || fours(a.add, a.lda, a.E, DT)));
        return check_hip(hipGetLastError(), "launch balance_gradient_kernel");
    }
    const int64_t groups = groups_of(a.T, a.E);
    note_kernel("balance_kernel", __PRETTY_FUNCTION__);
    if (groups == 1) {
        hipLaunchKernelGGL((balance_kernel<DT, LANES, R, true>), dim3(1), dim3(kThreads), 0, stream, a, workspace, pieces);
        return check_hip(hipGetLastError(), "launch balance_kernel");
    }
    hipLaunchKernelGGL((balance_kernel<DT, LANES, R, false>), dim3((unsigned)groups), dim3(kThreads), 0, stream, a, workspace, pieces);
    hipLaunchKernelGGL(balance_sum_kernel, dim3((unsigned)ceil_div(a.E, kSlice)), dim3(1024), 0, stream, a, workspace, (int)groups);
    return check_hip(hipGetLastError(), "launch balance_kernel");
}

template <int DT>
int launch_of(const BalanceArgs &a, void *workspace, hipStream_t stream)
{
    if (a.E <= 16) return launch_as<DT, 4, 4>(a, workspace, stream);
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
    if (groups == 1) return 0;
    return (size_t)(kMostSlices * 8 + 8 + groups * 8 + groups * E * 8);
}

int launch_balance(const BalanceArgs &a, int dtype, void *workspace, hipStream_t stream) { return launch(a, dtype, workspace, stream); }

int launch_balance_gradient(const BalanceArgs &a, int dtype, hipStream_t stream) { return launch(a, dtype, nullptr, stream); }

}  // namespace maddness

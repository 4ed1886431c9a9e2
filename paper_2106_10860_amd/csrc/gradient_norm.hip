// The norm over many tensors, and their scaling by it.  Both move bytes: the squares are summed in fp64 beside the loads.
//
// The tensors' places go with the launch, as arguments of the kernel, so that a captured graph holds them too; so many tensors to a launch.
#include "layers_common.h"

namespace maddness {
namespace {

constexpr int kTensors = 96, kThreads = 256, kChunk = kThreads * 64;      // elements that a workgroup takes at a time

struct Table {
    const void *data[kTensors];
    void *out[kTensors];
    int64_t count[kTensors];
    uint32_t end[kTensors];             // chunks of the tensors up to and with this one
    uint8_t types[kTensors];            // of data + 4 times that of out
    int n;
};

// The tensor that a chunk belongs to, and the chunk's first element.
__device__ __forceinline__ int tensor_of(const Table &t, uint32_t chunk, int64_t &first)
{
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (chunk < t.end[mid]) hi = mid;
        else lo = mid + 1;
    }
    first = (int64_t)(chunk - (lo ? t.end[lo - 1] : 0)) * kChunk;
    return lo;
}

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 32; d; d /= 2) x += __shfl_xor(x, d);
    return x;
}

// The sum over the workgroup's threads, in all of them.
__device__ __forceinline__ double group_sum(double x, double (&slots)[kThreads / 64])
{
    x = wave_sum(x);
    if (threadIdx.x % 64 == 0) slots[threadIdx.x / 64] = x;
    __syncthreads();
    x = slots[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) x += slots[w];
    return x;
}

template <int DT>
__device__ __forceinline__ void add_squares(const void *data, int64_t first, int64_t count, double &sum)
{
    if (first + kChunk <= count) {
        Raw<DT> raw[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) raw[p] = load_raw<DT>(data, first, (int64_t)(p * kThreads + threadIdx.x) * 8, count);
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            float v[8];
            widen<DT>(raw[p], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fma((double)v[i], (double)v[i], sum);
        }
    } else {
        for (int64_t i = first + threadIdx.x; i < count; i += kThreads) {
            const double v = (double)widen_at<DT>(data, i);
            sum = __builtin_fma(v, v, sum);
        }
    }
}

// Sums of squares of a launch's tensors: to partials[workgroup], or in addition to what is there.
__global__ __launch_bounds__(kThreads) void squares_kernel(Table t, double *partials, bool add)
{
    __shared__ double slots[kThreads / 64];
    double sum = 0.0;
    const uint32_t chunks = t.n ? t.end[t.n - 1] : 0;
    for (uint32_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
        int64_t first;
        const int i = tensor_of(t, chunk, first);
        switch (t.types[i] & 3) {
        case kF32: add_squares<kF32>(t.data[i], first, t.count[i], sum); break;
        case kF16: add_squares<kF16>(t.data[i], first, t.count[i], sum); break;
        default: add_squares<kBF16>(t.data[i], first, t.count[i], sum);
        }
    }
    sum = group_sum(sum, slots);
    if (threadIdx.x == 0) partials[blockIdx.x] = add ? partials[blockIdx.x] + sum : sum;
}

__device__ __forceinline__ float norm_of(const double *partials, int parts, double (&slots)[kThreads / 64])
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) sum += partials[i];
    return (float)sqrt(group_sum(sum, slots));
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double *partials, int parts, float *norm)
{
    __shared__ double slots[kThreads / 64];
    const float all = norm_of(partials, parts, slots);
    if (threadIdx.x == 0) *norm = all;
}

template <int DT, int OT>
__device__ __forceinline__ void scale_chunk(const void *data, void *out, int64_t first, int64_t count, float factor)
{
    if (first + kChunk <= count) {
        Raw<DT> raw[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) raw[p] = load_raw<DT>(data, first, (int64_t)(p * kThreads + threadIdx.x) * 8, count);
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            float v[8];
            widen<DT>(raw[p], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= factor;
            store_run<OT>(out, first + (int64_t)(p * kThreads + threadIdx.x) * 8, v);
        }
    } else {
        for (int64_t i = first + threadIdx.x; i < count; i += kThreads) store_as<OT>(out, i, widen_at<DT>(data, i) * factor);
    }
}

// Scales a launch's tensors; the norm is that of the sums of squares, which every workgroup adds up for itself (16 KiB from L2), or given.
__global__ __launch_bounds__(kThreads) void clip_kernel(Table t, const double *partials, int parts, float *norm, bool given, float max_norm)
{
    __shared__ double slots[kThreads / 64];
    float all;
    if (given) {
        all = *norm;
    } else {
        all = norm_of(partials, parts, slots);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm = all;
    }
    const float factor = all > max_norm && all <= 3.402823466e38f ? (float)((double)max_norm / (double)all) : 1.0f;
    const uint32_t chunks = t.n ? t.end[t.n - 1] : 0;
    for (uint32_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
        int64_t first;
        const int i = tensor_of(t, chunk, first);
        const int64_t count = t.count[i];
        const void *data = t.data[i];
        void *out = t.out[i];
        if (data == out && factor == 1.0f) continue;
        switch (t.types[i]) {
        case kF32 + 4 * kF32: scale_chunk<kF32, kF32>(data, out, first, count, factor); break;
        case kF32 + 4 * kF16: scale_chunk<kF32, kF16>(data, out, first, count, factor); break;
        case kF32 + 4 * kBF16: scale_chunk<kF32, kBF16>(data, out, first, count, factor); break;
        case kF16 + 4 * kF32: scale_chunk<kF16, kF32>(data, out, first, count, factor); break;
        case kF16 + 4 * kF16: scale_chunk<kF16, kF16>(data, out, first, count, factor); break;
        case kF16 + 4 * kBF16: scale_chunk<kF16, kBF16>(data, out, first, count, factor); break;
        case kBF16 + 4 * kF32: scale_chunk<kBF16, kF32>(data, out, first, count, factor); break;
        case kBF16 + 4 * kF16: scale_chunk<kBF16, kF16>(data, out, first, count, factor); break;
        default: scale_chunk<kBF16, kBF16>(data, out, first, count, factor);
        }
    }
}

// The next tensors from `from` on that have elements, up to a launch's number of them and 2^32 - 1 chunks.
Table next_table(const maddness_tensor *tensors, int64_t n, int64_t &from, bool outs)
{
    Table t;
    t.n = 0;
    uint64_t chunks = 0;
    for (; from < n && t.n < kTensors; ++from) {
        const maddness_tensor &one = tensors[from];
        if (one.count == 0) continue;
        chunks += (uint64_t)ceil_div(one.count, (int64_t)kChunk);
        if (chunks > 0xffffffffu) break;
        t.data[t.n] = one.data;
        t.out[t.n] = outs ? one.out : nullptr;
        t.count[t.n] = one.count;
        t.end[t.n] = (uint32_t)chunks;
        t.types[t.n] = (uint8_t)(one.dtype + 4 * (outs ? one.out_dtype : 0));
        ++t.n;
    }
    return t;
}

unsigned groups_of(uint32_t chunks) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(chunks, kNormPartials)); }

// All sums of squares; how many of the partials hold them.
int launch_squares(const maddness_tensor *tensors, int64_t n, double *partials, int &parts, hipStream_t stream)
{
    uint64_t chunks = 0;
    for (int64_t i = 0; i < n; ++i) chunks += (uint64_t)ceil_div(tensors[i].count, (int64_t)kChunk);
    parts = (int)groups_of((uint32_t)std::min<uint64_t>(chunks, kNormPartials));
    int64_t from = 0;
    bool add = false;
    do {
        const Table t = next_table(tensors, n, from, false);
        hipLaunchKernelGGL(squares_kernel, dim3((unsigned)parts), dim3(kThreads), 0, stream, t, partials, add);
        const int rc = check_hip(hipGetLastError(), "launch squares_kernel");
        if (rc != MADDNESS_OK) return rc;
        add = true;
    } while (from < n);
    return MADDNESS_OK;
}

}  // namespace

int launch_gradient_norm(const maddness_tensor *tensors, int64_t n, float *norm, double *partials, hipStream_t stream)
{
    int parts;
    note_kernel("squares_kernel", nullptr);
    const int rc = launch_squares(tensors, n, partials, parts, stream);
    if (rc != MADDNESS_OK) return rc;
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, stream, partials, parts, norm);
    return check_hip(hipGetLastError(), "launch norm_kernel");
}

int launch_clip(const maddness_tensor *tensors, int64_t n, float max_norm, float *norm, bool given, double *partials, hipStream_t stream)
{
    int parts = 0, rc;
    note_kernel(given ? "clip_kernel" : "squares_kernel", nullptr);
    if (!given && (rc = launch_squares(tensors, n, partials, parts, stream)) != MADDNESS_OK) return rc;
    int64_t from = 0;
    do {
        const Table t = next_table(tensors, n, from, true);
        if (t.n == 0 && given) break;
        hipLaunchKernelGGL(clip_kernel, dim3(groups_of(t.n ? t.end[t.n - 1] : 0)), dim3(kThreads), 0, stream, t, partials, parts, norm, given, max_norm);
        if ((rc = check_hip(hipGetLastError(), "launch clip_kernel")) != MADDNESS_OK) return rc;
    } while (from < n);
    return MADDNESS_OK;
}

}  // namespace maddness

// The norm over many tensors, and their scaling by it.  Both move bytes: the squares are summed in fp64 beside the loads.
//
// The tensors' places go with the launch, as arguments of the kernel, so that a captured graph holds them too; so many tensors to a launch.
#include "lanes.h"
#include "layers_common.h"

namespace maddness {
namespace {

constexpr int kTensors = 96, kThreads = 256;
// Elements that a workgroup takes at a time: eight pieces of 8 to a thread, or one where the elements would otherwise leave compute units without work (a
// million in 4 tensors: norm and scaling 4.1 and 6.2 us with eight, 3.6 and 5.3 with one).
constexpr int kMany = 8;
constexpr int chunk_of(int pieces) { return kThreads * 8 * pieces; }

struct Table {
    const void *data[kTensors];
    void *out[kTensors];
    int64_t count[kTensors];
    uint32_t end[kTensors];             // chunks of the tensors up to and with this one
    uint8_t types[kTensors];            // of data + 4 times that of out
    int n;
};

// The tensor that a chunk belongs to, and the chunk's first element.
template <int PIECES>
__device__ __forceinline__ int tensor_of(const Table &t, uint32_t chunk, int64_t &first)
{
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (chunk < t.end[mid]) hi = mid;
        else lo = mid + 1;
    }
    first = (int64_t)(chunk - (lo ? t.end[lo - 1] : 0)) * chunk_of(PIECES);
    return lo;
}

// The sum over the workgroup's threads, in all of them.
__device__ __forceinline__ double group_sum(double x, double (&slots)[kThreads / 64])
{
    x = over_lanes<64>(x, plus);
    if (threadIdx.x % 64 == 0) slots[threadIdx.x / 64] = x;
    __syncthreads();
    x = slots[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) x += slots[w];
    return x;
}

// In two sums, as one addition in fp64 waits for the other.
template <int DT, int PIECES>
__device__ __forceinline__ void add_squares(const void *data, int64_t first, int64_t count, double (&sum)[2])
{
    if (first + chunk_of(PIECES) <= count) {
        Raw<DT> raw[PIECES];
#pragma unroll
        for (int p = 0; p < PIECES; ++p) raw[p] = load_raw<DT>(data, first, (int64_t)(p * kThreads + threadIdx.x) * 8, count);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            float v[8];
            widen<DT>(raw[p], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i % 2] = __builtin_fma((double)v[i], (double)v[i], sum[i % 2]);
        }
    } else {
        for (int64_t i = first + threadIdx.x; i < count; i += kThreads) {
            const double v = (double)widen_at<DT>(data, i);
            sum[0] = __builtin_fma(v, v, sum[0]);
        }
    }
}

// Sums of squares of a launch's tensors: to partials[workgroup], or in addition to what is there.
template <int PIECES>
__global__ __launch_bounds__(kThreads) void squares_kernel(Table t, double *partials, bool add)
{
    __shared__ double slots[kThreads / 64];
    double sums[2] = {};
    const uint32_t chunks = t.n ? t.end[t.n - 1] : 0;
    for (uint32_t chunk = blockIdx.x; chunk < chunks; chunk += gridDim.x) {
        int64_t first;
        const int i = tensor_of<PIECES>(t, chunk, first);
        switch (t.types[i] & 3) {
        case kF32: add_squares<kF32, PIECES>(t.data[i], first, t.count[i], sums); break;
        case kF16: add_squares<kF16, PIECES>(t.data[i], first, t.count[i], sums); break;
        default: add_squares<kBF16, PIECES>(t.data[i], first, t.count[i], sums);
        }
    }
    const double sum = group_sum(sums[0] + sums[1], slots);
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

// A whole chunk's pieces as they are in memory.
template <int PIECES>
struct Chunk {
    uint32_t w[PIECES][8];
};

template <int DT, int PIECES>
__device__ __forceinline__ void load_chunk(const void *data, int64_t first, int64_t count, Chunk<PIECES> &c)
{
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const Raw<DT> raw = load_raw<DT>(data, first, (int64_t)(p * kThreads + threadIdx.x) * 8, count);
#pragma unroll
        for (int i = 0; i < 2 * elem_size(DT); ++i) c.w[p][i] = raw.w[i];
    }
}

// (One piece has been asked for before the norm was known; of more the first to come is scaled while the others do.)
template <int DT, int OT, int PIECES>
__device__ __forceinline__ void scale_chunk(const Chunk<PIECES> &asked, bool whole, const void *data, void *out, int64_t first, int64_t count, float factor)
{
    if (whole) {
        Chunk<PIECES> c = asked;
        if constexpr (PIECES > 1) load_chunk<DT>(data, first, count, c);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            Raw<DT> raw;
#pragma unroll
            for (int i = 0; i < 2 * elem_size(DT); ++i) raw.w[i] = c.w[p][i];
            float v[8];
            widen<DT>(raw, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= factor;
            const int64_t at = first + (int64_t)(p * kThreads + threadIdx.x) * 8;
            store_run<OT>(out, at, v);
        }
    } else {
        for (int64_t i = first + threadIdx.x; i < count; i += kThreads) store_as<OT>(out, i, widen_at<DT>(data, i) * factor);
    }
}

// The chunk that a workgroup is at.
template <int PIECES>
struct Asked {
    Chunk<PIECES> pieces;
    int tensor;
    int64_t first, count;
    bool whole;
};

template <int PIECES>
__device__ __forceinline__ Asked<PIECES> ask(const Table &t, uint32_t chunk)
{
    Asked<PIECES> a;
    a.tensor = tensor_of<PIECES>(t, chunk, a.first);
    a.count = t.count[a.tensor];
    a.whole = a.first + chunk_of(PIECES) <= a.count;
    if (PIECES == 1 && a.whole) {
        switch (t.types[a.tensor] & 3) {
        case kF32: load_chunk<kF32>(t.data[a.tensor], a.first, a.count, a.pieces); break;
        case kF16: load_chunk<kF16>(t.data[a.tensor], a.first, a.count, a.pieces); break;
        default: load_chunk<kBF16>(t.data[a.tensor], a.first, a.count, a.pieces);
        }
    }
    return a;
}

// Scales a launch's tensors; the norm is that of the sums of squares, which every workgroup adds up for itself (16 KiB from L2) while its first chunk comes, or given.
template <int PIECES>
__global__ __launch_bounds__(kThreads) void clip_kernel(Table t, const double *partials, int parts, float *norm, bool given, float max_norm)
{
    __shared__ double slots[kThreads / 64];
    const uint32_t chunks = t.n ? t.end[t.n - 1] : 0;
    Asked<PIECES> now{};
    if (blockIdx.x < chunks) now = ask<PIECES>(t, chunks - 1 - blockIdx.x);      // (from the end: what the sums read last may still be in the memory-side cache)
    float all;
    if (given) {
        all = *norm;
    } else {
        all = norm_of(partials, parts, slots);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm = all;
    }
    const float factor = all > max_norm && all <= 3.402823466e38f ? (float)((double)max_norm / (double)all) : 1.0f;
    for (uint32_t turn = blockIdx.x; turn < chunks;) {
        const void *data = t.data[now.tensor];
        void *out = t.out[now.tensor];
        if (data != out || factor != 1.0f) {
            switch (t.types[now.tensor]) {
            case kF32 + 4 * kF32: scale_chunk<kF32, kF32>(now.pieces, now.whole, data, out, now.first, now.count, factor); break;
            case kF32 + 4 * kF16: scale_chunk<kF32, kF16>(now.pieces, now.whole, data, out, now.first, now.count, factor); break;
            case kF32 + 4 * kBF16: scale_chunk<kF32, kBF16>(now.pieces, now.whole, data, out, now.first, now.count, factor); break;
            case kF16 + 4 * kF32: scale_chunk<kF16, kF32>(now.pieces, now.whole, data, out, now.first, now.count, factor); break;
            case kF16 + 4 * kF16: scale_chunk<kF16, kF16>(now.pieces, now.whole, data, out, now.first, now.count, factor); break;
            case kF16 + 4 * kBF16: scale_chunk<kF16, kBF16>(now.pieces, now.whole, data, out, now.first, now.count, factor); break;
            case kBF16 + 4 * kF32: scale_chunk<kBF16, kF32>(now.pieces, now.whole, data, out, now.first, now.count, factor); break;
            case kBF16 + 4 * kF16: scale_chunk<kBF16, kF16>(now.pieces, now.whole, data, out, now.first, now.count, factor); break;
            default: scale_chunk<kBF16, kBF16>(now.pieces, now.whole, data, out, now.first, now.count, factor);
            }
        }
        turn += gridDim.x;
        if (turn < chunks) now = ask<PIECES>(t, chunks - 1 - turn);
    }
}

// The next tensors from `from` on that have elements, up to a launch's number of them and 2^32 - 1 chunks.
Table next_table(const maddness_tensor *tensors, int64_t n, int64_t chunk, int64_t &from, bool outs)
{
    Table t;
    t.n = 0;
    uint64_t chunks = 0;
    for (; from < n && t.n < kTensors; ++from) {
        const maddness_tensor &one = tensors[from];
        if (one.count == 0) continue;
        chunks += (uint64_t)ceil_div(one.count, chunk);
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

unsigned groups_of(uint64_t chunks) { return (unsigned)std::max<uint64_t>(1, std::min<uint64_t>(chunks, kNormPartials)); }

// How the tensors are cut: pieces to a thread, and chunks of that size in all.
struct Cut {
    int pieces;
    uint64_t chunks;
    Cut(const maddness_tensor *tensors, int64_t n)
    {
        uint64_t few = 0, many = 0;
        for (int64_t i = 0; i < n; ++i) {
            few += (uint64_t)ceil_div(tensors[i].count, (int64_t)chunk_of(1));
            many += (uint64_t)ceil_div(tensors[i].count, (int64_t)chunk_of(kMany));
        }
        pieces = few <= kNormPartials ? 1 : kMany;
        chunks = pieces == 1 ? few : many;
    }
};

// All sums of squares; how many of the partials hold them.
int launch_squares(const maddness_tensor *tensors, int64_t n, const Cut &cut, double *partials, int &parts, hipStream_t stream)
{
    parts = (int)groups_of(cut.chunks);
    int64_t from = 0;
    bool add = false;
    do {
        const Table t = next_table(tensors, n, chunk_of(cut.pieces), from, false);
        const auto kernel = cut.pieces == 1 ? squares_kernel<1> : squares_kernel<kMany>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)parts), dim3(kThreads), 0, stream, t, partials, add);
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
    const int rc = launch_squares(tensors, n, Cut(tensors, n), partials, parts, stream);
    if (rc != MADDNESS_OK) return rc;
    hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kThreads), 0, stream, partials, parts, norm);
    return check_hip(hipGetLastError(), "launch norm_kernel");
}

int launch_clip(const maddness_tensor *tensors, int64_t n, float max_norm, float *norm, bool given, double *partials, hipStream_t stream)
{
    const Cut cut(tensors, n);
    int parts = 0, rc;
    note_kernel(given ? "clip_kernel" : "squares_kernel", nullptr);
    if (!given && (rc = launch_squares(tensors, n, cut, partials, parts, stream)) != MADDNESS_OK) return rc;
    int64_t from = 0;
    do {
        const Table t = next_table(tensors, n, chunk_of(cut.pieces), from, true);
        if (t.n == 0 && given) break;
        const auto kernel = cut.pieces == 1 ? clip_kernel<1> : clip_kernel<kMany>;
        hipLaunchKernelGGL(kernel, dim3(groups_of(t.n ? t.end[t.n - 1] : 0)), dim3(kThreads), 0, stream, t, partials, parts, norm, given, max_norm);
        if ((rc = check_hip(hipGetLastError(), "launch clip_kernel")) != MADDNESS_OK) return rc;
    } while (from < n);
    return MADDNESS_OK;
}

}  // namespace maddness

// The norm over many tensors, and their scaling by it.  Both move bytes: the squares are summed in fp64 beside the loads.  201 million bfloat16 gradients: squares 111 us (3.6 TB/s behind a
// scaling whose results are still on their way to memory, 4.9 without), scaling to fp32 228 (5.3 TB/s).
//
// The tensors' places go with the launch, as arguments of the kernel, so that a captured graph holds them too; so many tensors to a launch.
#include "lanes.h"
#include "layers_common.h"

namespace maddness {
namespace {

constexpr int kThreads = 256;
// Tensors to a launch: a table of them is read anew by every launch, entry after entry of a search where it is long; a short one comes at once.
constexpr int kFewTensors = 8, kManyTensors = 96;
// Elements that a workgroup takes at a time: eight pieces of 8 to a thread, or one where the elements would otherwise leave compute units without work (a
// million in 4 tensors: norm and scaling 4.1 and 6.2 us with eight, 3.6 and 5.3 with one).
constexpr int kMany = 8;
constexpr int chunk_of(int pieces) { return kThreads * 8 * pieces; }

template <int N>
struct Table {
    const void *data[N];
    void *out[N];
    int64_t count[N];
    uint32_t end[N];                    // chunks of the tensors up to and with this one; of those that are not there, of all
    uint8_t types[N];                   // of data + 4 times that of out
    uint32_t chunks;
};

// The tensor that a chunk belongs to.
struct Entry {
    const void *data;
    void *out;
    int64_t count, first;               // its elements, and the chunk's first one
    int types;
};

template <int PIECES, int N>
__device__ __forceinline__ Entry entry_of(const Table<N> &t, uint32_t chunk)
{
    Entry e;
    uint32_t before;
    if constexpr (N == kFewTensors) {
        // (all of it in registers: no load waits for another)
        e = Entry{t.data[0], t.out[0], t.count[0], 0, t.types[0]};
        before = 0;
#pragma unroll
        for (int i = 1; i < N; ++i) {
            const bool later = chunk >= t.end[i - 1];
            const void *data = t.data[i];
            void *out = t.out[i];
            const int64_t count = t.count[i];
            const int types = t.types[i];
            e.data = later ? data : e.data;
            e.out = later ? out : e.out;
            e.count = later ? count : e.count;
            e.types = later ? types : e.types;
            before = later ? t.end[i - 1] : before;
        }
    } else {
        int lo = 0, hi = N - 1;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (chunk < t.end[mid]) hi = mid;
            else lo = mid + 1;
        }
        e = Entry{t.data[lo], t.out[lo], t.count[lo], 0, t.types[lo]};
        before = lo ? t.end[lo - 1] : 0;
    }
    e.first = (int64_t)(chunk - before) * chunk_of(PIECES);
    return e;
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
template <int PIECES, int N>
__global__ __launch_bounds__(kThreads) void squares_kernel(Table<N> t, double *partials, bool add)
{
    __shared__ double slots[kThreads / 64];
    double sums[2] = {};
    for (uint32_t chunk = blockIdx.x; chunk < t.chunks; chunk += gridDim.x) {
        const Entry e = entry_of<PIECES>(t, chunk);
        switch (e.types & 3) {
        case kF32: add_squares<kF32, PIECES>(e.data, e.first, e.count, sums); break;
        case kF16: add_squares<kF16, PIECES>(e.data, e.first, e.count, sums); break;
        default: add_squares<kBF16, PIECES>(e.data, e.first, e.count, sums);
        }
    }
    const double sum = group_sum(sums[0] + sums[1], slots);
    if (threadIdx.x == 0) partials[blockIdx.x] = add ? partials[blockIdx.x] + sum : sum;
}

__device__ __forceinline__ double norm_of(const double *partials, int parts, double (&slots)[kThreads / 64])
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += kThreads) sum += partials[i];
    return sqrt(group_sum(sum, slots));
}

__global__ __launch_bounds__(kThreads) void norm_kernel(const double *partials, int parts, float *norm)
{
    __shared__ double slots[kThreads / 64];
    const double all = norm_of(partials, parts, slots);
    if (threadIdx.x == 0) *norm = (float)all;
}

// Eight elements as they are in memory, of a narrow type in the first half.
struct Piece {
    i32x4 lo, hi;
};

template <int DT>
__device__ __forceinline__ Piece load_piece(const void *data, int64_t at)
{
    using words = __attribute__((ext_vector_type(4), aligned(elem_size(DT)))) int;
    const words *from = reinterpret_cast<const words *>(static_cast<const char *>(data) + at * elem_size(DT));
    if constexpr (DT == kF32) return Piece{from[0], from[1]};
    else return Piece{from[0], i32x4{}};
}

template <int DT, int OT>
__device__ __forceinline__ void scale_piece(const Piece &piece, void *out, int64_t at, float factor)
{
    Raw<DT> raw;
#pragma unroll
    for (int i = 0; i < 2 * elem_size(DT); ++i) raw.w[i] = (uint32_t)(i < 4 ? piece.lo[i] : piece.hi[i % 4]);
    float v[8];
    widen<DT>(raw, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= factor;
    store_run<OT>(out, at, v);
}

// (One piece has been asked for before the norm was known.)
template <int DT, int OT, int PIECES>
__device__ __forceinline__ void scale_chunk(const Piece &asked, bool whole, const Entry &e, float factor)
{
    if (whole) {
        const int64_t at = e.first + (int64_t)threadIdx.x * 8;
        if constexpr (PIECES == 1) {
            scale_piece<DT, OT>(asked, e.out, at, factor);
        } else {
            Piece pieces[PIECES];
#pragma unroll
            for (int p = 0; p < PIECES; ++p) pieces[p] = load_piece<DT>(e.data, at + p * kThreads * 8);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) scale_piece<DT, OT>(pieces[p], e.out, at + p * kThreads * 8, factor);
        }
    } else {
        for (int64_t i = e.first + threadIdx.x; i < e.count; i += kThreads) store_as<OT>(e.out, i, widen_at<DT>(e.data, i) * factor);
    }
}

// Scales a launch's tensors; the norm is that of the sums of squares, which every workgroup adds up for itself (16 KiB from L2) while its first chunk comes, or given.
template <int PIECES, int N>
__global__ __launch_bounds__(kThreads) void clip_kernel(Table<N> t, const double *partials, int parts, float *norm, bool given, float max_norm)
{
    __shared__ double slots[kThreads / 64];
    Piece asked{};
    Entry now{};
    bool whole = false;
    auto turn_to = [&](uint32_t chunk) INLINE_LAMBDA {
        now = entry_of<PIECES>(t, chunk);
        whole = now.first + chunk_of(PIECES) <= now.count;
        if (PIECES == 1 && whole) {
            const int64_t at = now.first + (int64_t)threadIdx.x * 8;
            if ((now.types & 3) == kF32) asked = load_piece<kF32>(now.data, at);
            else asked = load_piece<kF16>(now.data, at);      // (bits, of either narrow type)
        }
    };
    if (blockIdx.x < t.chunks) turn_to(blockIdx.x);
    double all;
    if (given) {
        all = (double)*norm;
    } else {
        all = norm_of(partials, parts, slots);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)all;
    }
    // (of the norm as it was summed: rounded first it would put half a step more on every element)
    const float factor = all > (double)max_norm && (float)all <= 3.402823466e38f ? (float)((double)max_norm / all) : 1.0f;
    for (uint32_t chunk = blockIdx.x; chunk < t.chunks;) {
        if (now.data != now.out || factor != 1.0f) {
            switch (now.types) {
            case kF32 + 4 * kF32: scale_chunk<kF32, kF32, PIECES>(asked, whole, now, factor); break;
            case kF32 + 4 * kF16: scale_chunk<kF32, kF16, PIECES>(asked, whole, now, factor); break;
            case kF32 + 4 * kBF16: scale_chunk<kF32, kBF16, PIECES>(asked, whole, now, factor); break;
            case kF16 + 4 * kF32: scale_chunk<kF16, kF32, PIECES>(asked, whole, now, factor); break;
            case kF16 + 4 * kF16: scale_chunk<kF16, kF16, PIECES>(asked, whole, now, factor); break;
            case kF16 + 4 * kBF16: scale_chunk<kF16, kBF16, PIECES>(asked, whole, now, factor); break;
            case kBF16 + 4 * kF32: scale_chunk<kBF16, kF32, PIECES>(asked, whole, now, factor); break;
            case kBF16 + 4 * kF16: scale_chunk<kBF16, kF16, PIECES>(asked, whole, now, factor); break;
            default: scale_chunk<kBF16, kBF16, PIECES>(asked, whole, now, factor);
            }
        }
        chunk += gridDim.x;
        if (chunk < t.chunks) turn_to(chunk);
    }
}

// The next tensors from `from` on that have elements, up to a table's number of them and 2^32 - 1 chunks.
template <int N>
Table<N> next_table(const maddness_tensor *tensors, int64_t n, int64_t chunk, int64_t &from, bool outs)
{
    Table<N> t{};
    uint64_t chunks = 0;
    int entries = 0;
    for (; from < n && entries < N; ++from) {
        const maddness_tensor &one = tensors[from];
        if (one.count == 0) continue;
        const uint64_t more = (uint64_t)ceil_div(one.count, chunk);
        if (chunks + more > 0xffffffffu) break;
        chunks += more;
        t.data[entries] = one.data;
        t.out[entries] = outs ? one.out : nullptr;
        t.count[entries] = one.count;
        t.end[entries] = (uint32_t)chunks;
        t.types[entries] = (uint8_t)(one.dtype + 4 * (outs ? one.out_dtype : 0));
        ++entries;
    }
    for (; entries < N; ++entries) t.end[entries] = (uint32_t)chunks;
    t.chunks = (uint32_t)chunks;
    return t;
}

unsigned groups_of(uint64_t chunks) { return (unsigned)std::max<uint64_t>(1, std::min<uint64_t>(chunks, kNormPartials)); }

// How the tensors are cut: pieces to a thread, chunks of that size in all, and whether a short table holds them.
struct Cut {
    int pieces;
    uint64_t chunks;
    bool few_tensors;
    Cut(const maddness_tensor *tensors, int64_t n)
    {
        uint64_t few = 0, many = 0;
        for (int64_t i = 0; i < n; ++i) {
            few += (uint64_t)ceil_div(tensors[i].count, (int64_t)chunk_of(1));
            many += (uint64_t)ceil_div(tensors[i].count, (int64_t)chunk_of(kMany));
        }
        pieces = few <= kNormPartials ? 1 : kMany;
        chunks = pieces == 1 ? few : many;
        few_tensors = n <= kFewTensors;
    }
};

// Calls f with a table after the other: at least once.  (Only who has launched something asks for errors: an older call's may be waiting.)
template <int N, typename F>
int for_tables(const maddness_tensor *tensors, int64_t n, int pieces, bool outs, F f)
{
    int64_t from = 0;
    do {
        const Table<N> t = next_table<N>(tensors, n, chunk_of(pieces), from, outs);
        const int rc = f(t);
        if (rc != MADDNESS_OK) return rc;
    } while (from < n);
    return MADDNESS_OK;
}

template <int PIECES, int N>
int launch_squares_as(const maddness_tensor *tensors, int64_t n, double *partials, int parts, hipStream_t stream)
{
    bool add = false;
    return for_tables<N>(tensors, n, PIECES, false, [&](const Table<N> &t) {
        hipLaunchKernelGGL((squares_kernel<PIECES, N>), dim3((unsigned)parts), dim3(kThreads), 0, stream, t, partials, add);
        add = true;
        return check_hip(hipGetLastError(), "launch squares_kernel");
    });
}

template <int PIECES, int N>
int launch_clip_as(const maddness_tensor *tensors, int64_t n, const double *partials, int parts, float *norm, bool given, float max_norm, hipStream_t stream)
{
    return for_tables<N>(tensors, n, PIECES, true, [&](const Table<N> &t) {
        if (t.chunks == 0 && given) return (int)MADDNESS_OK;
        hipLaunchKernelGGL((clip_kernel<PIECES, N>), dim3(groups_of(t.chunks)), dim3(kThreads), 0, stream, t, partials, parts, norm, given, max_norm);
        return check_hip(hipGetLastError(), "launch clip_kernel");
    });
}

// All sums of squares; how many of the partials hold them.
int launch_squares(const maddness_tensor *tensors, int64_t n, const Cut &cut, double *partials, int &parts, hipStream_t stream)
{
    parts = (int)groups_of(cut.chunks);
    if (cut.few_tensors) {
        if (cut.pieces == 1) return launch_squares_as<1, kFewTensors>(tensors, n, partials, parts, stream);
        return launch_squares_as<kMany, kFewTensors>(tensors, n, partials, parts, stream);
    }
    if (cut.pieces == 1) return launch_squares_as<1, kManyTensors>(tensors, n, partials, parts, stream);
    return launch_squares_as<kMany, kManyTensors>(tensors, n, partials, parts, stream);
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
    if (cut.few_tensors) {
        if (cut.pieces == 1) return launch_clip_as<1, kFewTensors>(tensors, n, partials, parts, norm, given, max_norm, stream);
        return launch_clip_as<kMany, kFewTensors>(tensors, n, partials, parts, norm, given, max_norm, stream);
    }
    if (cut.pieces == 1) return launch_clip_as<1, kManyTensors>(tensors, n, partials, parts, norm, given, max_norm, stream);
    return launch_clip_as<kMany, kManyTensors>(tensors, n, partials, parts, norm, given, max_norm, stream);
}

}  // namespace maddness

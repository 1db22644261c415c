// The 2-norm of many gradients together, and clipping to it (include/placeto.h).
//
// Two passes over the gradients: the sum of squares, then the product with max_norm / norm; the second goes from the last
// chunk to the first, so that what the first has read last is found in the caches.  Bound by memory (two reads and a
// write).  The tensors come as a table by value, or as a list that is made of such tables first: a call needs nothing on
// the device that a captured graph or another stream could find changed.  (A pair of launches to a table of 128 tensors
// instead, 291 of them: 270 us; with the list 250.)
#include <algorithm>

#include "elements.h"
#include "losses.h"

namespace pl {
namespace {

struct Chunk {
    const void *src;
    void *dst;
    int n, dtype;
};

// The last tensor that begins at or in front of a chunk.  (Tensors without elements are not among them.)
__device__ __forceinline__ int tensor_of(const int32_t *first, int n, int chunk)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= chunk) lo = mid; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ Chunk chunk_of(const void *src, void *dst, int64_t numel, int dtype, int64_t at, int most)
{
    const int64_t bytes = at * (dtype == PL_F32 ? 4 : 2);
    return {static_cast<const char *>(src) + bytes, static_cast<char *>(dst) + bytes,
            static_cast<int>(min(static_cast<int64_t>(most), numel - at)), dtype};
}

// Chunks of a table, and of a list: the latter's offsets are searched in LDS where they fit.
struct TableChunks {
    const ClipTable &t;
    __device__ explicit TableChunks(const ClipTable &t) : t(t) {}
    __device__ int count() const { return t.first[t.n]; }
    __device__ Chunk operator()(int c) const
    {
        const int i = tensor_of(t.first, t.n, c);
        return chunk_of(t.src[i], t.dst[i], t.numel[i], t.dtype[i], static_cast<int64_t>(c - t.first[i]) * t.chunk, t.chunk);
    }
};
constexpr int kListInLds = 4096;
struct ListChunks {
    const ClipList &t;
    const int32_t *first;
    __device__ explicit ListChunks(const ClipList &t) : t(t), first(t.first)
    {
        __shared__ int32_t copy[kListInLds];
        if (t.n <= kListInLds) {
            for (int i = threadIdx.x; i < t.n; i += blockDim.x) copy[i] = t.first[i];
            __syncthreads();
            first = copy;
        }
    }
    __device__ int count() const { return t.chunks; }
    __device__ Chunk operator()(int c) const
    {
        const int i = tensor_of(first, t.n, c);
        const ClipTensor x = t.tensors[i];
        return chunk_of(x.src, x.dst, x.numel, static_cast<int>(x.dtype), static_cast<int64_t>(c - first[i]) * t.chunk, t.chunk);
    }
};
__device__ __forceinline__ TableChunks chunks_of(const ClipTable &t) { return TableChunks(t); }
__device__ __forceinline__ ListChunks chunks_of(const ClipList &t) { return ListChunks(t); }

// Squares of a slot in float64.
template <int N>
__device__ __forceinline__ double slot_squares(const float (&f)[N])
{
    double d = 0.0;
#pragma unroll
    for (int k = 0; k < N; ++k) d = __builtin_fma(static_cast<double>(f[k]), static_cast<double>(f[k]), d);
    return d;
}

// (kAhead loads of a thread are on their way together)
constexpr int kAhead = 4;

template <typename T, int THREADS>
__device__ __forceinline__ double chunk_squares(const Chunk &c)
{
    constexpr int N = Elem<T>::N;
    const Span<T> span(static_cast<const T *>(c.src), c.n);
    double a = 0.0;
    for (int i = threadIdx.x; i < span.whole; i += kAhead * THREADS) {
        uint4 v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) v[k] = span.load(i + k * THREADS);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k * THREADS < span.whole) {
                float f[N];
                Elem<T>::unpack(v[k], f);
                a += slot_squares<N>(f);
            }
    }
    if (const int e = span.edge(threadIdx.x); e >= 0) {
        const float f[1] = {Elem<T>::load(span.p + e)};
        a += slot_squares<1>(f);
    }
    return a;
}

template <int THREADS>
__device__ __forceinline__ double squares_of(const Chunk &c)
{
    return c.dtype == PL_BF16 ? chunk_squares<__bf16, THREADS>(c)
                              : c.dtype == PL_F16 ? chunk_squares<_Float16, THREADS>(c) : chunk_squares<float, THREADS>(c);
}

// Sum over the workgroup, known to all of its threads.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double wave[THREADS / 64];
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) v += wave[i];
    return v;
}

// max_norm / norm = m 2^e: the quotient of a tiny limit and a huge norm is no fp32 number, its products are.  One for a norm that
// is reported as infinite or NaN.
struct Factor {
    float m;
    int e;
    __device__ bool is_one() const { return m == 1.0f && e == 0; }
};

__device__ __forceinline__ Factor factor_of(double norm, float max_norm)
{
    Factor f{1.0f, 0};
    if (norm > max_norm && static_cast<float>(norm) < INFINITY) f.m = static_cast<float>(frexp(max_norm / norm, &f.e));
    return f;
}

template <typename T, int THREADS>
__device__ __forceinline__ void chunk_scale(const Chunk &c, const Factor &by)
{
    constexpr int N = Span<T>::N;
    const Span<T> span(static_cast<const T *>(c.src), c.n);
    T *o = static_cast<T *>(c.dst);
    if (by.is_one() && o == span.p) return;
    for (int i = threadIdx.x; i < span.whole; i += kAhead * THREADS) {
        uint4 v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) v[k] = span.load(i + k * THREADS);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k * THREADS < span.whole) {
                if (!by.is_one()) {
                    float f[N];
                    Elem<T>::unpack(v[k], f);
#pragma unroll
                    for (int j = 0; j < N; ++j) f[j] = ldexpf(f[j] * by.m, by.e);
                    v[k] = Elem<T>::pack(f);
                }
                stream_16(o + span.head + static_cast<uint32_t>(i + k * THREADS) * N, v[k]);
            }
    }
    if (const int e = span.edge(threadIdx.x); e >= 0) {
        const float f = Elem<T>::load(span.p + e);
        Elem<T>::store(o + e, by.is_one() ? f : ldexpf(f * by.m, by.e));
    }
}

template <int THREADS>
__device__ __forceinline__ void scale_chunk(const Chunk &c, const Factor &by)
{
    if (c.dtype == PL_BF16) chunk_scale<__bf16, THREADS>(c, by);
    else if (c.dtype == PL_F16) chunk_scale<_Float16, THREADS>(c, by);
    else chunk_scale<float, THREADS>(c, by);
}

template <typename Tensors>
__global__ __launch_bounds__(256) void k_clip_sums(Tensors t, double *__restrict__ sums)
{
    const auto chunks = chunks_of(t);
    double a = 0.0;
    for (int i = blockIdx.x; i < chunks.count(); i += gridDim.x) a += squares_of<256>(chunks(i));
    a = block_sum<256>(a);
    if (threadIdx.x == 0) sums[blockIdx.x] = a;
}

// The norm from the workgroups' sums, in an order that depends on their number alone.
__device__ __forceinline__ double norm_of(const double *__restrict__ sums, int n)
{
    double a = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) a += sums[i];
    return sqrt(block_sum<256>(a));
}

__global__ __launch_bounds__(256) void k_clip_norm(const double *__restrict__ sums, int n, float *__restrict__ out_norm)
{
    const double norm = norm_of(sums, n);
    if (threadIdx.x == 0) *out_norm = static_cast<float>(norm);
}

// Every workgroup takes the norm from the sums: 8 KiB out of the caches, instead of one more launch.
template <typename Tensors>
__global__ __launch_bounds__(256) void k_clip_scale(Tensors t, const double *__restrict__ sums, int n, float max_norm,
                                                    float *__restrict__ out_norm)
{
    const double norm = norm_of(sums, n);
    if (blockIdx.x == 0 && threadIdx.x == 0) *out_norm = static_cast<float>(norm);
    const Factor by = factor_of(norm, max_norm);
    const auto chunks = chunks_of(t);
    for (int i = chunks.count() - 1 - blockIdx.x; i >= 0; i -= gridDim.x) scale_chunk<256>(chunks(i), by);
}

// Everything in one launch by one workgroup.
__global__ __launch_bounds__(1024) void k_clip_small(ClipTable t, float max_norm, float *__restrict__ out_norm)
{
    const TableChunks chunks(t);
    double a = 0.0;
    for (int i = 0; i < chunks.count(); ++i) a += squares_of<1024>(chunks(i));
    const double norm = sqrt(block_sum<1024>(a));
    if (threadIdx.x == 0) *out_norm = static_cast<float>(norm);
    const Factor by = factor_of(norm, max_norm);
    for (int i = chunks.count() - 1; i >= 0; --i) scale_chunk<1024>(chunks(i), by);
}

__global__ __launch_bounds__(kClipTensors) void k_clip_list(ClipTable t, ClipList list, int at)
{
    const int i = threadIdx.x;
    if (i < t.n) {
        list.tensors[at + i] = {t.src[i], t.dst[i], t.numel[i], t.dtype[i]};
        list.first[at + i] = t.first[i];
    }
    if (i == 0) list.first[at + t.n] = t.first[t.n];
}

}  // namespace

void launch_clip_list(const ClipTable &t, const ClipList &list, int at, hipStream_t s)
{
    hipLaunchKernelGGL(k_clip_list, dim3(1), dim3(kClipTensors), 0, s, t, list, at);
}

template <typename Tensors>
void launch_clip(const Tensors &t, int64_t chunks, double *sums, float max_norm, bool scales, float *out_norm, hipStream_t s)
{
    const int blocks = static_cast<int>(std::min<int64_t>(chunks, kClipBlocks));
    if (blocks) hipLaunchKernelGGL(k_clip_sums<Tensors>, dim3(blocks), dim3(256), 0, s, t, sums);
    if (blocks && scales)
        hipLaunchKernelGGL(k_clip_scale<Tensors>, dim3(blocks), dim3(256), 0, s, t, sums, blocks, max_norm, out_norm);
    else
        hipLaunchKernelGGL(k_clip_norm, dim3(1), dim3(256), 0, s, sums, blocks, out_norm);
}
template void launch_clip(const ClipTable &, int64_t, double *, float, bool, float *, hipStream_t);
template void launch_clip(const ClipList &, int64_t, double *, float, bool, float *, hipStream_t);

void launch_clip_small(const ClipTable &t, float max_norm, float *out_norm, hipStream_t s)
{
    hipLaunchKernelGGL(k_clip_small, dim3(1), dim3(1024), 0, s, t, max_norm, out_norm);
}

}  // namespace pl

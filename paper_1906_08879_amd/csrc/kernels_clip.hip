// The 2-norm of many gradients together, and clipping to it (include/placeto.h).
//
// Two passes over the gradients: the sum of squares, then the product with max_norm / norm; the second goes from the last
// chunk to the first, so that what the first has read last is found in the caches.  Bound by memory (two reads and a
// write).  The tensors come as a table by value, so that a call needs nothing on the device that a captured graph or
// another stream could find changed.
#include <algorithm>

#include "elements.h"
#include "losses.h"

namespace pl {
namespace {

struct Chunk {
    int tensor, n;
    int64_t at;
};

// Chunk c of a table: the last tensor that begins at or in front of it.  (A tensor without elements is not in the table.)
__device__ __forceinline__ Chunk chunk_at(const ClipTable &t, int c)
{
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid; else hi = mid;
    }
    const int64_t at = static_cast<int64_t>(c - t.first[lo]) * t.chunk;
    return {lo, static_cast<int>(min(static_cast<int64_t>(t.chunk), t.numel[lo] - at)), at};
}

// Squares of a slot: in fp32 where their sum is well within its range, which all but wild or vanished gradients are (one
// conversion to a slot instead of one to an element, which took longer than the elements' bytes), else in float64.
template <int N>
__device__ __forceinline__ double slot_squares(const float (&f)[N])
{
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k) s = __builtin_fmaf(f[k], f[k], s);
    if (s > 0x1p-90f && s < 0x1p120f) return s;
    double d = 0.0;
#pragma unroll
    for (int k = 0; k < N; ++k) d = __builtin_fma(static_cast<double>(f[k]), static_cast<double>(f[k]), d);
    return d;
}

// (kAhead loads of a thread are on their way together)
constexpr int kAhead = 4;

template <typename T, int THREADS>
__device__ __forceinline__ double chunk_squares(const ClipTable &t, const Chunk &c)
{
    constexpr int N = Elem<T>::N;
    const Span<T> span(static_cast<const T *>(t.src[c.tensor]) + c.at, c.n);
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
__device__ __forceinline__ double squares_of(const ClipTable &t, int chunk)
{
    const Chunk c = chunk_at(t, chunk);
    const int dtype = t.dtype[c.tensor];
    return dtype == PL_BF16 ? chunk_squares<__bf16, THREADS>(t, c)
                            : dtype == PL_F16 ? chunk_squares<_Float16, THREADS>(t, c) : chunk_squares<float, THREADS>(t, c);
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

// max_norm / norm = m 2^e: the quotient of a tiny limit and a huge norm is no fp32 number, its products are.
struct Factor {
    float m;
    int e;
    __device__ bool is_one() const { return m == 1.0f && e == 0; }
};

__device__ __forceinline__ Factor factor_of(double norm, float max_norm)
{
    Factor f{1.0f, 0};
    if (norm > max_norm && norm < INFINITY) f.m = static_cast<float>(frexp(max_norm / norm, &f.e));
    return f;
}

template <typename T, int THREADS>
__device__ __forceinline__ void chunk_scale(const ClipTable &t, const Chunk &c, const Factor &by)
{
    constexpr int N = Span<T>::N;
    const Span<T> span(static_cast<const T *>(t.src[c.tensor]) + c.at, c.n);
    T *o = static_cast<T *>(t.dst[c.tensor]) + c.at;
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
__device__ __forceinline__ void scale_chunk(const ClipTable &t, int chunk, const Factor &by)
{
    const Chunk c = chunk_at(t, chunk);
    const int dtype = t.dtype[c.tensor];
    if (dtype == PL_BF16) chunk_scale<__bf16, THREADS>(t, c, by);
    else if (dtype == PL_F16) chunk_scale<_Float16, THREADS>(t, c, by);
    else chunk_scale<float, THREADS>(t, c, by);
}

__global__ __launch_bounds__(256) void k_clip_sums(ClipTable t, double *__restrict__ sums)
{
    double a = 0.0;
    for (int i = blockIdx.x; i < t.first[t.n]; i += gridDim.x) a += squares_of<256>(t, i);
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
__global__ __launch_bounds__(256) void k_clip_scale(ClipTable t, const double *__restrict__ sums, int n, float max_norm,
                                                    float *__restrict__ out_norm)
{
    const double norm = norm_of(sums, n);
    if (out_norm && blockIdx.x == 0 && threadIdx.x == 0) *out_norm = static_cast<float>(norm);
    const Factor by = factor_of(norm, max_norm);
    for (int i = t.first[t.n] - 1 - blockIdx.x; i >= 0; i -= gridDim.x) scale_chunk<256>(t, i, by);
}

// Everything in one launch by one workgroup.
__global__ __launch_bounds__(1024) void k_clip_small(ClipTable t, float max_norm, float *__restrict__ out_norm)
{
    double a = 0.0;
    for (int i = 0; i < t.first[t.n]; ++i) a += squares_of<1024>(t, i);
    const double norm = sqrt(block_sum<1024>(a));
    if (threadIdx.x == 0) *out_norm = static_cast<float>(norm);
    const Factor by = factor_of(norm, max_norm);
    for (int i = t.first[t.n] - 1; i >= 0; --i) scale_chunk<1024>(t, i, by);
}

}  // namespace

int clip_blocks(const ClipTable &t) { return std::min(t.first[t.n], kClipBlocks); }

void launch_clip_sums(const ClipTable &t, double *sums, hipStream_t s)
{
    if (clip_blocks(t)) hipLaunchKernelGGL(k_clip_sums, dim3(clip_blocks(t)), dim3(256), 0, s, t, sums);
}

void launch_clip_norm(const double *sums, int n_sums, float *out_norm, hipStream_t s)
{
    hipLaunchKernelGGL(k_clip_norm, dim3(1), dim3(256), 0, s, sums, n_sums, out_norm);
}

void launch_clip_scale(const ClipTable &t, const double *sums, int n_sums, float max_norm, float *out_norm, hipStream_t s)
{
    if (clip_blocks(t))
        hipLaunchKernelGGL(k_clip_scale, dim3(clip_blocks(t)), dim3(256), 0, s, t, sums, n_sums, max_norm, out_norm);
}

void launch_clip_small(const ClipTable &t, float max_norm, float *out_norm, hipStream_t s)
{
    hipLaunchKernelGGL(k_clip_small, dim3(1), dim3(1024), 0, s, t, max_norm, out_norm);
}

}  // namespace pl

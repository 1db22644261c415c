// The 2-norm of many gradients together, and clipping to it (include/placeto.h).
//
// Two passes over the gradients: squares summed in float64 (the square of any gradient fits, and
// the conversions and fused multiply-adds of an element cost less than its bytes), then the product with
// max_norm / norm.  The tensors come as a table by value, so that a call needs nothing on the device
// that a captured graph or another stream could find changed.
#include <algorithm>

#include "elements.h"
#include "losses.h"

namespace pl {
namespace {

struct Chunk {
    int tensor;
    int64_t at;
    int n;
};

// Chunk c of a table: the last tensor that begins at or in front of it.  (A tensor without elements has no chunk.)
__device__ __forceinline__ Chunk chunk_at(const ClipTable &t, int c)
{
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid; else hi = mid;
    }
    const int64_t at = static_cast<int64_t>(c - t.first[lo]) * kClipChunk;
    return {lo, at, static_cast<int>(min(kClipChunk, t.numel[lo] - at))};
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const ClipTable &t, const Chunk &c)
{
    constexpr int N = Elem<T>::N;
    const Row<T> row(static_cast<const T *>(t.src[c.tensor]) + c.at, 0, 0, c.n);
    double a = 0.0;
    for (int i = threadIdx.x; i < row.slots; i += 256) {
        float f[N];
        row.load(i, f, 0.0f);
#pragma unroll
        for (int k = 0; k < N; ++k) a = __builtin_fma(static_cast<double>(f[k]), static_cast<double>(f[k]), a);
    }
    return a;
}

__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double wave[4];
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = v;
    __syncthreads();
    return wave[0] + wave[1] + wave[2] + wave[3];
}

// max_norm / norm as mantissa and exponent: the quotient of a tiny limit and a huge norm is no fp32 number, its products are.
__device__ __forceinline__ ClipFactor factor_of(double norm, float max_norm)
{
    ClipFactor f{1.0f, 0};
    if (norm > max_norm && norm < INFINITY) {
        int e;
        f.m = static_cast<float>(frexp(max_norm / norm, &e));
        f.e = e;
    }
    return f;
}

__global__ __launch_bounds__(256) void k_clip_sums(ClipTable t, double *__restrict__ sums)
{
    double a = 0.0;
    for (int i = blockIdx.x; i < t.first[t.n]; i += gridDim.x) {
        const Chunk c = chunk_at(t, i);
        const int dtype = t.dtype[c.tensor];
        a += dtype == PL_BF16 ? chunk_squares<__bf16>(t, c) : dtype == PL_F16 ? chunk_squares<_Float16>(t, c) : chunk_squares<float>(t, c);
    }
    a = block_sum(a);
    if (threadIdx.x == 0) sums[blockIdx.x] = a;
}

__global__ __launch_bounds__(256) void k_clip_norm(const double *__restrict__ sums, int n, float max_norm, float *__restrict__ out_norm,
                                                   ClipFactor *__restrict__ factor)
{
    double a = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) a += sums[i];
    const double norm = sqrt(block_sum(a));
    if (threadIdx.x == 0) {
        *out_norm = static_cast<float>(norm);
        *factor = factor_of(norm, max_norm);
    }
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const ClipTable &t, const Chunk &c, ClipFactor by)
{
    constexpr int N = Elem<T>::N;
    const Row<T> row(static_cast<const T *>(t.src[c.tensor]) + c.at, 0, 0, c.n);
    T *o = static_cast<T *>(t.dst[c.tensor]) + c.at;
    const bool as_is = by.m == 1.0f && by.e == 0;
    if (as_is && o == row.p) return;
    for (int i = threadIdx.x; i < row.slots; i += 256) {
        float f[N];
        row.load(i, f, 0.0f);
        if (!as_is) {
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = ldexpf(f[k] * by.m, by.e);
        }
        store_slot(o, row.first(i), c.n, f);
    }
}

__global__ __launch_bounds__(256) void k_clip_scale(ClipTable t, const ClipFactor *__restrict__ factor)
{
    const ClipFactor f = *factor;
    for (int i = blockIdx.x; i < t.first[t.n]; i += gridDim.x) {
        const Chunk c = chunk_at(t, i);
        const int dtype = t.dtype[c.tensor];
        if (dtype == PL_BF16) chunk_scale<__bf16>(t, c, f);
        else if (dtype == PL_F16) chunk_scale<_Float16>(t, c, f);
        else chunk_scale<float>(t, c, f);
    }
}

}  // namespace

int clip_blocks(const ClipTable &t) { return std::min(t.first[t.n], kClipBlocks); }

void launch_clip_sums(const ClipTable &t, double *sums, hipStream_t s)
{
    if (clip_blocks(t)) hipLaunchKernelGGL(k_clip_sums, dim3(clip_blocks(t)), dim3(256), 0, s, t, sums);
}

void launch_clip_norm(const double *sums, int n_sums, float max_norm, float *out_norm, ClipFactor *factor, hipStream_t s)
{
    hipLaunchKernelGGL(k_clip_norm, dim3(1), dim3(256), 0, s, sums, n_sums, max_norm, out_norm, factor);
}

void launch_clip_scale(const ClipTable &t, const ClipFactor *factor, hipStream_t s)
{
    if (clip_blocks(t)) hipLaunchKernelGGL(k_clip_scale, dim3(clip_blocks(t)), dim3(256), 0, s, t, factor);
}

}  // namespace pl

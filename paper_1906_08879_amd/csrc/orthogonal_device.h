// What the kernels of the orthogonalised update share: matrices by groups of four elements of a row, and the direction.
#pragma once
#include "elements.h"
#include "orthogonal.h"

namespace pl {
namespace {

template <typename F>
__device__ __forceinline__ void for_type(int dtype, F f)
{
    if (dtype == PL_F32) f(float{});
    else if (dtype == PL_BF16) f(__bf16{});
    else f(_Float16{});
}

// Four elements of a row side by side, aligned to one of them, of which `left` are there.
template <typename T>
struct Four {
    typedef T vector __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};

template <typename T>
__device__ __forceinline__ void load_group(const void *p, int64_t at, int left, float (&v)[4])
{
    const T *from = static_cast<const T *>(p) + at;
    if (left >= 4) {
        const typename Four<T>::vector x = *reinterpret_cast<const typename Four<T>::vector *>(from);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = static_cast<float>(x[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < left ? static_cast<float>(from[e]) : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store_group(void *p, int64_t at, int left, const float (&v)[4])
{
    T *to = static_cast<T *>(p) + at;
    if (left >= 4) {
        typename Four<T>::vector x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = static_cast<T>(v[e]);
        *reinterpret_cast<typename Four<T>::vector *>(to) = x;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) to[e] = static_cast<T>(v[e]);
    }
}

// What is orthogonalised, from the new momentum and the gradient.
__device__ __forceinline__ float direction(const OrthCfg &cfg, bool momentum, float m, float g)
{
    if (!momentum) return g;
    return cfg.nesterov ? g + cfg.beta * m : m;
}

}  // namespace
}  // namespace pl

// Elements of the types that losses and gradients come in, 16 bytes at a time.
#pragma once
#include <cmath>
#include <cstdint>

#include "internal.h"

namespace pl {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));

typedef short shortx2 __attribute__((ext_vector_type(2)));
typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));

// Two 16-bit elements of a word side by side.
__device__ __forceinline__ uint32_t more_of_two(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(shortx2, a), __builtin_bit_cast(shortx2, b)));
}

__device__ __forceinline__ uint32_t less_of_two(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(ushortx2, a), __builtin_bit_cast(ushortx2, b)));
}
__device__ __forceinline__ uint32_t largest_of_two(uint32_t most, uint32_t least)
{
    return ((most & 0x8000u ? least : most) & 0xffffu) | ((most & 0x80000000u ? least : most) & 0xffff0000u);
}

template <typename T>
struct Elem;
template <>
struct Elem<float> {
    static constexpr int N = 4;        // elements of 16 bytes
    static __device__ void unpack(const uint4 &v, float (&f)[4])
    {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    static __device__ uint4 pack(const float (&f)[4])
    {
        return {__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
    }
    // The largest of values among which one is not negative has the largest bits as a signed number, the largest of
    // negative ones the least as an unsigned number: a word's worth of elements with an integer instruction each.
    static constexpr uint32_t kNone = 0x80000000u;       // `more` of nothing; `less` of nothing is 0xffffffff, a NaN
    static __device__ uint32_t more(uint32_t a, uint32_t b) { return static_cast<uint32_t>(max(static_cast<int32_t>(a), static_cast<int32_t>(b))); }
    static __device__ uint32_t less(uint32_t a, uint32_t b) { return min(a, b); }
    static __device__ float largest(uint32_t most, uint32_t least)
    {
        return __uint_as_float(static_cast<int32_t>(most) < 0 ? least : most);
    }
    static __device__ float load(const float *p) { return *p; }
    static __device__ void store(float *p, float f) { *p = f; }
};
template <>
struct Elem<__bf16> {
    static constexpr int N = 8;
    static __device__ void unpack(const uint4 &v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ uint4 pack(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){f[2 * i], f[2 * i + 1]}, bf16x2));
        return {w[0], w[1], w[2], w[3]};
    }
    static constexpr uint32_t kNone = 0x80008000u;
    static __device__ uint32_t more(uint32_t a, uint32_t b) { return more_of_two(a, b); }
    static __device__ uint32_t less(uint32_t a, uint32_t b) { return less_of_two(a, b); }
    static __device__ float largest(uint32_t most, uint32_t least)
    {
        const uint32_t a = largest_of_two(most, least);
        return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
    }
    static __device__ float load(const __bf16 *p) { return static_cast<float>(*p); }
    static __device__ void store(__bf16 *p, float f) { *p = static_cast<__bf16>(f); }
};
template <>
struct Elem<_Float16> {
    static constexpr int N = 8;
    static __device__ void unpack(const uint4 &v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const halfx2 h = __builtin_bit_cast(halfx2, w[i]);
            f[2 * i] = static_cast<float>(h.x);
            f[2 * i + 1] = static_cast<float>(h.y);
        }
    }
    static __device__ uint4 pack(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = __builtin_bit_cast(uint32_t, (halfx2){static_cast<_Float16>(f[2 * i]), static_cast<_Float16>(f[2 * i + 1])});
        return {w[0], w[1], w[2], w[3]};
    }
    static constexpr uint32_t kNone = 0x80008000u;
    static __device__ uint32_t more(uint32_t a, uint32_t b) { return more_of_two(a, b); }
    static __device__ uint32_t less(uint32_t a, uint32_t b) { return less_of_two(a, b); }
    static __device__ float largest(uint32_t most, uint32_t least)
    {
        const halfx2 a = __builtin_bit_cast(halfx2, largest_of_two(most, least));
        return fmaxf(static_cast<float>(a.x), static_cast<float>(a.y));
    }
    static __device__ float load(const _Float16 *p) { return static_cast<float>(*p); }
    static __device__ void store(_Float16 *p, float f) { *p = static_cast<_Float16>(f); }
};

// A row as slots of 16 aligned bytes: slot i holds elements i N - shift .. of the row, the first and
// the last slot may reach past its ends and are taken an element at a time.
template <typename T>
struct Row {
    static constexpr int N = Elem<T>::N;
    const T *p;
    int V, shift, slots;
    __device__ Row(const void *data, int64_t stride, int64_t row, int V) : p(static_cast<const T *>(data) + row * stride), V(V)
    {
        shift = static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
        slots = (V + shift + N - 1) / N;
    }
    __device__ int first(int slot) const { return slot * N - shift; }
    __device__ uint4 load(int slot, float outside) const
    {
        const int e = first(slot);
        if (e >= 0 && e + N <= V) return *reinterpret_cast<const uint4 *>(p + e);
        float f[N];
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = (e + i >= 0 && e + i < V) ? Elem<T>::load(p + e + i) : outside;
        return Elem<T>::pack(f);
    }
    __device__ void load(int slot, float (&f)[N], float outside) const { Elem<T>::unpack(load(slot, outside), f); }
};

// The same elements as `whole` slots within the row and up to 2 N - 2 elements in front of and behind them, one of
// which each of the first 2 N lanes can take (edge): loads of whole slots need no branch.
template <typename T>
struct Span {
    static constexpr int N = Elem<T>::N;
    const T *p;
    int V, head, whole;
    __device__ Span(const T *p, int V) : p(p), V(V)
    {
        const int shift = static_cast<int>((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
        head = shift ? min(N - shift, V) : 0;
        whole = (V - head) / N;
    }
    __device__ int tail() const { return head + whole * N; }
    __device__ int edge(int lane) const
    {
        if (lane < head) return lane;
        return lane >= N && lane < 2 * N && tail() + lane - N < V ? tail() + lane - N : -1;
    }
    // (slot < whole; past it the last one again)
    __device__ uint4 load(int slot) const
    {
        return *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p + head) + static_cast<uint32_t>(min(slot, whole - 1)) * 16u);
    }
};

// 16 bytes to or from an address that is aligned to its elements only (one instruction all the same, slower where a
// cache line ends within it).
typedef uint32_t words_at_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t words_at_4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
__device__ __forceinline__ void store_16(T *out, const uint4 &v)
{
    if (sizeof(T) == 4) *reinterpret_cast<words_at_4 *>(out) = words_at_4{v.x, v.y, v.z, v.w};
    else *reinterpret_cast<words_at_2 *>(out) = words_at_2{v.x, v.y, v.z, v.w};
}

// The same past the caches, which keep what they hold: for whole cache lines of a stream that is not read again soon.
template <typename T>
__device__ __forceinline__ void stream_16(T *out, const uint4 &v)
{
    if (sizeof(T) == 4) __builtin_nontemporal_store(words_at_4{v.x, v.y, v.z, v.w}, reinterpret_cast<words_at_4 *>(out));
    else __builtin_nontemporal_store(words_at_2{v.x, v.y, v.z, v.w}, reinterpret_cast<words_at_2 *>(out));
}

template <typename T>
__device__ __forceinline__ uint4 load_16(const T *in)
{
    if (sizeof(T) == 4) {
        const words_at_4 v = *reinterpret_cast<const words_at_4 *>(in);
        return {v.x, v.y, v.z, v.w};
    }
    const words_at_2 v = *reinterpret_cast<const words_at_2 *>(in);
    return {v.x, v.y, v.z, v.w};
}

template <typename T>
__device__ __forceinline__ void store_slot(T *out, int e, int V, const float (&f)[Elem<T>::N])
{
    constexpr int N = Elem<T>::N;
    if (e >= 0 && e + N <= V) {
        store_16(out + e, Elem<T>::pack(f));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i >= 0 && e + i < V) Elem<T>::store(out + e + i, f[i]);
    }
}

// Rows of a few aligned bytes.
template <int BYTES>
struct Words {
    static constexpr int N = BYTES / 4;
    uint32_t w[N];
    __device__ void load(const void *p)
    {
        if constexpr (BYTES == 4) w[0] = *static_cast<const uint32_t *>(p);
        if constexpr (BYTES == 8) *this = from(*static_cast<const uint2 *>(p));
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const uint4 v = static_cast<const uint4 *>(p)[i];
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        }
    }
    __device__ void store(void *p) const
    {
        if constexpr (BYTES == 4) *static_cast<uint32_t *>(p) = w[0];
        if constexpr (BYTES == 8) *static_cast<uint2 *>(p) = {w[0], w[1]};
        if constexpr (BYTES >= 16) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) static_cast<uint4 *>(p)[i] = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
        }
    }
    static __device__ Words from(const uint2 &v)
    {
        Words r;
        r.w[0] = v.x; r.w[1] = v.y;
        return r;
    }
};

template <typename T, int CAP>
__device__ __forceinline__ void unpack_words(const uint32_t *w, float *f)
{
#pragma unroll
    for (int j = 0; j < CAP; ++j) {
        if constexpr (sizeof(T) == 4) f[j] = __uint_as_float(w[j]);
        else f[j] = static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(w[j / 2] >> (16 * (j % 2)))));
    }
}

template <typename T, int CAP>
__device__ __forceinline__ void pack_words(const float *f, uint32_t *w)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < CAP; ++j) w[j] = __float_as_uint(f[j]);
    } else {
#pragma unroll
        for (int j = 0; j < CAP; j += 2)
            w[j / 2] = __builtin_bit_cast(uint16_t, static_cast<T>(f[j])) |
                       static_cast<uint32_t>(__builtin_bit_cast(uint16_t, static_cast<T>(f[j + 1]))) << 16;
    }
}

template <typename F>
void by_type(int dtype, F &&f)
{
    if (dtype == PL_BF16) f(__bf16{});
    else if (dtype == PL_F16) f(_Float16{});
    else f(float{});
}

}  // namespace
}  // namespace pl

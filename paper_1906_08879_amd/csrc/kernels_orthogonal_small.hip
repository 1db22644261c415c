// The orthogonalised update of matrices of few rows (include/placeto.h): everything in one workgroup, one launch for many matrices; long ones
// of up to 32 rows in parts.
//
// Up to 32 rows the iteration goes over the short side alone, in float64: with A_0 = X X', step i has B_i = a I + b A_i + c A_i^2 and
// A_{i+1} = B_i A_i B_i, and X ends as (B_n .. B_1) X.  All of them are polynomials of A_0, symmetric, and trade places in a product.  X is read twice,
// once for A_0 and once for the result, whatever the number of steps.  In float64 nothing is lost by it (the factors' product has entries up to 485 beside
// results of 1, which fp32 would leave with 10^-4 of nearly dependent rows): results are off by their last rounding, 3e-8 of the factor's
// norm, where fp32 products leave 1e-6 and products of two halves (kernels_orthogonal.hip) up to 2.9e-6 with few rows.  Bound by the two products with X on
// the float64 matrix cores (64 multiply-adds a cycle of a CU) and, in between, by the latency of three short products a step: 16 x 4096 takes 38 us (in
// halves, step by step, 104), 32 x 2048 49 (116); in parts 32 x 100000 45 (531) and 32 x 1048576 122 (1692), 3.3 TB/s.
//
// With 33 to 64 rows, and up to 1024 columns, X lies in registers: a wave has 16 NB columns as 16 x 16 parts, of
// which a lane holds column lane % 16, rows 4 (lane / 16) .. + 3, in the two halves that kernels_orthogonal.hip explains.  That is both
// what a product on the matrix cores (16 x 16 x 16) leaves and what the next one takes as its right operand: B X needs no movement of X.  X X' takes X as both operands
// along the columns, that is the parts transposed: fed as a left operand and multiplied by the unit matrix, a part comes out
// transposed, exactly.  The waves' sums of X X' are added in LDS, two by two in a fixed order; A and B are kept there.
//
// Bound by the conversions between the two halves and fp32, beside the products, of the matrix with the most columns: the 24 matrices
// of a policy network, up to 896 x 64, take 114 us in one launch, five iterations of 21 us; in tiles of several workgroups an iteration of
// 65 rows and more is three launches one behind another, of 9 to 14 us each.
#include <algorithm>

#include "orthogonal_device.h"

namespace pl {
namespace {

typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float4_t __attribute__((ext_vector_type(4)));

// W elements side by side, aligned to one of them.
template <typename T, int W>
struct Group {
    typedef T vector __attribute__((ext_vector_type(W), aligned(sizeof(T))));
    static __device__ void load(const void *p, int64_t i, float (&v)[W])
    {
        const vector x = *reinterpret_cast<const vector *>(static_cast<const T *>(p) + i);
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = static_cast<float>(x[e]);
    }
    static __device__ void store(void *p, int64_t i, const float (&v)[W])
    {
        vector x;
#pragma unroll
        for (int e = 0; e < W; ++e) x[e] = static_cast<T>(v[e]);
        *reinterpret_cast<vector *>(static_cast<T *>(p) + i) = x;
    }
};

struct Part {                          // of a matrix, 16 x 16
    half4 hi, lo;
};

__device__ __forceinline__ Part part_of(const float4_t &v)
{
    Part p;
    p.hi = __builtin_convertvector(v, half4);
    float4_t rest;
#pragma unroll
    for (int e = 0; e < 4; ++e) rest[e] = __builtin_fmaf(static_cast<float>(p.hi[e]), -1.0f, v[e]);
    p.lo = __builtin_convertvector(rest, half4);
    return p;
}

// p f + v, a fused multiply-add with each half (which takes it as it is).
__device__ __forceinline__ float4_t add_part(const Part &p, float f, float4_t v)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(static_cast<float>(p.hi[e]), f, __builtin_fmaf(static_cast<float>(p.lo[e]), f, v[e]));
    return v;
}

__device__ __forceinline__ float4_t product(const half4 &a, const half4 &b, const float4_t &c) { return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float4_t product(const Part &a, const Part &b, const float4_t &c)
{
    return product(a.lo, b.hi, product(a.hi, b.lo, product(a.hi, b.hi, c)));
}

typedef _Float16 half8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ half8 beside(const half4 &a, const half4 &b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// Two products at once: in 16 x 16 x 32 a lane has eight places of the axis that is summed over, four of each part.
__device__ __forceinline__ float4_t product(const Part &a, const Part &a2, const Part &b, const Part &b2, float4_t c)
{
    const half8 ah = beside(a.hi, a2.hi), bh = beside(b.hi, b2.hi);
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, bh, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(ah, beside(b.lo, b2.lo), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(beside(a.lo, a2.lo), bh, c, 0, 0, 0);
}

constexpr int KB = 4;                  // parts of the rows: 33 to 64 of them

// Symmetric matrices in LDS, 16 KB rows of both halves; rows are an odd number of 8-byte words apart.
struct Square {
    static constexpr int K = KB * 16, PITCH = K + 4;
    _Float16 hi[K][PITCH], lo[K][PITCH];
    // Rows 16 i + lane % 16, columns 16 j + 4 (lane / 16) ..: part (i, j) as an operand.
    __device__ Part at(int i, int j, int lane) const
    {
        const int r = i * 16 + (lane & 15), c = j * 16 + (lane >> 4) * 4;
        return {*reinterpret_cast<const half4 *>(&hi[r][c]), *reinterpret_cast<const half4 *>(&lo[r][c])};
    }
    // Part (i, j) of a result, to both sides of the diagonal.
    __device__ void set(int i, int j, int lane, const Part &p)
    {
        const int c = j * 16 + (lane & 15), r = i * 16 + (lane >> 4) * 4;
        *reinterpret_cast<half4 *>(&hi[c][r]) = p.hi;
        *reinterpret_cast<half4 *>(&lo[c][r]) = p.lo;
        if (i == j) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            hi[r + e][c] = p.hi[e];
            lo[r + e][c] = p.lo[e];
        }
    }
};

constexpr int kWaves = 8;
constexpr int kGroups = 8;             // of a matrix' elements that a thread has on their way at a time

struct SmallShared {
    static constexpr int PAIRS = KB * (KB + 1) / 2;
    Square A, B;
    float4_t added[kWaves / 2][PAIRS][64];
    double sums[kWaves];
};

template <int NB>
__device__ __forceinline__ void update_small(const OrthSmallTable &t, const OrthSmall &o, SmallShared &sh)
{
    constexpr int PAIRS = SmallShared::PAIRS;
    Square &A = sh.A, &B = sh.B;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool tall = o.rows > o.cols;
    const int quad = lane >> 4;
    // Momentum and direction, in the order of the matrix, and from there to the parts through memory (fp32, columns of X one behind
    // another, with zeros to whole parts): a loop over elements for every type, instead of every type in code that is unrolled
    // over the parts.
    float *u = static_cast<float *>(o.room);
    constexpr int pitch = KB * 16;
    for (int i = tid; i < kWaves * NB * 4 * pitch; i += kWaves * 64) reinterpret_cast<float4_t *>(u)[i] = float4_t{};
    __syncthreads();
    auto at = [&](int r, int c) { return tall ? r * pitch + c : c * pitch + r; };
    double sum = 0.0;
    // over the matrix in groups of W elements of a row: f(row, column)
    auto each_group = [&](auto width, auto f) {
        constexpr int W = decltype(width)::value;
        const uint32_t groups = o.cols / W, all = o.rows * groups, magic = groups > 1 ? 0xffffffffu / groups + 1 : 0;   // (exact below 2^16)
        for (uint32_t i0 = tid; i0 < all; i0 += kGroups * kWaves * 64) {
            int r[kGroups], c[kGroups];
#pragma unroll
            for (int p = 0; p < kGroups; ++p) {            // (past the end the last group again, which does no harm but in sums)
                const uint32_t i = min(i0 + p * kWaves * 64, all - 1);
                r[p] = groups > 1 ? __umulhi(i, magic) : i;
                c[p] = static_cast<int>(i - r[p] * groups) * W;
            }
            f(r, c, static_cast<int>(min<uint32_t>(kGroups, (all - i0 + kWaves * 64 - 1) / (kWaves * 64))));
        }
    };
    auto start = [&](auto type, auto width) {
        using T = decltype(type);
        constexpr int W = decltype(width)::value;
        each_group(width, [&](const int (&r)[kGroups], const int (&c)[kGroups], int count) {
            float v[kGroups][W], m[kGroups][W];
#pragma unroll
            for (int p = 0; p < kGroups; ++p) Group<T, W>::load(o.grad, static_cast<int64_t>(r[p]) * o.grad_stride + c[p], v[p]);
            if (o.momentum) {
#pragma unroll
                for (int p = 0; p < kGroups; ++p) Group<float, W>::load(o.momentum, static_cast<int64_t>(r[p]) * o.momentum_stride + c[p], m[p]);
            }
#pragma unroll
            for (int p = 0; p < kGroups; ++p) {
                if (p >= count) break;
                if (o.momentum) {
#pragma unroll
                    for (int e = 0; e < W; ++e) m[p][e] = t.cfg.beta * m[p][e] + v[p][e];
                    if (o.new_momentum) Group<float, W>::store(o.new_momentum, static_cast<int64_t>(r[p]) * o.new_momentum_stride + c[p], m[p]);
#pragma unroll
                    for (int e = 0; e < W; ++e) v[p][e] = t.cfg.nesterov ? v[p][e] + t.cfg.beta * m[p][e] : m[p][e];
                }
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    u[at(r[p], c[p] + e)] = v[p][e];
                    sum += static_cast<double>(v[p][e]) * v[p][e];
                }
            }
        });
    };
    const bool by_four = o.cols % 4 == 0;
    for_type(o.grad_dtype, [&](auto type) {
        if (by_four) start(type, std::integral_constant<int, 4>{});
        else start(type, std::integral_constant<int, 1>{});
    });
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if (lane == 0) sh.sums[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kWaves; ++w) sum += sh.sums[w];
    // nothing but zeros stays zero; a norm that is no number makes the whole matrix none
    const double norm = sqrt(sum) + t.cfg.eps, factor = norm == 0.0 ? 0.0 : norm < INFINITY ? t.x_scale / norm : NAN;
    const float4_t *mine = reinterpret_cast<const float4_t *>(u + (wave * NB * 16 + (lane & 15)) * pitch + quad * 4);
    Part x[KB][NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
#pragma unroll
        for (int i = 0; i < KB; ++i) {
            float4_t f = mine[j * 4 * pitch + i * 4];
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = f[e] == 0.0f ? 0.0f : static_cast<float>(f[e] * factor);
            x[i][j] = part_of(f);
            asm volatile("" : "+v"(x[i][j].hi), "+v"(x[i][j].lo));
        }
        if (j % 2) __builtin_amdgcn_sched_barrier(0);        // (two columns of parts after the others, here and below: their registers)
    }
    half4 unit;
#pragma unroll
    for (int e = 0; e < 4; ++e) unit[e] = (lane & 15) == quad * 4 + e ? static_cast<_Float16>(1.0f) : static_cast<_Float16>(0.0f);

#pragma unroll 1
    for (int s = 0; s < t.n_steps; ++s) {
        const OrthStep st = t.step[s];
        // A = X X'
        float4_t acc[PAIRS] = {};
        constexpr int J = NB > 1 ? 2 : 1;            // columns of parts at once
#pragma unroll
        for (int j = 0; j < NB; j += J) {
            Part y[J][KB];                           // transposed
#pragma unroll
            for (int q = 0; q < J; ++q)
#pragma unroll
                for (int i = 0; i < KB; ++i) {
                    const float4_t none = {};
                    const float4_t hi = product(x[i][j + q].hi, unit, none), lo = product(x[i][j + q].lo, unit, none);
                    y[q][i] = {__builtin_convertvector(hi, half4), __builtin_convertvector(lo, half4)};
                }
#pragma unroll
            for (int a = 0, p = 0; a < KB; ++a)
#pragma unroll
                for (int b = 0; b <= a; ++b, ++p) {
                    if constexpr (J == 2) acc[p] = product(y[0][a], y[1][a], y[0][b], y[1][b], acc[p]);
                    else acc[p] = product(y[0][a], y[0][b], acc[p]);
                }
            __builtin_amdgcn_sched_barrier(0);
        }
        for (int half = kWaves / 2; half; half >>= 1) {
            if (wave >= half && wave < 2 * half)
#pragma unroll
                for (int p = 0; p < PAIRS; ++p) sh.added[wave - half][p][lane] = acc[p];
            __syncthreads();
            if (wave < half)
#pragma unroll
                for (int p = 0; p < PAIRS; ++p) acc[p] += sh.added[wave][p][lane];
            __syncthreads();
        }
        if (wave == 0) {
#pragma unroll
            for (int a = 0, at = 0; a < KB; ++a)
#pragma unroll
                for (int b = 0; b <= a; ++b, ++at) A.set(a, b, lane, part_of(acc[at] * st.gram));
        }
        __syncthreads();
        // B = a I + b A + c A A
        for (int p = wave; p < PAIRS; p += kWaves) {
            int a = 0;
            while ((a + 1) * (a + 2) / 2 <= p) ++a;
            const int b = p - a * (a + 1) / 2;
            float4_t sq = {};
#pragma unroll
            for (int c = 0; c < KB; c += 2) sq = product(A.at(a, c, lane), A.at(a, c + 1, lane), A.at(b, c, lane), A.at(b, c + 1, lane), sq);
            // (the part itself from across the diagonal, four rows of a column side by side)
            float4_t sum = add_part(A.at(b, a, lane), st.linear, sq * st.square);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += a == b && (lane & 15) == quad * 4 + e ? st.unit : 0.0f;
            B.set(a, b, lane, part_of(sum));
        }
        __syncthreads();
        // X = B X
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            float4_t d[KB] = {};
            int from = lane;
            asm volatile("" : "+v"(from));           // (B is read again: kept over the columns it would take 64 registers)
#pragma unroll
            for (int i = 0; i < KB; ++i) {
#pragma unroll
                for (int c = 0; c < KB; c += 2) d[i] = product(B.at(i, c, from), B.at(i, c + 1, from), x[c][j], x[c + 1][j], d[i]);
                if (NB == 8) __builtin_amdgcn_sched_barrier(0);      // (and of B)
            }
#pragma unroll
            for (int i = 0; i < KB; ++i) {
                x[i][j] = part_of(d[i] * st.next);
                // (the halves alone go on to the next step: without this their conversions do too)
                asm volatile("" : "+v"(x[i][j].hi), "+v"(x[i][j].lo));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    float4_t *result = const_cast<float4_t *>(mine);
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < KB; ++i)
            result[j * 4 * pitch + i * 4] = add_part(x[i][j], t.per_last, float4_t{});
    __syncthreads();
    auto finish = [&](void *to, const void *weight, uint32_t to_stride, auto type, auto width) {
        using T = decltype(type);
        constexpr int W = decltype(width)::value;
        each_group(width, [&](const int (&r)[kGroups], const int (&c)[kGroups], int count) {
            float v[kGroups][W], w[kGroups][W];
#pragma unroll
            for (int p = 0; p < kGroups; ++p)
#pragma unroll
                for (int e = 0; e < W; ++e) v[p][e] = u[at(r[p], c[p] + e)];
            if (weight) {
#pragma unroll
                for (int p = 0; p < kGroups; ++p) Group<T, W>::load(weight, static_cast<int64_t>(r[p]) * o.weight_stride + c[p], w[p]);
            }
#pragma unroll
            for (int p = 0; p < kGroups; ++p) {
                if (p >= count) break;
#pragma unroll
                for (int e = 0; e < W; ++e) v[p][e] = weight ? t.cfg.lr_decay * w[p][e] - t.cfg.lr * o.scale * v[p][e] : v[p][e];
                Group<T, W>::store(to, static_cast<int64_t>(r[p]) * to_stride + c[p], v[p]);
            }
        });
    };
    auto finish_by_type = [&](void *to, const void *weight, uint32_t to_stride, int dtype) {
        for_type(dtype, [&](auto type) {
            if (by_four) finish(to, weight, to_stride, type, std::integral_constant<int, 4>{});
            else finish(to, weight, to_stride, type, std::integral_constant<int, 1>{});
        });
    };
    if (o.out) finish_by_type(o.out, nullptr, o.out_stride, o.out_dtype);
    if (o.new_weight) finish_by_type(o.new_weight, o.weight, o.new_weight_stride, o.weight_dtype);
}

// ---- up to 32 rows: over the short side, in float64
#define INLINE __attribute__((always_inline))        // (a lambda that is left as a call would take the table of matrices to memory)
typedef double double4_t __attribute__((ext_vector_type(4)));

// 16 x 16 x 4: operands i = lane % 16, k = lane / 16; results rows 4 r + lane / 16, column lane % 16.
__device__ __forceinline__ double4_t product(double a, double b, const double4_t &c) { return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0); }

constexpr int kPending = 4;            // steps of a wave whose loads are on their way together

template <int THIN>
struct ThinShared {
    static constexpr int K = THIN * 16, TILES = THIN * (THIN + 1) / 2;
    typedef double Symmetric[K][K + 1];
    Symmetric A;
    union {
        struct {
            Symmetric B, Q[2], C;
        };
        double4_t added[kWaves][TILES][64];
    };
};

// W elements of a row side by side, of which `left` are there: gradient and momentum, then what is orthogonalised.
template <int W>
struct Source {
    float v[W], m[W];
};

template <typename T, int W>
__device__ __forceinline__ void read_some(const void *p, int64_t at, int left, float (&x)[W])
{
    if constexpr (W == 4) load_group<T>(p, at, left, x);
    else x[0] = left > 0 ? static_cast<float>(static_cast<const T *>(p)[at]) : 0.0f;
}

// What is orthogonalised, of a set of sources: each(f) calls f(source, row, column, left) for all of them.  FIRST: the new momentum goes to where it is
// kept, from where the second pass takes it.
template <bool FIRST, typename Each>
__device__ __forceinline__ void read_all(const OrthCfg &cfg, const OrthSmall &o, Each each)
{
    const bool momentum = o.momentum, kept = o.new_momentum, again = !FIRST && kept;
    if (momentum) {
        const float *from = again ? o.new_momentum : o.momentum;
        const int64_t stride = again ? o.new_momentum_stride : o.momentum_stride;
        each([&](auto &x, int r, int c, int left) INLINE { read_some<float>(from, r * stride + c, left, x.m); });
    }
    for_type(o.grad_dtype, [&](auto type) INLINE {
        each([&](auto &x, int r, int c, int left) INLINE { read_some<decltype(type)>(o.grad, static_cast<int64_t>(r) * o.grad_stride + c, left, x.v); });
    });
    if (!momentum) return;
    each([&](auto &x, int r, int c, int left) INLINE {
        constexpr int W = sizeof(x.v) / sizeof(float);
#pragma unroll
        for (int e = 0; e < W; ++e) x.m[e] = again ? x.m[e] : cfg.beta * x.m[e] + x.v[e];
        if (FIRST && kept) {
            const int64_t at = static_cast<int64_t>(r) * o.new_momentum_stride + c;
            if constexpr (W == 4) store_group<float>(o.new_momentum, at, left, x.m);
            else if (left > 0) o.new_momentum[at] = x.m[0];
        }
#pragma unroll
        for (int e = 0; e < W; ++e) x.v[e] = direction(cfg, true, x.m[e], x.v[e]);
    });
}

// Results, four side by side each, to `out` and into the weights.
template <typename Each>
__device__ __forceinline__ void write_all(const OrthCfg &cfg, const OrthSmall &o, Each each)
{
    if (o.out)
        for_type(o.out_dtype, [&](auto type) INLINE {
            each([&](const float (&v)[4], float (&)[4], int r, int c, int left) INLINE {
                if (left > 0) store_group<decltype(type)>(o.out, static_cast<int64_t>(r) * o.out_stride + c, left, v);
            });
        });
    if (o.new_weight)
        for_type(o.weight_dtype, [&](auto type) INLINE {
            typedef decltype(type) T;
            each([&](const float (&)[4], float (&w)[4], int r, int c, int left) INLINE { load_group<T>(o.weight, static_cast<int64_t>(r) * o.weight_stride + c, left, w); });
            each([&](const float (&v)[4], float (&w)[4], int r, int c, int left) INLINE {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = cfg.lr_decay * w[e] - cfg.lr * o.scale * v[e];
                if (left > 0) store_group<T>(o.new_weight, static_cast<int64_t>(r) * o.new_weight_stride + c, left, w);
            });
        });
}

// X X' of the columns c0 .. c1 of X, 16 to a wave at a time.
template <int THIN>
__device__ __forceinline__ void gram_of(const OrthCfg &cfg, const OrthSmall &o, int c0, int c1, double4_t (&acc)[ThinShared<THIN>::TILES])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, quad = lane >> 4;
    const bool tall = o.rows > o.cols;
    const int k = tall ? o.cols : o.rows;
    auto add = [&](auto element) INLINE {                           // element(part of the rows, r): row r16 of it, one of four columns
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int a = 0, p = 0; a < THIN; ++a)
#pragma unroll
                for (int b = 0; b <= a; ++b, ++p) acc[p] = product(static_cast<double>(element(a, r)), static_cast<double>(element(b, r)), acc[p]);
    };
    for (int c = c0 + wave * 16; c < c1; c += kPending * kWaves * 16) {
        if (!tall) {                                         // (a lane's four columns side by side: the order of a sum's terms is free)
            Source<4> u[kPending][THIN];
            auto each = [&](auto f) INLINE {
#pragma unroll
                for (int p = 0; p < kPending; ++p)
#pragma unroll
                    for (int a = 0; a < THIN; ++a) {
                        const int row = a * 16 + r16, col = c + p * kWaves * 16 + quad * 4;
                        f(u[p][a], row, col, row < k ? c1 - col : 0);
                    }
            };
            read_all<true>(cfg, o, each);
#pragma unroll
            for (int p = 0; p < kPending; ++p) add([&](int a, int r) INLINE { return u[p][a].v[r]; });
        } else {
            Source<1> u[kPending][THIN][4];
            auto each = [&](auto f) INLINE {
#pragma unroll
                for (int p = 0; p < kPending; ++p)
#pragma unroll
                    for (int a = 0; a < THIN; ++a)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int row = c + p * kWaves * 16 + r * 4 + quad, col = a * 16 + r16;
                            f(u[p][a][r], row, col, row < c1 && col < k ? 1 : 0);
                        }
            };
            read_all<true>(cfg, o, each);
#pragma unroll
            for (int p = 0; p < kPending; ++p) add([&](int a, int r) INLINE { return u[p][a][r].v[0]; });
        }
    }
}

// A part of X X' to both sides of the diagonal.
template <int THIN>
__device__ __forceinline__ void put_gram(ThinShared<THIN> &sh, int tile, int lane, const double4_t &sum)
{
    const int a = tile ? 1 : 0, b = tile == 2 ? 1 : 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = a * 16 + r * 4 + (lane >> 4), j = b * 16 + (lane & 15);
        sh.A[i][j] = sum[r];
        if (a != b) sh.A[j][i] = sum[r];
    }
}

// From U U' in A: 1 / norm, and of the iteration on U / norm the product of all its factors.
template <int THIN>
__device__ __forceinline__ const typename ThinShared<THIN>::Symmetric &iterate(const OrthSmallTable &t, ThinShared<THIN> &sh, double *per_norm)
{
    constexpr int K = ThinShared<THIN>::K, SQ = THIN * THIN;
    typedef typename ThinShared<THIN>::Symmetric Symmetric;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r16 = lane & 15, quad = lane >> 4;
    double trace = lane < K ? sh.A[lane % K][lane % K] : 0.0;
#pragma unroll
    for (int d = 32; d; d >>= 1) trace += __shfl_xor(trace, d);
    // nothing but zeros stays zero; a norm that is no number makes the whole matrix none
    const double norm = sqrt(trace) + t.cfg.eps, f = norm == 0.0 ? 0.0 : norm < INFINITY ? 1.0 / norm : NAN;
    *per_norm = f;
    __syncthreads();
    for (int e = tid; e < K * K; e += kWaves * 64) sh.A[e / K][e % K] *= f * f;
    __syncthreads();
    auto tile = [&](const Symmetric &m, const Symmetric &n, int i, int j) INLINE {
        double4_t even = {}, odd = {};                   // (two chains of products, each half as long)
#pragma unroll
        for (int c = 0; c < K; c += 8) {
            even = product(m[i * 16 + r16][c + quad], n[j * 16 + r16][c + quad], even);
            odd = product(m[i * 16 + r16][c + 4 + quad], n[j * 16 + r16][c + 4 + quad], odd);
        }
        return even + odd;
    };
    auto put = [&](Symmetric &to, int i, int j, const double4_t &v) INLINE {
#pragma unroll
        for (int r = 0; r < 4; ++r) to[i * 16 + r * 4 + quad][j * 16 + r16] = v[r];
    };
    const int i = wave % SQ / THIN, j = wave % THIN;
    int now = 0;
#pragma unroll 1
    for (int s = 0; s < t.n_steps; ++s) {
        const double a = t.iteration[s][0], b = t.iteration[s][1], c = t.iteration[s][2];
        const bool last = s + 1 == t.n_steps;
        if (wave < SQ) {
            double4_t v = tile(sh.A, sh.A, i, j);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = i * 16 + r * 4 + quad, col = j * 16 + r16;
                v[r] = c * v[r] + b * sh.A[row][col] + (row == col ? a : 0.0);
            }
            put(sh.B, i, j, v);
        }
        __syncthreads();
        if (wave < SQ) {
            double4_t v;
            if (s == 0) {
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = sh.B[i * 16 + r * 4 + quad][j * 16 + r16];
            } else {
                v = tile(sh.B, sh.Q[now], i, j);
            }
            put(sh.Q[now ^ 1], i, j, v);
        } else if (wave < 2 * SQ && !last) {
            put(sh.C, i, j, tile(sh.B, sh.A, i, j));
        }
        __syncthreads();
        if (wave < SQ && !last) put(sh.A, i, j, tile(sh.C, sh.B, i, j));
        now ^= 1;
        __syncthreads();
    }
    return sh.Q[now];
}

// The columns c0 .. c1 of Q X.  A wave reads all rows of its columns before it writes them (out may be grad).
template <int THIN>
__device__ __forceinline__ void apply_to(const OrthCfg &cfg, const OrthSmall &o, const typename ThinShared<THIN>::Symmetric &Q, double f, int c0, int c1)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, quad = lane >> 4;
    const bool tall = o.rows > o.cols;
    const int k = tall ? o.cols : o.rows;
    double q[THIN][4][THIN];                                 // of rows [part][r] the rows [part] of the result
    if (!tall) {
        // X' Q: a lane has the columns 4 r16 .. of the rows 4 r + quad, and then of row r16 the columns 4 (4 r + quad) ..
#pragma unroll
        for (int a = 0; a < THIN; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < THIN; ++i) q[a][r][i] = Q[a * 16 + r * 4 + quad][i * 16 + r16] * f;
        for (int c = c0 + wave * 64; c < c1; c += kWaves * 64) {
            Source<4> u[THIN][4];
            auto each = [&](auto g) INLINE {
#pragma unroll
                for (int a = 0; a < THIN; ++a)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = a * 16 + r * 4 + quad, col = c + r16 * 4;
                        g(u[a][r], row, col, row < k ? c1 - col : 0);
                    }
            };
            read_all<false>(cfg, o, each);
#pragma unroll
            for (int i = 0; i < THIN; ++i) {
                double4_t d[4] = {};
#pragma unroll
                for (int a = 0; a < THIN; ++a)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) d[e] = product(static_cast<double>(u[a][r].v[e]), q[a][r][i], d[e]);
                float v[4][4], w[4][4];
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[r][e] = static_cast<float>(d[e][r]);
                write_all(cfg, o, [&](auto g) INLINE {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = i * 16 + r16, col = c + (r * 4 + quad) * 4;
                        g(v[r], w[r], row, col, row < k ? c1 - col : 0);
                    }
                });
            }
        }
    } else {
        // Q X: a lane has the rows 4 quad .. of column r16, before and after (row 4 r + quad of a product is row 4 quad + r of the result)
#pragma unroll
        for (int a = 0; a < THIN; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < THIN; ++i) q[a][r][i] = Q[i * 16 + (r16 & 3) * 4 + (r16 >> 2)][a * 16 + quad * 4 + r] * f;
        for (int c = c0 + wave * 16; c < c1; c += kPending * kWaves * 16) {
            Source<4> u[kPending][THIN];
            auto each = [&](auto g) INLINE {
#pragma unroll
                for (int p = 0; p < kPending; ++p)
#pragma unroll
                    for (int a = 0; a < THIN; ++a) {
                        const int row = c + p * kWaves * 16 + r16, col = a * 16 + quad * 4;
                        g(u[p][a], row, col, row < c1 ? k - col : 0);
                    }
            };
            read_all<false>(cfg, o, each);
            float v[kPending][THIN][4], w[kPending][THIN][4];
#pragma unroll
            for (int p = 0; p < kPending; ++p)
#pragma unroll
                for (int i = 0; i < THIN; ++i) {
                    double4_t d = {};
#pragma unroll
                    for (int a = 0; a < THIN; ++a)
#pragma unroll
                        for (int r = 0; r < 4; ++r) d = product(q[a][r][i], static_cast<double>(u[p][a].v[r]), d);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[p][i][e] = static_cast<float>(d[e]);
                }
            write_all(cfg, o, [&](auto g) INLINE {
#pragma unroll
                for (int p = 0; p < kPending; ++p)
#pragma unroll
                    for (int i = 0; i < THIN; ++i) {
                        const int row = c + p * kWaves * 16 + r16, col = i * 16 + quad * 4;
                        g(v[p][i], w[p][i], row, col, row < c1 ? k - col : 0);
                    }
            });
        }
    }
}

// The waves' sums of X X' added in their order: out(tile, lane, sum).
template <int THIN, typename F>
__device__ __forceinline__ void add_waves(ThinShared<THIN> &sh, const double4_t (&acc)[ThinShared<THIN>::TILES], F out)
{
    constexpr int TILES = ThinShared<THIN>::TILES;
    const int tid = threadIdx.x;
#pragma unroll
    for (int p = 0; p < TILES; ++p) sh.added[tid >> 6][p][tid & 63] = acc[p];
    __syncthreads();
    for (int e = tid; e < TILES * 64; e += kWaves * 64) {
        double4_t sum = sh.added[0][e >> 6][e & 63];
        for (int w = 1; w < kWaves; ++w) sum += sh.added[w][e >> 6][e & 63];
        out(e >> 6, e & 63, sum);
    }
    __syncthreads();
}

template <int THIN>
__device__ __forceinline__ void update_thin(const OrthSmallTable &t, const OrthSmall &o, ThinShared<THIN> &sh)
{
    const int n = max(o.rows, o.cols);
    double4_t acc[ThinShared<THIN>::TILES] = {};
    gram_of<THIN>(t.cfg, o, 0, n, acc);
    add_waves<THIN>(sh, acc, [&](int tile, int lane, const double4_t &sum) INLINE { put_gram<THIN>(sh, tile, lane, sum); });
    double f;
    const auto &Q = iterate<THIN>(t, sh, &f);
    apply_to<THIN>(t.cfg, o, Q, f, 0, n);
}

// LISTED: from a list in memory instead of the table (a choice made on the device cost 15% of the policy network's 115 us).
template <bool LISTED>
__global__ __launch_bounds__(kWaves * 64) void k_orth_small(OrthSmallTable t, const OrthSmall *__restrict__ list)
{
    __shared__ union {
        SmallShared of_64;
        ThinShared<1> of_16;
        ThinShared<2> of_32;
    } sh;
    const OrthSmall &o = LISTED ? list[blockIdx.x] : t.m[blockIdx.x];
    const int n = max(o.rows, o.cols), k = min(o.rows, o.cols);
    if (k <= 16) update_thin<1>(t, o, sh.of_16);
    else if (k <= kOrthThin) update_thin<2>(t, o, sh.of_32);
    else if (n <= 16 * kWaves) update_small<1>(t, o, sh.of_64);
    else if (n <= 64 * kWaves) update_small<4>(t, o, sh.of_64);
    else update_small<8>(t, o, sh.of_64);
}

__global__ __launch_bounds__(256) void k_orth_small_list(OrthSmallTable t, OrthSmall *__restrict__ list, int at)
{
    static_assert(sizeof(OrthSmall) % 4 == 0, "copied by words");
    const uint32_t *from = reinterpret_cast<const uint32_t *>(t.m);
    uint32_t *to = reinterpret_cast<uint32_t *>(list + at);
    for (uint32_t i = threadIdx.x; i < t.n * sizeof(OrthSmall) / 4; i += 256) to[i] = from[i];
}

// ---- long ones of up to 32 rows, in parts: the parts' X X', then their sum and the iteration, then the parts' results.  A matrix' room has
// a tile of 16 x 16 behind the other of every part's X X' (as the lanes have them), then those of the factors' product over the norm.
struct LongPart {
    const OrthSmall *o;
    int part, parts, c0, c1;
};

__device__ __forceinline__ int parts_of(const OrthSmall &o, int *columns)
{
    const int n = max(o.rows, o.cols);
    *columns = orth_part(n);
    return (n + *columns - 1) / *columns;
}

// The part that a workgroup has: the last matrix whose parts begin at or in front of it.
__device__ __forceinline__ LongPart part_of(const OrthSmall *list, int count, int id)
{
    int in_front = 0;
    for (int i0 = 0; i0 < count; i0 += 64) {
        const int i = i0 + (threadIdx.x & 63);
        in_front += __popcll(__ballot(i < count && list[min(i, count - 1)].first <= id));
    }
    LongPart p;
    p.o = list + (in_front - 1);
    p.part = id - p.o->first;
    int columns;
    p.parts = parts_of(*p.o, &columns);
    p.c0 = p.part * columns;
    p.c1 = min(max(p.o->rows, p.o->cols), p.c0 + columns);
    return p;
}

typedef double double4_room __attribute__((ext_vector_type(4), aligned(16)));

// f(16 or 32 rows)
template <typename F>
__device__ __forceinline__ void by_rows(const OrthSmall &o, F f)
{
    if (min(o.rows, o.cols) <= 16) f(std::integral_constant<int, 1>{});
    else f(std::integral_constant<int, 2>{});
}

union LongShared {
    ThinShared<1> of_16;
    ThinShared<2> of_32;
    template <int THIN>
    __device__ ThinShared<THIN> &get()
    {
        if constexpr (THIN == 1) return of_16;
        else return of_32;
    }
};

template <bool LISTED>
__global__ __launch_bounds__(kWaves * 64) void k_orth_long_gram(OrthSmallTable t, const OrthSmall *__restrict__ list, int count)
{
    __shared__ LongShared sh;
    const LongPart p = part_of(LISTED ? list : t.m, count, blockIdx.x);
    by_rows(*p.o, [&](auto thin) INLINE {
        constexpr int THIN = decltype(thin)::value, TILES = ThinShared<THIN>::TILES;
        double4_t acc[TILES] = {};
        gram_of<THIN>(t.cfg, *p.o, p.c0, p.c1, acc);
        double4_room *to = static_cast<double4_room *>(p.o->room) + static_cast<int64_t>(p.part) * (TILES * 64);
        add_waves<THIN>(sh.get<THIN>(), acc, [&](int tile, int lane, const double4_t &sum) INLINE { to[tile * 64 + lane] = sum; });
    });
}

template <bool LISTED>
__global__ __launch_bounds__(kWaves * 64) void k_orth_long_iterate(OrthSmallTable t, const OrthSmall *__restrict__ list)
{
    __shared__ LongShared sh;
    const OrthSmall &o = LISTED ? list[blockIdx.x] : t.m[blockIdx.x];
    by_rows(o, [&](auto thin) INLINE {
        constexpr int THIN = decltype(thin)::value, TILES = ThinShared<THIN>::TILES, K = ThinShared<THIN>::K;
        ThinShared<THIN> &mine = sh.get<THIN>();
        int columns;
        const int parts = parts_of(o, &columns), tid = threadIdx.x;
        const double4_room *from = static_cast<const double4_room *>(o.room);
        for (int e = tid; e < TILES * 64; e += kWaves * 64) {
            double4_t sum = {};
#pragma unroll 8
            for (int p = 0; p < parts; ++p) sum += from[p * (TILES * 64) + e];
            put_gram<THIN>(mine, e >> 6, e & 63, sum);
        }
        __syncthreads();
        double f;
        const auto &Q = iterate<THIN>(t, mine, &f);
        double *to = static_cast<double *>(o.room) + static_cast<int64_t>(parts) * (TILES * 256);
        for (int e = tid; e < K * K; e += kWaves * 64) to[e] = Q[e / K][e % K] * f;
    });
}

template <bool LISTED>
__global__ __launch_bounds__(kWaves * 64) void k_orth_long_apply(OrthSmallTable t, const OrthSmall *__restrict__ list, int count)
{
    __shared__ LongShared sh;
    const LongPart p = part_of(LISTED ? list : t.m, count, blockIdx.x);
    by_rows(*p.o, [&](auto thin) INLINE {
        constexpr int THIN = decltype(thin)::value, TILES = ThinShared<THIN>::TILES, K = ThinShared<THIN>::K;
        ThinShared<THIN> &mine = sh.get<THIN>();
        const double *from = static_cast<const double *>(p.o->room) + static_cast<int64_t>(p.parts) * (TILES * 256);
        for (int e = threadIdx.x; e < K * K; e += kWaves * 64) mine.A[e / K][e % K] = from[e];
        __syncthreads();
        apply_to<THIN>(t.cfg, *p.o, mine.A, 1.0, p.c0, p.c1);
    });
}

}  // namespace

void launch_orth_small_list(const OrthSmallTable &t, OrthSmall *list, int at, hipStream_t s)
{
    hipLaunchKernelGGL(k_orth_small_list, dim3(1), dim3(256), 0, s, t, list, at);
}

void launch_orth_small(const OrthSmallTable &t, const OrthSmall *list, int count, hipStream_t s)
{
    hipLaunchKernelGGL(list ? k_orth_small<true> : k_orth_small<false>, dim3(count), dim3(kWaves * 64), 0, s, t, list);
}

void launch_orth_long(const OrthSmallTable &t, const OrthSmall *list, int count, int parts, hipStream_t s)
{
    const dim3 block(kWaves * 64);
    hipLaunchKernelGGL(list ? k_orth_long_gram<true> : k_orth_long_gram<false>, dim3(parts), block, 0, s, t, list, count);
    hipLaunchKernelGGL(list ? k_orth_long_iterate<true> : k_orth_long_iterate<false>, dim3(count), block, 0, s, t, list);
    hipLaunchKernelGGL(list ? k_orth_long_apply<true> : k_orth_long_apply<false>, dim3(parts), block, 0, s, t, list, count);
}

}  // namespace pl

// The orthogonalised update of matrices (include/placeto.h): momentum, norm, Newton-Schulz iteration and step.
//
// With X of k rows and n >= k columns, an iteration is A = X X', B = a I + b A + c A A, X := B X.  A and B are symmetric: of their
// tiles those on and below the diagonal are computed and the others copied across it.  All three products take both operands by
// rows along the axis that they sum over, for which X is kept as k rows of n and as n rows of k; the last product computes X' and
// writes both.
//
// Every operand v is held as two fp16 numbers, v s = hi + lo with a power of two s, hi = fp16(v s), lo = fp16(v s - hi): 22 bits,
// and a product is hi hi + hi lo + lo hi on the matrix cores with fp32 sums; the dropped lo lo is 2^-22 of it.  The iteration
// raises the smallest singular values by up to a^steps (485 for the usual five) against the largest, and errors with them: one
// fp16 or bf16 product instead of three would leave factors that are off by 2^-11 a^steps where the matrix is nearly of low rank.
// s puts the largest number that an operand can hold at 2^14 (fp16 ends at 2^16), known on the host from the iteration's factors
// and ||X|| <= 1; what it leaves below the last bit of lo is 2^-38 of that number.
//
// Bound by the matrix cores where matrices are large: 8192 x 4096 takes 6.0 ms, of which three products at the rate of the card's library
// (1.40 PFLOP/s of fp16) would take 5.15, with 67 to 73% of the matrix cores' cycles busy; 16 of 1024 x 1024 with eight of 4096 x 1024 3.1
// ms against 1.93 (53%: a tile's 32 blocks lie between a beginning and an end that nothing overlaps).  By the steps' dependence on one
// another where they are small: 226 us for three of 1111 x 333 with others, 24 launches of 2 to 14 us.  Tiles of 64 to 256 by the sizes
// (OrthKind).
#include <algorithm>

#include "orthogonal_device.h"

namespace pl {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float4_t __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(256) void k_orth_list(OrthTable t, OrthMatrix *__restrict__ list, int at)
{
    const uint32_t *from = reinterpret_cast<const uint32_t *>(t.m);
    uint32_t *to = reinterpret_cast<uint32_t *>(list + at);
    for (uint32_t i = threadIdx.x; i < t.n * sizeof(OrthMatrix) / 4; i += 256) to[i] = from[i];
}

// The matrix that workgroup `id` belongs to, by one of the numbers of workgroups: 64 of them looked at together.
template <typename First>
__device__ __forceinline__ int matrix_of(const OrthMatrix *list, int n, int id, First first)
{
    int in_front = 0;
    for (int i0 = 0; i0 < n; i0 += 64) {
        const int i = i0 + (threadIdx.x & 63);
        in_front += __popcll(__ballot(i < n && first(list[i < n ? i : 0]) <= id));
    }
    return in_front - 1;
}

// ---- the new momentum, and sums of squares of the direction: eight groups of four elements to a thread at a time
constexpr int kSumGroups = 8;

__global__ __launch_bounds__(256) void k_orth_momentum(const OrthMatrix *__restrict__ list, int n_matrices, OrthCfg cfg)
{
    const OrthMatrix &o = list[matrix_of(list, n_matrices, blockIdx.x, [](const OrthMatrix &m) { return m.first_sum; })];
    const uint32_t part = blockIdx.x - o.first_sum, tid = threadIdx.x;
    // rows behind one another are one
    const uint32_t cols = o.cols;
    const bool whole = o.grad_stride == o.cols && (!o.momentum || o.momentum_stride == o.cols) && (!o.new_momentum || o.new_momentum_stride == o.cols);
    const uint32_t elements = o.rows * cols, width = whole ? elements : cols, by = (width + 3) / 4, all = whole ? by : by * o.rows;
    double sum = 0.0;
    for_type(o.grad_dtype, [&](auto type) {
        using T = decltype(type);
        for (uint32_t i0 = part * (256 * kSumGroups) + tid; i0 < all; i0 += o.sum_parts * (256 * kSumGroups)) {
            float v[kSumGroups][4], m[kSumGroups][4];
            uint32_t row[kSumGroups], col[kSumGroups];
            int left[kSumGroups];
#pragma unroll
            for (int p = 0; p < kSumGroups; ++p) {
                const uint32_t i = i0 + p * 256;
                row[p] = whole ? 0 : i / by;
                col[p] = (i - row[p] * by) * 4;
                left[p] = i < all ? static_cast<int>(min(4u, width - col[p])) : 0;
            }
#pragma unroll
            for (int p = 0; p < kSumGroups; ++p) load_group<T>(o.grad, row[p] * o.grad_stride + col[p], left[p], v[p]);
            if (o.momentum) {
#pragma unroll
                for (int p = 0; p < kSumGroups; ++p) load_group<float>(o.momentum, row[p] * o.momentum_stride + col[p], left[p], m[p]);
#pragma unroll
                for (int p = 0; p < kSumGroups; ++p) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) m[p][e] = cfg.beta * m[p][e] + v[p][e];
                    if (o.new_momentum) store_group<float>(o.new_momentum, row[p] * o.new_momentum_stride + col[p], left[p], m[p]);
                }
            }
#pragma unroll
            for (int p = 0; p < kSumGroups; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const double u = direction(cfg, o.momentum != nullptr, m[p][e], v[p][e]);
                    sum += u * u;                        // (what is not there is zero)
                }
        }
    });
    __shared__ double wave[4];
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((tid & 63) == 0) wave[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) o.sums[part] = (wave[0] + wave[1]) + (wave[2] + wave[3]);
}

struct Halves {
    _Float16 hi, lo;
};

__device__ __forceinline__ Halves halves_of(float v)
{
    Halves h;
    h.hi = static_cast<_Float16>(v);
    h.lo = static_cast<_Float16>(v - static_cast<float>(h.hi));
    return h;
}

__device__ __forceinline__ int64_t half_at(int64_t row, int pad, int col)
{
    return row * 2 * pad + (col / kOrthBlock) * (2 * kOrthBlock) + col % kOrthBlock;
}

// ---- the matrix over its norm, by rows and by columns
__global__ __launch_bounds__(256) void k_orth_layout(const OrthMatrix *__restrict__ list, int n_matrices, OrthCfg cfg, float x_scale)
{
    constexpr int T = kOrthLayout, GROUPS = T * T / 4 / 256;
    __shared__ float tile[T][T + 1];
    __shared__ double factor;
    const OrthMatrix &o = list[matrix_of(list, n_matrices, blockIdx.x, [](const OrthMatrix &m) { return m.first_layout; })];
    const int id = blockIdx.x - o.first_layout, tid = threadIdx.x;
    const int across = (o.cols + T - 1) / T, r0 = id / across * T, c0 = id % across * T;
    float v[GROUPS][4];
    for_type(o.grad_dtype, [&](auto type) {
        using E = decltype(type);
        float m[GROUPS][4];
        const float *old = o.new_momentum ? o.new_momentum : o.momentum;
        const int64_t old_stride = o.new_momentum ? o.new_momentum_stride : o.momentum_stride;
#pragma unroll
        for (int p = 0; p < GROUPS; ++p) {
            const int i = p * 256 + tid, r = r0 + i / (T / 4), c = c0 + i % (T / 4) * 4, left = r < o.rows ? o.cols - c : 0;
            load_group<E>(o.grad, r * o.grad_stride + c, left, v[p]);
            if (o.momentum) load_group<float>(old, r * old_stride + c, left, m[p]);
        }
        if (o.momentum) {
#pragma unroll
            for (int p = 0; p < GROUPS; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[p][e] = direction(cfg, true, o.new_momentum ? m[p][e] : cfg.beta * m[p][e] + v[p][e], v[p][e]);
        }
    });
    if (tid < 64) {
        double sum = 0.0;
        for (int i = tid; i < o.sum_parts; i += 64) sum += o.sums[i];
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        // nothing but zeros stays zero; a norm that is no number makes the whole matrix none
        const double norm = sqrt(sum) + cfg.eps;
        if (tid == 0) factor = norm == 0.0 ? 0.0 : norm < INFINITY ? x_scale / norm : NAN;
    }
    __syncthreads();
    const double f = factor;
#pragma unroll
    for (int p = 0; p < GROUPS; ++p) {
        const int i = p * 256 + tid, r = i / (T / 4), c = i % (T / 4) * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e) tile[r][c + e] = r0 + r < o.rows && c0 + c + e < o.cols ? static_cast<float>(v[p][e] * f) : 0.0f;
    }
    __syncthreads();
    _Float16 *by_row = o.tall ? o.xt[0] : o.x, *by_col = o.tall ? o.x : o.xt[0];
    const int row_pad = o.tall ? o.k_pad : o.n_pad, col_pad = o.tall ? o.n_pad : o.k_pad;
    auto put = [&](_Float16 *to, int64_t at, auto value) {
        half4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const Halves h = halves_of(value(e));
            hi[e] = h.hi;
            lo[e] = h.lo;
        }
        *reinterpret_cast<half4 *>(to + at) = hi;
        *reinterpret_cast<half4 *>(to + at + kOrthBlock) = lo;
    };
#pragma unroll
    for (int p = 0; p < GROUPS; ++p) {
        const int i = p * 256 + tid, u = i / (T / 4), w = i % (T / 4) * 4;
        if (r0 + u < o.rows && c0 + w < row_pad) put(by_row, half_at(r0 + u, row_pad, c0 + w), [&](int e) { return tile[u][w + e]; });
        if (c0 + u < o.cols && r0 + w < col_pad) put(by_col, half_at(c0 + u, col_pad, r0 + w), [&](int e) { return tile[w + e][u]; });
    }
}

// ---- products
enum { GRAM, SQUARE, STEP, LAST };

// What a workgroup of a product has: TILE x TILE of a result, a half of the rows and a half or a quarter of the columns to a wave.
template <int TILE>
struct Shape {
    static constexpr int ACROSS = TILE > 128 ? 4 : 2, WAVES = 2 * ACROSS, THREADS = WAVES * 64;
    static constexpr int MI = TILE / 2 / 16, NJ = TILE / ACROSS / 16;
    // Blocks that are loaded at a time.  Tiles of 64 multiply for less time than a load takes: X X' of 333 x 1111 22.4 us with one, 18.3
    // with two; for tiles of 128 two change nothing.
    static constexpr int DEEP = TILE == 64 ? 2 : 1;
    static constexpr int OPERAND = TILE * 128;           // bytes of one operand's rows at one block of 32
    static constexpr int LOADED = 2 * DEEP * OPERAND;    // bytes of what is loaded at a time: blocks of both operands
    // results on their way out: floats from a row to the next (lanes of 16 columns and every eighth row meet 64 banks)
    static constexpr int STAGE = TILE / 2, PITCH = TILE + 2;
    static constexpr int LDS = 2 * LOADED > STAGE * PITCH * 4 ? 2 * LOADED : STAGE * PITCH * 4;
};

// The rows of an operand from row0 on, one block of 32 elements (both halves, 128 bytes) of each at a time: eight rows to a wave's load,
// 16 bytes to a lane.  Row r's bytes 16 c .. lie at 16 (c ^ r % 8), so that the lanes' reads below, of one c in 16 rows, meet
// every bank.
template <int TILE>
struct Rows {
    static constexpr int LOADS = TILE / 8 / Shape<TILE>::WAVES;
    const char *base;                  // of the first row's next block
    uint32_t at[LOADS];                // (2^21 columns of 4 bytes, 256 rows)
    __device__ Rows(const _Float16 *from, int row0, int rows, int64_t row_halves, int block, int wave, int lane)
    {
        const int chunk = (lane & 7) ^ (lane >> 3);
        base = reinterpret_cast<const char *>(from + row0 * row_halves + block * (2 * kOrthBlock));
#pragma unroll
        for (int g = 0; g < LOADS; ++g) {
            const int row = min((g * Shape<TILE>::WAVES + wave) * 8 + (lane >> 3), rows - 1 - row0);
            at[g] = row * static_cast<uint32_t>(row_halves * 2) + chunk * 16;
        }
    }
    __device__ void next(char *lds, int wave)
    {
#pragma unroll
        for (int g = 0; g < LOADS; ++g)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t *)(base + at[g]),
                                             (__attribute__((address_space(3))) uint32_t *)(lds + (g * Shape<TILE>::WAVES + wave) * 1024), 16, 0, 0);
        base += 4 * kOrthBlock;
    }
};

__device__ __forceinline__ half8 read_half(const char *lds, int row, int chunk)
{
    return *reinterpret_cast<const half8 *>(lds + row * 128 + ((chunk ^ (row & 7)) << 4));
}

// Waits for this wave's loads from memory alone, and for its reads of LDS alone.
constexpr int kLoads = 0x0f70, kReads = 0xc07f;

__device__ __forceinline__ void end_turn()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Both halves of a number in a word, and back.
__device__ __forceinline__ uint32_t word_of(float v)
{
    const Halves h = halves_of(v);
    return __builtin_bit_cast(uint16_t, h.hi) | static_cast<uint32_t>(__builtin_bit_cast(uint16_t, h.lo)) << 16;
}

__device__ __forceinline__ void store_words(_Float16 *to, int64_t at, const uint32_t (&w)[8])
{
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        hi[e] = (w[2 * e] & 0xffffu) | w[2 * e + 1] << 16;
        lo[e] = w[2 * e] >> 16 | (w[2 * e + 1] & 0xffff0000u);
    }
    *reinterpret_cast<uint4 *>(to + at) = {hi[0], hi[1], hi[2], hi[3]};
    *reinterpret_cast<uint4 *>(to + at + kOrthBlock) = {lo[0], lo[1], lo[2], lo[3]};
}

// The result's rows from r0 on (columns of x) and columns from c0 on (rows of x), from LDS: out and weights.
template <int TILE>
__device__ __forceinline__ void write_out(const OrthMatrix &o, const OrthCfg &cfg, const float *stage, int r0, int c0)
{
    using S = Shape<TILE>;
    const int wide = o.tall ? TILE : S::STAGE, high = o.tall ? S::STAGE : TILE, by = wide / 4;       // in the order of the matrix
    const int row0 = o.tall ? r0 : c0, col0 = o.tall ? c0 : r0, n_rows = min(high, o.rows - row0), n_cols = min(wide, o.cols - col0);
    const int step = o.tall ? 1 : S::PITCH, down = o.tall ? S::PITCH : 1;
    auto go = [&](auto type, void *to, int64_t to_stride, const void *weight) {
        using T = decltype(type);
        for (int s = threadIdx.x; s < n_rows * by; s += S::THREADS) {
            const int r = s / by, c = (s - r * by) * 4, left = n_cols - c;
            if (left <= 0) continue;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = stage[r * down + (c + e) * step];
            if (weight) {
                float w[4];
                load_group<T>(weight, (row0 + r) * o.weight_stride + col0 + c, left, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = cfg.lr_decay * w[e] - cfg.lr * o.scale * v[e];
            }
            store_group<T>(to, (row0 + r) * to_stride + col0 + c, left, v);
        }
    };
    if (o.out) for_type(o.out_dtype, [&](auto type) { go(type, o.out, o.out_stride, nullptr); });
    if (o.new_weight) for_type(o.weight_dtype, [&](auto type) { go(type, o.new_weight, o.new_weight_stride, o.weight); });
}

constexpr bool symmetric(int phase) { return phase == GRAM || phase == SQUARE; }

// Which tile of a result a workgroup has.  Of symmetric ones (0, 0), (1, 0), (1, 1), (2, 0) ...
template <int TILE, int PHASE>
__device__ __forceinline__ void place_tile(const OrthMatrix &o, int tile, int *ti, int *tj)
{
    if (symmetric(PHASE)) {
        *ti = static_cast<int>((sqrtf(8.0f * tile + 1.0f) - 1.0f) * 0.5f);
        while (*ti * (*ti + 1) / 2 > tile) --*ti;
        while ((*ti + 1) * (*ti + 2) / 2 <= tile) ++*ti;
        *tj = tile - *ti * (*ti + 1) / 2;
    } else {
        const int across = (o.k + TILE - 1) / TILE;
        *ti = tile / across;
        *tj = tile - *ti * across;
    }
}

// The sums of a tile to where they belong.  `lds`: Shape::LDS bytes that nobody reads any more.
template <int TILE, int PHASE>
__device__ __forceinline__ void finish_tile(const OrthMatrix &o, const OrthCfg &cfg, const OrthStep &st, int from, int ti, int tj,
                                            const float4_t (&acc)[Shape<TILE>::MI][Shape<TILE>::NJ], char *lds)
{
    using S = Shape<TILE>;
    constexpr bool kSym = symmetric(PHASE);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave / S::ACROSS * (S::MI * 16), wj = wave % S::ACROSS * (S::NJ * 16), r16 = lane & 15, quad = lane >> 4;
    const int rows = kSym ? o.k : o.n, i0 = ti * TILE, j0 = tj * TILE;
    // Results go out by way of LDS, half of the tile's rows at a time, so that whole cache lines are read and written: 8 elements to a
    // thread, four threads to the 32 that lie together.  First by columns, where the part of A that is added is read, for X or across
    // the diagonal; then, as words, by rows.
    float *stage = reinterpret_cast<float *>(lds);
    const float factor = PHASE == GRAM ? st.gram : PHASE == SQUARE ? st.square : st.next;
    for (int h = 0; h < TILE; h += S::STAGE) {
        __syncthreads();
        if (wi == h) {
#pragma unroll
            for (int i = 0; i < S::MI; ++i)
#pragma unroll
                for (int j = 0; j < S::NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) stage[(i * 16 + quad * 4 + e) * S::PITCH + wj + j * 16 + r16] = acc[i][j][e] * factor;
        }
        __syncthreads();
        const int r0 = i0 + h;
        constexpr int kTasks = S::STAGE / 8 * TILE, kBatch = 4;
        for (int t0 = tid; t0 < kTasks; t0 += kBatch * S::THREADS) {
            half8 hi[kBatch], lo[kBatch];
            int64_t to[kBatch];
            bool in[kBatch];
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {       // (what is added, for all of them before it is waited for)
                const int t = t0 + b * S::THREADS, r = (t / (4 * TILE) * 4 + t % 4) * 8, c = j0 + t / 4 % TILE;
                in[b] = t < kTasks && c < o.k && r0 + r < (kSym ? o.k_pad : o.n_pad);
                to[b] = half_at(c, kSym ? o.k_pad : o.n_pad, r0 + r);
                if (PHASE == SQUARE && in[b]) {
                    const _Float16 *old = o.a + to[b];
                    hi[b] = *reinterpret_cast<const half8 *>(old);
                    lo[b] = *reinterpret_cast<const half8 *>(old + kOrthBlock);
                }
            }
#pragma unroll
            for (int b = 0; b < kBatch; ++b) {
                if (!in[b]) continue;
                const int t = t0 + b * S::THREADS, r = (t / (4 * TILE) * 4 + t % 4) * 8, u = t / 4 % TILE;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = stage[(r + e) * S::PITCH + u];
                if (PHASE == SQUARE) {
                    const int c = j0 + u - r0 - r;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[e] += st.linear * (static_cast<float>(hi[b][e]) + static_cast<float>(lo[b][e]));
                        v[e] += c == e ? st.unit : 0.0f;
                    }
                }
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = PHASE == LAST ? __float_as_uint(v[e]) : r0 + r + e < rows ? word_of(v[e]) : 0u;
                if (PHASE != LAST) store_words(kSym ? (PHASE == GRAM ? o.a : o.b) : o.x, to[b], w);
#pragma unroll
                for (int e = 0; e < 8; ++e) stage[(r + e) * S::PITCH + u] = __uint_as_float(w[e]);
            }
        }
        if (kSym && ti == tj) continue;
        __syncthreads();
        if (PHASE == LAST) {
            write_out<TILE>(o, cfg, stage, r0, j0);
            continue;
        }
        for (int t = tid; t < S::STAGE * (TILE / 8); t += S::THREADS) {
            const int r = t / (TILE / 8), u = t % (TILE / 8) * 8;
            if (r0 + r >= rows || j0 + u >= o.k_pad) continue;
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const uint2 two = *reinterpret_cast<const uint2 *>(stage + r * S::PITCH + u + e);
                w[e] = two.x;
                w[e + 1] = two.y;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = j0 + u + e < o.k ? w[e] : 0u;     // (columns that nobody has computed)
            store_words(PHASE == GRAM ? o.a : PHASE == SQUARE ? o.b : o.xt[from ^ 1], half_at(r0 + r, o.k_pad, j0 + u), w);
        }
    }
}

template <int TILE, int PHASE>
__global__ __launch_bounds__(Shape<TILE>::THREADS, 2) void k_orth_product(const OrthMatrix *__restrict__ list, int n_matrices, OrthCfg cfg,
                                                                          OrthStep st, int from)
{
    using S = Shape<TILE>;
    constexpr bool kSym = symmetric(PHASE);
    __shared__ __align__(16) char lds[S::LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wi = wave / S::ACROSS * (S::MI * 16), wj = wave % S::ACROSS * (S::NJ * 16), r16 = lane & 15, quad = lane >> 4;
    constexpr int kind = PHASE == LAST ? STEP : PHASE;
    int which = matrix_of(list, n_matrices, blockIdx.x, [](const OrthMatrix &m) { return m.first[kind]; }), tile = blockIdx.x - list[which].first[kind];
    // Eight matrices of the same sides take turns, so that all tiles of one go to one die (workgroups go round them) and meet in its cache:
    // 16 of 1024 x 1024 and eight of 4096 x 1024 read 259 MB for X X' instead of 1458, in 170 us instead of 216.
    const int run = list[which].run, eight = which - (run & 7);
    if (eight + 8 <= n_matrices && list[eight + 7].run == (run | 7)) {
        tile = blockIdx.x - list[eight].first[kind];
        which = eight + (tile & 7);
        tile >>= 3;
    }
    const OrthMatrix &o = list[which];
    int part = 0, depth = PHASE == GRAM ? o.n_pad : o.k_pad, blocks = depth / kOrthBlock;
    constexpr bool kParts = PHASE == GRAM && TILE == kOrthSplitTile;
    if (kParts && o.n_parts > 1) {
        part = tile % o.n_parts;
        tile /= o.n_parts;
        blocks = min(o.part_blocks, blocks - part * o.part_blocks);
    }
    const int loads = (blocks + S::DEEP - 1) / S::DEEP;
    int ti, tj;
    place_tile<TILE, PHASE>(o, tile, &ti, &tj);
    const int rows = kSym ? o.k : o.n;           // of the result
    const _Float16 *P = PHASE == GRAM ? o.x : PHASE == SQUARE ? o.a : o.xt[from], *Q = PHASE == GRAM ? o.x : PHASE == SQUARE ? o.a : o.b;
    const int i0 = ti * TILE, j0 = tj * TILE;
    const int64_t row_halves = 2 * static_cast<int64_t>(depth);

    float4_t acc[S::MI][S::NJ] = {};
    const int first = kParts && o.n_parts > 1 ? part * o.part_blocks : 0;
    Rows<TILE> of_p(P, i0, rows, row_halves, first, wave, lane), of_q(Q, j0, o.k, row_halves, first, wave, lane);
    auto load = [&](int s) {
#pragma unroll
        for (int d = 0; d < S::DEEP; ++d) {
            if (S::DEEP > 1 && s * S::DEEP + d >= blocks) break;
            of_p.next(lds + (s & 1) * S::LOADED + 2 * d * S::OPERAND, wave);
            of_q.next(lds + (s & 1) * S::LOADED + (2 * d + 1) * S::OPERAND, wave);
        }
    };
    load(0);
    __builtin_amdgcn_s_waitcnt(kLoads);
    __syncthreads();
    // Two waves of a SIMD, one of each half of the workgroup (`behind`), take turns: one reads from LDS while the other multiplies.  A
    // turn ends at a barrier; the half behind begins one later and the other waits one more at the end.  A wave loads its share of
    // what comes next as soon as both halves have read what lies there, two turns before it is read.
    const bool turns = S::WAVES == 8, behind = turns && wave >= S::WAVES / 2;
    if (behind) {
        if (loads > 1) load(1);
        end_turn();
    }
    for (int s = 0; s < loads; ++s) {
        const char *now = lds + (s & 1) * S::LOADED;
        // (all reads in front of the next loads: a read behind one waits for it)
        half8 p[S::DEEP][S::MI][2], q[S::DEEP][S::NJ][2];
#pragma unroll
        for (int d = 0; d < S::DEEP; ++d) {
            if (S::DEEP > 1 && s * S::DEEP + d >= blocks) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int j = 0; j < S::NJ; ++j) q[d][j][h] = read_half(now + (2 * d + 1) * S::OPERAND, wj + j * 16 + r16, h * 4 + quad);
#pragma unroll
                for (int i = 0; i < S::MI; ++i) p[d][i][h] = read_half(now + 2 * d * S::OPERAND, wi + i * 16 + r16, h * 4 + quad);
            }
        }
        if (!behind && s + 1 < loads) load(s + 1);
        if (turns) {
            __builtin_amdgcn_s_waitcnt(kReads);
            if (behind) __builtin_amdgcn_s_waitcnt(kLoads);
            end_turn();
            if (behind && s + 2 < loads) load(s + 2);
            __builtin_amdgcn_s_setprio(1);
        }
#pragma unroll
        for (int d = 0; d < S::DEEP; ++d) {
            if (S::DEEP > 1 && s * S::DEEP + d >= blocks) break;
#pragma unroll
            for (int h = 0; h < 3; ++h)              // hi hi, hi lo, lo hi
#pragma unroll
                for (int i = 0; i < S::MI; ++i)
#pragma unroll
                    for (int j = 0; j < S::NJ; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[d][i][h == 2], q[d][j][h == 1], acc[i][j], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);           // (the products stay in front of the wait for the next block)
        if (turns) {
            __builtin_amdgcn_s_setprio(0);
            if (!behind) __builtin_amdgcn_s_waitcnt(kLoads);
            end_turn();
        } else {
            __builtin_amdgcn_s_waitcnt(kLoads);
            __syncthreads();
        }
    }
    if (turns && !behind) end_turn();
    if (kParts && o.n_parts > 1) {
        float4_t *to = reinterpret_cast<float4_t *>(o.parts) + (static_cast<int64_t>(tile) * o.n_parts + part) * (S::MI * S::NJ * S::THREADS);
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) to[(i * S::NJ + j) * S::THREADS + tid] = acc[i][j];
        return;
    }
    finish_tile<TILE, PHASE>(o, cfg, st, from, ti, tj, acc, lds);
}

// X X' from sums over parts of the long axis, in their order (a call: 128 x 4096 307 us without, 156 with it; 256 x 16384 1060 and 285).
__global__ __launch_bounds__(Shape<kOrthSplitTile>::THREADS) void k_orth_join(const OrthMatrix *__restrict__ list, int n_matrices, OrthCfg cfg, OrthStep st)
{
    using S = Shape<kOrthSplitTile>;
    __shared__ __align__(16) char lds[S::STAGE * S::PITCH * 4];
    const OrthMatrix &o = list[matrix_of(list, n_matrices, blockIdx.x, [](const OrthMatrix &m) { return m.first_join; })];
    const int tile = blockIdx.x - o.first_join;
    const float4_t *parts = reinterpret_cast<const float4_t *>(o.parts) + static_cast<int64_t>(tile) * o.n_parts * (S::MI * S::NJ * S::THREADS) + threadIdx.x;
    float4_t acc[S::MI][S::NJ] = {};
#pragma unroll 4
    for (int p = 0; p < o.n_parts; ++p)
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) acc[i][j] += parts[(p * S::MI * S::NJ + i * S::NJ + j) * S::THREADS];
    int ti, tj;
    place_tile<kOrthSplitTile, GRAM>(o, tile, &ti, &tj);
    finish_tile<kOrthSplitTile, GRAM>(o, cfg, st, 0, ti, tj, acc, lds);
}

}  // namespace

void launch_orth_list(const OrthTable &t, OrthMatrix *list, int at, hipStream_t s)
{
    hipLaunchKernelGGL(k_orth_list, dim3(1), dim3(256), 0, s, t, list, at);
}

void launch_orth_start(const OrthMatrix *list, const OrthGrid &grid, const OrthCfg &cfg, float x_scale, hipStream_t s)
{
    hipLaunchKernelGGL(k_orth_momentum, dim3(static_cast<uint32_t>(grid.sums)), dim3(256), 0, s, list, grid.n_matrices, cfg);
    hipLaunchKernelGGL(k_orth_layout, dim3(static_cast<uint32_t>(grid.layouts)), dim3(256), 0, s, list, grid.n_matrices, cfg, x_scale);
}

namespace {

template <int PHASE>
void launch_product(const OrthMatrix *list, const OrthGrid &g, const OrthCfg &cfg, const OrthStep &step, int from, hipStream_t s)
{
    const OrthWork &w = g.work[PHASE == LAST ? STEP : PHASE];
    const auto go = [&](auto tile) {
        constexpr int TILE = decltype(tile)::value;
        hipLaunchKernelGGL((k_orth_product<TILE, PHASE>), dim3(static_cast<uint32_t>(w.tiles)), dim3(Shape<TILE>::THREADS), 0, s, list, g.n_matrices,
                           cfg, step, from);
    };
    if (w.kind == 3) go(std::integral_constant<int, kOrthKinds[3].tile>{});
    else if (w.kind == 2) go(std::integral_constant<int, kOrthKinds[2].tile>{});
    else if (w.kind == 1) go(std::integral_constant<int, kOrthKinds[1].tile>{});
    else go(std::integral_constant<int, kOrthKinds[0].tile>{});
}

}  // namespace

void launch_orth_step(const OrthMatrix *list, const OrthGrid &g, const OrthCfg &cfg, const OrthStep &step, int number, bool last, hipStream_t s)
{
    launch_product<GRAM>(list, g, cfg, step, 0, s);
    if (g.joins)
        hipLaunchKernelGGL(k_orth_join, dim3(static_cast<uint32_t>(g.joins)), dim3(Shape<kOrthSplitTile>::THREADS), 0, s, list, g.n_matrices, cfg, step);
    launch_product<SQUARE>(list, g, cfg, step, 0, s);
    if (last) launch_product<LAST>(list, g, cfg, step, number & 1, s);
    else launch_product<STEP>(list, g, cfg, step, number & 1, s);
}

}  // namespace pl

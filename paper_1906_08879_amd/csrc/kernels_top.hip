// The most likely actions of rows of logits (include/placeto.h), with log probabilities and entropies.
//
// Softmax parts of a row as in kernels_losses.hip, x_j = (z_j - m) log2 e / T.  Actions are ordered by (z, lower index), one whole
// number of 64 bits: the float's bits turned so that they order like its values, then the index counted down.  No two are equal, so
// that an action's place in the list is the number of greater ones, whatever order they are found in.
//
// One pass over memory, four ways of it by the width:
//   up to 16                   a row to a thread, in registers
//   up to 128, many rows       a row to a lane, in LDS (by_lanes)
//   up to 4096 bf16            a row to a wave, up to 8192 (or a slice of a longer one) to a workgroup, in registers
//   longer                     streamed, two steps at a time; few rows or very long ones in slices, whose lists a second kernel joins
// A line is taken that the list's last logit cannot lie below: the top-th largest of the maxima of threads or slots.  What reaches it
// (a few more than `top` where logits lie at random) goes to LDS, where each counts the greater ones.  Rows where too much reaches the line
// (equal logits, fewer than `top` that are allowed) or that hold NaN take their top-th number by its digits instead, with seven passes
// over the row in cache.
// Bound by memory from 8192 logits on, and by the list's own work below: 64 of 65536 bf16 in 4096 rows 122 us, 4.4 TB/s; 2 of 8 fp32 in
// 799744 rows 10 us; 20 of one row of 131072, two launches, 15 us, of which reading takes less than one.
#include <algorithm>
#include <cmath>

#include "rows.h"

namespace pl {
namespace {

__device__ __forceinline__ uint32_t order_of(float z)
{
    const uint32_t b = __float_as_uint(z + 0.0f);        // (-0 counts as 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order); }
__device__ __forceinline__ uint64_t entry_of(float z, int action)
{
    return static_cast<uint64_t>(order_of(z)) << 32 | (0xffffffffu - static_cast<uint32_t>(action));
}
__device__ __forceinline__ int action_of(uint64_t entry) { return static_cast<int>(0xffffffffu - static_cast<uint32_t>(entry)); }
__device__ __forceinline__ float logit_of(uint64_t entry) { return value_of(static_cast<uint32_t>(entry >> 32)); }

// log p of a logit from its row's sums.
struct RowLog {
    float m, s, log_s, per, per2, lowest;
    __device__ float operator()(float z) const
    {
        const float d = z - (m == -INFINITY ? 0.0f : m);
        if (!(s > 0.0f)) return NAN;                     // (nothing is allowed; a logit is no number)
        if (z == lowest && d * per2 < kNoChance) return -INFINITY;
        return d * per - log_s;
    }
};

__device__ __forceinline__ RowLog row_log(const TopArgs &g, const Sums &a)
{
    return {a.m, a.s, kLn2 * log2f(a.s), g.per, g.per2, lowest_of(g.x.dtype)};
}

__device__ __forceinline__ float entropy_of(const Sums &a) { return a.s == 0.0f ? NAN : kLn2 * (log2f(a.s) - a.t * reciprocal(a.s)); }

// What a row has besides its list.
template <typename T>
__device__ __forceinline__ void finish_scores(const TopArgs &g, int64_t n, const Sums &a, const RowLog &log_p)
{
    if (g.out_logp) {
        const int act = g.actions[n];
        g.out_logp[n] = act >= 0 && act < g.x.V ? log_p(Elem<T>::load(static_cast<const T *>(g.x.data) + n * g.x.stride + act)) : NAN;
    }
    if (g.out_entropy) g.out_entropy[n] = entropy_of(a);
}

struct TopScale {
    float m, per2;
    __device__ float operator()(float z) const { return (z - m) * per2; }
};

__device__ __forceinline__ Sums rebased_by(const Sums &a, float m, float per2)
{
    if (a.s == 0.0f) return {m, 0.0f, 0.0f};
    const float d = (a.m - m) * per2, e = exp2_of(d);
    return {m, a.s * e, e * (a.t + fmaxf(d, kLowest) * a.s)};
}

// ---- narrow rows: a row to a thread
template <typename T, int CAP, bool WHOLE>
__global__ __launch_bounds__(256) void k_top_narrow(TopArgs g)
{
    extern __shared__ float tile[];
    const int V = WHOLE ? CAP : g.x.V, pitch = V | 1, tid = threadIdx.x;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 256, n = n0 + tid;
    const int count = static_cast<int>(min(int64_t{256}, g.x.n - n0));
    float z[CAP];
    if (WHOLE) {
        if (tid < count) {
            Words<CAP * sizeof(T)> words;
            words.load(static_cast<const T *>(g.x.data) + n * g.x.stride);
            unpack_words<T, CAP>(words.w, z);
        }
    } else {
        narrow_tile<T, false>(g.x.data, g.x.stride, n0, count, V, g.magic, pitch, tile);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < CAP; ++j)
            if (j < V) z[j] = tile[tid * pitch + j];
    }
    if (tid >= count) return;
    auto each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < CAP; ++j)
            if (WHOLE || j < V) f(j, z[j]);
    };
    Sums a;
    each([&](int, float v) { a.m = fmaxf(a.m, v); });
    const TopScale x{ref_of(a.m).m, g.per2};
    each([&](int, float v) {
        const float y = x(v), e = exp2_of(y);
        a.s += e;
        a.t += e * fmaxf(y, kLowest);
    });
    const RowLog log_p = row_log(g, a);
    // the largest below the one before, as often as asked for
    uint64_t before = ~uint64_t{0};
    for (int i = 0; i < g.top; ++i) {
        uint64_t best = 0;
        each([&](int j, float v) {
            const uint64_t e = entry_of(v, j + 1);           // (from 1 on: a NaN of all bits at action 0 is below the first `before` too)
            if (e < before && e > best) best = e;
        });
        g.out_top[n * g.top + i] = action_of(best) - 1;
        if (g.out_top_logp) g.out_top_logp[n * g.top + i] = log_p(logit_of(best));
        before = best;
    }
    finish_scores<T>(g, n, a, log_p);
}

// ---- many rows of some more actions: a row to a lane still, in LDS
template <typename T>
__global__ __launch_bounds__(64) void k_top_lane(TopArgs g)
{
    extern __shared__ float tile[];
    const int V = g.x.V, pitch = V | 1, tid = threadIdx.x;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 64, n = n0 + tid;
    const int count = static_cast<int>(min(int64_t{64}, g.x.n - n0));
    narrow_tile<T, false, 64>(g.x.data, g.x.stride, n0, count, V, g.magic, pitch, tile);
    __syncthreads();
    if (tid >= count) return;
    float *z = tile + tid * pitch;
    Sums a;
#pragma unroll 8
    for (int j = 0; j < V; ++j) a.m = fmaxf(a.m, z[j]);
    const TopScale x{ref_of(a.m).m, g.per2};
#pragma unroll 8
    for (int j = 0; j < V; ++j) {
        const float v = z[j], y = x(v), e = exp2_of(y);
        a.s += e;
        a.t += e * fmaxf(y, kLowest);
        z[j] = __uint_as_float(max(order_of(v), 1u));    // (its bits from here on)
    }
    const RowLog log_p = row_log(g, a);
    // the largest, the first one of equals, as often as asked for, and 0 in its place
    for (int i = 0; i < g.top; ++i) {
        uint32_t best = 0;
        int at = 0;
#pragma unroll 8
        for (int j = 0; j < V; ++j) {
            const uint32_t o = __float_as_uint(z[j]);
            at = o > best ? j : at;
            best = max(o, best);
        }
        z[at] = 0.0f;
        g.out_top[n * g.top + i] = at;
        if (g.out_top_logp) g.out_top_logp[n * g.top + i] = log_p(value_of(best));
    }
    finish_scores<T>(g, n, a, log_p);
}

// ---- wider rows
template <int KEPT>
struct TopShared {
    static constexpr int kKept = KEPT;
    uint64_t entry[KEPT];
    uint32_t count[256];               // of a digit's values
    uint64_t cut;
    int kept, need;
};

// Whether a row's element counts for f: whole slots, then the elements in front of and behind them.
template <typename T, int THREADS, typename F>
__device__ __forceinline__ void each_element(const Span<T> &row, int begin, int end, bool with_edge, F f)
{
    constexpr int N = Elem<T>::N;
    for (int i0 = begin; i0 < end; i0 += THREADS) {
        const int i = i0 + static_cast<int>(threadIdx.x);
        float z[N];
        if (i < end) Elem<T>::unpack(row.load(i), z);
#pragma unroll
        for (int j = 0; j < N; ++j) f(i < end, i < end ? z[j] : 0.0f, row.head + i * N + j);
    }
    if (with_edge) {
        const int e = row.edge(threadIdx.x);
        f(e >= 0, e >= 0 ? Elem<T>::load(row.p + e) : 0.0f, e);
    }
}

// The `top` first entries of a part of a row into sh.entry, by the digits of the last one of them.
template <typename T, int THREADS, typename Shared>
__device__ __forceinline__ void select_by_digits(const Span<T> &row, int begin, int end, bool with_edge, int top, Shared &sh)
{
    const int tid = threadIdx.x;
    uint64_t prefix = 0, above = 0;
    int need = top;
    for (int shift = 56; shift >= 0; shift -= 8) {
        if (shift == 24) {                               // (an index has 24 bits: the digit above them is full)
            prefix |= uint64_t{0xff} << 24;
            above |= uint64_t{0xff} << 24;
            continue;
        }
        __syncthreads();
        for (int i = tid; i < 256; i += THREADS) sh.count[i] = 0;
        __syncthreads();
        each_element<T, THREADS>(row, begin, end, with_edge, [&](bool is, float z, int at) {
            const uint64_t e = entry_of(z, at);
            const bool mine = is && (e & above) == prefix;
            const uint32_t digit = static_cast<uint32_t>(e >> shift) & 0xff;
            // most often the lanes have one digit in common
            const uint64_t active = __ballot(mine);
            if (active == 0) return;
            const uint32_t first = __builtin_amdgcn_readlane(digit, __ffsll(static_cast<unsigned long long>(active)) - 1);
            const uint64_t same = __ballot(mine && digit == first);
            if (mine) {
                if (digit != first) atomicAdd(&sh.count[digit], 1u);
                else if (__popcll(same & ((uint64_t{1} << (tid & 63)) - 1)) == 0) atomicAdd(&sh.count[first], static_cast<uint32_t>(__popcll(same)));
            }
        });
        __syncthreads();
        if (tid == 0) {
            int d = 255, left = need;
            for (; d > 0 && static_cast<int>(sh.count[d]) < left; --d) left -= sh.count[d];
            sh.cut = prefix | static_cast<uint64_t>(d) << shift;
            sh.need = left;
        }
        __syncthreads();
        prefix = sh.cut;
        need = sh.need;
        above |= uint64_t{0xff} << shift;
    }
    __syncthreads();
    if (tid == 0) sh.kept = 0;
    __syncthreads();
    each_element<T, THREADS>(row, begin, end, with_edge, [&](bool is, float z, int at) {
        const uint64_t e = entry_of(z, at);
        if (is && e >= prefix) sh.entry[min(atomicAdd(&sh.kept, 1), Shared::kKept - 1)] = e;
    });
    __syncthreads();
}

// The place of every kept entry among them: out(place, entry) for the first `top`.
template <int THREADS, typename Shared, typename F>
__device__ __forceinline__ void rank_kept(const Shared &sh, int kept, int top, F out)
{
    for (int i = threadIdx.x; i < kept; i += THREADS) {
        const uint64_t mine = sh.entry[i];
        int place = 0;
#pragma unroll 8
        for (int j = 0; j < kept; ++j) place += sh.entry[j] > mine;
        if (place < top) out(place, mine);
    }
}

// Kept entries that are many more than `top`, down to those from the top-th on: each counts the greater ones among all that are left, so
// that their number goes into the time twice.  By the first wave, an entry's upper 32 bits in a register of a lane.
template <int THREADS, typename Shared>
__device__ __forceinline__ void thin_kept(Shared &sh, int top)
{
    constexpr int MINE = Shared::kKept / 64;
    const int kept = sh.kept, lane = threadIdx.x & 63;
    __syncthreads();                                     // (the first wave writes the number that the others have come here by)
    if (kept < top + 64) return;
    if (threadIdx.x < 64) {
        uint32_t mine[MINE];
#pragma unroll
        for (int w = 0; w < MINE; ++w) mine[w] = w * 64 + lane < kept ? static_cast<uint32_t>(sh.entry[w * 64 + lane] >> 32) : 0;
        uint32_t line = 0;
        for (int b = 31; b >= 0; --b) {
            const uint32_t next = line | 1u << b;
            int reach = 0;
#pragma unroll
            for (int w = 0; w < MINE; ++w) reach += __popcll(__ballot(mine[w] >= next));
            if (reach >= top) line = next;
        }
        int left = 0;
#pragma unroll
        for (int w = 0; w < MINE; ++w) {                 // (an entry goes to a place that has been read)
            const bool in = w * 64 + lane < kept && mine[w] >= line;
            const uint64_t with = __ballot(in), e = in ? sh.entry[w * 64 + lane] : 0;
            if (in) sh.entry[left + __popcll(with & ((uint64_t{1} << lane) - 1))] = e;
            left += __popcll(with);
        }
        if (lane == 0) sh.kept = left;
    }
    __syncthreads();
}

// What follows from a row's or a slice's sums and kept entries.
template <typename T, int THREADS, typename Shared>
__device__ __forceinline__ void finish_list(const TopArgs &g, int64_t n, const Sums &a, const Shared &sh, int top)
{
    const int kept = min(sh.kept, Shared::kKept);
    if (g.slices == 1) {
        const RowLog log_p = row_log(g, a);
        rank_kept<THREADS>(sh, kept, top, [&](int place, uint64_t e) {
            g.out_top[n * g.top + place] = action_of(e);
            if (g.out_top_logp) g.out_top_logp[n * g.top + place] = log_p(logit_of(e));
        });
        if (threadIdx.x == 0) finish_scores<T>(g, n, a, log_p);
    } else {
        const int64_t slice = n * g.slices + blockIdx.y;
        rank_kept<THREADS>(sh, kept, top, [&](int place, uint64_t e) { g.lists[slice * g.top + place] = e; });
        for (int i = top + static_cast<int>(threadIdx.x); i < g.top; i += THREADS) g.lists[slice * g.top + i] = 0;
        if (threadIdx.x == 0) g.parts[slice] = {a.m, a.s, a.t};
    }
}

// A row, or a slice of one, in the registers of a wave or of a workgroup.  LONG: for lists of more than kShortTop, whose thinning takes
// registers (35 more of 68, and 40% of the time of lists of one in 4104 logits, so that shorter ones go without).
template <typename T, int THREADS, int CH, int KEPT, bool LONG>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(4))) void k_top_row(TopArgs g)
{
    constexpr int N = Elem<T>::N, WAVES = THREADS / 64;
    __shared__ TopShared<KEPT> sh;
    __shared__ float most_of[THREADS];
    __shared__ RowPart part[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int64_t n = blockIdx.x; n < g.x.n; n += gridDim.x) {
        const Span<T> row(static_cast<const T *>(g.x.data) + n * g.x.stride, g.x.V);
        const int per = (row.whole + g.slices - 1) / g.slices, begin = min(row.whole, per * static_cast<int>(blockIdx.y)), end = min(row.whole, begin + per);
        const bool with_edge = blockIdx.y == 0;
        uint4 v[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if (begin + k * THREADS < end) v[k] = row.load(min(begin + k * THREADS + tid, end - 1));
        const int edge = with_edge ? row.edge(tid) : -1;
        const float z_edge = edge >= 0 ? Elem<T>::load(row.p + edge) : -INFINITY;
        if (tid == 0) sh.kept = 0;
        uint32_t most = Elem<T>::kNone, least = 0xffffffffu;
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if (begin + k * THREADS + tid < end) add_words<T>(v[k], most, least);
        const bool some = begin + tid < end;
        const float mine = fmaxf(z_edge, some ? Elem<T>::largest(most, least) : -INFINITY);
        Sums a;
        a.m = max_of<64>(mine);
        const TopScale x{ref_of(a.m).m, g.per2};
        if (edge >= 0) a.s += exp2_of(x(z_edge));
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (begin + k * THREADS + tid < end) {
                float f[N];
                Elem<T>::unpack(v[k], f);
#pragma unroll
                for (int j = 0; j < N; ++j) a.s += exp2_of(x(f[j]));
            }
            keep_packed(v[k]);
        }
        if (g.out_entropy) {                             // (few rows have it wanted: the exponentials are taken again)
            auto add_t = [&](float z) {
                const float y = x(z);
                a.t += exp2_of(y) * fmaxf(y, kLowest);
            };
            if (edge >= 0) add_t(z_edge);
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (begin + k * THREADS + tid < end) {
                    uint4 w = v[k];
                    keep_packed(w);
                    float f[N];
                    Elem<T>::unpack(w, f);
#pragma unroll
                    for (int j = 0; j < N; ++j) add_t(f[j]);
                }
        }
        a.s = sum_of<64>(a.s);
        a.t = sum_of<64>(a.t);
        most_of[tid] = mine;
        if (lane == 0) part[wave] = {a.m, a.s, a.t};
        __syncthreads();
        {
            Sums of;
            if (lane < WAVES) of = {part[lane].m, part[lane].s, part[lane].t};
            const float m = max_of<64>(of.m);
            const Sums x = rebased_by(of, ref_of(m).m, g.per2);
            a = {m, sum_of<64>(x.s), sum_of<64>(x.t)};
        }
        // the highest line that `top` of the threads' maxima reach, to the upper 20 bits of their numbers; of a single wave, whose maxima
        // are few beside a long list, that `top` of its slots' maxima or of its elements reach
        uint32_t line = 0;
        if (THREADS == 64 && (g.top > 16 || (CH == 1 && g.top * N > g.x.V))) {
            constexpr int KEYS = CH == 1 ? N : CH;
            uint32_t key[KEYS + 1];
            key[KEYS] = order_of(z_edge);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const bool is = begin + k * THREADS + tid < end;
                if (CH == 1) {
                    float f[N];
                    Elem<T>::unpack(v[0], f);
#pragma unroll
                    for (int j = 0; j < N; ++j) key[j % KEYS] = is ? order_of(f[j]) : 0;
                } else {
                    keep_packed(v[k]);
                    uint32_t slot_most = Elem<T>::kNone, slot_least = 0xffffffffu;
                    add_words<T>(v[k], slot_most, slot_least);
                    key[k] = is ? order_of(Elem<T>::largest(slot_most, slot_least)) : 0;
                }
            }
            for (int b = 31; b >= 12; --b) {
                const uint32_t next = line | 1u << b;
                int reach = 0;
#pragma unroll
                for (int i = 0; i <= KEYS; ++i) reach += __popcll(__ballot(key[i] >= next));
                if (reach >= g.top) line = next;
            }
        } else {
            uint32_t key[WAVES];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) key[w] = order_of(most_of[w * 64 + lane]);
            for (int b = 31; b >= 12; --b) {
                const uint32_t next = line | 1u << b;
                int reach = 0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) reach += __popcll(__ballot(key[w] >= next));
                if (reach >= g.top) line = next;
            }
        }
        // (a line below all numbers is minus infinity, or where `some` threads have nothing)
        const float z_line = line <= order_of(-INFINITY) ? -INFINITY : value_of(line);
        auto keep = [&](float z, int at) {
            if (z >= z_line) {
                const int i = atomicAdd(&sh.kept, 1);
                if (i < KEPT) sh.entry[i] = entry_of(z, at);
            }
        };
        if (mine >= z_line && a.s > 0.0f) {
            if (edge >= 0) keep(z_edge, edge);
            int from = begin + tid;
            asm volatile("" : "+v"(from));               // (the slots' numbers are taken anew, their registers are the row's)
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                keep_packed(v[k]);
                uint32_t slot_most = Elem<T>::kNone, slot_least = 0xffffffffu;
                add_words<T>(v[k], slot_most, slot_least);
                if (from + k * THREADS < end && Elem<T>::largest(slot_most, slot_least) >= z_line) {
                    const int at = row.head + (from + k * THREADS) * N;
                    const uint32_t words[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll 1
                    for (int w = 0; w < 4; ++w) {        // (rarely more than one of them)
                        const uint4 one{w == 0 ? words[0] : w == 1 ? words[1] : w == 2 ? words[2] : words[3], 0, 0, 0};
                        float f[N];
                        Elem<T>::unpack(one, f);
#pragma unroll
                        for (int j = 0; j < N / 4; ++j) keep(f[j], at + w * (N / 4) + j);
                    }
                }
            }
        }
        __syncthreads();
        const int here = (end - begin) * N + (with_edge ? g.x.V - row.whole * N : 0), top = min(g.top, here);
        if (sh.kept > KEPT || sh.kept < top) select_by_digits<T, THREADS>(row, begin, end, with_edge, top, sh);
        else if (LONG) thin_kept<THREADS>(sh, top);
        finish_list<T, THREADS>(g, n, a, sh, top);
        __syncthreads();
    }
}

// Long rows, or slices of them, streamed: a line comes from the first step (2048 slots), and slots that reach it go to LDS whole, from all
// steps; a second line comes from their maxima, and only what reaches that is taken apart and ordered (64 of 65536 bf16, 4096 rows: 122 us).  Wave by wave some lane reaches
// the first line nearly always: taking elements apart at once (with the row in registers, or streamed) cost 4096 rows of 65536 bf16
// 187 us.
constexpr int kStreamSlots = 8;        // of a thread in a step

template <typename T, bool WITH_T, bool LONG>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4))) void k_top_stream(TopArgs g)
{
    constexpr int N = Elem<T>::N, STEP = kStreamSlots * 256;
    constexpr int kSlotsKept = LONG ? 1024 : 512;        // (a list of 128 has 710 of them in 65536 logits on the average, one of 64 about 360)
    __shared__ TopShared<1024> sh;
    __shared__ uint4 slots[kSlotsKept];
    __shared__ int32_t slot_at[kSlotsKept], n_slots;
    __shared__ float most_of[256], second_line;
    __shared__ RowPart part[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int64_t n = blockIdx.x; n < g.x.n; n += gridDim.x) {
        const Span<T> row(static_cast<const T *>(g.x.data) + n * g.x.stride, g.x.V);
        const int per = (row.whole + g.slices - 1) / g.slices, begin = min(row.whole, per * static_cast<int>(blockIdx.y)), end = min(row.whole, begin + per);
        const bool with_edge = blockIdx.y == 0;
        uint4 next[kStreamSlots];
        if (begin < end) {
#pragma unroll
            for (int k = 0; k < kStreamSlots; ++k) next[k] = row.load(min(begin + tid + k * 256, end - 1));
        }
        const int edge = with_edge ? row.edge(tid) : -1;
        const float z_edge = edge >= 0 ? Elem<T>::load(row.p + edge) : -INFINITY;
        if (tid == 0) sh.kept = n_slots = 0;
        Sums a;                                          // of this thread, relative to its own maximum
        float z_line = -INFINITY;
        auto raise = [&](float m) {
            if (!(m > a.m)) return;
            if (a.s != 0.0f) {
                const float d = (a.m - m) * g.per2, e = exp2_of(d);
                if (WITH_T) a.t = e * (a.t + fmaxf(d, kLowest) * a.s);
                a.s *= e;
            }
            a.m = m;
        };
        auto add_one = [&](float z) {
            const float y = (z - ref_of(a.m).m) * g.per2, e = exp2_of(y);
            a.s += e;
            if (WITH_T) a.t += e * fmaxf(y, kLowest);
        };
        // the highest line that `top` of the maxima reach, to the upper 20 bits of their numbers; per lane MINE of them
        auto line_of = [&](const auto &key) {
            constexpr int MINE = sizeof(key) / sizeof(key[0]);
            uint32_t line = 0;
            for (int b = 31; b >= 12; --b) {
                const uint32_t higher = line | 1u << b;
                int reach = 0;
#pragma unroll
                for (int w = 0; w < MINE; ++w) reach += __popcll(__ballot(key[w] >= higher));
                if (reach >= g.top) line = higher;
            }
            return line <= order_of(-INFINITY) ? -INFINITY : value_of(line);
        };
        for (int i = begin; i == begin || i < end; i += STEP) {
            uint4 v[kStreamSlots];
#pragma unroll
            for (int k = 0; k < kStreamSlots; ++k) v[k] = next[k];
            if (i + STEP < end) {
#pragma unroll
                for (int k = 0; k < kStreamSlots; ++k) next[k] = row.load(min(i + STEP + tid + k * 256, end - 1));
            }
            float most = -INFINITY;
            if (i + tid < end) {
                uint32_t words_most = Elem<T>::kNone, words_least = 0xffffffffu;
#pragma unroll
                for (int k = 0; k < kStreamSlots; ++k)
                    if (i + tid + k * 256 < end) add_words<T>(v[k], words_most, words_least);
                most = Elem<T>::largest(words_most, words_least);
            }
            if (i == begin) most = fmaxf(most, z_edge);
            raise(most);
            if (i == begin && edge >= 0) add_one(z_edge);
#pragma unroll
            for (int k = 0; k < kStreamSlots; ++k) {
                if (i + tid + k * 256 < end) {
                    float f[N];
                    Elem<T>::unpack(v[k], f);
#pragma unroll
                    for (int j = 0; j < N; ++j) add_one(f[j]);
                }
                keep_packed(v[k]);
            }
            if (i == begin) {
                most_of[tid] = most;
                __syncthreads();
                uint32_t key[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) key[w] = order_of(most_of[w * 64 + lane]);
                z_line = line_of(key);
            }
            if (most >= z_line) {
                int from = i + tid;
                asm volatile("" : "+v"(from));           // (the slots' numbers are taken anew)
#pragma unroll
                for (int k = 0; k < kStreamSlots; ++k) {
                    keep_packed(v[k]);
                    uint32_t slot_most = Elem<T>::kNone, slot_least = 0xffffffffu;
                    add_words<T>(v[k], slot_most, slot_least);
                    if (from + k * 256 < end && Elem<T>::largest(slot_most, slot_least) >= z_line) {
                        const int at = atomicAdd(&n_slots, 1);
                        if (at < kSlotsKept) {
                            slots[at] = v[k];
                            slot_at[at] = row.head + (from + k * 256) * N;
                        }
                    }
                }
            }
        }
        {
            const float m = max_of<64>(a.m);
            const Sums x = rebased_by(a, ref_of(m).m, g.per2);
            const float s = sum_of<64>(x.s), t = sum_of<64>(x.t);
            if (lane == 0) part[wave] = {m, s, t};
        }
        __syncthreads();
        {
            Sums of;
            if (lane < 4) of = {part[lane].m, part[lane].s, part[lane].t};
            const float m = max_of<64>(of.m);
            const Sums x = rebased_by(of, ref_of(m).m, g.per2);
            a = {m, sum_of<64>(x.s), sum_of<64>(x.t)};
        }
        const int here = (end - begin) * N + (with_edge ? g.x.V - row.whole * N : 0), top = min(g.top, here), count = n_slots;
        const bool fits = count <= kSlotsKept && a.s > 0.0f;         // (NaN is above no line)
        if (fits) {
            if (wave == 0) {
                uint32_t key[kSlotsKept / 64];
#pragma unroll
                for (int w = 0; w < kSlotsKept / 64; ++w) {
                    key[w] = 0;
                    if (w * 64 + lane < count) {
                        uint32_t slot_most = Elem<T>::kNone, slot_least = 0xffffffffu;
                        add_words<T>(slots[w * 64 + lane], slot_most, slot_least);
                        key[w] = order_of(Elem<T>::largest(slot_most, slot_least));
                    }
                }
                const float line = line_of(key);
                if (lane == 0) second_line = fmaxf(line, z_line);
            }
            __syncthreads();
            const float line = second_line;
            auto keep = [&](float z, int at) {
                if (z >= line) {
                    const int i = atomicAdd(&sh.kept, 1);
                    if (i < sh.kKept) sh.entry[i] = entry_of(z, at);
                }
            };
            if (edge >= 0) keep(z_edge, edge);
            for (int i = tid; i < count; i += 256) {
                float f[N];
                Elem<T>::unpack(slots[i], f);
                const int at = slot_at[i];
#pragma unroll
                for (int j = 0; j < N; ++j) keep(f[j], at + j);
            }
            __syncthreads();
        }
        if (!fits || sh.kept > sh.kKept || sh.kept < top) select_by_digits<T, 256>(row, begin, end, with_edge, top, sh);
        finish_list<T, 256>(g, n, a, sh, top);
        __syncthreads();
    }
}

// The lists of a row's slices together.  (Zeros end a list that is shorter than `top`.)
template <typename T>
__global__ __launch_bounds__(256) void k_top_join(TopArgs g)
{
    __shared__ TopShared<kTopKept> sh;
    __shared__ uint64_t best[PL_MAX_TOP];
    const int tid = threadIdx.x, lane = tid & 63;
    for (int64_t n = blockIdx.x; n < g.x.n; n += gridDim.x) {
        const uint64_t *lists = g.lists + n * g.slices * g.top;
        Sums a;
        float m = -INFINITY;
        bool none = false;
        for (int i = lane; i < g.slices; i += 64) {
            const RowPart of = g.parts[n * g.slices + i];
            m = fmaxf(m, of.m);
            none = none || of.m != of.m;
        }
        a.m = __any(none) ? NAN : max_of<64>(m);
        for (int i = lane; i < g.slices; i += 64) {
            const RowPart of = g.parts[n * g.slices + i];
            const Sums x = rebased_by({of.m, of.s, of.t}, ref_of(a.m).m, g.per2);
            a.s += x.s;
            a.t += x.t;
        }
        a.s = sum_of<64>(a.s);
        a.t = sum_of<64>(a.t);
        // rounds: the best so far and as many lists as there is room for
        const int group = (kTopKept - PL_MAX_TOP) / g.top;
        int have = 0;
        for (int l0 = 0; l0 < g.slices; l0 += group) {
            const int lists_now = min(group, g.slices - l0);
            if (tid == 0) sh.kept = have;
            for (int i = tid; i < have; i += 256) sh.entry[i] = best[i];
            __syncthreads();
            // left out: what `top` entries are above, of those kept so far or of these lists, whose first `ahead` of each are `top` together
            const int ahead = (g.top + lists_now - 1) / lists_now - 1;
            uint64_t line = ~uint64_t{0};
            for (int i = lane; i < lists_now; i += 64) line = min(line, lists[static_cast<int64_t>(l0 + i) * g.top + ahead]);
#pragma unroll
            for (int d = 32; d; d >>= 1) line = min(line, static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(line), d)));
            line = max(line == 0 ? uint64_t{0} : line - 1, have == g.top ? best[g.top - 1] : 0);
            for (int i = tid; i < lists_now * g.top; i += 256) {
                const uint64_t e = lists[static_cast<int64_t>(l0) * g.top + i];
                if (e > line) sh.entry[atomicAdd(&sh.kept, 1)] = e;
            }
            __syncthreads();
            const int kept = sh.kept;
            rank_kept<256>(sh, kept, g.top, [&](int place, uint64_t e) { best[place] = e; });
            have = min(kept, g.top);
            __syncthreads();
        }
        const RowLog log_p = row_log(g, a);
        for (int i = tid; i < g.top; i += 256) {
            g.out_top[n * g.top + i] = action_of(best[i]);
            if (g.out_top_logp) g.out_top_logp[n * g.top + i] = log_p(logit_of(best[i]));
        }
        if (tid == 0) finish_scores<T>(g, n, a, log_p);
        __syncthreads();
    }
}

constexpr int kShortTop = 64;

// A lane takes top V steps whatever the number of rows, a wave about as long for any width.  Calls, us, a row to a lane against one to a
// wave: the first 16 of 64 bf16, 16384 rows 30 against 22, 65536 32 against 79; all of 64, 65536 rows 100 against 122; 64 of 128, 65536
// rows 184 against 124; 1 of 17, 3.9 million rows 64 against 2990.
bool by_lanes(const LogitsView &x, int top)
{
    const int64_t steps = static_cast<int64_t>(top) * x.V;
    return x.V <= kLaneRow && steps <= 4096 && x.n >= 8192 + 16 * steps;
}

int slots_of(const LogitsView &x) { return x.dtype == PL_F32 ? (x.V + 3) / 4 : (x.V + 7) / 8; }

}  // namespace

TopWorkspace carve_top_workspace(void *base, const LogitsView &x, int top)
{
    TopWorkspace w;
    constexpr int kMost = 8192;                  // slots of a workgroup: what it keeps above the first step's line grows with them
    const int slots = slots_of(x);
    if (x.n > 0 && slots > kMost) w.slices = (slots + kMost - 1) / kMost;
    if (x.n > 0 && x.n < 64 && x.V >= 32768)
        w.slices = std::max(w.slices, static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({1024 / x.n, x.V / 8192, kMaxSlices}))));
    const size_t lists = w.slices > 1 ? static_cast<size_t>(x.n) * w.slices : 0;
    w.parts = static_cast<RowPart *>(base);
    const size_t at = (lists * sizeof(RowPart) + 15) / 16 * 16;
    w.lists = base ? reinterpret_cast<uint64_t *>(static_cast<char *>(base) + at) : nullptr;
    w.bytes = std::max<size_t>(16, at + lists * top * sizeof(uint64_t));
    return w;
}

void launch_top(TopArgs a, const TopWorkspace &ws, hipStream_t s)
{
    a.slices = ws.slices;
    a.parts = ws.parts;
    a.lists = ws.lists;
    by_type(a.x.dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int W = 4 / sizeof(T);
        if (a.x.V <= kNarrow) {
            const size_t bytes = a.x.V * sizeof(T), align = std::min<size_t>(bytes, 16);
            const bool whole = reinterpret_cast<uintptr_t>(a.x.data) % align == 0 && a.x.stride * sizeof(T) % align == 0;
            const dim3 grid(static_cast<uint32_t>((a.x.n + 255) / 256));
            const size_t lds = 256 * (a.x.V | 1) * sizeof(float);
            if (whole && bytes == 8) hipLaunchKernelGGL((k_top_narrow<T, 2 * W, true>), grid, dim3(256), 0, s, a);
            else if (whole && bytes == 16) hipLaunchKernelGGL((k_top_narrow<T, 4 * W, true>), grid, dim3(256), 0, s, a);
            else if (whole && bytes == 32) hipLaunchKernelGGL((k_top_narrow<T, 8 * W, true>), grid, dim3(256), 0, s, a);
            else hipLaunchKernelGGL((k_top_narrow<T, kNarrow, false>), grid, dim3(256), lds, s, a);
            return;
        }
        if (by_lanes(a.x, a.top)) {
            hipLaunchKernelGGL(k_top_lane<T>, dim3(static_cast<uint32_t>((a.x.n + 63) / 64)), dim3(64), 64 * (a.x.V | 1) * sizeof(float), s, a);
            return;
        }
        const int slots = (slots_of(a.x) + a.slices - 1) / a.slices;
        const uint32_t rows = static_cast<uint32_t>(std::min<int64_t>(a.x.n, 1 << 22));
        const dim3 grid(rows, a.slices);
        // (rows of a wave in turn: a workgroup for each would take as long to begin as to do)
        const dim3 waves(std::min<uint32_t>(rows, 1 << 13), a.slices);
        const bool longer = a.top > kShortTop;
        auto launch = [&](auto kernel, dim3 blocks, int threads) { hipLaunchKernelGGL(kernel, blocks, dim3(threads), 0, s, a); };
        if (slots <= 64) launch(k_top_row<T, 64, 1, 512, false>, waves, 64);
        else if (slots <= 64 * 4) launch(k_top_row<T, 64, 4, 1024, true>, grid, 64);
        else if (slots <= 64 * 8) launch(k_top_row<T, 64, 8, 1024, true>, grid, 64);
        else if (slots <= 256 * 4) launch(longer ? k_top_row<T, 256, 4, kTopKept, true> : k_top_row<T, 256, 4, kTopKept, false>, grid, 256);
        // (slices of few rows are done sooner in registers, with a barrier less: 37 rows of 50001 fp16 12.5 us as a call, streamed 14.7)
        else if (a.slices > 1 && slots <= 256 * 8) launch(longer ? k_top_row<T, 256, 8, kTopKept, true> : k_top_row<T, 256, 8, kTopKept, false>, grid, 256);
        else if (a.out_entropy) launch(longer ? k_top_stream<T, true, true> : k_top_stream<T, true, false>, grid, 256);
        else launch(longer ? k_top_stream<T, false, true> : k_top_stream<T, false, false>, grid, 256);
        if (a.slices > 1) hipLaunchKernelGGL(k_top_join<T>, dim3(rows), dim3(256), 0, s, a);
    });
}

}  // namespace pl

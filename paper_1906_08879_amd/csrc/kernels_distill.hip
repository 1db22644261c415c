// The loss against a teacher that is known by a list of actions in every row (include/placeto.h), with the gradient of the logits.
//
// With x_j = (z_j - m) / T, the row's maximum m, the sum R of e^x over the actions outside the list and S = R + the sum over the
// list: ln p_j = x_j - ln S, p_rest = R / S, and the gradient is e^{x_j} A outside the list, A = w / T (F - r / p_rest) / S.
// R is summed over the actions outside the list themselves, which are told apart by a bit for every element: as 1 - sum p it
// would be lost where the policy gives the list nearly everything.  Where it gives them less still, R leaves fp32 relative to the row's
// maximum, and so does r / p_rest: rows with a tail whose R is below 2^-40 (DistillArgs::least) take it again, relative to the largest of the
// others themselves, and their gradients too: e^{x_j} (F p_rest - r) / R with exponents that end at 0.  (A call of 512 actions a row takes 2% longer
// for looking, where no row does.)  What there is of a list, up to 128 entries, is done in float64 by
// one wave: values are small differences of log probabilities, and with S = R + list an error of R takes part in them only by
// p_rest - r.  Gradients at listed actions, F p - q, are differences as well.
//
// A row lies in the registers of a wave or a workgroup between its sums and its gradient (one read, one write), in a thread's up to
// 16 actions, in a lane's part of LDS up to 128 where there are many rows (by_lanes); the listed actions' gradients are then written once more
// by the thread that has written them.  Few long rows, and those too long for 960 threads, take a pass for the sums and one for the
// gradient.  A wave beside those that hold the row does the list (its float64 in their registers would spill theirs).
// Bound by memory from some thousand logits on (lists of 64, 8192 rows of 65536 bf16: 343 to 357 us on six cards, 6.0 to 6.3 TB/s; 4104 rows of 50001: 158 us, 5.2), below
// that by the list's float64 (lists of 3 of 8 fp32, 799744 rows: 33 us, where the bytes take 15).
#include <algorithm>
#include <cmath>

#include "rows.h"

namespace pl {
namespace {

struct Scale {
    float m, per2;
    __device__ float operator()(float z) const { return (z - m) * per2; }
};

// e^x to 10^-11 of it: 2^n times the series of e^{r ln 2} to the ninth power, n the whole number next to x log2 e and r the rest,
// |r| <= 1/2.  (The results end in fp32; exp of the library is several times as long.)
__device__ __forceinline__ double exp_of(double x)
{
    x = x < -1e4 ? -1e4 : x > 1e4 ? 1e4 : x;             // (NaN stays)
    const double y = x * 1.4426950408889634, n = rint(y), r = (y - n) * 0.6931471805599453;
    double s = 1.0 / 362880.0;
    s = fma(s, r, 1.0 / 40320.0);
    s = fma(s, r, 1.0 / 5040.0);
    s = fma(s, r, 1.0 / 720.0);
    s = fma(s, r, 1.0 / 120.0);
    s = fma(s, r, 1.0 / 24.0);
    s = fma(s, r, 1.0 / 6.0);
    s = fma(s, r, 0.5);
    s = fma(s, r, 1.0);
    s = fma(s, r, 1.0);
    return ldexp(s, static_cast<int>(n));
}

// ln x to about as much: from x = m 2^e the fp32 logarithm y and a step of Newton's from it, y + (x e^-y - 1), whose error is half the
// square of the first one's.
__device__ __forceinline__ double log_of(double x)
{
    int e;
    const double m = frexp(x, &e), y = 0.6931471805599453 * (static_cast<double>(log2f(static_cast<float>(m))) + e);
    return y + (x * exp_of(-y) - 1.0);
}

// ---- a row's list: entries i and i + 64 are those of lane i of one wave
struct Read {
    int id[2];                         // action; -1: left out
    float lq[2], z[2];
};

__device__ __forceinline__ void read_list(Read &r, const DistillArgs &g, int64_t n, int lane)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = lane + 64 * h;
        r.id[h] = -1;
        r.lq[h] = r.z[h] = -INFINITY;
        if (i < g.k) {
            r.id[h] = g.top[n * g.k + i];
            r.lq[h] = g.top_logp[n * g.k + i];
        }
    }
}

template <typename T>
__device__ __forceinline__ void read_logits(Read &r, const DistillArgs &g, int64_t n)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (r.id[h] < 0 || r.id[h] >= g.x.V || r.lq[h] == -INFINITY) r.id[h] = -1;
        else r.z[h] = Elem<T>::load(static_cast<const T *>(g.x.data) + n * g.x.stride + r.id[h]);
    }
}

// The list in LDS, where one wave goes over it.
struct List {
    double q[PL_MAX_TOP], e[PL_MAX_TOP];
    float lq[PL_MAX_TOP], z[PL_MAX_TOP], inside[PL_MAX_TOP];     // inside: the gradient at the first entry of an action
    int32_t id[PL_MAX_TOP], first[PL_MAX_TOP];
};

// Between writes and reads of different lanes of the wave.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Entries whose action the policy does not allow are left out.
__device__ __forceinline__ void keep_list(List &l, const Read &r, float m, const DistillArgs &g, int lane)
{
    const Scale x{m == -INFINITY ? 0.0f : m, g.per2};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = lane + 64 * h;
        if (i >= g.k) continue;
        const bool masked = r.z[h] == -INFINITY || (r.z[h] == lowest_of(g.x.dtype) && x(r.z[h]) < kNoChance);
        l.id[i] = masked ? -1 : r.id[h];
        l.lq[i] = r.lq[h];
        l.z[i] = r.z[h];
        l.first[i] = l.id[i] >= 0;
    }
    wave_sync();
}

// Which entries are the first of their action; whether any is not.
__device__ __forceinline__ bool mark_first(List &l, int lane, int k)
{
    bool again = false;
#pragma unroll 1
    for (int i = lane; i < k; i += 64) {
        const int id = l.id[i];
        bool first = id >= 0;
#pragma unroll 4
        for (int j = 0; j < i; ++j) first = first && l.id[j] != id;
        l.first[i] = first;
        again = again || (id >= 0 && !first);
    }
    wave_sync();
    return __any(again);
}

// The sum of e^x over the allowed actions outside the list (0: there are none), relative to the row's maximum or to one that is lower by
// `down` (< 0, in units of T), `least` = e^down.
struct Rest {
    double sum, down, least;
};

__device__ __forceinline__ Rest rest_below(const DistillArgs &g, double sum, float m, float most)
{
    const double down = (static_cast<double>(most) - m) * g.per;
    return {sum, down, exp_of(down)};
}

// What follows for a row from its maximum, its rest, and the list.
struct RowResult {
    double value, mass, share;
    float A;                           // e^x A: the gradient of the others, x as in their sum
};

__device__ __forceinline__ double tail_mass(double mass, double rest, int tail)
{
    return tail && rest > 0.0 && mass < 1.0 ? 1.0 - mass : 0.0;
}

// Sums over a list: of q, of e^x, and of q (ln q - x).
struct ListSums {
    double mass, list, cross;
};

__device__ __forceinline__ ListSums sum_list(const DistillArgs &g, List &l, int lane, float m)
{
    const double base = m == -INFINITY ? 0.0 : static_cast<double>(m);
    ListSums s{0.0, 0.0, 0.0};
#pragma unroll 1
    for (int i = lane; i < g.k; i += 64) {
        if (l.id[i] < 0) continue;
        const double lq = l.lq[i], x = (static_cast<double>(l.z[i]) - base) * g.per, q = exp_of(lq), e = exp_of(x);
        l.q[i] = q;
        l.e[i] = e;
        s.mass += q;
        s.cross += q * (lq - x);
        if (l.first[i]) s.list += e;
    }
    return {wave_sum(s.mass), wave_sum(s.list), wave_sum(s.cross)};
}

__device__ __forceinline__ RowResult finish_list(const DistillArgs &g, List &l, int lane, const ListSums &sums, const Rest &rest, float weight, bool repeated)
{
    const double mass = sums.mass, list = sums.list, S = fma(rest.sum, rest.least, list);
    RowResult r{0.0, mass, 0.0, 0.0f};
    if (S == 0.0) return r;                              // (nothing is allowed: nothing is listed either)
    const double per_S = 1.0 / S, tail = tail_mass(mass, rest.sum, g.tail), F = mass + tail, ratio = tail > 0.0 ? tail / rest.sum : 0.0;
    r.value = sums.cross + mass * log_of(S);
    if (tail > 0.0) r.value += tail * (log_of(ratio * S) - rest.down);
    r.share = list * per_S;
    const double scale = static_cast<double>(weight) * g.grad_scale * g.per;
    r.A = static_cast<float>(scale * (F * (rest.least * per_S) - ratio));
    wave_sync();
#pragma unroll 1
    for (int i = lane; i < g.k; i += 64) {
        if (!l.first[i]) continue;
        double q = l.q[i];
        if (repeated) {                                  // all entries of the action
            q = 0.0;
            const int id = l.id[i];
            for (int j = 0; j < g.k; ++j)
                if (l.id[j] == id) q += l.q[j];
        }
        l.inside[i] = static_cast<float>(scale * (F * (l.e[i] * per_S) - q));
    }
    return r;
}

__device__ __forceinline__ float weight_of(const DistillArgs &g, int seq)
{
    return g.w.weights ? g.w.weights[seq] : g.w.weight_at ? *g.w.weight_at : g.w.weight;
}

// What a row gives besides its gradient, by one wave.
__device__ __forceinline__ void row_outputs(const DistillArgs &g, int64_t n, int lane, const List &l, const RowResult &r, float weight,
                                            double (&acc)[3])
{
    if (g.out_coeff) {
        const double scale = static_cast<double>(weight) * g.grad_scale * g.per;
        for (int i = lane; i < g.k; i += 64) g.out_coeff[n * g.k + i] = l.id[i] >= 0 ? static_cast<float>(scale * l.q[i]) : 0.0f;
    }
    if (lane == 0 && g.out_values) g.out_values[n] = static_cast<float>(r.value);
    acc[0] += weight * r.value;
    acc[1] += weight * r.mass;
    acc[2] += weight * r.share;
}

__device__ __forceinline__ void row_nothing(const DistillArgs &g, int64_t n, int lane)
{
    if (g.out_coeff)
        for (int i = lane; i < g.k; i += 64) g.out_coeff[n * g.k + i] = 0.0f;
    if (lane == 0 && g.out_values) g.out_values[n] = 0.0f;
}

// ---- the loss from the workgroups' sums, in their order
__global__ __launch_bounds__(1024) void k_distill_stats(const double *__restrict__ sums, int blocks, float *__restrict__ out)
{
    const int tid = threadIdx.x;
    double a = 0.0;                              // of sum tid & 3
#pragma unroll 8
    for (int64_t i = tid; i < static_cast<int64_t>(blocks) * 4; i += 1024) a += sums[i];
#pragma unroll
    for (int o = 32; o >= 4; o >>= 1) a += __shfl_xor(a, o);
    __shared__ double last[16][4];
    if ((tid & 63) < 4) last[tid >> 6][tid & 3] = a;
    __syncthreads();
    if (tid < 3) {
        double v = 0.0;
        for (int w = 0; w < 16; ++w) v += last[w][tid];
        out[tid] = static_cast<float>(v);
    }
}

// A workgroup's sums, or the loss itself where nobody else has a part.
__device__ __forceinline__ void block_out(const DistillArgs &g, int i, double v)
{
    if (gridDim.x == 1) {
        if (i < 3) g.out_stats[i] = static_cast<float>(v);
    } else {
        g.sums[static_cast<size_t>(blockIdx.x) * 4 + i] = v;
    }
}

// ---- narrow rows: a row to a thread.  (Four waves to a SIMD: with 132 registers instead of 128, three, 200000 rows of 16 bf16 37.6 us instead
// of 34.9.)
template <typename T, int CAP, bool WHOLE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(WHOLE ? 4 : 1))) void k_distill_narrow(DistillArgs g)
{
    extern __shared__ float tile[];
    __shared__ double sums[4][4];
    const int V = WHOLE ? CAP : g.x.V, pitch = V | 1, tid = threadIdx.x;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 256, n = n0 + tid;
    const int count = static_cast<int>(min(int64_t{256}, g.x.n - n0));
    double acc[3] = {0.0, 0.0, 0.0};
    Place at{0, false};
    if (tid < count) at = place_of(g.rows, n);
    float z[CAP];
    if (WHOLE) {
        if (at.counts) {
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
    auto each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < CAP; ++j)
            if (WHOLE || j < V) f(j, z[j]);
    };
    float grad[CAP];
#pragma unroll
    for (int j = 0; j < CAP; ++j) grad[j] = 0.0f;
    if (at.counts) {
        float m = -INFINITY;
        each([&](int, float v) { m = fmaxf(m, v); });
        const double base = m == -INFINITY ? 0.0 : static_cast<double>(m);
        const Scale x{static_cast<float>(base), g.per2};
        const float weight = weight_of(g, at.seq), low = lowest_of(g.x.dtype);
        uint32_t allowed = 0;
        each([&](int j, float v) { allowed |= (v == -INFINITY || (v == low && x(v) < kNoChance) ? 0u : 1u) << j; });
        // the list: q and e^x of every action that it has
        uint32_t listed = 0;
        double q[CAP], e_listed[CAP], mass = 0.0, list = 0.0, cross = 0.0;
#pragma unroll
        for (int j = 0; j < CAP; ++j) q[j] = e_listed[j] = 0.0;
        for (int i = 0; i < g.k; ++i) {
            const int id = g.top[n * g.k + i];
            const float lq = g.top_logp[n * g.k + i];
            if (id < 0 || id >= V || lq == -INFINITY || !(allowed >> id & 1)) continue;
            float mine = z[0];
#pragma unroll
            for (int j = 1; j < CAP; ++j)
                if (WHOLE || j < V) mine = j == id ? z[j] : mine;
            const double p = exp_of(lq), y = (static_cast<double>(mine) - base) * g.per, e = exp_of(y);
            mass += p;
            cross += p * (lq - y);
            if (!(listed >> id & 1)) list += e;
            listed |= 1u << id;
#pragma unroll
            for (int j = 0; j < CAP; ++j) {
                q[j] += j == id ? p : 0.0;
                e_listed[j] = j == id ? e : e_listed[j];
            }
        }
        const uint32_t others = allowed & ~listed;
        Scale y = x;                             // of the others
        auto e_other = [&](int j, float v) { return others >> j & 1 ? exp2_of(y(v)) : 0.0f; };
        float sum = 0.0f;
        each([&](int j, float v) { sum += e_other(j, v); });
        double down = 0.0, least = 1.0;
        if (sum < g.least && others) {
            y.m = -INFINITY;
            each([&](int j, float v) { y.m = others >> j & 1 ? fmaxf(y.m, v) : y.m; });
            down = (static_cast<double>(y.m) - base) * g.per;
            least = exp_of(down);
            sum = 0.0f;
            each([&](int j, float v) { sum += e_other(j, v); });
        }
        const double rest = sum;
        const double S = rest * least + list, per_s = S == 0.0 ? 0.0 : 1.0 / S, tail = tail_mass(mass, rest, g.tail), F = mass + tail,
                     ratio = tail > 0.0 ? tail / rest : 0.0;
        double value = cross + mass * log_of(S);
        if (tail > 0.0) value += tail * (log_of(ratio * S) - down);
        if (S == 0.0) value = 0.0;
        const double scale = static_cast<double>(weight) * g.grad_scale * g.per;
        const float A = S == 0.0 ? 0.0f : static_cast<float>(scale * (F * (least * per_s) - ratio));
        if (g.out_grad) {
            each([&](int j, float v) {
                if (listed >> j & 1) grad[j] = static_cast<float>(scale * (F * (e_listed[j] * per_s) - q[j]));
                else grad[j] = e_other(j, v) * A;
            });
        }
        if (g.out_values) g.out_values[n] = static_cast<float>(value);
        acc[0] = weight * value;
        acc[1] = weight * mass;
        acc[2] = weight * list * per_s;
        if (g.out_coeff)
            for (int i = 0; i < g.k; ++i) {
                const int id = g.top[n * g.k + i];
                const float lq = g.top_logp[n * g.k + i];
                const bool in = id >= 0 && id < V && lq != -INFINITY && (allowed >> id & 1);
                g.out_coeff[n * g.k + i] = in ? static_cast<float>(scale * exp_of(lq)) : 0.0f;
            }
    } else if (tid < count) {
        if (g.out_values) g.out_values[n] = 0.0f;
        if (g.out_coeff)
            for (int i = 0; i < g.k; ++i) g.out_coeff[n * g.k + i] = 0.0f;
    }
    if (g.out_grad) {
        if (WHOLE) {
            if (tid < count) {
                Words<CAP * sizeof(T)> words;
                pack_words<T, CAP>(grad, words.w);
                words.store(static_cast<T *>(g.out_grad) + n * g.grad_stride);
            }
        } else {
#pragma unroll
            for (int j = 0; j < CAP; ++j)
                if (j < V) tile[tid * pitch + j] = grad[j];
            __syncthreads();
            narrow_tile<T, true>(g.out_grad, g.grad_stride, n0, count, V, g.magic, pitch, tile);
        }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const double v = wave_sum(acc[i]);
        if ((tid & 63) == 0) sums[tid >> 6][i] = v;
    }
    __syncthreads();
    if (tid < 4) block_out(g, tid, tid < 3 ? (sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]) : 0.0);
}

// ---- many rows of some more actions: a row to a lane still, in LDS
template <typename T>
__global__ __launch_bounds__(64) void k_distill_lane(DistillArgs g)
{
    extern __shared__ float tile[];
    const int V = g.x.V, pitch = V | 1, tid = threadIdx.x;
    double acc[3] = {0.0, 0.0, 0.0};
    for (int64_t n0 = static_cast<int64_t>(blockIdx.x) * 64; n0 < g.x.n; n0 += static_cast<int64_t>(gridDim.x) * 64) {
        const int64_t n = n0 + tid;
        const int count = static_cast<int>(min(int64_t{64}, g.x.n - n0));
        narrow_tile<T, false, 64>(g.x.data, g.x.stride, n0, count, V, g.magic, pitch, tile);
        __syncthreads();
        Place at{0, false};
        if (tid < count) at = place_of(g.rows, n);
        float *z = tile + tid * pitch;
        if (at.counts) {
            float m = -INFINITY;
#pragma unroll 8
            for (int j = 0; j < V; ++j) m = fmaxf(m, z[j]);
            const double base = m == -INFINITY ? 0.0 : static_cast<double>(m);
            const Scale x{static_cast<float>(base), g.per2};
            const float weight = weight_of(g, at.seq), low = lowest_of(g.x.dtype);
            const double scale = static_cast<double>(weight) * g.grad_scale * g.per;
            // the list; a bit for every action that it has
            uint64_t listed_low = 0, listed_high = 0;
            auto bit_of = [&](int j) { return (j < 64 ? listed_low : listed_high) >> (j & 63) & 1; };
            double mass = 0.0, list = 0.0, cross = 0.0, value = 0.0, F = 0.0, per_s = 0.0;
            bool again = false;
#pragma unroll 1
            for (int pass = 0; pass < (g.out_grad ? 2 : 1); ++pass) {    // the sums; the gradients from them
                for (int i = 0; i < g.k; ++i) {
                    const int id = g.top[n * g.k + i];
                    const float lq = g.top_logp[n * g.k + i];
                    float coeff = 0.0f;
                    bool in = id >= 0 && id < V && lq != -INFINITY;
                    if (in) {
                        const float mine = z[id];
                        in = pass ? bit_of(id) : !(mine == -INFINITY || (mine == low && x(mine) < kNoChance));
                        if (in) {
                            const double y = (static_cast<double>(mine) - base) * g.per, e = exp_of(y);
                            double p = 0.0;
                            int j = i;                   // all entries of the action, at its first one
#pragma unroll 1
                            do
                                if (g.top[n * g.k + j] == id) p += exp_of(g.top_logp[n * g.k + j]);
                            while (++j < g.k && pass && again);
                            const uint64_t low_bit = id < 64 ? uint64_t{1} << id : 0, high_bit = id < 64 ? 0 : uint64_t{1} << (id - 64);
                            if (pass) {
                                z[id] = static_cast<float>(scale * (F * (e * per_s) - p));
                                listed_low &= ~low_bit;
                                listed_high &= ~high_bit;
                            } else {
                                mass += p;
                                cross += p * (lq - y);
                                if (bit_of(id)) again = true;
                                else list += e;
                                listed_low |= low_bit;
                                listed_high |= high_bit;
                                coeff = static_cast<float>(scale * p);
                            }
                        }
                    }
                    if (!pass && g.out_coeff) g.out_coeff[n * g.k + i] = coeff;
                }
                if (pass) break;
                Scale y = x;                         // of the others
                double rest = 0.0, down = 0.0, least = 1.0;
                auto sum_rest = [&]() {
                    rest = 0.0;
#pragma unroll 4
                    for (int j = 0; j < V; ++j) rest += bit_of(j) ? 0.0f : exp2_of(y(z[j]));
                };
                sum_rest();
                if (rest < g.least) {
                    float most = -INFINITY;
#pragma unroll 1
                    for (int j = 0; j < V; ++j) {
                        if (bit_of(j)) continue;
                        if (z[j] == low && x(low) < kNoChance) z[j] = -INFINITY;
                        most = fmaxf(most, z[j]);
                    }
                    if (most != -INFINITY) {
                        y.m = most;
                        down = (static_cast<double>(most) - base) * g.per;
                        least = exp_of(down);
                        sum_rest();
                    }
                }
                const double S = rest * least + list;
                per_s = S == 0.0 ? 0.0 : 1.0 / S;
                const double p_rest = rest * per_s, tail = tail_mass(mass, rest, g.tail);
                F = mass + tail;
                value = cross;
#pragma unroll 1
                for (int l = 0; l < (tail > 0.0 ? 2 : 1); ++l) value += (l ? tail : mass) * (log_of(l ? tail / p_rest : S) - (l ? down : 0.0));
                if (S == 0.0) value = 0.0;
                const float A = S == 0.0 ? 0.0f : static_cast<float>(scale * (F * least - (tail > 0.0 ? tail / p_rest : 0.0)) * per_s);
                if (g.out_grad) {
#pragma unroll 4
                    for (int j = 0; j < V; ++j)
                        if (!bit_of(j)) z[j] = S == 0.0 ? 0.0f : exp2_of(y(z[j])) * A;
                }
            }
            if (g.out_values) g.out_values[n] = static_cast<float>(value);
            acc[0] += weight * value;
            acc[1] += weight * mass;
            acc[2] += weight * list * per_s;
        } else if (tid < count) {
            if (g.out_grad)
                for (int j = 0; j < V; ++j) z[j] = 0.0f;
            if (g.out_values) g.out_values[n] = 0.0f;
            if (g.out_coeff)
                for (int i = 0; i < g.k; ++i) g.out_coeff[n * g.k + i] = 0.0f;
        }
        __syncthreads();
        if (g.out_grad) {
            narrow_tile<T, true, 64>(g.out_grad, g.grad_stride, n0, count, V, g.magic, pitch, tile);
            __syncthreads();
        }
    }
    const double sums[3] = {wave_sum(acc[0]), wave_sum(acc[1]), wave_sum(acc[2])};
    if (tid < 4) block_out(g, tid, tid == 0 ? sums[0] : tid == 1 ? sums[1] : tid == 2 ? sums[2] : 0.0);
}

// ---- wider rows.  A bit for every element of the slots at hand, and the listed actions by the threads that have them.
template <int THREADS, int CH, int N>
struct Marks {
    static constexpr int kSlots = THREADS * CH, kWords = kSlots * N / 32 + 1;
    uint32_t bits[kWords];             // the last one: of the elements in front of and behind the slots
    int32_t head[THREADS], next[PL_MAX_TOP];     // the entries of a thread's elements, chained; -1 ends them
    __device__ void clear()
    {
        for (int i = threadIdx.x; i < kWords; i += THREADS) bits[i] = 0;
        head[threadIdx.x] = -1;
    }
    // Number of the bit of an element, and the thread that has the element; -1: none of the slots from `begin` to `end`.
    static __device__ int bit_of(int e, int row_head, int row_tail, int begin, int end, bool with_edge, int *thread)
    {
        if (e < row_head || e >= row_tail) {
            *thread = e < row_head ? e : N + (e - row_tail);
            return with_edge ? kSlots * N + *thread : -1;
        }
        const int slot = (e - row_head) / N - begin;
        *thread = static_cast<int>(static_cast<uint32_t>(max(slot, 0)) % THREADS);
        return slot >= 0 && slot < end - begin ? slot * N + (e - row_head) % N : -1;
    }
    // by one wave; whether an action was marked before
    __device__ bool mark(int bit) { return atomicOr(&bits[bit >> 5], 1u << (bit & 31)) >> (bit & 31) & 1; }
    __device__ void link(int i, int thread) { next[i] = atomicExch(&head[thread], i); }
    __device__ uint32_t of_slot(int slot) const { return bits[slot * N / 32] >> (slot * N % 32) & ((1u << N) - 1); }
    __device__ bool of_edge(int lane) const { return bits[kWords - 1] >> lane & 1; }
};

// Sum of e^x over the unmarked elements of a slot.
template <int N>
__device__ __forceinline__ float unmarked_sum(const float (&f)[N], uint32_t marks, const Scale &x)
{
    float s = 0.0f;
    if (__any(marks != 0)) {
#pragma unroll
        for (int j = 0; j < N; ++j) s += marks >> j & 1 ? 0.0f : exp2_of(x(f[j]));
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) s += exp2_of(x(f[j]));
    }
    return s;
}

// The gradient of a slot and of an element: e^x A.
template <typename T>
__device__ __forceinline__ void write_slot(T *out, const uint4 &v, float A, const Scale &x)
{
    constexpr int N = Elem<T>::N;
    float f[N];
    Elem<T>::unpack(v, f);
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = A == 0.0f ? 0.0f : exp2_of(x(f[j])) * A;
    stream_16(out, Elem<T>::pack(f));
}

// The elements of a slot that are masked or listed as -infinity, which has no part in a sum; and the maximum of the others.
template <typename T>
__device__ __forceinline__ void leave_others(uint4 &v, uint32_t marks, float masked, float &most)
{
    constexpr int N = Elem<T>::N;
    float f[N];
    Elem<T>::unpack(v, f);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        f[j] = marks >> j & 1 || f[j] == masked ? -INFINITY : f[j];
        most = fmaxf(most, f[j]);
    }
    v = Elem<T>::pack(f);
}

// THREADS threads have the row in registers, CH slots each; one more wave has the list.  Its float64 arithmetic runs beside the sums,
// and needs registers that the others hold the row in: in one of them 130 to 220 bytes a thread were spilled.
template <typename T, int THREADS, int CH>
__global__ __launch_bounds__(THREADS + 64) __attribute__((amdgpu_waves_per_eu(4))) void k_distill_row(DistillArgs g)
{
    constexpr int N = Elem<T>::N, WAVES = THREADS / 64;
    __shared__ Marks<THREADS, CH, N> marks;
    __shared__ List list;
    __shared__ float most_of[WAVES], rest_of[WAVES];
    __shared__ struct __align__(8) {
        float A;
        int again;                                   // the others' sum is taken again
    } shared;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    auto row_most = [&]() { return max_of<64>(most_of[lane < WAVES ? lane : 0]); };
    if (wave == WAVES) {                             // (the barriers of both branches answer one another)
        double acc[3] = {0.0, 0.0, 0.0};
        for (int64_t n = blockIdx.x; n < g.x.n; n += gridDim.x) {
            const Place place = place_of(g.rows, n);
            if (!place.counts) {
                row_nothing(g, n, lane);
                continue;
            }
            const Span<T> row(static_cast<const T *>(g.x.data) + n * g.x.stride, g.x.V);
            Read read;
            read_list(read, g, n, lane);
            read_logits<T>(read, g, n);
            const float weight = weight_of(g, place.seq);
            __syncthreads();                         // the maximum; marks are clear
            const float m = row_most();
            keep_list(list, read, m, g, lane);
            bool again = false;
#pragma unroll 1
            for (int i = lane; i < g.k; i += 64)
                if (list.id[i] >= 0) {
                    int thread;
                    again = marks.mark(marks.bit_of(list.id[i], row.head, row.tail(), 0, row.whole, true, &thread)) || again;
                    marks.next[i] = thread;
                }
            const bool repeated = __any(again);
            __syncthreads();                         // the marks
            if (repeated) mark_first(list, lane, g.k);
            const ListSums sums = sum_list(g, list, lane, m);
            __syncthreads();                         // the sums of the others
            auto rest_sum = [&]() { return wave_sum(lane < WAVES ? static_cast<double>(rest_of[lane]) : 0.0); };
            Rest rest{rest_sum(), 0.0, 1.0};
            bool given_up = g.tail && rest.sum < g.least;
            if (given_up && g.k >= g.x.V) {          // (not where all actions are listed)
                int listed = 0;
                for (int i = lane; i < PL_MAX_TOP; i += 64) listed += __popcll(__ballot(i < g.k && list.first[i]));
                given_up = listed < g.x.V;
            }
            if (__builtin_expect(given_up, false)) {
                if (lane == 0) shared.again = 1;
                __syncthreads();                     // (the others wait here for what follows from their sums)
                __syncthreads();                     // their own maximum
                const float most = row_most();
                __syncthreads();                     // their sums
                if (most != -INFINITY) rest = rest_below(g, rest_sum(), m, most);
            }
            const RowResult r = finish_list(g, list, lane, sums, rest, weight, repeated);
            if (lane == 0) {
                shared.A = r.A;
                shared.again = 0;
            }
#pragma unroll 1
            for (int i = lane; i < g.k; i += 64)
                if (list.first[i]) marks.link(i, marks.next[i]);
            __syncthreads();                         // the gradient's factor and entries
            row_outputs(g, n, lane, list, r, weight, acc);
            __syncthreads();                         // the row is written
        }
        if (lane == 0) {
            for (int i = 0; i < 3; ++i) block_out(g, i, acc[i]);
            block_out(g, 3, 0.0);
        }
        return;
    }
    int tid = threadIdx.x;
    for (int64_t n = blockIdx.x; n < g.x.n; n += gridDim.x) {
        asm volatile("" : "+v"(tid));                // (addresses are taken anew for every row)
        const Span<T> row(static_cast<const T *>(g.x.data) + n * g.x.stride, g.x.V);
        T *out = g.out_grad ? static_cast<T *>(g.out_grad) + n * g.grad_stride : nullptr;
        const int edge = row.edge(tid), whole = row.whole;
        if (!place_of(g.rows, n).counts) {
            if (out) {
#pragma unroll
                for (int k = 0; k < CH; ++k)
                    if (k * THREADS + tid < whole) stream_16(out + row.head + (k * THREADS + tid) * N, uint4{0, 0, 0, 0});
                if (edge >= 0) Elem<T>::store(out + edge, 0.0f);
            }
            continue;
        }
        uint4 v[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if (k * THREADS < whole) v[k] = row.load(k * THREADS + tid);
        float z_edge = edge >= 0 ? Elem<T>::load(row.p + edge) : -INFINITY;
        marks.clear();
        uint32_t most = Elem<T>::kNone, least = 0xffffffffu;
#pragma unroll
        for (int k = 0; k < CH; ++k)
            if (k * THREADS < whole) add_words<T>(v[k], most, least);
        const float wave_most = max_of<64>(fmaxf(z_edge, whole > 0 ? Elem<T>::largest(most, least) : -INFINITY));
        if (lane == 0) most_of[wave] = wave_most;
        __syncthreads();
        Scale x{ref_of(row_most()).m, g.per2};
        __syncthreads();
        float rest = edge >= 0 && !marks.of_edge(tid) ? exp2_of(x(z_edge)) : 0.0f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (k * THREADS + tid < whole) {
                float f[N];
                Elem<T>::unpack(v[k], f);
                rest += unmarked_sum<N>(f, marks.of_slot(k * THREADS + tid), x);
            }
            keep_packed(v[k]);
        }
        rest = sum_of<64>(rest);
        if (lane == 0) rest_of[wave] = rest;
        __syncthreads();
        __syncthreads();
        float A = shared.A;
        if (g.tail && __builtin_expect(shared.again, 0)) {
            const float low = lowest_of(g.x.dtype), masked = x(low) < kNoChance ? low : -INFINITY;
            float most = -INFINITY;
            if (edge >= 0) {
                if (marks.of_edge(tid) || z_edge == masked) z_edge = -INFINITY;
                most = z_edge;
            }
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                keep_packed(v[k]);
                if (k * THREADS + tid < whole) leave_others<T>(v[k], marks.of_slot(k * THREADS + tid), masked, most);
            }
            most = max_of<64>(most);
            if (lane == 0) most_of[wave] = most;
            __syncthreads();
            most = row_most();
            if (most != -INFINITY) {                 // (else there are none, and their sum was 0)
                x.m = most;
                rest = edge >= 0 ? exp2_of(x(z_edge)) : 0.0f;
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    keep_packed(v[k]);
                    if (k * THREADS + tid < whole) {
                        float f[N];
                        Elem<T>::unpack(v[k], f);
                        rest += unmarked_sum<N>(f, 0, x);
                    }
                }
                rest = sum_of<64>(rest);
                if (lane == 0) rest_of[wave] = rest;
            }
            __syncthreads();
            __syncthreads();
            A = shared.A;
        }
        if (out) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                keep_packed(v[k]);
                if (k * THREADS + tid < whole) write_slot<T>(out + row.head + static_cast<uint32_t>(k * THREADS + tid) * N, v[k], A, x);
            }
            if (edge >= 0) Elem<T>::store(out + edge, A == 0.0f ? 0.0f : exp2_of(x(z_edge)) * A);
            // the listed actions' gradients, once more by the threads that have written them
            for (int i = marks.head[tid]; i >= 0; i = marks.next[i]) Elem<T>::store(out + list.id[i], list.inside[i]);
        }
        __syncthreads();
    }
}

// ---- rows in slices: sums over the unlisted actions, then what follows from them, then the gradient
constexpr int kPartSlots = 8;          // of a thread in a step

// Of a part's actions outside the list the sum relative to its largest logit, listed or not; where that is below `least`, or the
// part lies near the type's lowest value, relative to their own maximum, without those at the lowest value, which are counted: whether they are masked
// goes by the row's maximum.
template <typename T>
__global__ __launch_bounds__(256) void k_distill_part(DistillArgs g)
{
    constexpr int N = Elem<T>::N, STEP = kPartSlots * 256;
    __shared__ Marks<256, kPartSlots, N> marks;
    __shared__ RowPart part[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int64_t n = blockIdx.x; n < g.x.n; n += gridDim.x) {
        if (!place_of(g.rows, n).counts) continue;
        const Span<T> row(static_cast<const T *>(g.x.data) + n * g.x.stride, g.x.V);
        const int per = (row.whole + g.slices - 1) / g.slices, begin = min(row.whole, per * static_cast<int>(blockIdx.y)), end = min(row.whole, begin + per);
        const bool with_edge = blockIdx.y == 0;
        const int edge = with_edge ? row.edge(tid) : -1;
        const float z_edge = edge >= 0 ? Elem<T>::load(row.p + edge) : -INFINITY;
        auto set_marks = [&](int b0, int b1) {
            marks.clear();
            __syncthreads();
            for (int i = tid; i < g.k; i += 256) {
                const int id = g.top[n * g.k + i];
                int thread;
                if (id >= 0 && id < g.x.V && g.top_logp[n * g.k + i] != -INFINITY) {
                    const int bit = marks.bit_of(id, row.head, row.tail(), b0, b1, with_edge && b0 == begin, &thread);
                    if (bit >= 0) marks.mark(bit);
                }
            }
            __syncthreads();
        };
        float m = -INFINITY;
        double s = 0.0;                              // of this thread, relative to m
        for (int b0 = begin; b0 == begin || b0 < end; b0 += STEP) {
            const int b1 = min(end, b0 + STEP);
            uint4 v[kPartSlots];
#pragma unroll
            for (int k = 0; k < kPartSlots; ++k)
                if (b0 + k * 256 + tid < b1) v[k] = row.load(b0 + k * 256 + tid);
            set_marks(b0, b1);
            uint32_t most = Elem<T>::kNone, least = 0xffffffffu;
#pragma unroll
            for (int k = 0; k < kPartSlots; ++k)
                if (b0 + k * 256 + tid < b1) add_words<T>(v[k], most, least);
            float next = fmaxf(m, b0 + tid < b1 ? Elem<T>::largest(most, least) : -INFINITY);
            if (b0 == begin) next = fmaxf(next, z_edge);
            const Scale x{ref_of(next).m, g.per2};
            if (s != 0.0) s *= exp2_of(x(m));
            m = next;
            float add = b0 == begin && edge >= 0 && !marks.of_edge(tid) ? exp2_of(x(z_edge)) : 0.0f;
#pragma unroll
            for (int k = 0; k < kPartSlots; ++k)
                if (b0 + k * 256 + tid < b1) {
                    float f[N];
                    Elem<T>::unpack(v[k], f);
                    add += unmarked_sum<N>(f, marks.of_slot(k * 256 + tid), x);
                }
            s += add;
            __syncthreads();
        }
        const float wave_m = max_of<64>(m);
        s = wave_sum(s == 0.0 ? 0.0 : s * exp2_of((m - ref_of(wave_m).m) * g.per2));
        if (lane == 0) part[wave] = {wave_m, static_cast<float>(s), 0.0f};
        __syncthreads();
        const float all = fmaxf(fmaxf(part[0].m, part[1].m), fmaxf(part[2].m, part[3].m)), low = lowest_of(g.x.dtype);
        double sum = 0.0;
        for (int w = 0; w < 4; ++w)
            if (part[w].s != 0.0f) sum += static_cast<double>(part[w].s) * exp2_of((part[w].m - ref_of(all).m) * g.per2);
        DistillPart of{all, all, static_cast<float>(sum), 0.0f};
        if (g.tail && all != -INFINITY && (sum < g.least || !((low - all) * g.per2 < kNoChance))) {
            of.base = -INFINITY;
            of.s = 0.0f;
#pragma unroll 1
            for (int pass = 0; pass < 2; ++pass) {   // the maximum and the number of the lowest; the sum
                const Scale x{ref_of(of.base).m, g.per2};
                float most = -INFINITY, add = 0.0f;
                auto take = [&](float z) {
                    if (z != low) most = fmaxf(most, z);
                    add += pass ? (z == low ? 0.0f : exp2_of(x(z))) : z == low ? 1.0f : 0.0f;
                };
#pragma unroll 1
                for (int b0 = begin; b0 == begin || b0 < end; b0 += STEP) {
                    const int b1 = min(end, b0 + STEP);
                    __syncthreads();
                    set_marks(b0, b1);
                    if (b0 == begin && edge >= 0 && !marks.of_edge(tid)) take(z_edge);
#pragma unroll 2
                    for (int i = b0 + tid; i < b1; i += 256) {
                        float f[N];
                        Elem<T>::unpack(row.load(i), f);
                        const uint32_t marked = marks.of_slot(i - b0);
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            if (!(marked >> j & 1)) take(f[j]);
                    }
                }
                most = max_of<64>(most);
                add = sum_of<64>(add);
                if (lane == 0) part[wave] = {most, add, 0.0f};
                __syncthreads();
                of.base = fmaxf(fmaxf(part[0].m, part[1].m), fmaxf(part[2].m, part[3].m));
                (pass ? of.s : of.lowest) = (part[0].s + part[1].s) + (part[2].s + part[3].s);
            }
        }
        if (tid == 0) g.parts[n * g.slices + blockIdx.y] = of;
        __syncthreads();
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_distill_finish(DistillArgs g)
{
    __shared__ double sums[4][4];
    __shared__ List lists[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    double acc[3] = {0.0, 0.0, 0.0};
    for (int64_t n = static_cast<int64_t>(blockIdx.x) * 4 + wave; n < g.x.n; n += static_cast<int64_t>(gridDim.x) * 4) {
        const Place place = place_of(g.rows, n);
        RowGrad rg{0.0f, 0.0f, 0.0f, 0.0f};
        List &list = lists[wave];
        if (place.counts) {
            Read read;
            read_list(read, g, n, lane);
            float m = -INFINITY;
            for (int i = lane; i < g.slices; i += 64) m = fmaxf(m, g.parts[n * g.slices + i].m);
            read_logits<T>(read, g, n);
            m = max_of<64>(m);
            // the sum of the others relative to `to`
            const float low = lowest_of(g.x.dtype);
            auto sum_rest = [&](float to, bool with_lowest) {
                const Scale x{ref_of(to).m, g.per2};
                double sum = 0.0;
                for (int i = lane; i < g.slices; i += 64) {
                    const DistillPart of = g.parts[n * g.slices + i];
                    if (of.s != 0.0f) sum += static_cast<double>(of.s) * exp2_of(x(of.base));
                    if (of.lowest != 0.0f && with_lowest) sum += static_cast<double>(of.lowest) * exp2_of(x(low));
                }
                return wave_sum(sum);
            };
            Rest rest{sum_rest(m, true), 0.0, 1.0};
            float base = m;
            const bool given_up = rest.sum < g.least, masked = Scale{ref_of(m).m, g.per2}(low) < kNoChance;
            if (given_up) {
                float most = -INFINITY;
                for (int i = lane; i < g.slices; i += 64) {
                    const DistillPart of = g.parts[n * g.slices + i];
                    if (of.s != 0.0f) most = fmaxf(most, of.base);
                    if (of.lowest != 0.0f && !masked) most = fmaxf(most, low);
                }
                most = max_of<64>(most);
                if (most != -INFINITY) rest = rest_below(g, sum_rest(base = most, !masked), m, most);
            }
            keep_list(list, read, m, g, lane);
            const bool repeated = mark_first(list, lane, g.k);
            const float weight = weight_of(g, place.seq);
            const RowResult r = finish_list(g, list, lane, sum_list(g, list, lane, m), rest, weight, repeated);
            row_outputs(g, n, lane, list, r, weight, acc);
            rg = {base, r.A, given_up && masked ? 1.0f : 0.0f, 0.0f};
        } else {
            row_nothing(g, n, lane);
        }
        if (g.out_grad) {
            if (lane == 0) g.row_grad[n] = rg;
            for (int i = lane; i < g.k; i += 64) {
                const bool first = place.counts && list.first[i];
                g.at[n * g.k + i] = first ? list.id[i] : -1;
                g.inside[n * g.k + i] = first ? list.inside[i] : 0.0f;
            }
        }
    }
    if (lane < 4) sums[wave][lane] = lane == 0 ? acc[0] : lane == 1 ? acc[1] : lane == 2 ? acc[2] : 0.0;
    __syncthreads();
    if (tid < 4) block_out(g, tid, (sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid]));
}

constexpr int kGradChunk = 4;          // slots of a thread

template <typename T>
__global__ __launch_bounds__(256) void k_distill_grad(DistillArgs g, int chunks)
{
    constexpr int N = Elem<T>::N, STEP = kGradChunk * 256;
    __shared__ Marks<256, kGradChunk, N> marks;
    __shared__ int32_t at[PL_MAX_TOP];
    __shared__ float inside[PL_MAX_TOP];
    const int tid = threadIdx.x;
    const int64_t ids = g.x.n * chunks;
    for (int64_t id = blockIdx.x; id < ids; id += gridDim.x) {
        const int64_t n = id / chunks;
        const int chunk = static_cast<int>(id - n * chunks);
        const RowGrad rg = g.row_grad[n];
        const Span<T> row(static_cast<const T *>(g.x.data) + n * g.x.stride, g.x.V);
        T *out = static_cast<T *>(g.out_grad) + n * g.grad_stride;
        const int b0 = chunk * STEP, b1 = min(row.whole, b0 + STEP), edge = chunk == 0 ? row.edge(tid) : -1;
        uint4 v[kGradChunk];
#pragma unroll
        for (int k = 0; k < kGradChunk; ++k)
            if (b0 + k * 256 + tid < b1) v[k] = row.load(b0 + k * 256 + tid);
        float z_edge = edge >= 0 ? Elem<T>::load(row.p + edge) : 0.0f;
        if (rg.B != 0.0f) {                          // (actions at the lowest value are masked)
            const float low = lowest_of(g.x.dtype);
            float most = 0.0f;
#pragma unroll
            for (int k = 0; k < kGradChunk; ++k)
                if (b0 + k * 256 + tid < b1) leave_others<T>(v[k], 0, low, most);
            if (z_edge == low) z_edge = -INFINITY;
        }
        marks.head[tid] = -1;
        __syncthreads();
        if (tid < g.k) {
            const int e = g.at[n * g.k + tid];
            int thread;
            if (e >= 0 && marks.bit_of(e, row.head, row.tail(), b0, b1, chunk == 0, &thread) >= 0) {
                at[tid] = e;
                inside[tid] = g.inside[n * g.k + tid];
                marks.link(tid, thread);
            }
        }
        __syncthreads();
        const Scale x{ref_of(rg.m).m, g.per2};
#pragma unroll
        for (int k = 0; k < kGradChunk; ++k)
            if (b0 + k * 256 + tid < b1) write_slot<T>(out + row.head + static_cast<uint32_t>(b0 + k * 256 + tid) * N, v[k], rg.A, x);
        if (edge >= 0) Elem<T>::store(out + edge, rg.A == 0.0f ? 0.0f : exp2_of(x(z_edge)) * rg.A);
        for (int i = marks.head[tid]; i >= 0; i = marks.next[i]) Elem<T>::store(out + at[i], inside[i]);
        __syncthreads();
    }
}

// A lane takes its list's entries one by one, a wave about as long for any row.  Calls, us, a row to a lane against one to a wave: lists
// of 5 of 17 bf16, 4096 rows 19 against 16, 16384 19 against 39; 16 of 100, 16384 rows 59 against 39, 65536 69 against 137; 64 of 64,
// whose lists are more than a CU's cache, a million rows 3740 against 2160; 5 of 17, 3.9 million rows 390 against 7810.
bool by_lanes(const LogitsView &x, int k) { return x.V <= kLaneRow && k <= 32 && x.n >= 8192 + 1024 * k + 64 * x.V; }

int slots_of(const LogitsView &x) { return x.dtype == PL_F32 ? (x.V + 3) / 4 : (x.V + 7) / 8; }
constexpr int kRowSlots = 960 * 18;    // of the widest row that a workgroup keeps

constexpr int kRowBlocks = 4096;       // workgroups that go over the rows: 14 of two waves to a CU, and more

// As for the policy loss: rows are cut into slices where there are few of them.
bool in_slices(const LogitsView &x) { return (x.n < 64 && x.V >= 32768) || slots_of(x) > kRowSlots; }

}  // namespace

DistillWorkspace carve_distill_workspace(void *base, const LogitsView &x, const RowsView &rows, int k)
{
    DistillWorkspace w;
    w.loss = carve_loss_workspace(base, x, rows);
    size_t pos = (w.loss.bytes + 15) / 16 * 16;
    const size_t n = in_slices(x) ? static_cast<size_t>(x.n) * k : 0, parts = in_slices(x) ? static_cast<size_t>(x.n) * w.loss.slices : 0;
    w.parts = base ? reinterpret_cast<DistillPart *>(static_cast<char *>(base) + pos) : nullptr;
    pos += parts * sizeof(DistillPart);
    w.at = base ? reinterpret_cast<int32_t *>(static_cast<char *>(base) + pos) : nullptr;
    pos += (n * 4 + 15) / 16 * 16;
    w.inside = base ? reinterpret_cast<float *>(static_cast<char *>(base) + pos) : nullptr;
    pos += (n * 4 + 15) / 16 * 16;
    w.sums = base ? reinterpret_cast<double *>(static_cast<char *>(base) + pos) : nullptr;
    pos += static_cast<size_t>(std::max<int64_t>(kRowBlocks, (x.n + 255) / 256)) * 4 * sizeof(double);
    w.bytes = pos;
    return w;
}

void launch_distill(DistillArgs a, int reduction, const DistillWorkspace &ws, hipStream_t s)
{
    a.w = launch_row_weights(a.x, a.rows, reduction, ws.loss, s);
    a.sums = ws.sums;
    int blocks = 0;
    if (a.x.n > 0)
        by_type(a.x.dtype, [&](auto t) {
            using T = decltype(t);
            constexpr int W = 4 / sizeof(T), N = Elem<T>::N;
            auto over_rows = [&](auto kernel, int threads) {
                blocks = static_cast<int>(std::min<int64_t>(a.x.n, kRowBlocks));
                hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), 0, s, a);
            };
            if (a.x.V <= kNarrow) {
                const size_t bytes = a.x.V * sizeof(T), align = std::min<size_t>(bytes, 16);
                const bool whole = (reinterpret_cast<uintptr_t>(a.x.data) | reinterpret_cast<uintptr_t>(a.out_grad)) % align == 0 &&
                                   a.x.stride * sizeof(T) % align == 0 && (!a.out_grad || a.grad_stride * sizeof(T) % align == 0);
                const size_t lds = 256 * (a.x.V | 1) * sizeof(float);
                blocks = static_cast<int>((a.x.n + 255) / 256);
                auto go = [&](auto kernel, size_t bytes_lds) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(256), bytes_lds, s, a); };
                if (whole && bytes == 8) go(k_distill_narrow<T, 2 * W, true>, 0);
                else if (whole && bytes == 16) go(k_distill_narrow<T, 4 * W, true>, 0);
                else if (whole && bytes == 32) go(k_distill_narrow<T, 8 * W, true>, 0);
                else go(k_distill_narrow<T, kNarrow, false>, lds);
                return;
            }
            if (by_lanes(a.x, a.k)) {
                blocks = static_cast<int>(std::min<int64_t>((a.x.n + 63) / 64, kRowBlocks));
                hipLaunchKernelGGL(k_distill_lane<T>, dim3(blocks), dim3(64), 64 * (a.x.V | 1) * sizeof(float), s, a);
                return;
            }
            const int slots = slots_of(a.x);
            if (!in_slices(a.x)) {
                if (slots <= 64) over_rows(k_distill_row<T, 64, 1>, 128);
                else if (slots <= 64 * 4) over_rows(k_distill_row<T, 64, 4>, 128);
                else if (slots <= 192 * 8) over_rows(k_distill_row<T, 192, 8>, 256);
                else if (slots <= 448 * 8) over_rows(k_distill_row<T, 448, 8>, 512);
                else if (slots <= 448 * 20) over_rows(k_distill_row<T, 448, 20>, 512);
                else over_rows(k_distill_row<T, 960, 18>, 1024);
                return;
            }
            a.parts = ws.parts;
            a.slices = ws.loss.slices;
            a.row_grad = ws.loss.grad;
            a.at = ws.at;
            a.inside = ws.inside;
            const uint32_t rows = static_cast<uint32_t>(std::min<int64_t>(a.x.n, 1 << 16));
            hipLaunchKernelGGL(k_distill_part<T>, dim3(rows, a.slices), dim3(256), 0, s, a);
            blocks = static_cast<int>(std::min<int64_t>((a.x.n + 3) / 4, kRowBlocks));
            hipLaunchKernelGGL(k_distill_finish<T>, dim3(blocks), dim3(256), 0, s, a);
            if (a.out_grad) {
                const int chunks = std::max(1, (a.x.V / N + kGradChunk * 256 - 1) / (kGradChunk * 256));
                hipLaunchKernelGGL(k_distill_grad<T>, dim3(static_cast<uint32_t>(std::min<int64_t>(a.x.n * chunks, 1 << 20))), dim3(256), 0, s, a, chunks);
            }
        });
    if (blocks != 1) hipLaunchKernelGGL(k_distill_stats, dim3(1), dim3(1024), 0, s, ws.sums, blocks, a.out_stats);
}

}  // namespace pl

// Losses on rows of logits (include/placeto.h): log probabilities of actions, the clipped policy loss
// and the preference loss, with the gradient of the logits.
//
// For a row z with maximum m, in powers of two: x_j = (z_j - m) log2 e, s = sum_j 2^{x_j} and t = sum_j 2^{x_j} x_j give
//     l = log pi(a) = (z_a - m) - ln 2 log2 s,      H = ln 2 (log2 s - t / s),
// and with w c = d loss / d l and -w g = d loss / d H the gradient of logit j is
//     w [ c (1[j = a] - p_j) + g p_j (log p_j + H) ] = 2^{x_j} (A + B x_j) + C 1[j = a],
//     C = w c,  B = ln 2 w g / s,  A = (-w c + w g (H - ln s)) / s.
// z_j - m is taken before it is scaled: it is exact near the maximum, however far the row lies from zero, so that a
// probability close to 1 has a logarithm close to 0 (one fused multiply-add for both leaves that at 1e-7).
#include <algorithm>
#include <cmath>

#include "elements.h"
#include "losses.h"

namespace pl {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr double kAddsNothing = INFINITY;   // in place of the l of a row that adds nothing to its sequence
constexpr float kLowest = -300.0f;     // 2^-300 is 0 in fp32: an x below it stands for -infinity, whose product with 0 is NaN
constexpr float kNoChance = -150.0f;   // 2^-150 rounds to 0 in fp32: an action at the type's lowest value is masked below it

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// z -> x of a maximum m.  (A row of -infinity alone has sums of 0.)
struct Ref {
    float m;
    __device__ float operator()(float z) const { return (z - m) * kLog2e; }
};
__device__ __forceinline__ Ref ref_of(float m) { return {m == -INFINITY ? 0.0f : m}; }

// ---- over 4 lanes, 16 lanes (a DPP row) and a wave
template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}

__device__ __forceinline__ float max_of_4(float v)
{
    v = fmaxf(v, dpp<0xb1>(v));        // within four lanes: the neighbour, then the other pair
    return fmaxf(v, dpp<0x4e>(v));
}

__device__ __forceinline__ float sum_of_4(float v)
{
    v += dpp<0xb1>(v);
    return v + dpp<0x4e>(v);
}

__device__ __forceinline__ float max_of_16(float v)
{
    v = fmaxf(v, dpp<0x128>(v));       // rotations within the row by 8, 4, 2, 1
    v = fmaxf(v, dpp<0x124>(v));
    v = fmaxf(v, dpp<0x122>(v));
    return fmaxf(v, dpp<0x121>(v));
}

__device__ __forceinline__ float sum_of_16(float v)
{
    v += dpp<0x128>(v);
    v += dpp<0x124>(v);
    v += dpp<0x122>(v);
    return v + dpp<0x121>(v);
}

__device__ __forceinline__ float lane_value(float v, int lane)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

template <int LANES>
__device__ __forceinline__ float max_of(float v)
{
    if (LANES == 4) return max_of_4(v);
    v = max_of_16(v);
    if (LANES == 16) return v;
    return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}

template <int LANES>
__device__ __forceinline__ float sum_of(float v)
{
    if (LANES == 4) return sum_of_4(v);
    v = sum_of_16(v);
    if (LANES == 16) return v;
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

// ---- maximum and sums of a row
struct Sums {
    float m = -INFINITY, s = 0.0f, t = 0.0f;
};

// What a holds, relative to the maximum of b.  Sums without a probability (s = 0) say nothing.
__device__ __forceinline__ Sums rebased(const Sums &a, float m, const Ref &to)
{
    if (a.s == 0.0f) return {m, 0.0f, 0.0f};
    const float d = to(ref_of(a.m).m), e = exp2_of(d);
    return {m, a.s * e, e * (a.t + fmaxf(d, kLowest) * a.s)};
}

template <int LANES>
__device__ __forceinline__ Sums merge_of(const Sums &a)
{
    const float m = max_of<LANES>(a.m);
    const Sums x = rebased(a, m, ref_of(m));
    return {m, sum_of<LANES>(x.s), sum_of<LANES>(x.t)};
}

// ---- rows and sequences
struct Place {
    int seq;
    bool counts;
};

__device__ __forceinline__ Place place_of(const RowsView &r, int64_t n)
{
    Place p{0, true};
    if (r.order == PL_ROWS_PACKED) {
        int lo = 0, hi = r.S;                    // the last sequence that begins at or in front of the row
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (r.bounds[mid] <= n) lo = mid; else hi = mid;
        }
        p.seq = lo;
        p.counts = r.bounds[lo] <= n && n < r.bounds[lo + 1];
    } else {
        const int q = r.order == PL_ROWS_BY_STEP ? r.S : r.L;
        const int u = r.magic ? static_cast<int>(__umulhi(static_cast<uint32_t>(n), r.magic) >> r.shift) : static_cast<int>(n);
        const int v = static_cast<int>(n) - u * q;
        p.seq = r.order == PL_ROWS_BY_STEP ? v : u;
        const int step = r.order == PL_ROWS_BY_STEP ? u : v;
        if (r.bounds) p.counts = step < r.bounds[p.seq];
    }
    if (r.mask && p.counts) p.counts = r.mask[n] != 0;
    return p;
}

// l of a row from its fp32 maximum and sum, not rounded itself: sums over a sequence, whose difference to another one's counts, are
// off by what s is off (some units of 2^-24), not by that of l's own size.
__device__ __forceinline__ double exact_l(const Sums &a, float z_a)
{
    return (static_cast<double>(z_a) - a.m) - log(static_cast<double>(a.s));
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// 1 / s to an ulp, for s that is neither tiny nor huge.
__device__ __forceinline__ float reciprocal(float s)
{
    const float r = __builtin_amdgcn_rcpf(s);
    return __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r);
}

__device__ __forceinline__ float lowest_of(int dtype) { return dtype == PL_F32 ? -0x1.fffffep127f : dtype == PL_BF16 ? -0x1.fep127f : -65504.0f; }

// l, H and log s of a row from its sums; a row without an allowed action has l = NaN, an action of probability zero
// l = -infinity.
__device__ __forceinline__ void finish_row(const Sums &a, float z_a, bool action_ok, float &l, float &H, float &log_s)
{
    const float log2_s = log2f(a.s);
    log_s = kLn2 * log2_s;
    H = kLn2 * (log2_s - a.t * reciprocal(a.s));
    l = action_ok ? (z_a - a.m) - log_s : NAN;
    if (a.s == 0.0f) H = l = NAN;
}

struct PolicyRow {
    float c = 0.0f, g = 0.0f;          // - d loss / d l, - d loss / d H, without the gradient's scale
    float sur = 0.0f, kl = 0.0f, H = 0.0f, cut = 0.0f;
};

// What a row has besides its logits, read before they are waited for.
struct RowIn {
    Place p;
    int act = -1;
    float adv = 0.0f, old = 0.0f, ref = 0.0f, w = 0.0f;    // w: PASS_POLICY the row's weight, PASS_PREF_GRAD d loss / d l
};

__device__ __forceinline__ void policy_in(RowIn &in, const PolicyArgs &a, int64_t n)
{
    in.adv = a.advantages[a.advantage_per_seq ? in.p.seq : n];
    if (a.old_logp) in.old = a.old_logp[n];
    if (a.ref_logp) in.ref = a.ref_logp[n];
    in.w = a.weights ? a.weights[in.p.seq] : a.weight_at ? *a.weight_at : a.weight;
}

// Value and derivatives of a row that counts and adds something.
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs &a, const RowIn &in, float l, float H)
{
    PolicyRow r;
    float ratio = a.old_logp ? expf(l - in.old) : (l == l ? 1.0f : l);
    if (in.adv == 0.0f && ratio == INFINITY) ratio = 0.0f;       // no advantage, whatever the ratio: not 0 times infinity
    const bool cut = in.adv > 0.0f ? ratio > 1.0f + a.clip_high : (in.adv < 0.0f && ratio < 1.0f - a.clip_low);
    const float held = cut ? (in.adv > 0.0f ? 1.0f + a.clip_high : 1.0f - a.clip_low) : ratio;
    r.sur = in.w * (-in.adv * held);
    r.c = cut ? 0.0f : in.adv * ratio;
    if (a.ref_logp) {
        const float d = in.ref - l, e = expm1f(d);
        r.kl = in.w * (e - d);
        r.c += a.kl_coeff != 0.0f ? a.kl_coeff * e : 0.0f;   // (e may be infinite; the same below)
    }
    r.c *= in.w;
    r.g = in.w * a.entropy_coeff;
    r.H = in.w * H;
    r.cut = cut ? in.w : 0.0f;
    return r;
}

__device__ __forceinline__ RowGrad grad_of(const PolicyRow &r, const PolicyArgs &a, const Sums &sums, float H, float log_s)
{
    const float c = -r.c * a.grad_scale, g = r.g * a.grad_scale;
    const float per = reciprocal(sums.s);
    return {sums.m, (-c + g * (H - log_s)) * per, kLn2 * g * per, c};
}

// 2^x (A + B x) of a slot
template <int N>
__device__ __forceinline__ void grad_slot(float (&f)[N], const RowGrad &g, const Ref &ref)
{
    if (g.B == 0.0f) {
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = exp2_of(ref(f[j])) * g.A;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float x = ref(f[j]);
            f[j] = exp2_of(x) * (g.A + g.B * fmaxf(x, kLowest));
        }
    }
}

__device__ __forceinline__ void policy_stats_out(const double (&v)[4], float kl_coeff, float entropy_coeff, float *out)
{
    out[0] = static_cast<float>(v[0] + (kl_coeff != 0.0f ? kl_coeff * v[1] : 0.0) - entropy_coeff * v[2]);
    for (int i = 0; i < 4; ++i) out[1 + i] = static_cast<float>(v[i]);
}

// ---- the loss from the workgroups' sums, in their order
__global__ __launch_bounds__(1024) void k_policy_stats(const double *__restrict__ sums, int blocks, float kl_coeff,
                                                       float entropy_coeff, float *__restrict__ out)
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
    if (tid == 0) {
        double v[4] = {0.0, 0.0, 0.0, 0.0};
        for (int w = 0; w < 16; ++w)
            for (int i = 0; i < 4; ++i) v[i] += last[w][i];
        policy_stats_out(v, kl_coeff, entropy_coeff, out);
    }
}

// ---- the gradient of the logits, an element at a time, kGradSlots slots of a row to a wave.  For a preference a row takes
// its sequence's d loss / d l (seq_coeff) first.
constexpr int kGradSlots = 256;

struct GradArgs {
    LogitsView x;
    const int32_t *actions;
    const RowGrad *grad;
    void *out;
    int64_t out_stride;
    int chunks;                        // waves to a row
    RowsView rows;                     // with seq_coeff
    const float *seq_coeff;
    float *out_coeff;
    float grad_scale;
};

template <typename T>
__global__ __launch_bounds__(256) void k_row_grad(GradArgs a)
{
    constexpr int N = Elem<T>::N;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
    const int64_t ids = a.x.n * a.chunks;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + wave; i < ids; i += static_cast<int64_t>(gridDim.x) * 4) {
        const int64_t id = ids - 1 - i;              // from the last row to the first: what the pass before has read last first
        const int64_t n = id / a.chunks;
        const int chunk = static_cast<int>(id - n * a.chunks);
        RowGrad g = a.grad[n];
        if (a.seq_coeff) {
            const Place at = place_of(a.rows, n);
            const float c = at.counts && g.A != 0.0f ? a.grad_scale * a.seq_coeff[at.seq] : 0.0f;
            g.A = c == 0.0f ? 0.0f : -c * g.A;
            g.C = c;
            if (a.out_coeff && chunk == 0 && lane == 0) a.out_coeff[n] = -c;
        }
        if (!a.out) continue;
        const Span<T> row(static_cast<const T *>(a.x.data) + n * a.x.stride, a.x.V);
        T *o = static_cast<T *>(a.out) + n * a.out_stride;
        const bool none = g.A == 0.0f && g.B == 0.0f && g.C == 0.0f;
        const int act = none ? -1 : a.actions[n], edge = chunk == 0 ? row.edge(lane) : -1;
        const Ref ref = ref_of(g.m);
        uint4 v[kGradSlots / 64];
        float z_edge = 0.0f;
        const int first = chunk * kGradSlots + lane;
        if (!none) {
#pragma unroll
            for (int k = 0; k < kGradSlots / 64; ++k) v[k] = row.load(first + k * 64);
            if (edge >= 0) z_edge = Elem<T>::load(row.p + edge);
        }
#pragma unroll
        for (int k = 0; k < kGradSlots / 64; ++k) {
            const int slot = first + k * 64, e = row.head + slot * N;
            if (slot < row.whole) {
                float f[N];
                if (none) {
#pragma unroll
                    for (int j = 0; j < N; ++j) f[j] = 0.0f;
                } else {
                    Elem<T>::unpack(v[k], f);
                    grad_slot<N>(f, g, ref);
                    if (act >= e && act < e + N) {
#pragma unroll
                        for (int j = 0; j < N; ++j) f[j] += e + j == act ? g.C : 0.0f;
                    }
                }
                stream_16(o + e, Elem<T>::pack(f));
            }
        }
        if (edge >= 0) {
            float f[1] = {z_edge};
            grad_slot<1>(f, g, ref);
            Elem<T>::store(o + edge, none ? 0.0f : f[0] + (edge == act ? g.C : 0.0f));
        }
    }
}

// Rows of a sequence that its bounds leave.
__device__ __forceinline__ int bounded_length(const RowsView &rows, int q)
{
    if (rows.order == PL_ROWS_PACKED)
        return static_cast<int>(max(int64_t{0}, min(rows.n, static_cast<int64_t>(rows.bounds[q + 1])) - max(0, rows.bounds[q])));
    return rows.bounds ? min(rows.L, max(0, rows.bounds[q])) : rows.L;
}

// ---- sequences: sums of l and l - ref over the rows that count, and their number (with logp == nullptr: the
// number only)
struct SeqSum {
    double l = 0.0, ratio = 0.0;
    int n = 0;
};

// Steps i, i + by, ... below `end` of sequence q.
__device__ __forceinline__ SeqSum add_steps(const RowsView &rows, const double *__restrict__ logp, const float *__restrict__ ref, int q,
                                            int64_t i, int64_t end, int by)
{
    SeqSum s;
    const int64_t step = rows.order == PL_ROWS_BY_STEP ? rows.S : 1;
    const int64_t first = rows.order == PL_ROWS_PACKED ? max(0, rows.bounds[q])
                                                       : rows.order == PL_ROWS_BY_STEP ? q : static_cast<int64_t>(q) * rows.L;
    // (eight rows at a time, their loads together: past the end the last one again)
    for (; i < end; i += 8 * by) {
        double l[8];
        float r[8];
        bool in[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t at = i + k * by, n = first + min(at, end - 1) * step;
            in[k] = at < end && (!rows.mask || rows.mask[n]);
            l[k] = logp ? logp[n] : 0.0;
            r[k] = logp && ref ? ref[n] : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            s.n += in[k];
            if (in[k] && l[k] != kAddsNothing) {
                s.l += l[k];
                s.ratio += l[k] - r[k];
            }
        }
    }
    return s;
}

// Sums over the threads of a workgroup whose numbers are equal modulo lanes_s, for the first lanes_s of them.
template <int THREADS>
__device__ __forceinline__ SeqSum sum_abreast(SeqSum s, int lanes_s)
{
    __shared__ double l[THREADS], ratio[THREADS];
    __shared__ int n[THREADS];
    const int tid = threadIdx.x;
    __syncthreads();
    l[tid] = s.l;
    ratio[tid] = s.ratio;
    n[tid] = s.n;
    for (int o = THREADS / 2; o >= lanes_s; o >>= 1) {
        __syncthreads();
        if (tid < o) {
            l[tid] += l[tid + o];
            ratio[tid] += ratio[tid + o];
            n[tid] += n[tid + o];
        }
    }
    return {l[tid], ratio[tid], n[tid]};
}

// Part blockIdx.y of every sequence: lanes_s sequences and 256 / lanes_s of their rows side by side.
__global__ __launch_bounds__(256) void k_seq_sums(RowsView rows, const double *__restrict__ logp, const float *__restrict__ ref,
                                                  int lanes_s, double *__restrict__ part, int32_t *__restrict__ part_n)
{
    const int tid = threadIdx.x, ls = tid & (lanes_s - 1), abreast = 256 / lanes_s;
    const int q = blockIdx.x * lanes_s + ls;
    SeqSum s;
    if (q < rows.S) {
        const int64_t len = bounded_length(rows, q), per = (len + gridDim.y - 1) / gridDim.y;
        s = add_steps(rows, logp, ref, q, per * blockIdx.y + tid / lanes_s, min(len, per * (blockIdx.y + 1)), abreast);
    }
    s = sum_abreast<256>(s, lanes_s);
    if (tid < lanes_s && q < rows.S) {
        const size_t at = static_cast<size_t>(blockIdx.y) * rows.S + q;
        if (part) {
            part[at * 2] = s.l;
            part[at * 2 + 1] = s.ratio;
        }
        part_n[at] = s.n;
    }
}

// Sums of the parts of every sequence, sixteen lanes to one (one workgroup).  Without parts the numbers of rows are those of
// the bounds.  And the weights of rows: `weight` of any, `weights` of those of each sequence.
__global__ __launch_bounds__(1024) void k_seq_totals(RowsView r, int seq_parts, const double *__restrict__ part,
                                                     const int32_t *__restrict__ part_n, double *__restrict__ seq_sum,
                                                     int32_t *__restrict__ seq_n, float *__restrict__ weight,
                                                     float *__restrict__ weights)
{
    __shared__ int32_t wave[16][2];
    const int tid = threadIdx.x, S = r.S;
    int rows = 0, seqs = 0;
    if (!part_n) {
        for (int q = tid; q < S; q += 1024) {
            const int c = bounded_length(r, q);
            seq_n[q] = c;
            rows += c;
            seqs += c > 0;
        }
    } else {
        const int lane = tid & 15;
        for (int q = tid >> 4; q < S; q += 64) {
            double a = 0.0, b = 0.0;
            int c = 0;
#pragma unroll 4
            for (int i = lane; i < seq_parts; i += 16) {
                const size_t at = static_cast<size_t>(i) * S + q;
                if (part) {
                    a += part[at * 2];
                    b += part[at * 2 + 1];
                }
                c += part_n[at];
            }
#pragma unroll
            for (int o = 8; o; o >>= 1) {
                a += __shfl_xor(a, o);
                b += __shfl_xor(b, o);
                c += __shfl_xor(c, o);
            }
            if (lane == 0) {
                if (part) {
                    seq_sum[q * 2] = a;
                    seq_sum[q * 2 + 1] = b;
                }
                seq_n[q] = c;
                rows += c;
                seqs += c > 0;
            }
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        rows += __shfl_xor(rows, o);
        seqs += __shfl_xor(seqs, o);
    }
    if ((tid & 63) == 0) {
        wave[tid >> 6][0] = rows;
        wave[tid >> 6][1] = seqs;
    }
    __syncthreads();
    rows = seqs = 0;
    for (int i = 0; i < 16; ++i) {
        rows += wave[i][0];
        seqs += wave[i][1];
    }
    if (weight && tid == 0) *weight = rows > 0 ? 1.0f / static_cast<float>(rows) : 0.0f;
    if (weights)
        for (int q = tid; q < S; q += 1024) {
            const int c = seq_n[q];
            weights[q] = c > 0 ? static_cast<float>(1.0 / (static_cast<double>(seqs) * c)) : 0.0f;
        }
}

// The weights of few rows under a mask in one launch by one workgroup (instead of two), a row to a thread.
__global__ __launch_bounds__(1024) void k_weights(RowsView r, float *__restrict__ weight, float *__restrict__ weights)
{
    __shared__ int32_t bounds[kMiddleSeqs + 1];
    __shared__ uint32_t count[kMiddleSeqs];
    __shared__ int32_t wave[16];
    const int tid = threadIdx.x;
    uint8_t mask[8];                                     // of eight rows, 1024 apart
    auto read_mask = [&](int64_t i) {
#pragma unroll
        for (int k = 0; k < 8; ++k) mask[k] = r.mask[min(i + k * 1024, r.n - 1)];
    };
    read_mask(tid);
    if (r.bounds)
        for (int q = tid; q < r.S + (r.order == PL_ROWS_PACKED); q += 1024) bounds[q] = r.bounds[q];
    for (int q = tid; q < r.S; q += 1024) count[q] = 0;
    __syncthreads();
    RowsView in_lds = r;
    if (r.bounds) in_lds.bounds = bounds;
    in_lds.mask = nullptr;
    int n = 0;
    for (int64_t i = tid; i < r.n; i += 8 * 1024) {
        if (i != tid) read_mask(i);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + k * 1024 < r.n && mask[k]) {
                const Place p = place_of(in_lds, i + k * 1024);
                n += p.counts;
                if (weights && p.counts) atomicAdd(&count[p.seq], 1u);       // (whole numbers: their order does not matter)
            }
    }
    auto total = [&](int v) {
#pragma unroll
        for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
        __syncthreads();
        if ((tid & 63) == 0) wave[tid >> 6] = v;
        __syncthreads();
        v = 0;
        for (int i = 0; i < 16; ++i) v += wave[i];
        return v;
    };
    if (!weights) {
        n = total(n);
        if (tid == 0) *weight = n > 0 ? 1.0f / static_cast<float>(n) : 0.0f;
        return;
    }
    __syncthreads();
    int seqs = 0;
    for (int q = tid; q < r.S; q += 1024) seqs += count[q] > 0;
    seqs = total(seqs);
    for (int q = tid; q < r.S; q += 1024)
        weights[q] = count[q] > 0 ? static_cast<float>(1.0 / (static_cast<double>(seqs) * count[q])) : 0.0f;
}

// ---- pairs: margins, the loss, and d loss / d s of every sequence
struct Pair {
    int a, b;
    bool ok;
};

__device__ __forceinline__ Pair pair_at(const PrefArgs &p, int S, int i)
{
    Pair r{2 * i, 2 * i + 1, true};
    if (p.pairs) {
        r.a = p.pairs[2 * i];
        r.b = p.pairs[2 * i + 1];
        r.ok = r.a >= 0 && r.a < S && r.b >= 0 && r.b < S;
    }
    return r;
}

__device__ __forceinline__ double seq_ratio(const PrefArgs &p, const double *seq_sum, const int32_t *seq_n, int q, int which)
{
    const double v = seq_sum[q * 2 + which];
    return p.average && seq_n[q] > 0 ? v / seq_n[q] : v;
}

__device__ __forceinline__ float d_margin(float m, float eps)
{
    return eps / (1.0f + expf(-m)) - (1.0f - eps) / (1.0f + expf(m));
}

__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.0f) + log1pf(expf(-fabsf(x))) + (x != x ? x : 0.0f); }

// (A margin may be infinite: a term without weight is left out, not 0 times infinity.)
__device__ __forceinline__ float pair_loss(float m, float eps)
{
    return (eps != 1.0f ? (1.0f - eps) * softplus(-m) : 0.0f) + (eps != 0.0f ? eps * softplus(m) : 0.0f);
}

// d loss / d s of the THREADS / kTeam sequences from q0 on, kTeam lanes to each: with a list of pairs they go over all of
// them, THREADS at a time through LDS, and add those of their sequence; without one a sequence is in one pair.  `first`:
// the loss and the margins as well.
constexpr int kTeam = 8;

template <int THREADS>
__device__ __forceinline__ void pairs_of(const PrefArgs &p, int S, int q0, bool first, const double *seq_sum, const int32_t *seq_n,
                                         float *__restrict__ seq_coeff, float *__restrict__ out_stats)
{
    __shared__ int4 tile[THREADS];
    __shared__ double wave[THREADS / 64][3];
    const int tid = threadIdx.x, lane = tid & (kTeam - 1), q = q0 + tid / kTeam;
    double loss = 0.0, right = 0.0, valid = 0.0, coeff = 0.0;
    auto margin = [&](const Pair &pr) {
        return static_cast<float>(p.beta * (seq_ratio(p, seq_sum, seq_n, pr.a, 1) - seq_ratio(p, seq_sum, seq_n, pr.b, 1)));
    };
    if (p.pairs || first)
        for (int i0 = 0; i0 < p.n_pairs; i0 += THREADS) {
            const int i = i0 + tid;
            Pair pr{-1, -1, false};
            float m = NAN, g = 0.0f;
            if (i < p.n_pairs) {
                pr = pair_at(p, S, i);
                if (pr.ok) {
                    m = margin(pr);
                    g = d_margin(m, p.smoothing);
                    if (first) loss += pair_loss(m, p.smoothing);
                    right += m > 0.0f;
                    valid += 1.0;
                }
                if (first && p.out_margins) p.out_margins[i] = m;
            }
            if (!p.pairs) continue;
            __syncthreads();
            tile[tid] = {pr.ok ? pr.a : -1, pr.ok ? pr.b : -1, __float_as_int(g), 0};
            __syncthreads();
            const int n = min(THREADS, p.n_pairs - i0);
#pragma unroll 8
            for (int k = lane; k < n; k += kTeam) {
                const int4 e = tile[k];
                if (e.x == q || e.y == q) coeff += (e.x == q ? __int_as_float(e.z) : 0.0f) - (e.y == q ? __int_as_float(e.z) : 0.0f);
            }
        }
    if (p.pairs || first) {                              // (the same for the whole workgroup)
        __shared__ double all[3];
        if (first) {
            loss = wave_sum(loss);
            right = wave_sum(right);
        }
        valid = wave_sum(valid);
        __syncthreads();
        if ((tid & 63) == 0) {
            wave[tid >> 6][0] = loss;
            wave[tid >> 6][1] = right;
            wave[tid >> 6][2] = valid;
        }
        __syncthreads();
        if (tid < 3) {
            double v = 0.0;
#pragma unroll
            for (int w = 0; w < THREADS / 64; ++w) v += wave[w][tid];
            all[tid] = v;
        }
        __syncthreads();
        loss = all[0];
        right = all[1];
        valid = all[2];
    }
    if (!p.pairs) valid = p.n_pairs;
    const double per = valid > 0.0 ? 1.0 / valid : 0.0;
    if (first && tid == 0) {
        out_stats[0] = static_cast<float>(loss * per);
        out_stats[1] = static_cast<float>(right * per);
    }
#pragma unroll
    for (int o = kTeam / 2; o; o >>= 1) coeff += __shfl_xor(coeff, o);
    if (lane == 0 && q < S) {
        if (!p.pairs && (q >> 1) < p.n_pairs) {
            const float g = d_margin(margin(Pair{q & ~1, q | 1, true}), p.smoothing);
            coeff = (q & 1) ? -g : g;
        }
        coeff *= per * p.beta;
        if (p.average && seq_n[q] > 0) coeff /= seq_n[q];
        seq_coeff[q] = static_cast<float>(coeff);
        if (p.out_seq_logp) p.out_seq_logp[q] = static_cast<float>(seq_ratio(p, seq_sum, seq_n, q, 0));
    }
}

__global__ __launch_bounds__(256) void k_pairs(PrefArgs p, int S, const double *__restrict__ seq_sum, const int32_t *__restrict__ seq_n,
                                               float *__restrict__ seq_coeff, float *__restrict__ out_stats)
{
    pairs_of<256>(p, S, blockIdx.x * (256 / kTeam), blockIdx.x == 0, seq_sum, seq_n, seq_coeff, out_stats);
}

// Few rows and sequences: the sums of sequences and the pairs in one launch by one workgroup (instead of three).
__global__ __launch_bounds__(1024) void k_pref_middle(RowsView rows, PrefArgs p, const double *__restrict__ logp, int lanes_s,
                                                      float *__restrict__ seq_coeff, float *__restrict__ out_stats)
{
    static_assert(kPairSeqs <= 1024 / kTeam, "all sequences at once");
    __shared__ double seq_sum[2 * kPairSeqs];
    __shared__ int32_t seq_n[kPairSeqs];
    const int tid = threadIdx.x;
    if (rows.order == PL_ROWS_BY_STEP) {
        for (int q0 = 0; q0 < rows.S; q0 += lanes_s) {
            const int q = q0 + (tid & (lanes_s - 1));
            SeqSum s;
            if (q < rows.S) s = add_steps(rows, logp, p.ref_logp, q, tid / lanes_s, bounded_length(rows, q), 1024 / lanes_s);
            s = sum_abreast<1024>(s, lanes_s);
            if (tid < lanes_s && q < rows.S) {
                seq_sum[q * 2] = s.l;
                seq_sum[q * 2 + 1] = s.ratio;
                seq_n[q] = s.n;
            }
        }
    } else {                                             // a wave to a sequence
        for (int q = tid >> 6; q < rows.S; q += 16) {
            SeqSum s = add_steps(rows, logp, p.ref_logp, q, tid & 63, bounded_length(rows, q), 64);
            s.l = wave_sum(s.l);
            s.ratio = wave_sum(s.ratio);
#pragma unroll
            for (int o = 32; o; o >>= 1) s.n += __shfl_xor(s.n, o);
            if ((tid & 63) == 0) {
                seq_sum[q * 2] = s.l;
                seq_sum[q * 2 + 1] = s.ratio;
                seq_n[q] = s.n;
            }
        }
    }
    __syncthreads();
    pairs_of<1024>(p, rows.S, 0, true, seq_sum, seq_n, seq_coeff, out_stats);
}

// What a kernel that takes whole rows does with them.
enum RowPass { PASS_LOGP, PASS_POLICY, PASS_PREF_FORWARD, PASS_PREF_GRAD };

struct RowArgs {
    LogitsView x;
    RowsView rows;
    uint32_t magic;                    // e / V = high word of e * magic (narrow rows)
    const int32_t *actions;
    float *out_logp, *out_entropy;
    PolicyArgs policy;                 // PASS_POLICY
    double *sums;
    float *out_stats;
    double *logp;                      // PASS_PREF_FORWARD
    RowGrad *grad;
    const float *seq_coeff;            // PASS_PREF_GRAD
    float *out_coeff;
    float grad_scale;
    void *out_grad;                    // both gradients
    int64_t grad_stride;
};

template <int PASS>
__device__ __forceinline__ void read_in(const RowArgs &g, int64_t n, RowIn &in)
{
    if (!in.p.counts) return;
    if (PASS == PASS_POLICY) policy_in(in, g.policy, n);
    if (PASS == PASS_PREF_GRAD) in.w = g.grad_scale * g.seq_coeff[in.p.seq];
}

// What follows from a row's sums: outputs, the row's part of the loss (added to `acc`) and its gradient.  `first`: this
// thread writes the row's outputs and keeps its part.
template <int PASS>
__device__ __forceinline__ RowGrad finish_pass(const RowArgs &g, int64_t n, const RowIn &in, const Sums &a, float z_a, bool first,
                                               double *acc)
{
    float l = 0.0f, H = 0.0f, log_s = 0.0f;
    bool live = false;
    if (in.p.counts) {
        const bool ok = in.act >= 0 && in.act < g.x.V;
        if (z_a == lowest_of(g.x.dtype) && ref_of(a.m)(z_a) < kNoChance) z_a = -INFINITY;
        finish_row(a, z_a, ok, l, H, log_s);
        live = ok && l != -INFINITY && a.s != 0.0f;
    }
    RowGrad rg{a.m, 0.0f, 0.0f, 0.0f};
    if (PASS == PASS_POLICY) {
        PolicyRow r;
        if (live) {
            r = policy_row(g.policy, in, l, H);
            rg = grad_of(r, g.policy, a, H, log_s);
        }
        if (first) {
            acc[0] += r.sur;
            acc[1] += r.kl;
            acc[2] += r.H;
            acc[3] += r.cut;
            if (g.policy.out_coeff) g.policy.out_coeff[n] = r.c * g.policy.grad_scale;
            if (g.policy.out_entropy_coeff) g.policy.out_entropy_coeff[n] = r.g * g.policy.grad_scale;
        }
    }
    if (PASS == PASS_PREF_GRAD) {
        const float c = live ? in.w : 0.0f;
        rg.C = c;
        rg.A = c == 0.0f ? 0.0f : -c * reciprocal(a.s);
        if (first && g.out_coeff) g.out_coeff[n] = -c;
    } else if (first) {
        if (g.out_logp) g.out_logp[n] = l;
        if (g.out_entropy) g.out_entropy[n] = H;
    }
    if (PASS == PASS_PREF_FORWARD && first) {
        g.logp[n] = live ? exact_l(a, z_a) : kAddsNothing;
        if (g.grad) g.grad[n] = {a.m, live ? 1.0f / a.s : 0.0f, 0.0f, 0.0f};
    }
    return rg;
}

// The workgroup's part of the loss: into `sums`, or the loss itself where nobody else has a part.  wave[i][.]: wave i's.
__device__ __forceinline__ void finish_sums(const RowArgs &g, const double (*wave)[4], int waves)
{
    if (threadIdx.x >= 4) return;
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    if (gridDim.x == 1) {
        if (threadIdx.x) return;
        for (int w = 0; w < waves; ++w)
            for (int i = 0; i < 4; ++i) v[i] += wave[w][i];
        policy_stats_out(v, g.policy.ref_logp ? g.policy.kl_coeff : 0.0f, g.policy.entropy_coeff, g.out_stats);
    } else {
        for (int w = 0; w < waves; ++w) v[0] += wave[w][threadIdx.x];
        g.sums[static_cast<size_t>(blockIdx.x) * 4 + threadIdx.x] = v[0];
    }
}

// The same from a part of every thread; sums[i]: sum i's.
__device__ __forceinline__ void finish_block_sums(const RowArgs &g, double (*sums)[256])
{
    const int tid = threadIdx.x, i = tid >> 6, lane = tid & 63;      // wave i takes sum i
    const double v = wave_sum((sums[i][lane] + sums[i][lane + 64]) + (sums[i][lane + 128] + sums[i][lane + 192]));
    if (gridDim.x > 1) {
        if (lane == 0) g.sums[static_cast<size_t>(blockIdx.x) * 4 + i] = v;
    } else {
        if (lane == 0) sums[i][0] = v;
        __syncthreads();
        if (tid == 0) {
            const double all[4] = {sums[0][0], sums[1][0], sums[2][0], sums[3][0]};
            policy_stats_out(all, g.policy.ref_logp ? g.policy.kl_coeff : 0.0f, g.policy.entropy_coeff, g.out_stats);
        }
    }
}

// ---- narrow rows (up to kNarrow actions): a row per thread, 256 rows through LDS, everything in one pass.
// The rows' elements go in and out in the order they lie in memory, whatever their number; rows are an odd number
// of words apart in LDS, so that the lanes' walks along their rows meet 32 different banks.
// The elements of rows [n0, n0 + count) into the tile or out of it, in 16-byte slots where the rows lie behind one another.
template <typename T, bool STORE>
__device__ __forceinline__ void narrow_tile(const void *data, int64_t stride, int64_t n0, int count, int V, uint32_t magic, int pitch,
                                            float *tile)
{
    constexpr int N = Elem<T>::N;
    const int tid = threadIdx.x;
    auto row_at = [&](int e) { return V == 1 ? e : static_cast<int>(__umulhi(static_cast<uint32_t>(e), magic)); };
    if (stride == V) {
        T *base = static_cast<T *>(const_cast<void *>(data)) + n0 * V;
        const int total = count * V;
        const Row<T> all(base, 0, 0, total);
        for (int i = tid; i < all.slots; i += 256) {
            float f[N];
            const int e = all.first(i);
            if (!STORE) all.load(i, f, 0.0f);
            int r = row_at(max(e, 0)), c = max(e, 0) - r * V;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                if (e + k >= 0 && e + k < total) {
                    if (STORE) f[k] = tile[r * pitch + c];
                    else tile[r * pitch + c] = f[k];
                    if (++c == V) {
                        c = 0;
                        ++r;
                    }
                }
            }
            if (STORE) store_slot(base, e, total, f);
        }
    } else {
        for (int i = tid; i < count * V; i += 256) {
            const int r = row_at(i), c = i - r * V;
            T *p = static_cast<T *>(const_cast<void *>(data)) + (n0 + r) * stride + c;
            if (STORE) Elem<T>::store(p, tile[r * pitch + c]);
            else tile[r * pitch + c] = Elem<T>::load(p);
        }
    }
}

// The thread keeps its row in CAP registers.  WHOLE: rows of CAP actions are 4, 8, 16 or 32 aligned bytes, which
// the thread reads and writes itself, without LDS.
template <typename T, int PASS, int CAP, bool WHOLE>
__global__ __launch_bounds__(256) void k_narrow(RowArgs g)
{
    constexpr bool kGrad = PASS == PASS_POLICY || PASS == PASS_PREF_GRAD;
    extern __shared__ float tile[];
    __shared__ double sums[PASS == PASS_POLICY ? 4 : 1][256];
    const int V = WHOLE ? CAP : g.x.V, pitch = V | 1, tid = threadIdx.x;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * 256, n = n0 + tid;
    const int count = static_cast<int>(min(int64_t{256}, g.x.n - n0));
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    RowIn in;
    in.p.counts = false;
    if (tid < count) {
        in.p = place_of(g.rows, n);
        if (in.p.counts) in.act = g.actions[n];
        read_in<PASS>(g, n, in);
    }
    float reg[CAP];
    float *z = tile + tid * pitch;
    // f(j, logit j) for every action
    auto each = [&](auto f) {
#pragma unroll
        for (int j = 0; j < CAP; ++j)
            if (WHOLE || j < V) f(j, reg[j]);
    };
    if (WHOLE) {
        if (in.p.counts) {
            Words<CAP * sizeof(T)> words;
            words.load(static_cast<const T *>(g.x.data) + n * g.x.stride);
            unpack_words<T, CAP>(words.w, reg);
        }
    } else {
        narrow_tile<T, false>(g.x.data, g.x.stride, n0, count, V, g.magic, pitch, tile);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < CAP; ++j)
            if (j < V) reg[j] = z[j];
    }
    if (tid < count) {
        Sums a;
        float z_a = 0.0f;
        if (in.p.counts) {
            each([&](int, float v) { a.m = fmaxf(a.m, v); });
            const Ref ref = ref_of(a.m);
            each([&](int j, float v) {
                const float x = ref(v), e = exp2_of(x);
                a.s += e;
                a.t += e * fmaxf(x, kLowest);
                if (j == in.act) z_a = v;
            });
        }
        const RowGrad rg = finish_pass<PASS>(g, n, in, a, z_a, true, acc);
        if (kGrad && g.out_grad) {
            const bool none = rg.A == 0.0f && rg.B == 0.0f && rg.C == 0.0f;
            const Ref ref = ref_of(rg.m);
            auto gradient = [&](int j, float v) {
                float f[1] = {v};
                grad_slot<1>(f, rg, ref);
                return none ? 0.0f : f[0] + (j == in.act ? rg.C : 0.0f);
            };
            if (WHOLE) {
                float f[CAP];
#pragma unroll
                for (int j = 0; j < CAP; ++j) f[j] = gradient(j, reg[j]);
                Words<CAP * sizeof(T)> words;
                pack_words<T, CAP>(f, words.w);
                words.store(static_cast<T *>(g.out_grad) + n * g.grad_stride);
            } else {
                each([&](int j, float v) { z[j] = gradient(j, v); });
            }
        }
    }
    if (kGrad && !WHOLE && g.out_grad) {
        __syncthreads();
        narrow_tile<T, true>(g.out_grad, g.grad_stride, n0, count, V, g.magic, pitch, tile);
    }
    if (PASS == PASS_POLICY) {
        for (int i = 0; i < 4; ++i) sums[i][tid] = acc[i];
        __syncthreads();
        finish_block_sums(g, sums);
    }
}

// The words of a slot into the candidates for the largest logit.
template <typename T>
__device__ __forceinline__ void add_words(const uint4 &v, uint32_t &most, uint32_t &least)
{
    most = Elem<T>::more(Elem<T>::more(Elem<T>::more(Elem<T>::more(most, v.x), v.y), v.z), v.w);
    least = Elem<T>::less(Elem<T>::less(Elem<T>::less(Elem<T>::less(least, v.x), v.y), v.z), v.w);
}

// The slot stays in its four registers: without this the compiler keeps every unpacked value from one use to the next.
__device__ __forceinline__ void keep_packed(uint4 &v) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }

// ---- rows of middling width: LANES lanes to a row, R rows of a lane one behind another, all of them in its registers; what
// follows from the sums of the workgroup's rows is done a row to a thread, as for narrow rows: with a wave to a row it
// took most of the time (131072 rows of 256 floats: 122 us, against 74; 56 with slots from the row's start).
// A row is cut into slots of 16 bytes from its start, aligned or not; the last one is the row's last 16 bytes, some of which
// the slot before has too: they are left out of the sums, and their gradient is written twice, the same.
// STREAM: the gradient goes past the caches, where every row of it begins at a multiple of 16 bytes (65536 rows of 512
// floats: 53 us against 64); lines that several stores fill in parts are better put together in them (671040 rows of 100
// bf16: 167 us against 91).
template <typename T, int LANES, int CH, int R, int PASS, bool STREAM>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4))) void k_group(RowArgs g)
{
    constexpr int N = Elem<T>::N, ABREAST = 256 / LANES, ROWS = ABREAST * R;
    constexpr bool kGrad = PASS == PASS_POLICY || PASS == PASS_PREF_GRAD;
    static_assert(ROWS <= 256, "a thread to a row");
    __shared__ RowPart part[ROWS];
    __shared__ RowGrad grads[ROWS];
    __shared__ int acts[ROWS];
    __shared__ bool counts[ROWS];
    __shared__ double sums[PASS == PASS_POLICY ? 4 : 1][256];
    const int tid = threadIdx.x, lane = tid & (LANES - 1), V = g.x.V;
    const int mine = LANES == 64 ? __builtin_amdgcn_readfirstlane(tid >> 6) : tid / LANES;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * ROWS;
    const int rows = static_cast<int>(min(int64_t{ROWS}, g.x.n - n0));
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    RowIn in;
    in.p.counts = false;
    float z_a = 0.0f;
    if (tid < rows) {
        in.p = place_of(g.rows, n0 + tid);
        if (in.p.counts) in.act = g.actions[n0 + tid];
        read_in<PASS>(g, n0 + tid, in);
        if (in.act >= 0 && in.act < V) z_a = Elem<T>::load(static_cast<const T *>(g.x.data) + (n0 + tid) * g.x.stride + in.act);
        counts[tid] = in.p.counts;
        if (kGrad) acts[tid] = in.act;
    }
    __syncthreads();
    // first element of slot k of this lane; the elements of it that the slot before has
    auto start = [&](int k) { return min((k * LANES + lane) * N, V - N); };
    auto twice = [&](int k) { return (k * LANES + lane) * N - start(k); };
    uint4 v[R * CH];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = i * ABREAST + mine;
        if (r < rows && counts[r]) {
            const T *row = static_cast<const T *>(g.x.data) + (n0 + r) * g.x.stride;
#pragma unroll
            for (int k = 0; k < CH; ++k) v[i * CH + k] = load_16(row + start(k));
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int r = i * ABREAST + mine;
        if (r < rows && counts[r]) {
            Sums a;
            uint32_t most = Elem<T>::kNone, least = 0xffffffffu;
#pragma unroll
            for (int k = 0; k < CH; ++k) add_words<T>(v[i * CH + k], most, least);
            a.m = max_of<LANES>(Elem<T>::largest(most, least));
            const Ref ref = ref_of(a.m);
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if ((k * LANES + lane) * N < V) {
                    float f[N];
                    Elem<T>::unpack(v[i * CH + k], f);
                    if (V % N) {
                        const int skip = twice(k);
#pragma unroll
                        for (int j = 0; j < N; ++j) f[j] = j < skip ? -INFINITY : f[j];
                    }
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const float x = ref(f[j]), e = exp2_of(x);
                        a.s += e;
                        if (PASS == PASS_POLICY || PASS == PASS_LOGP) a.t += e * fmaxf(x, kLowest);
                    }
                }
            a.s = sum_of<LANES>(a.s);
            if (PASS == PASS_POLICY || PASS == PASS_LOGP) a.t = sum_of<LANES>(a.t);
            if (lane == 0) part[r] = {a.m, a.s, a.t};
        }
        if (kGrad) {
#pragma unroll
            for (int k = 0; k < CH; ++k) keep_packed(v[i * CH + k]);
        }
    }
    __syncthreads();
    if (tid < rows) {
        const RowPart of = part[tid];
        grads[tid] = finish_pass<PASS>(g, n0 + tid, in, in.p.counts ? Sums{of.m, of.s, of.t} : Sums{}, z_a, true, acc);
    }
    if (PASS == PASS_POLICY) {
        for (int i = 0; i < 4; ++i) sums[i][tid] = acc[i];
    }
    __syncthreads();
    if (kGrad && g.out_grad) {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int r = i * ABREAST + mine;
            if (r >= rows) continue;
            const RowGrad rg = grads[r];
            const Ref ref = ref_of(rg.m);
            const bool none = rg.A == 0.0f && rg.B == 0.0f && rg.C == 0.0f;
            const int act = none ? -1 : acts[r];
            T *o = static_cast<T *>(g.out_grad) + (n0 + r) * g.grad_stride;
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if ((k * LANES + lane) * N < V) {
                    const int e = start(k);
                    float f[N];
                    if (none) {
#pragma unroll
                        for (int j = 0; j < N; ++j) f[j] = 0.0f;
                    } else {
                        Elem<T>::unpack(v[i * CH + k], f);
                        grad_slot<N>(f, rg, ref);
                        if (act >= e && act < e + N) {
#pragma unroll
                            for (int j = 0; j < N; ++j) f[j] += e + j == act ? rg.C : 0.0f;
                        }
                    }
                    if (STREAM) stream_16(o + e, Elem<T>::pack(f));
                    else store_16(o + e, Elem<T>::pack(f));
                }
        }
    }
    if constexpr (PASS == PASS_POLICY) finish_block_sums(g, sums);
}

// ---- wider rows that fit in the registers of LANES threads: read once, the maximum and the sums of every wave, those of
// the row in its first wave, the gradient from the registers.  Bound by memory: a pass that reads the row again for its
// gradient moves a half more.
// A lane holds CH slots of 16 aligned bytes, LANES apart, and one of the up to 2 N - 2 elements in front of the first and
// behind the last whole slot.  Loads are predicated, with one value or -infinity in place of the others, so that all of
// them are on their way before the first is waited for.
// In launches of one width or another that were tried for rows of 32768 to 65536 bf16, workgroups of 256 and 512 threads with
// sixteen slots to a lane came out first: several of them are on a compute unit, one loading while another computes
// (8192 rows of 32768: 217 to 232 us; with 1024 threads and eight slots 272).
template <typename T, int LANES, int CH, int PASS>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) __attribute__((amdgpu_waves_per_eu(4))) void k_rows(RowArgs g)
{
    static_assert(LANES == 64 || LANES >= 256, "a wave or a workgroup to a row");
    constexpr int N = Elem<T>::N, ROWS = LANES < 256 ? 256 / LANES : 1, WAVES = LANES / 64;
    constexpr bool kGrad = PASS == PASS_POLICY;
    __shared__ RowPart part[WAVES];
    __shared__ RowGrad shared_grad;
    __shared__ double loss[ROWS][4];               // of the rows that these lanes have had
    const int tid = threadIdx.x;
    int lane = tid & (LANES - 1);
    const int V = g.x.V;
    const int mine = WAVES == 1 ? __builtin_amdgcn_readfirstlane(tid >> 6) : 0;
    if (PASS == PASS_POLICY && lane < 4) loss[mine][lane] = 0.0;
    if (PASS == PASS_POLICY) __syncthreads();
    for (int64_t n = static_cast<int64_t>(blockIdx.x) * ROWS + mine; n < g.x.n; n += static_cast<int64_t>(gridDim.x) * ROWS) {
        asm volatile("" : "+v"(lane));               // the slots' offsets are taken anew: kept over the rows they would cost CH registers
        const Span<T> row(static_cast<const T *>(g.x.data) + n * g.x.stride, V);
        const int head = row.head, whole = row.whole, edge = row.edge(lane);
        RowIn in;
        in.p = place_of(g.rows, n);
        if (in.p.counts) in.act = g.actions[n];
        const int act = in.act;
        const bool acts = act >= 0 && act < V;
        uint4 v[CH];
        float z_edge = -INFINITY, z_a = 0.0f;
        Sums a;
        if (in.p.counts) {
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (k * LANES < whole) v[k] = row.load(k * LANES + lane);
            if (edge >= 0) z_edge = Elem<T>::load(row.p + edge);
            if (acts) z_a = Elem<T>::load(row.p + act);
            uint32_t most = Elem<T>::kNone, least = 0xffffffffu;
#pragma unroll
            for (int k = 0; k < CH; ++k)
                if (k * LANES < whole) add_words<T>(v[k], most, least);
            a.m = max_of<64>(fmaxf(z_edge, Elem<T>::largest(most, least)));
            const Ref ref = ref_of(a.m);
            auto add_all = [&](auto with_t) {
                auto add_one = [&](float z) {
                    const float x = ref(z), e = exp2_of(x);
                    a.s += e;
                    if (with_t) a.t += e * fmaxf(x, kLowest);
                };
                if (edge >= 0) add_one(z_edge);
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    if (k * LANES + lane < whole) {
                        float f[N];
                        Elem<T>::unpack(v[k], f);
#pragma unroll
                        for (int j = 0; j < N; ++j) add_one(f[j]);
                    }
                    if (kGrad) keep_packed(v[k]);
                }
                a.s = sum_of<64>(a.s);
                if (with_t) a.t = sum_of<64>(a.t);
            };
            if (PASS == PASS_POLICY || (PASS == PASS_LOGP && g.out_entropy)) add_all(std::true_type{});
            else add_all(std::false_type{});
        }
        if (WAVES == 1 || tid < 64) read_in<PASS>(g, n, in);
        RowGrad rg;
        if (WAVES > 1) {
            if ((tid & 63) == 0) part[tid >> 6] = {a.m, a.s, a.t};
            __syncthreads();
            if (tid < 64) {
                const RowPart of = part[lane < WAVES ? lane : 0];
                a = merge_of<64>(lane < WAVES ? Sums{of.m, of.s, of.t} : Sums{});
                rg = finish_pass<PASS>(g, n, in, a, z_a, tid == 0, loss[0]);
                if (tid == 0) shared_grad = rg;
            }
            __syncthreads();
            rg = shared_grad;
        } else {
            rg = finish_pass<PASS>(g, n, in, a, z_a, lane == 0, loss[mine]);
        }
        if (kGrad && g.out_grad) {
            T *o = static_cast<T *>(g.out_grad) + n * g.grad_stride;
            const bool none = rg.A == 0.0f && rg.B == 0.0f && rg.C == 0.0f;
            const Ref ref = ref_of(rg.m);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                keep_packed(v[k]);
                if (k * LANES + lane < whole) {
                    float f[N];
                    if (none) {
#pragma unroll
                        for (int j = 0; j < N; ++j) f[j] = 0.0f;
                    } else {
                        Elem<T>::unpack(v[k], f);
                        grad_slot<N>(f, rg, ref);
                    }
                    stream_16(o + head + static_cast<uint32_t>(k * LANES + lane) * N, Elem<T>::pack(f));
                }
            }
            if (edge >= 0) {
                float f[1] = {z_edge};
                grad_slot<1>(f, rg, ref);
                Elem<T>::store(o + edge, none ? 0.0f : f[0]);
            }
            // the action's own logit: written once more by the lane that has written it
            if (!none && acts) {
                const int slot = (act - head) / N;
                if (act >= head && act < row.tail() ? lane == (slot & (LANES - 1)) : edge == act) {
                    float f[1] = {z_a};
                    grad_slot<1>(f, rg, ref);
                    Elem<T>::store(o + act, f[0] + rg.C);
                }
            }
        }
    }
    if (PASS == PASS_POLICY) {
        __syncthreads();
        finish_sums(g, loss, ROWS);
    }
}

// ---- long rows, or slices of them where there are few, that are only read: a workgroup to a row (slice), a few slots of a
// lane on their way while the ones before are added.  A lane's sums are fp32 over a step (16 or 32 logits) and float64 over the
// steps: in fp32 alone equal logits all round the same way (rows of 2^22 of them: log probabilities off by 2e-4).  Its x are relative
// to a logit that the largest it has seen exceeds by kRise at most, and to the largest in the end: scaled at every step
// that rises a little, the sums would be rounded the same way as often (a rise of 0.2 over 2^22 logits: off by 2e-5).
constexpr int kStreamSlots = 4;
constexpr float kRise = 4.0f;

template <typename T, bool WITH_T>
__device__ __forceinline__ Sums stream_sums(const Span<T> &row, int begin, int end, bool with_edge)
{
    constexpr int N = Elem<T>::N, STEP = kStreamSlots * 256;
    const int tid = threadIdx.x;
    Sums a;                                              // of a step, and
    double s = 0.0, t = 0.0;                             // of the steps before, both relative to a.m
    float most_seen = -INFINITY;
    Ref ref = ref_of(a.m);
    auto rebase = [&](float m) {                         // (as `rebased`, between two steps)
        const Ref to = ref_of(m);
        if (s != 0.0) {
            const float d = to(ref.m), e = exp2_of(d);
            t = e * (t + fmaxf(d, kLowest) * s);
            s *= e;
        }
        a.m = m;
        ref = to;
    };
    auto add_one = [&](float z) {
        const float x = ref(z), e = exp2_of(x);
        a.s += e;
        if (WITH_T) a.t += e * fmaxf(x, kLowest);
    };
    auto end_step = [&]() {
        s += a.s;
        if (WITH_T) t += a.t;
        a.s = a.t = 0.0f;
    };
    uint4 next[kStreamSlots];
    if (begin < end) {
#pragma unroll
        for (int k = 0; k < kStreamSlots; ++k) next[k] = row.load(min(begin + tid + k * 256, end - 1));
    }
    if (with_edge) {
        const int e = row.edge(tid);
        const float z = e >= 0 ? Elem<T>::load(row.p + e) : -INFINITY;
        if (z > a.m) rebase(z);
        most_seen = z;
        if (e >= 0) add_one(z);
        end_step();
    }
    for (int i = begin + tid; i - tid < end; i += STEP) {
        uint4 v[kStreamSlots];
#pragma unroll
        for (int k = 0; k < kStreamSlots; ++k) v[k] = next[k];
        if (i - tid + STEP < end) {
#pragma unroll
            for (int k = 0; k < kStreamSlots; ++k) next[k] = row.load(min(i + STEP + k * 256, end - 1));
        }
        uint32_t most = Elem<T>::kNone, least = 0xffffffffu;
#pragma unroll
        for (int k = 0; k < kStreamSlots; ++k) add_words<T>(v[k], most, least);
        const float m = Elem<T>::largest(most, least);
        most_seen = fmaxf(most_seen, m);
        if (m > a.m + kRise) rebase(m);
#pragma unroll
        for (int k = 0; k < kStreamSlots; ++k)
            if (i + k * 256 < end) {
                float f[N];
                Elem<T>::unpack(v[k], f);
#pragma unroll
                for (int j = 0; j < N; ++j) add_one(f[j]);
            }
        end_step();
    }
    if (most_seen > a.m) rebase(most_seen);
    return merge_of<64>(Sums{a.m, static_cast<float>(s), static_cast<float>(t)});
}

// PASS_LOGP and PASS_PREF_FORWARD of whole rows, or (slices > 1) the sums of the slices.
template <typename T, int PASS>
__global__ __launch_bounds__(256) void k_stream(RowArgs g, RowPart *__restrict__ parts, int slices, bool with_t)
{
    __shared__ RowPart part[4];
    const int tid = threadIdx.x;
    for (int64_t n = blockIdx.x; n < g.x.n; n += gridDim.x) {
        RowIn in;
        in.p = place_of(g.rows, n);
        const Span<T> row(static_cast<const T *>(g.x.data) + n * g.x.stride, g.x.V);
        Sums a;
        float z_a = 0.0f;
        if (in.p.counts) {
            if (parts == nullptr) {
                in.act = g.actions[n];
                if (in.act >= 0 && in.act < g.x.V) z_a = Elem<T>::load(row.p + in.act);
            }
            const int per = (row.whole + slices - 1) / slices, begin = per * blockIdx.y, end = min(row.whole, begin + per);
            a = with_t ? stream_sums<T, true>(row, begin, end, blockIdx.y == 0) : stream_sums<T, false>(row, begin, end, blockIdx.y == 0);
            if ((tid & 63) == 0) part[tid >> 6] = {a.m, a.s, a.t};
        }
        __syncthreads();
        if (tid < 64 && in.p.counts) {
            const RowPart of = part[tid & 3];
            a = merge_of<64>(tid < 4 ? Sums{of.m, of.s, of.t} : Sums{});
        }
        if (tid < 64) {
            if (parts == nullptr) {
                double none[4];
                finish_pass<PASS>(g, n, in, a, z_a, tid == 0, none);
            } else if (in.p.counts && tid == 0) {
                parts[n * slices + blockIdx.y] = {a.m, a.s, a.t};
            }
        }
        __syncthreads();
    }
}

// What follows from the slices of rows: a thread to a row of one slice, a wave to a row of several.
template <typename T, int PASS, int LANES>
__global__ __launch_bounds__(256) void k_finish(RowArgs g, const RowPart *__restrict__ parts, int slices)
{
    __shared__ double sums[PASS == PASS_POLICY ? 4 : 1][256];
    const int tid = threadIdx.x, lane = tid & (LANES - 1);
    const int64_t n = static_cast<int64_t>(blockIdx.x) * (256 / LANES) + tid / LANES;
    double acc[4] = {0.0, 0.0, 0.0, 0.0};
    if (n < g.x.n) {
        RowIn in;
        in.p = place_of(g.rows, n);
        Sums a;
        float z_a = 0.0f;
        if (in.p.counts) {
            in.act = g.actions[n];
            read_in<PASS>(g, n, in);
            if (lane < slices) {
                const RowPart of = parts[n * slices + lane];
                a = {of.m, of.s, of.t};
            }
            if (in.act >= 0 && in.act < g.x.V) z_a = Elem<T>::load(static_cast<const T *>(g.x.data) + n * g.x.stride + in.act);
            if constexpr (LANES > 1) a = merge_of<LANES>(a);
        }
        const RowGrad rg = finish_pass<PASS>(g, n, in, a, z_a, lane == 0, acc);
        if (PASS == PASS_POLICY && g.grad && lane == 0) g.grad[n] = rg;
    }
    if constexpr (PASS == PASS_POLICY) {
        for (int i = 0; i < 4; ++i) sums[i][tid] = acc[i];
        __syncthreads();
        finish_block_sums(g, sums);
    }
}

// Slots of 16 bytes in a row, the last one begun; those of the rows that k_narrow and k_group take, and the rows of a workgroup of k_group.
constexpr int kGroupSlots = 256;
int row_slots(const LogitsView &x) { return x.dtype == PL_F32 ? (x.V + 3) / 4 : (x.V + 7) / 8; }
int group_rows(int slots) { return slots <= 16 ? 256 : slots <= 32 ? 128 : slots <= 64 ? 64 : slots <= 128 ? 32 : 16; }

// Whether rows are cut into slices for a workgroup each, with a launch or two more, rather than taken whole.  Kernels of one call,
// bf16, whole rows against slices: log probabilities of 63 rows of 16384 4.3 us against 5.8, of 32768 5.8 against 6.0, of 131072
// 13.7 against 7.6, of one row of 32768 5.2 against 5.1; loss and gradient of 63 rows of 16384 9.4 against 12.6, of 32768 11.9
// against 12.6, of 131072 22.4 against 17.8; of 128 rows of 131072 24.0 against 28.2.
bool few_rows(const LogitsView &x) { return x.n < 64 && x.V >= 32768; }

int row_blocks(int64_t n) { return static_cast<int>((n + kRowsPerBlock - 1) / kRowsPerBlock); }

// Rows in slices: their sums into ws.parts, and what follows from them.
template <int PASS>
int launch_slices(const RowArgs &g, const LossWorkspace &ws, bool with_t, hipStream_t s)
{
    const int blocks = static_cast<int>(ws.slices > 1 ? (g.x.n + 3) / 4 : row_blocks(g.x.n));
    by_type(g.x.dtype, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((k_stream<T, PASS_LOGP>), dim3(static_cast<uint32_t>(std::min<int64_t>(g.x.n, 2048)), ws.slices), dim3(256), 0, s,
                           g, ws.parts, ws.slices, with_t);
        if (ws.slices > 1) hipLaunchKernelGGL((k_finish<T, PASS, 64>), dim3(blocks), dim3(256), 0, s, g, ws.parts, ws.slices);
        else hipLaunchKernelGGL((k_finish<T, PASS, 1>), dim3(blocks), dim3(256), 0, s, g, ws.parts, 1);
    });
    return blocks;
}

void launch_grad(GradArgs a, hipStream_t s)
{
    by_type(a.x.dtype, [&](auto t) {
        using T = decltype(t);
        a.chunks = a.out ? (a.x.V / Elem<T>::N + kGradSlots - 1) / kGradSlots : 1;
        hipLaunchKernelGGL(k_row_grad<T>, dim3(static_cast<uint32_t>(std::min<int64_t>((a.x.n * a.chunks + 3) / 4, 1 << 22))), dim3(256), 0,
                           s, a);
    });
}

// Whether one workgroup does the sums of sequences and the pairs: where the sequences are few, whatever the pairs.  By step, its
// threads share a sequence's rows; otherwise a wave has a sequence to itself.  Kernels of one call, four logits a row, one workgroup
// against two launches or three: by step 64 sequences of 30 rows 12.1 us against 11.6, of 200 rows 14.0 against 15.7 (and 19 against
// 25 as a call), with 4096 pairs 57 against 67, with 131072 1390 against 1662, but 512 sequences of 4 rows 26 against 12, with 4096 pairs
// 168 against 54; packed, 16 sequences of 100 rows 13.2 against 13.6, 64 of 30 20.4 against 14.1.
bool middle_fits(const RowsView &rows)
{
    return rows.order == PL_ROWS_BY_STEP ? rows.S <= kPairSeqs && rows.n <= kMiddleRows : rows.S <= kPairSeqs / 4 && rows.n <= kMiddleRows / 16;
}

GradArgs grad_args(const LogitsView &x, const int32_t *actions, const LossWorkspace &ws, void *out, int64_t out_stride)
{
    GradArgs a{};
    a.x = x;
    a.actions = actions;
    a.grad = ws.grad;
    a.out = out;
    a.out_stride = out_stride;
    return a;
}

// Sequences side by side in a workgroup of k_seq_sums: neighbouring rows of PL_ROWS_BY_STEP are of neighbouring
// sequences, of the other orders of one.
int seq_lanes(const RowsView &rows)
{
    int lanes = 1;
    if (rows.order == PL_ROWS_BY_STEP)
        while (lanes < 64 && lanes < rows.S) lanes *= 2;
    return lanes;
}

// Sums and numbers of rows of every sequence.
void launch_seq_sums(const RowsView &rows, const double *logp, const float *ref, const LossWorkspace &ws, hipStream_t s)
{
    const int lanes_s = seq_lanes(rows);
    const bool whole = ws.seq_parts == 1;
    hipLaunchKernelGGL(k_seq_sums, dim3((rows.S + lanes_s - 1) / lanes_s, ws.seq_parts), dim3(256), 0, s, rows, logp, ref,
                       lanes_s, whole ? ws.seq_sum : ws.seq_part, whole ? ws.seq_n : ws.seq_part_n);
    if (!whole)
        hipLaunchKernelGGL(k_seq_totals, dim3(1), dim3(1024), 0, s, rows, ws.seq_parts, ws.seq_part, ws.seq_part_n, ws.seq_sum, ws.seq_n,
                           nullptr, nullptr);
}

// Whether one workgroup counts the rows under a mask.  A call on rows of four logits, one workgroup against two launches: 16 sequences
// of 512 rows 9.7 us against 12.3 (by step), of 2048 14.6 against 12.3; packed 12.6 against 12.7 and 26 against 13.  The second
// launch has sixteen lanes for a sequence: 1024 of 32 rows 14.5 against 26.8 (by step), packed 41 against 29.
bool weights_fit(const RowsView &rows)
{
    return rows.S <= kMiddleSeqs && rows.n <= 8192 + (rows.order == PL_ROWS_PACKED ? 0 : 24 * static_cast<int64_t>(rows.S));
}

// The weights of rows whose number is found on the device.
void launch_weights(const RowsView &rows, bool by_seqs, const LossWorkspace &ws, hipStream_t s)
{
    const int lanes_s = seq_lanes(rows);
    if (rows.mask && weights_fit(rows)) {
        hipLaunchKernelGGL(k_weights, dim3(1), dim3(1024), 0, s, rows, by_seqs ? nullptr : ws.weight, by_seqs ? ws.weights : nullptr);
        return;
    }
    if (rows.mask)
        hipLaunchKernelGGL(k_seq_sums, dim3((rows.S + lanes_s - 1) / lanes_s, ws.seq_parts), dim3(256), 0, s, rows, nullptr, nullptr,
                           lanes_s, nullptr, ws.seq_part_n);
    hipLaunchKernelGGL(k_seq_totals, dim3(1), dim3(1024), 0, s, rows, ws.seq_parts, nullptr, rows.mask ? ws.seq_part_n : nullptr, nullptr,
                       ws.seq_n, by_seqs ? nullptr : ws.weight, by_seqs ? ws.weights : nullptr);
}

RowArgs row_args(const LogitsView &x, const RowsView &rows, const int32_t *actions)
{
    RowArgs g{};
    g.x = x;
    g.rows = rows;
    g.actions = actions;
    g.magic = x.V > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / x.V + 1) : 0;
    return g;
}

// Whole rows in one pass (k_narrow, k_group, k_rows), and how many workgroups take them; 0 where they do not fit or where there are
// so few of them that a row is better cut into slices.
template <int PASS>
int launch_rows(const RowArgs &g, hipStream_t s)
{
    int blocks = 0;

    by_type(g.x.dtype, [&](auto t) {
        using T = decltype(t);
        const int slots = row_slots(g.x), whole_slots = g.x.V / Elem<T>::N;
        auto launch = [&](auto kernel, int64_t grid, int threads, size_t lds) {
            blocks = static_cast<int>(grid);
            hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), lds, s, g);
        };
        // kernels whose workgroups take `rows` rows each, and kernels whose workgroups go over the rows
        auto go = [&](auto kernel, int rows, size_t lds = 0) { launch(kernel, (g.x.n + rows - 1) / rows, 256, lds); };
        auto go_over = [&](auto kernel, int rows, int threads) {
            launch(kernel, std::min<int64_t>((g.x.n + rows - 1) / rows, kMaxSumBlocks), threads, 0);
        };
        auto group = [&](auto f) {
            if constexpr (PASS == PASS_POLICY || PASS == PASS_PREF_GRAD) {
                const bool at_16 = reinterpret_cast<uintptr_t>(g.out_grad) % 16 == 0 && g.grad_stride * sizeof(T) % 16 == 0;
                if (at_16) return f(std::true_type{});
            }
            f(std::false_type{});
        };
        if (g.x.V <= kNarrow) {
            constexpr int W = 4 / sizeof(T);             // elements of a word
            const size_t bytes = g.x.V * sizeof(T), align = std::min<size_t>(bytes, 16);
            const bool whole = (reinterpret_cast<uintptr_t>(g.x.data) | reinterpret_cast<uintptr_t>(g.out_grad)) % align == 0 &&
                               g.x.stride * sizeof(T) % align == 0 && (!g.out_grad || g.grad_stride * sizeof(T) % align == 0);
            const size_t lds = 256 * (g.x.V | 1) * sizeof(float);
            if (whole && bytes == 4 && sizeof(T) == 2) go(k_narrow<T, PASS, 2, true>, 256);
            else if (whole && bytes == 8) go(k_narrow<T, PASS, 2 * W, true>, 256);
            else if (whole && bytes == 16) go(k_narrow<T, PASS, 4 * W, true>, 256);
            else if (whole && bytes == 32) go(k_narrow<T, PASS, 8 * W, true>, 256);
            else go(k_narrow<T, PASS, kNarrow, false>, 256, lds);
        }
        else if (slots <= 4) group([&](auto stream) { go(k_group<T, 4, 1, 4, PASS, decltype(stream)::value>, group_rows(slots)); });
        else if (slots <= 8) group([&](auto stream) { go(k_group<T, 4, 2, 4, PASS, decltype(stream)::value>, group_rows(slots)); });
        else if (slots <= 16) group([&](auto stream) { go(k_group<T, 4, 4, 4, PASS, decltype(stream)::value>, group_rows(slots)); });
        else if (slots <= 32) group([&](auto stream) { go(k_group<T, 16, 2, 8, PASS, decltype(stream)::value>, group_rows(slots)); });
        else if (slots <= 64) group([&](auto stream) { go(k_group<T, 16, 4, 4, PASS, decltype(stream)::value>, group_rows(slots)); });
        else if (slots <= 128) group([&](auto stream) { go(k_group<T, 16, 8, 2, PASS, decltype(stream)::value>, group_rows(slots)); });
        else if (slots <= 256) group([&](auto stream) { go(k_group<T, 64, 4, 4, PASS, decltype(stream)::value>, group_rows(slots)); });
        if constexpr (PASS != PASS_PREF_GRAD) {
            if (slots <= kGroupSlots || few_rows(g.x)) return;
            if constexpr (PASS == PASS_POLICY) {
                if (whole_slots <= 64 * 16) go_over(k_rows<T, 64, 16, PASS>, 4, 256);
                else if (whole_slots <= 256 * 16) go_over(k_rows<T, 256, 16, PASS>, 1, 256);
                else if (whole_slots <= 512 * 16) go_over(k_rows<T, 512, 16, PASS>, 1, 512);
                else if (whole_slots <= 1024 * 16) go_over(k_rows<T, 1024, 16, PASS>, 1, 1024);
            } else if (whole_slots <= 64 * 12) {
                // (rows that are only read: 22336 of 3001 bf16 32 us, streamed 47; 8384 of 8000: 31 us, streamed 26)
                go_over(k_rows<T, 64, 12, PASS>, 4, 256);
            } else {
                blocks = static_cast<int>(std::min<int64_t>(g.x.n, 1 << 22));
                hipLaunchKernelGGL((k_stream<T, PASS>), dim3(blocks), dim3(256), 0, s, g, nullptr, 1, g.out_entropy != nullptr);
            }
        }
    });
    return blocks;
}

}  // namespace

LossWorkspace carve_loss_workspace(void *base, const LogitsView &x, const RowsView &rows)
{
    LossWorkspace w;
    size_t pos = 0;
    auto take = [&](auto *&p, size_t count) {
        using T = std::remove_reference_t<decltype(*p)>;
        p = base ? reinterpret_cast<T *>(static_cast<char *>(base) + pos) : nullptr;
        pos += (count * sizeof(T) + 15) / 16 * 16;
    };
    const size_t n = static_cast<size_t>(x.n), S = static_cast<size_t>(rows.S);
    // a thousand workgroups where the rows are fewer, of 8192 logits at least
    if (x.n > 0)    // (the workspace does not depend on which kernels run)
        w.slices = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({1024 / x.n, x.V / 8192, kMaxSlices})));
    // eight rows to a thread of k_seq_sums, as long as the workgroups are few
    const int64_t longest = rows.order == PL_ROWS_PACKED ? rows.n / rows.S : rows.L;
    const int64_t per_part = 8 * (256 / seq_lanes(rows)), groups = (rows.S + seq_lanes(rows) - 1) / seq_lanes(rows);
    w.seq_parts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({(longest + per_part - 1) / per_part, kMaxSeqParts, 2048 / groups})));
    take(w.parts, n * w.slices);
    take(w.grad, n);
    take(w.logp, n);
    take(w.seq_part, S * w.seq_parts * 2);
    take(w.seq_part_n, S * w.seq_parts);
    take(w.seq_sum, S * 2);
    take(w.seq_n, S);
    take(w.seq_coeff, S);
    take(w.weights, S);
    take(w.weight, 1);
    const int slots = row_slots(x);
    const int64_t sum_blocks = slots <= kGroupSlots ? (x.n + group_rows(slots) - 1) / group_rows(slots) : row_blocks(x.n);
    take(w.sums, static_cast<size_t>(std::max<int64_t>(sum_blocks, kMaxSumBlocks)) * 4);
    w.bytes = pos;
    return w;
}

void launch_action_logp(const LogitsView &x, const RowsView &rows, const int32_t *actions, float *out_logp, float *out_entropy,
                        const LossWorkspace &ws, hipStream_t s)
{
    RowArgs g = row_args(x, rows, actions);
    g.out_logp = out_logp;
    g.out_entropy = out_entropy;
    if (!launch_rows<PASS_LOGP>(g, s)) launch_slices<PASS_LOGP>(g, ws, out_entropy != nullptr, s);
}

void launch_policy_loss(const LogitsView &x, const RowsView &rows, const PolicyArgs &args, int reduction, float *out_stats,
                        void *out_grad, int64_t grad_stride, const LossWorkspace &ws, hipStream_t s)
{
    PolicyArgs a = args;
    if (x.n > 0 && reduction != PL_REDUCE_SUM) {
        if (rows.all) {
            a.weight = static_cast<float>(1.0 / static_cast<double>(x.n));   // sequences of equal length: the same for both
        } else {
            launch_weights(rows, reduction == PL_REDUCE_SEQS, ws, s);
            (reduction == PL_REDUCE_SEQS ? a.weights : a.weight_at) = reduction == PL_REDUCE_SEQS ? ws.weights : ws.weight;
        }
    }
    int blocks = 0;
    if (x.n > 0) {
        RowArgs g = row_args(x, rows, a.actions);
        g.policy = a;
        g.out_logp = a.out_logp;
        g.out_entropy = a.out_entropy;
        g.sums = ws.sums;
        g.out_stats = out_stats;
        g.out_grad = out_grad;
        g.grad_stride = grad_stride;
        blocks = launch_rows<PASS_POLICY>(g, s);
        if (!blocks) {
            g.grad = out_grad ? ws.grad : nullptr;
            blocks = launch_slices<PASS_POLICY>(g, ws, true, s);
            if (out_grad) launch_grad(grad_args(x, a.actions, ws, out_grad, grad_stride), s);
        }
        if (blocks == 1) return;                 // the kernel has written the loss
    }
    hipLaunchKernelGGL(k_policy_stats, dim3(1), dim3(1024), 0, s, ws.sums, blocks, a.ref_logp ? a.kl_coeff : 0.0f,
                       a.entropy_coeff, out_stats);
}

void launch_preference_loss(const LogitsView &x, const RowsView &rows, const PrefArgs &a, float *out_stats, void *out_grad,
                            int64_t grad_stride, const LossWorkspace &ws, hipStream_t s)
{
    RowArgs g = row_args(x, rows, a.actions);
    g.out_logp = a.out_logp;
    g.logp = ws.logp;
    g.grad = ws.grad;
    // rows that are read fast again whole need nothing kept of them
    const bool again = row_slots(x) <= kGroupSlots;
    if (again) g.grad = nullptr;
    if (x.n > 0 && !launch_rows<PASS_PREF_FORWARD>(g, s)) launch_slices<PASS_PREF_FORWARD>(g, ws, false, s);
    if (middle_fits(rows)) {
        hipLaunchKernelGGL(k_pref_middle, dim3(1), dim3(1024), 0, s, rows, a, ws.logp, seq_lanes(rows), ws.seq_coeff, out_stats);
    } else {
        launch_seq_sums(rows, ws.logp, a.ref_logp, ws, s);
        hipLaunchKernelGGL(k_pairs, dim3((rows.S + 256 / kTeam - 1) / (256 / kTeam)), dim3(256), 0, s, a, rows.S, ws.seq_sum, ws.seq_n,
                           ws.seq_coeff, out_stats);
    }
    if (x.n == 0 || (!out_grad && !a.out_coeff)) return;
    if (again) {
        g.out_coeff = a.out_coeff;
        g.seq_coeff = ws.seq_coeff;
        g.grad_scale = a.grad_scale;
        g.out_grad = out_grad;
        g.grad_stride = grad_stride;
        launch_rows<PASS_PREF_GRAD>(g, s);
    } else {
        GradArgs ga = grad_args(x, a.actions, ws, out_grad, grad_stride);
        ga.rows = rows;
        ga.seq_coeff = ws.seq_coeff;
        ga.out_coeff = a.out_coeff;
        ga.grad_scale = a.grad_scale;
        launch_grad(ga, s);
    }
}

}  // namespace pl

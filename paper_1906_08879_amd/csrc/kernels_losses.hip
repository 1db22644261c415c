// Losses on rows of logits (include/placeto.h): log probabilities of actions, the clipped policy loss
// and the preference loss, with the gradient of the logits.
//
// For a row z with maximum m:  s = sum_j e^{z_j - m},  t = sum_j e^{z_j - m} (z_j - m)  give
//     l = log pi(a) = (z_a - m) - log s,      H = log s - t / s,
// and with w c = d loss / d l and -w g = d loss / d H the gradient of logit j is
//     w [ c (1[j = a] - p_j) + g p_j (log p_j + H) ] = e^{z_j - m} (A + B (z_j - m)) + C 1[j = a],
//     C = w c,  B = w g / s,  A = (-w c + w g (H - log s)) / s.
// z - m is taken before it is scaled, so rows of a type's lowest value, and rows far from zero, lose nothing.
#include <algorithm>
#include <cmath>

#include "elements.h"
#include "losses.h"

namespace pl {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLowest = -200.0f;     // e^-200 is 0 in fp32: z - m below it stands for -infinity, whose product with 0 is NaN

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// ---- maximum and sums of a row
struct Sums {
    float m = -INFINITY, s = 0.0f, t = 0.0f;
};

// The sums of both parts, relative to the larger maximum.  A part without a probability (s = 0) says nothing.
__device__ __forceinline__ Sums merge(const Sums &a, const Sums &b)
{
    if (a.s == 0.0f) return b;
    if (b.s == 0.0f) return a;
    Sums r;
    r.m = fmaxf(a.m, b.m);
    const float da = fmaxf(a.m - r.m, kLowest), db = fmaxf(b.m - r.m, kLowest);
    const float ea = exp_of(a.m - r.m), eb = exp_of(b.m - r.m);
    r.s = a.s * ea + b.s * eb;
    r.t = ea * (a.t + da * a.s) + eb * (b.t + db * b.s);
    return r;
}

template <int N>
__device__ __forceinline__ void add(Sums &a, const float (&f)[N])
{
    float m = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, f[i]);
    if (m == -INFINITY) {                        // nothing but -infinity and NaN so far
#pragma unroll
        for (int i = 0; i < N; ++i) a.s += (f[i] != f[i]) ? f[i] : 0.0f;
        return;
    }
    if (m != a.m) {
        const float d = a.m - m;
        if (a.s != 0.0f) {
            const float e = exp_of(d);
            a.t = e * (a.t + fmaxf(d, kLowest) * a.s);
            a.s *= e;
        }
        a.m = m;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = f[i] - m, e = exp_of(d);
        a.s += e;
        a.t += e * fmaxf(d, kLowest);
    }
}

__device__ __forceinline__ Sums wave_merge(Sums a)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        Sums b;
        b.m = __shfl_xor(a.m, o);
        b.s = __shfl_xor(a.s, o);
        b.t = __shfl_xor(a.t, o);
        a = merge(a, b);
    }
    return a;
}

__device__ __forceinline__ Sums merged_parts(const RowPart *parts, int slices)
{
    Sums a{parts[0].m, parts[0].s, parts[0].t};
    for (int i = 1; i < slices; ++i) a = merge(a, Sums{parts[i].m, parts[i].s, parts[i].t});
    return a;
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
        const int u = static_cast<int>(static_cast<uint32_t>(n) / static_cast<uint32_t>(q)), v = static_cast<int>(n) - u * q;
        p.seq = r.order == PL_ROWS_BY_STEP ? v : u;
        const int step = r.order == PL_ROWS_BY_STEP ? u : v;
        if (r.bounds) p.counts = step < r.bounds[p.seq];
    }
    if (r.mask && p.counts) p.counts = r.mask[n] != 0;
    return p;
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// l and H of a row from its sums; a row without an allowed action has l = NaN, an action of probability zero l = -infinity.
__device__ __forceinline__ void finish_row(const Sums &a, float z_a, bool action_ok, float &l, float &H, float &log_s)
{
    log_s = logf(a.s);
    H = log_s - a.t / a.s;
    l = action_ok ? (z_a - a.m) - log_s : NAN;
    if (a.s == 0.0f) H = l = NAN;
}

// ---- one slice of a row per workgroup: its maximum and sums
template <typename T>
__global__ __launch_bounds__(256) void k_row_parts(LogitsView x, RowsView rows, RowPart *__restrict__ parts, int slices)
{
    const int64_t n = blockIdx.x;
    const int tid = threadIdx.x;
    __shared__ RowPart wave[4];
    if (!place_of(rows, n).counts) return;
    const Row<T> row(x.data, x.stride, n, x.V);
    const int per = (row.slots + slices - 1) / slices;
    const int end = min(row.slots, per * (static_cast<int>(blockIdx.y) + 1));
    Sums a;
    for (int i = per * blockIdx.y + tid; i < end; i += 256) {
        float f[Elem<T>::N];
        row.load(i, f, -INFINITY);
        add(a, f);
    }
    a = wave_merge(a);
    if ((tid & 63) == 0) wave[tid >> 6] = {a.m, a.s, a.t};
    __syncthreads();
    if (tid == 0) {
        a = merged_parts(wave, 4);
        parts[n * slices + blockIdx.y] = {a.m, a.s, a.t};
    }
}

template <typename T>
__device__ __forceinline__ float logit(const LogitsView &x, int64_t n, int a)
{
    return Elem<T>::load(static_cast<const T *>(x.data) + n * x.stride + a);
}

// ---- one row per thread: log probabilities, and what the gradient of a preference needs
template <typename T>
__global__ __launch_bounds__(kRowsPerBlock) void k_finish_logp(LogitsView x, RowsView rows, const int32_t *__restrict__ actions,
                                                               const RowPart *__restrict__ parts, int slices,
                                                               float *__restrict__ out_logp, float *__restrict__ out_entropy,
                                                               float *__restrict__ logp, RowGrad *__restrict__ grad)
{
    const int64_t n = static_cast<int64_t>(blockIdx.x) * kRowsPerBlock + threadIdx.x;
    if (n >= x.n) return;
    float l = 0.0f, H = 0.0f;
    RowGrad g{0.0f, 0.0f, 0.0f, 0.0f};
    if (place_of(rows, n).counts) {
        const Sums a = merged_parts(parts + n * slices, slices);
        const int act = actions[n];
        const bool ok = act >= 0 && act < x.V;
        float log_s;
        finish_row(a, ok ? logit<T>(x, n, act) : 0.0f, ok, l, H, log_s);
        g.m = a.m;
        g.A = (ok && l != -INFINITY) ? 1.0f / a.s : 0.0f;   // 0: the row adds nothing
        if (a.s == 0.0f) g.A = 0.0f;
    }
    if (out_logp) out_logp[n] = l;
    if (logp) logp[n] = l;
    if (out_entropy) out_entropy[n] = H;
    if (grad) grad[n] = g;
}

// Weight of a row that counts.
__device__ __forceinline__ float row_weight(const RowsView &rows, int reduction, const RowTotals *totals, const int32_t *seq_n,
                                            int seq)
{
    if (reduction == PL_REDUCE_SUM) return 1.0f;
    if (reduction == PL_REDUCE_ROWS) return 1.0f / static_cast<float>(rows.all ? static_cast<int32_t>(rows.n) : totals->rows);
    if (rows.all) return static_cast<float>(1.0 / (static_cast<double>(rows.S) * rows.L));
    return static_cast<float>(1.0 / (static_cast<double>(totals->seqs) * seq_n[seq]));
}

struct PolicyRow {
    float c = 0.0f, g = 0.0f;          // - d loss / d l, - d loss / d H, without the gradient's scale
    float sur = 0.0f, kl = 0.0f, H = 0.0f, cut = 0.0f;
};

// Value and derivatives of a row that counts and adds something.
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs &a, int64_t n, int seq, float l, float H, float w)
{
    PolicyRow r;
    const float adv = a.advantages[a.advantage_per_seq ? seq : n];
    const float ratio = a.old_logp ? expf(l - a.old_logp[n]) : (l == l ? 1.0f : l);
    const bool cut = adv > 0.0f ? ratio > 1.0f + a.clip_high : (adv < 0.0f && ratio < 1.0f - a.clip_low);
    const float held = cut ? (adv > 0.0f ? 1.0f + a.clip_high : 1.0f - a.clip_low) : ratio;
    r.sur = w * (-adv * held);
    r.c = cut ? 0.0f : adv * ratio;
    if (a.ref_logp) {
        const float d = a.ref_logp[n] - l, e = expm1f(d);
        r.kl = w * (e - d);
        r.c += a.kl_coeff * e;
    }
    r.c *= w;
    r.g = w * a.entropy_coeff;
    r.H = w * H;
    r.cut = cut ? w : 0.0f;
    return r;
}

__device__ __forceinline__ RowGrad grad_of(const PolicyRow &r, const PolicyArgs &a, const Sums &sums, float H, float log_s)
{
    const float c = -r.c * a.grad_scale, g = r.g * a.grad_scale;
    return {sums.m, (-c + g * (H - log_s)) / sums.s, g / sums.s, c};
}

template <typename T>
__global__ __launch_bounds__(kRowsPerBlock) void k_finish_policy(LogitsView x, RowsView rows, PolicyArgs args,
                                                                 const RowPart *__restrict__ parts, int slices,
                                                                 const RowTotals *__restrict__ totals,
                                                                 const int32_t *__restrict__ seq_n, RowGrad *__restrict__ grad,
                                                                 double *__restrict__ sums)
{
    const int64_t n = static_cast<int64_t>(blockIdx.x) * kRowsPerBlock + threadIdx.x;
    const int tid = threadIdx.x;
    __shared__ double wave[4][4];
    PolicyRow r;
    if (n < x.n) {
        float l = 0.0f, H = 0.0f;
        RowGrad g{0.0f, 0.0f, 0.0f, 0.0f};
        const Place p = place_of(rows, n);
        if (p.counts) {
            const Sums a = merged_parts(parts + n * slices, slices);
            const int act = args.actions[n];
            const bool ok = act >= 0 && act < x.V;
            float log_s;
            finish_row(a, ok ? logit<T>(x, n, act) : 0.0f, ok, l, H, log_s);
            if (ok && l != -INFINITY && a.s != 0.0f) {
                r = policy_row(args, n, p.seq, l, H, row_weight(rows, args.reduction, totals, seq_n, p.seq));
                g = grad_of(r, args, a, H, log_s);
            }
        }
        if (grad) grad[n] = g;
        if (args.out_logp) args.out_logp[n] = l;
        if (args.out_entropy) args.out_entropy[n] = H;
        if (args.out_coeff) args.out_coeff[n] = r.c * args.grad_scale;
        if (args.out_entropy_coeff) args.out_entropy_coeff[n] = r.g * args.grad_scale;
    }
    const double v[4] = {wave_sum(r.sur), wave_sum(r.kl), wave_sum(r.H), wave_sum(r.cut)};
    if ((tid & 63) == 0)
        for (int i = 0; i < 4; ++i) wave[tid >> 6][i] = v[i];
    __syncthreads();
    if (tid < 4) sums[static_cast<size_t>(blockIdx.x) * 4 + tid] = wave[0][tid] + wave[1][tid] + wave[2][tid] + wave[3][tid];
}

// ---- the loss from the workgroups' sums, in their order
__global__ __launch_bounds__(256) void k_policy_stats(const double *__restrict__ sums, int blocks, float kl_coeff,
                                                      float entropy_coeff, float *__restrict__ out)
{
    __shared__ double wave[4][4];
    const int tid = threadIdx.x;
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    for (int b = tid; b < blocks; b += 256)
        for (int i = 0; i < 4; ++i) v[i] += sums[static_cast<size_t>(b) * 4 + i];
    for (int i = 0; i < 4; ++i) {
        v[i] = wave_sum(v[i]);
        if ((tid & 63) == 0) wave[tid >> 6][i] = v[i];
    }
    __syncthreads();
    if (tid == 0) {
        for (int i = 0; i < 4; ++i) v[i] = wave[0][i] + wave[1][i] + wave[2][i] + wave[3][i];
        out[0] = static_cast<float>(v[0] + kl_coeff * v[1] - entropy_coeff * v[2]);
        for (int i = 0; i < 4; ++i) out[1 + i] = static_cast<float>(v[i]);
    }
}

// ---- the gradient of the logits, an element at a time
template <typename T>
__global__ __launch_bounds__(256) void k_row_grad(LogitsView x, const int32_t *__restrict__ actions,
                                                  const RowGrad *__restrict__ grad, T *out, int64_t out_stride)
{
    constexpr int N = Elem<T>::N;
    const int64_t n = blockIdx.x;
    const RowGrad g = grad[n];
    const Row<T> row(x.data, x.stride, n, x.V);
    T *o = out + n * out_stride;
    const bool aligned = (reinterpret_cast<uintptr_t>(o) & 15) == (reinterpret_cast<uintptr_t>(row.p) & 15);
    const bool none = g.A == 0.0f && g.B == 0.0f && g.C == 0.0f;
    const int act = none ? -1 : actions[n];
    for (int i = blockIdx.y * 256 + threadIdx.x; i < row.slots; i += gridDim.y * 256) {
        float f[N];
        const int e = row.first(i);
        if (none) {
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = 0.0f;
        } else {
            row.load(i, f, -INFINITY);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float d = f[k] - g.m;
                f[k] = exp_of(d) * (g.B == 0.0f ? g.A : g.A + g.B * fmaxf(d, kLowest)) + (e + k == act ? g.C : 0.0f);
            }
        }
        store_slot(o, aligned, e, x.V, f);
    }
}

// ---- sequences: sums of l and l - ref over the rows that count, and their number (with logp == nullptr: the
// number only), of part blockIdx.y of every sequence.  64 / lanes_s rows of a sequence side by side in a wave.
__global__ __launch_bounds__(256) void k_seq_sums(RowsView rows, const float *__restrict__ logp, const float *__restrict__ ref,
                                                  const RowGrad *__restrict__ grad, int lanes_s, double *__restrict__ part,
                                                  int32_t *__restrict__ part_n)
{
    __shared__ double sum[256][2];
    __shared__ int32_t cnt[256];
    const int tid = threadIdx.x, ls = tid % lanes_s, ms = tid / lanes_s, rows_abreast = 256 / lanes_s;
    const int q = blockIdx.x * lanes_s + ls;
    double a = 0.0, b = 0.0;
    int c = 0;
    if (q < rows.S) {
        int64_t first, step = 1, len;
        if (rows.order == PL_ROWS_PACKED) {
            first = max(0, rows.bounds[q]);
            len = max(int64_t{0}, min(rows.n, static_cast<int64_t>(rows.bounds[q + 1])) - first);
        } else {
            len = rows.bounds ? min(rows.L, max(0, rows.bounds[q])) : rows.L;
            first = rows.order == PL_ROWS_BY_STEP ? q : static_cast<int64_t>(q) * rows.L;
            if (rows.order == PL_ROWS_BY_STEP) step = rows.S;
        }
        const int64_t per = (len + gridDim.y - 1) / gridDim.y, end = min(len, per * (blockIdx.y + 1));
        for (int64_t i = per * blockIdx.y + ms; i < end; i += rows_abreast) {
            const int64_t n = first + i * step;
            if (rows.mask && !rows.mask[n]) continue;
            ++c;
            if (!logp) continue;
            const float l = logp[n];
            if (grad && grad[n].A == 0.0f) continue;     // (a NaN from NaN logits is not 0)
            a += l;
            b += ref ? static_cast<double>(l) - ref[n] : l;
        }
    }
    sum[tid][0] = a;
    sum[tid][1] = b;
    cnt[tid] = c;
    __syncthreads();
    if (tid < lanes_s && q < rows.S) {
        for (int i = 1; i < rows_abreast; ++i) {
            a += sum[i * lanes_s + tid][0];
            b += sum[i * lanes_s + tid][1];
            c += cnt[i * lanes_s + tid];
        }
        const size_t at = static_cast<size_t>(blockIdx.y) * rows.S + q;
        if (part) {
            part[at * 2] = a;
            part[at * 2 + 1] = b;
        }
        part_n[at] = c;
    }
}

// Sums of the parts of every sequence, and over all sequences (one workgroup).
__global__ __launch_bounds__(1024) void k_seq_totals(int S, int seq_parts, const double *__restrict__ part,
                                                     const int32_t *__restrict__ part_n, double *__restrict__ seq_sum,
                                                     int32_t *__restrict__ seq_n, RowTotals *__restrict__ totals)
{
    __shared__ int32_t wave[16][2];
    const int tid = threadIdx.x;
    int rows = 0, seqs = 0;
    for (int q = tid; q < S; q += 1024) {
        double a = 0.0, b = 0.0;
        int c = 0;
        for (int i = 0; i < seq_parts; ++i) {
            const size_t at = static_cast<size_t>(i) * S + q;
            if (part) {
                a += part[at * 2];
                b += part[at * 2 + 1];
            }
            c += part_n[at];
        }
        if (part) {
            seq_sum[q * 2] = a;
            seq_sum[q * 2 + 1] = b;
        }
        seq_n[q] = c;
        rows += c;
        seqs += c > 0;
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
    if (tid == 0) {
        for (int i = 1; i < 16; ++i) {
            rows += wave[i][0];
            seqs += wave[i][1];
        }
        *totals = {rows, seqs};
    }
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

// A thread per sequence; every workgroup goes over all pairs, 256 at a time through LDS, and adds those of its sequences in
// the pairs' order.  The first workgroup adds up the loss.
__global__ __launch_bounds__(256) void k_pairs(PrefArgs p, int S, const double *__restrict__ seq_sum,
                                               const int32_t *__restrict__ seq_n, float *__restrict__ seq_coeff,
                                               float *__restrict__ out_stats)
{
    __shared__ int sa[256], sb[256];
    __shared__ float sg[256];
    __shared__ double wave[4][3];
    const int tid = threadIdx.x, q = blockIdx.x * 256 + tid;
    double loss = 0.0, right = 0.0, valid = 0.0, coeff = 0.0;
    for (int i0 = 0; i0 < p.n_pairs; i0 += 256) {
        const int i = i0 + tid;
        Pair pr{-1, -1, false};
        float m = NAN, g = 0.0f;
        if (i < p.n_pairs) {
            pr = pair_at(p, S, i);
            if (pr.ok) {
                m = static_cast<float>(p.beta * (seq_ratio(p, seq_sum, seq_n, pr.a, 1) - seq_ratio(p, seq_sum, seq_n, pr.b, 1)));
                g = d_margin(m, p.smoothing);
                loss += (1.0f - p.smoothing) * softplus(-m) + p.smoothing * softplus(m);
                right += m > 0.0f;
                valid += 1.0;
            }
            if (blockIdx.x == 0 && p.out_margins) p.out_margins[i] = m;
        }
        __syncthreads();
        sa[tid] = pr.ok ? pr.a : -1;
        sb[tid] = pr.ok ? pr.b : -1;
        sg[tid] = g;
        __syncthreads();
        const int n = min(256, p.n_pairs - i0);
        for (int k = 0; k < n; ++k) {
            if (sa[k] == q) coeff += sg[k];
            if (sb[k] == q) coeff -= sg[k];
        }
    }
    loss = wave_sum(loss);
    right = wave_sum(right);
    valid = wave_sum(valid);
    if ((tid & 63) == 0) {
        wave[tid >> 6][0] = loss;
        wave[tid >> 6][1] = right;
        wave[tid >> 6][2] = valid;
    }
    __syncthreads();
    valid = wave[0][2] + wave[1][2] + wave[2][2] + wave[3][2];
    const double per = valid > 0.0 ? 1.0 / valid : 0.0;
    if (blockIdx.x == 0 && tid == 0) {
        out_stats[0] = static_cast<float>((wave[0][0] + wave[1][0] + wave[2][0] + wave[3][0]) * per);
        out_stats[1] = static_cast<float>((wave[0][1] + wave[1][1] + wave[2][1] + wave[3][1]) * per);
    }
    if (q < S) {
        coeff *= per * p.beta;
        if (p.average && seq_n[q] > 0) coeff /= seq_n[q];
        seq_coeff[q] = static_cast<float>(coeff);
        if (p.out_seq_logp) p.out_seq_logp[q] = static_cast<float>(seq_ratio(p, seq_sum, seq_n, q, 0));
    }
}

// Every row takes its sequence's d loss / d l.
__global__ __launch_bounds__(kRowsPerBlock) void k_pref_rows(RowsView rows, PrefArgs p, const float *__restrict__ seq_coeff,
                                                             RowGrad *__restrict__ grad)
{
    const int64_t n = static_cast<int64_t>(blockIdx.x) * kRowsPerBlock + threadIdx.x;
    if (n >= rows.n) return;
    RowGrad g = grad[n];
    const Place at = place_of(rows, n);
    float c = 0.0f;
    if (at.counts && g.A != 0.0f) c = p.grad_scale * seq_coeff[at.seq];
    g.A = c == 0.0f ? 0.0f : -c * g.A;
    g.C = c;
    grad[n] = g;
    if (p.out_coeff) p.out_coeff[n] = -c;
}

int row_blocks(int64_t n) { return static_cast<int>((n + kRowsPerBlock - 1) / kRowsPerBlock); }

void launch_parts(const LogitsView &x, const RowsView &rows, const LossWorkspace &ws, hipStream_t s)
{
    by_type(x.dtype, [&](auto t) {
        hipLaunchKernelGGL(k_row_parts<decltype(t)>, dim3(static_cast<uint32_t>(x.n), ws.slices), dim3(256), 0, s, x, rows, ws.parts,
                           ws.slices);
    });
}

void launch_grad(const LogitsView &x, const int32_t *actions, const LossWorkspace &ws, void *out, int64_t out_stride, hipStream_t s)
{
    by_type(x.dtype, [&](auto t) {
        using T = decltype(t);
        const int slots = x.V / Elem<T>::N + 2, per_block = 256 * 4;
        hipLaunchKernelGGL(k_row_grad<T>, dim3(static_cast<uint32_t>(x.n), std::min((slots + per_block - 1) / per_block, 1024)),
                           dim3(256), 0, s, x, actions, ws.grad, static_cast<T *>(out), out_stride);
    });
}

void launch_seq_sums(const RowsView &rows, const float *logp, const float *ref, const LossWorkspace &ws, hipStream_t s)
{
    // neighbouring rows of PL_ROWS_BY_STEP are of neighbouring sequences, of the other orders of one
    int lanes_s = 1;
    if (rows.order == PL_ROWS_BY_STEP)
        while (lanes_s < 64 && lanes_s < rows.S) lanes_s *= 2;
    hipLaunchKernelGGL(k_seq_sums, dim3((rows.S + lanes_s - 1) / lanes_s, ws.seq_parts), dim3(256), 0, s, rows, logp, ref,
                       logp ? ws.grad : nullptr, lanes_s, logp ? ws.seq_part : nullptr, ws.seq_part_n);
    hipLaunchKernelGGL(k_seq_totals, dim3(1), dim3(1024), 0, s, rows.S, ws.seq_parts, logp ? ws.seq_part : nullptr, ws.seq_part_n,
                       ws.seq_sum, ws.seq_n, ws.totals);
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
    if (x.n > 0)
        w.slices = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({1024 / x.n, x.V / 8192, kMaxSlices})));
    const int64_t longest = rows.order == PL_ROWS_PACKED ? rows.n : rows.L;
    w.seq_parts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(longest / 2048, kMaxSeqParts)));
    take(w.parts, n * w.slices);
    take(w.grad, n);
    take(w.logp, n);
    take(w.seq_part, S * w.seq_parts * 2);
    take(w.seq_part_n, S * w.seq_parts);
    take(w.seq_sum, S * 2);
    take(w.seq_n, S);
    take(w.seq_coeff, S);
    take(w.totals, 1);
    take(w.sums, static_cast<size_t>(row_blocks(x.n)) * 4);
    w.bytes = pos;
    return w;
}

void launch_action_logp(const LogitsView &x, const int32_t *actions, float *out_logp, float *out_entropy,
                        const LossWorkspace &ws, hipStream_t s)
{
    RowsView rows;
    rows.n = x.n;
    rows.L = static_cast<int>(x.n);
    launch_parts(x, rows, ws, s);
    by_type(x.dtype, [&](auto t) {
        hipLaunchKernelGGL(k_finish_logp<decltype(t)>, dim3(row_blocks(x.n)), dim3(kRowsPerBlock), 0, s, x, rows, actions, ws.parts,
                           ws.slices, out_logp, out_entropy, nullptr, nullptr);
    });
}

void launch_policy_loss(const LogitsView &x, const RowsView &rows, const PolicyArgs &a, float *out_stats, void *out_grad,
                        int64_t grad_stride, const LossWorkspace &ws, hipStream_t s)
{
    if (x.n > 0) {
        if (!rows.all && a.reduction != PL_REDUCE_SUM)
            launch_seq_sums(rows, nullptr, nullptr, ws, s);
        launch_parts(x, rows, ws, s);
        by_type(x.dtype, [&](auto t) {
            hipLaunchKernelGGL(k_finish_policy<decltype(t)>, dim3(row_blocks(x.n)), dim3(kRowsPerBlock), 0, s, x, rows, a, ws.parts,
                               ws.slices, ws.totals, ws.seq_n, out_grad ? ws.grad : nullptr, ws.sums);
        });
    }
    hipLaunchKernelGGL(k_policy_stats, dim3(1), dim3(256), 0, s, ws.sums, row_blocks(x.n), a.ref_logp ? a.kl_coeff : 0.0f,
                       a.entropy_coeff, out_stats);
    if (x.n > 0 && out_grad) launch_grad(x, a.actions, ws, out_grad, grad_stride, s);
}

void launch_preference_loss(const LogitsView &x, const RowsView &rows, const PrefArgs &a, float *out_stats, void *out_grad,
                            int64_t grad_stride, const LossWorkspace &ws, hipStream_t s)
{
    if (x.n > 0) {
        launch_parts(x, rows, ws, s);
        by_type(x.dtype, [&](auto t) {
            hipLaunchKernelGGL(k_finish_logp<decltype(t)>, dim3(row_blocks(x.n)), dim3(kRowsPerBlock), 0, s, x, rows, a.actions,
                               ws.parts, ws.slices, a.out_logp, nullptr, ws.logp, ws.grad);
        });
    }
    launch_seq_sums(rows, ws.logp, a.ref_logp, ws, s);
    hipLaunchKernelGGL(k_pairs, dim3((rows.S + 255) / 256), dim3(256), 0, s, a, rows.S, ws.seq_sum, ws.seq_n, ws.seq_coeff, out_stats);
    if (x.n > 0 && (out_grad || a.out_coeff)) {
        hipLaunchKernelGGL(k_pref_rows, dim3(row_blocks(x.n)), dim3(kRowsPerBlock), 0, s, rows, a, ws.seq_coeff, ws.grad);
        if (out_grad) launch_grad(x, a.actions, ws, out_grad, grad_stride, s);
    }
}

}  // namespace pl

// C ABI of the losses on rows of logits and of gradient clipping (include/placeto.h): checks of the arguments, views and
// workspaces.
#include <algorithm>
#include <cmath>

#include "losses.h"

namespace pl {
namespace {

size_t element_size(int dtype) { return dtype == PL_F32 ? 4 : 2; }
bool dtype_ok(int dtype) { return dtype == PL_F32 || dtype == PL_BF16 || dtype == PL_F16; }
bool aligned_to(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

int view_logits(const pl_logits *in, LogitsView *x)
{
    if (!in) return fail(PL_ERR_NULL, "logits is NULL");
    if (!dtype_ok(in->dtype)) return fail(PL_ERR_SHAPE, "unknown type of logits");
    if (in->n_actions < 1 || in->n_actions > kMaxActions) return fail(PL_ERR_SHAPE, "n_actions must be 1 .. 2^24");
    if (in->n_rows < 0 || in->n_rows > std::numeric_limits<int32_t>::max()) return fail(PL_ERR_SHAPE, "n_rows must be 0 .. 2^31 - 1");
    if (in->row_stride < in->n_actions || in->row_stride > (int64_t{1} << 31))
        return fail(PL_ERR_SHAPE, "row_stride must be n_actions .. 2^31");
    x->data = in->data;
    x->n = in->n_rows;
    x->stride = in->row_stride;
    x->V = in->n_actions;
    x->dtype = in->dtype;
    return PL_OK;
}

int view_rows(const pl_rows *in, const LogitsView &x, RowsView *r)
{
    static const pl_rows one_sequence{1, PL_ROWS_BY_SEQ, nullptr, nullptr};
    *r = RowsView{};
    r->n = x.n;
    if (!in) in = &one_sequence;
    if (in->order < PL_ROWS_BY_SEQ || in->order > PL_ROWS_PACKED) return fail(PL_ERR_SHAPE, "unknown order of rows");
    if (in->n_seqs < 1 || in->n_seqs > (1 << 23)) return fail(PL_ERR_SHAPE, "n_seqs must be 1 .. 2^23");
    r->S = in->n_seqs;
    r->order = in->order;
    if (in->order == PL_ROWS_PACKED) {
        if (!in->bounds) return fail(PL_ERR_NULL, "packed rows need the offsets of their sequences");
    } else {
        if (x.n % in->n_seqs) return fail(PL_ERR_SHAPE, "n_rows must be a multiple of n_seqs");
        r->L = static_cast<int>(x.n / in->n_seqs);
    }
    // division by a constant: with 2^(b-1) < q <= 2^b, n / q = n * ceil(2^(31+b) / q) / 2^(31+b) for every n < 2^31
    const uint32_t q = in->order == PL_ROWS_BY_STEP ? static_cast<uint32_t>(r->S) : static_cast<uint32_t>(r->L);
    if (q > 1) {
        int b = 1;
        while ((uint64_t{1} << b) < q) ++b;
        r->magic = static_cast<uint32_t>(((uint64_t{1} << (31 + b)) + q - 1) / q);
        r->shift = b - 1;
    }
    r->bounds = in->bounds;
    r->mask = in->mask;
    r->all = !in->bounds && !in->mask;
    return PL_OK;
}

int check_call(const LogitsView &x, const RowsView &rows, const int32_t *actions, const void *out_grad, int64_t grad_stride,
               void *workspace, size_t workspace_bytes, LossWorkspace *ws)
{
    if (x.n > 0 && (!x.data || !actions)) return fail(PL_ERR_NULL, "logits and actions are required");
    const size_t e = element_size(x.dtype);
    if (!aligned_to(x.data, e) || !aligned_to(out_grad, e)) return fail(PL_ERR_SHAPE, "logits and out_grad must be aligned to their elements");
    if (out_grad && (grad_stride < x.V || grad_stride > (int64_t{1} << 31))) return fail(PL_ERR_SHAPE, "grad_stride must be n_actions .. 2^31");
    if (out_grad == x.data && out_grad && grad_stride != x.stride) return fail(PL_ERR_SHAPE, "in place, grad_stride must be row_stride");
    if (!workspace) return fail(PL_ERR_NULL, "workspace is NULL");
    if (!aligned_to(workspace, 16)) return fail(PL_ERR_SHAPE, "workspace must be aligned to 16 bytes");
    *ws = carve_loss_workspace(workspace, x, rows);
    if (ws->bytes > workspace_bytes) return fail(PL_ERR_SHAPE, "workspace holds fewer bytes than pl_loss_workspace names");
    return PL_OK;
}

// ---- learning from another policy
int check_temperature(double t)
{
    if (!(t >= 0x1p-20 && t <= 0x1p20)) return fail(PL_ERR_SHAPE, "temperature must be 2^-20 .. 2^20");
    return PL_OK;
}

int check_top(int32_t n_top, int32_t most)
{
    if (n_top < 1 || n_top > PL_MAX_TOP || n_top > most) return fail(PL_ERR_SHAPE, "n_top must be 1 .. 128, and at most n_actions where actions are looked for");
    return PL_OK;
}

uint32_t narrow_magic(int V) { return V > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / V + 1) : 0; }
constexpr double kLog2e = 1.4426950408889634;

}  // namespace
}  // namespace pl

using namespace pl;

extern "C" {

size_t pl_loss_workspace(const pl_logits *logits, const pl_rows *rows, int32_t n_pairs)
{
    LogitsView x;
    RowsView r;
    if (n_pairs < 0 || view_logits(logits, &x)) return 0;
    // (offsets need not be there yet)
    pl_rows sized{};
    const int32_t none = 0;
    if (rows) {
        sized = *rows;
        if (!sized.bounds) sized.bounds = &none;
    }
    if (view_rows(rows ? &sized : nullptr, x, &r)) return 0;
    return carve_loss_workspace(nullptr, x, r).bytes;
}

int pl_action_logp(const pl_logits *logits, const int32_t *actions, float *out_logp, float *out_entropy,
                   void *workspace, size_t workspace_bytes, void *stream)
{
    LogitsView x;
    RowsView rows;
    LossWorkspace ws;
    if (int rc = view_logits(logits, &x)) return rc;
    if (x.n == 0) return PL_OK;
    if (int rc = view_rows(nullptr, x, &rows)) return rc;
    if (int rc = check_call(x, rows, actions, nullptr, 0, workspace, workspace_bytes, &ws)) return rc;
    if (!out_logp) return fail(PL_ERR_NULL, "out_logp is required");
    launch_action_logp(x, rows, actions, out_logp, out_entropy, ws, static_cast<hipStream_t>(stream));
    PL_HIP(hipGetLastError());
    return PL_OK;
}

int pl_clipped_policy_loss(const pl_logits *logits, const pl_rows *rows_in, const pl_policy_loss_cfg *cfg,
                           const int32_t *actions, const float *advantages, const float *old_logp,
                           const float *ref_logp, float *out_stats, void *out_grad, int64_t grad_stride,
                           float *out_logp, float *out_entropy, float *out_coeff, float *out_entropy_coeff,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    LogitsView x;
    RowsView rows;
    LossWorkspace ws;
    if (int rc = view_logits(logits, &x)) return rc;
    if (int rc = view_rows(rows_in, x, &rows)) return rc;
    if (!cfg) return fail(PL_ERR_NULL, "cfg is NULL");
    if (!(cfg->clip_low >= 0.0f && cfg->clip_low <= 1.0f) || !(cfg->clip_high >= 0.0f))
        return fail(PL_ERR_SHAPE, "clip_low must be 0 .. 1 and clip_high not negative");
    if (!std::isfinite(cfg->kl_coeff) || !std::isfinite(cfg->entropy_coeff) || !std::isfinite(cfg->grad_scale))
        return fail(PL_ERR_SHAPE, "kl_coeff, entropy_coeff and grad_scale must be finite");
    if (cfg->reduction < PL_REDUCE_ROWS || cfg->reduction > PL_REDUCE_SUM) return fail(PL_ERR_SHAPE, "unknown reduction");
    if (cfg->advantage_per_seq != 0 && cfg->advantage_per_seq != 1) return fail(PL_ERR_SHAPE, "advantage_per_seq must be 0 or 1");
    if (int rc = check_call(x, rows, actions, out_grad, grad_stride, workspace, workspace_bytes, &ws)) return rc;
    if (!out_stats || (x.n > 0 && !advantages)) return fail(PL_ERR_NULL, "advantages and out_stats are required");
    const PolicyArgs a{actions, advantages, old_logp, ref_logp, out_logp, out_entropy, out_coeff, out_entropy_coeff,
                       cfg->clip_low, cfg->clip_high, cfg->kl_coeff, cfg->entropy_coeff, cfg->grad_scale,
                       cfg->advantage_per_seq, 1.0f, nullptr, nullptr};
    launch_policy_loss(x, rows, a, cfg->reduction, out_stats, out_grad, grad_stride, ws, static_cast<hipStream_t>(stream));
    PL_HIP(hipGetLastError());
    return PL_OK;
}

int pl_preference_loss(const pl_logits *logits, const pl_rows *rows_in, const pl_preference_cfg *cfg,
                       const int32_t *actions, const float *ref_logp, int32_t n_pairs, const int32_t *pairs,
                       float *out_stats, void *out_grad, int64_t grad_stride, float *out_logp,
                       float *out_seq_logp, float *out_margins, float *out_coeff, void *workspace,
                       size_t workspace_bytes, void *stream)
{
    LogitsView x;
    RowsView rows;
    LossWorkspace ws;
    if (int rc = view_logits(logits, &x)) return rc;
    if (int rc = view_rows(rows_in, x, &rows)) return rc;
    if (!cfg) return fail(PL_ERR_NULL, "cfg is NULL");
    if (!(cfg->beta >= 0.0f) || !std::isfinite(cfg->beta)) return fail(PL_ERR_SHAPE, "beta must be finite and not negative");
    if (!(cfg->label_smoothing >= 0.0f && cfg->label_smoothing <= 1.0f)) return fail(PL_ERR_SHAPE, "label_smoothing must be 0 .. 1");
    if (!std::isfinite(cfg->grad_scale)) return fail(PL_ERR_SHAPE, "grad_scale must be finite");
    if (cfg->average != 0 && cfg->average != 1) return fail(PL_ERR_SHAPE, "average must be 0 or 1");
    if (n_pairs < 0 || n_pairs > (1 << 24)) return fail(PL_ERR_SHAPE, "n_pairs must be 0 .. 2^24");
    if (!pairs && n_pairs > 0 && (rows.S % 2 || n_pairs != rows.S / 2))
        return fail(PL_ERR_SHAPE, "without a list of pairs n_pairs must be n_seqs / 2 (n_seqs even)");
    if (int rc = check_call(x, rows, actions, out_grad, grad_stride, workspace, workspace_bytes, &ws)) return rc;
    if (!out_stats) return fail(PL_ERR_NULL, "out_stats is required");
    const PrefArgs a{actions, ref_logp, out_logp, out_seq_logp, out_margins, out_coeff, pairs,
                     cfg->beta, cfg->label_smoothing, cfg->grad_scale, cfg->average, n_pairs};
    launch_preference_loss(x, rows, a, out_stats, out_grad, grad_stride, ws, static_cast<hipStream_t>(stream));
    PL_HIP(hipGetLastError());
    return PL_OK;
}

size_t pl_top_workspace(const pl_logits *logits, int32_t n_top)
{
    LogitsView x;
    if (view_logits(logits, &x) || check_top(n_top, x.V)) return 0;
    return carve_top_workspace(nullptr, x, n_top).bytes;
}

int pl_top_actions(const pl_logits *logits, double temperature, int32_t n_top, int32_t *out_top, float *out_top_logp,
                   const int32_t *actions, float *out_logp, float *out_entropy, void *workspace, size_t workspace_bytes,
                   void *stream)
{
    LogitsView x;
    if (int rc = view_logits(logits, &x)) return rc;
    if (int rc = check_temperature(temperature)) return rc;
    if (int rc = check_top(n_top, x.V)) return rc;
    if (!actions != !out_logp) return fail(PL_ERR_NULL, "actions and out_logp go together");
    if (x.n == 0) return PL_OK;
    if (!x.data || !out_top) return fail(PL_ERR_NULL, "logits and out_top are required");
    if (!aligned_to(x.data, element_size(x.dtype))) return fail(PL_ERR_SHAPE, "logits must be aligned to their elements");
    if (!workspace) return fail(PL_ERR_NULL, "workspace is NULL");
    if (!aligned_to(workspace, 16)) return fail(PL_ERR_SHAPE, "workspace must be aligned to 16 bytes");
    const TopWorkspace ws = carve_top_workspace(workspace, x, n_top);
    if (ws.bytes > workspace_bytes) return fail(PL_ERR_SHAPE, "workspace holds fewer bytes than pl_top_workspace names");
    TopArgs a{};
    a.x = x;
    a.actions = actions;
    a.out_top = out_top;
    a.out_top_logp = out_top_logp;
    a.out_logp = out_logp;
    a.out_entropy = out_entropy;
    a.top = n_top;
    a.per = static_cast<float>(1.0 / temperature);
    a.per2 = static_cast<float>(kLog2e / temperature);
    a.magic = narrow_magic(x.V);
    launch_top(a, ws, static_cast<hipStream_t>(stream));
    PL_HIP(hipGetLastError());
    return PL_OK;
}

size_t pl_distill_workspace(const pl_logits *logits, const pl_rows *rows, int32_t n_top)
{
    LogitsView x;
    RowsView r;
    if (pl_loss_workspace(logits, rows, 0) == 0 || view_logits(logits, &x) || check_top(n_top, PL_MAX_TOP)) return 0;
    pl_rows sized{};
    const int32_t none = 0;
    if (rows) {
        sized = *rows;
        if (!sized.bounds) sized.bounds = &none;
    }
    if (view_rows(rows ? &sized : nullptr, x, &r)) return 0;
    return carve_distill_workspace(nullptr, x, r, n_top).bytes;
}

int pl_distill_loss(const pl_logits *logits, const pl_rows *rows_in, const pl_distill_cfg *cfg, int32_t n_top, const int32_t *top,
                    const float *top_logp, float *out_stats, void *out_grad, int64_t grad_stride, float *out_values,
                    float *out_coeff, void *workspace, size_t workspace_bytes, void *stream)
{
    LogitsView x;
    RowsView rows;
    LossWorkspace loss;
    if (int rc = view_logits(logits, &x)) return rc;
    if (int rc = view_rows(rows_in, x, &rows)) return rc;
    if (!cfg) return fail(PL_ERR_NULL, "cfg is NULL");
    if (int rc = check_temperature(cfg->temperature)) return rc;
    if (!std::isfinite(cfg->grad_scale)) return fail(PL_ERR_SHAPE, "grad_scale must be finite");
    if (cfg->reduction < PL_REDUCE_ROWS || cfg->reduction > PL_REDUCE_SUM) return fail(PL_ERR_SHAPE, "unknown reduction");
    if (cfg->tail != 0 && cfg->tail != 1) return fail(PL_ERR_SHAPE, "tail must be 0 or 1");
    if (out_coeff && cfg->tail) return fail(PL_ERR_SHAPE, "out_coeff is that of a loss without tail");
    if (int rc = check_top(n_top, PL_MAX_TOP)) return rc;
    if (int rc = check_call(x, rows, top, out_grad, grad_stride, workspace, workspace_bytes, &loss)) return rc;
    if (!out_stats || (x.n > 0 && !top_logp)) return fail(PL_ERR_NULL, "top_logp and out_stats are required");
    const DistillWorkspace ws = carve_distill_workspace(workspace, x, rows, n_top);
    if (ws.bytes > workspace_bytes) return fail(PL_ERR_SHAPE, "workspace holds fewer bytes than pl_distill_workspace names");
    DistillArgs a{};
    a.x = x;
    a.rows = rows;
    a.top = top;
    a.top_logp = top_logp;
    a.k = n_top;
    a.tail = cfg->tail;
    a.per = 1.0 / cfg->temperature;
    a.per2 = static_cast<float>(kLog2e / cfg->temperature);
    a.grad_scale = cfg->grad_scale;
    // from 2^-40 on, what of a sum is below 2^-126 does not matter, and r / p_rest times the gradients' scale stays in fp32
    if (cfg->tail) a.least = static_cast<float>(std::max(0x1p-40, std::fabs(static_cast<double>(cfg->grad_scale)) / cfg->temperature * 0x1p-124));
    a.out_grad = out_grad;
    a.grad_stride = grad_stride;
    a.out_values = out_values;
    a.out_coeff = out_coeff;
    a.out_stats = out_stats;
    a.magic = narrow_magic(x.V);
    launch_distill(a, cfg->reduction, ws, static_cast<hipStream_t>(stream));
    PL_HIP(hipGetLastError());
    return PL_OK;
}

// Sums of the workgroups, and the list of the tensors where they do not go by value.
size_t pl_clip_gradients_workspace(int32_t n_tensors)
{
    if (n_tensors < 0) return 0;
    const size_t n = static_cast<size_t>(n_tensors), list = n > kClipTensors ? n * sizeof(ClipTensor) + (n + 1) * sizeof(int32_t) : 0;
    return kClipBlocks * sizeof(double) + (list + 15) / 16 * 16;
}

int pl_clip_gradients(int32_t n_tensors, void *const *grads, void *const *clipped, const int64_t *numel,
                      const int32_t *dtype, float max_norm, float *out_norm, void *workspace,
                      size_t workspace_bytes, void *stream)
{
    if (n_tensors < 0) return fail(PL_ERR_SHAPE, "n_tensors must not be negative");
    if (!(max_norm >= 0.0f)) return fail(PL_ERR_SHAPE, "max_norm must not be negative");
    if (!out_norm || !workspace || (n_tensors > 0 && (!grads || !numel || !dtype)))
        return fail(PL_ERR_NULL, "grads, numel, dtype, out_norm and workspace are required");
    if (!aligned_to(workspace, 16)) return fail(PL_ERR_SHAPE, "workspace must be aligned to 16 bytes");
    if (workspace_bytes < pl_clip_gradients_workspace(n_tensors))
        return fail(PL_ERR_SHAPE, "workspace holds fewer bytes than pl_clip_gradients_workspace names");
    bool scales = max_norm < INFINITY;           // whether anything is written but the norm
    int64_t total = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
        if (numel[i] < 0 || numel[i] > (int64_t{1} << 40) || total > (int64_t{1} << 40))
            return fail(PL_ERR_SHAPE, "numel must not be negative, and all tensors together have at most 2^40 elements");
        if (!dtype_ok(dtype[i])) return fail(PL_ERR_SHAPE, "unknown type of a gradient");
        total += numel[i];
        if (numel[i] == 0) continue;
        const size_t e = element_size(dtype[i]);
        if (!grads[i] || (clipped && !clipped[i])) return fail(PL_ERR_NULL, "a gradient or its result is NULL");
        if (!aligned_to(grads[i], e) || (clipped && !aligned_to(clipped[i], e)))
            return fail(PL_ERR_SHAPE, "gradients must be aligned to their elements");
        scales = scales || (clipped && clipped[i] != grads[i]);
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    double *sums = static_cast<double *>(workspace);
    // chunks of eight slots to a thread, as long as there are fewer of them than workgroups; a workgroup that does all alone
    // takes a tensor at a time
    const bool small = n_tensors <= 4 && total <= kClipSmall;
    const int chunk = static_cast<int>(small ? kClipSmall : std::min<int64_t>(kClipChunk, std::max<int64_t>(2048, total / kClipBlocks / 2048 * 2048)));
    // tables of the tensors, without the empty ones
    int32_t next = 0;
    int64_t chunks = 0;
    auto table = [&]() {
        ClipTable t;
        t.n = 0;
        t.chunk = chunk;
        t.first[0] = static_cast<int32_t>(chunks);
        for (; next < n_tensors && t.n < kClipTensors; ++next) {
            if (numel[next] == 0) continue;
            t.src[t.n] = grads[next];
            t.dst[t.n] = clipped ? clipped[next] : grads[next];
            t.numel[t.n] = numel[next];
            t.dtype[t.n] = static_cast<uint8_t>(dtype[next]);
            chunks += (numel[next] + chunk - 1) / chunk;
            t.first[++t.n] = static_cast<int32_t>(chunks);
        }
        return t;
    };
    ClipTable t = table();
    if (next == n_tensors) {
        if (small) launch_clip_small(t, max_norm, out_norm, s);
        else launch_clip(t, chunks, sums, max_norm, scales, out_norm, s);
    } else {
        ClipList list;
        list.tensors = reinterpret_cast<ClipTensor *>(sums + kClipBlocks);
        list.first = reinterpret_cast<int32_t *>(list.tensors + n_tensors);
        list.n = 0;
        list.chunk = chunk;
        for (;; t = table()) {
            launch_clip_list(t, list, list.n, s);
            list.n += t.n;
            if (next == n_tensors) break;
        }
        list.chunks = static_cast<int32_t>(chunks);
        launch_clip(list, chunks, sums, max_norm, scales, out_norm, s);
    }
    PL_HIP(hipGetLastError());
    return PL_OK;
}

}  // extern "C"

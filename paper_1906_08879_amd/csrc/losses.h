// Internal declarations of the losses on rows of logits and of gradient clipping (include/placeto.h):
// what their entry points hand to the kernels.
#pragma once
#include <cstddef>
#include <cstdint>

#include "internal.h"

namespace pl {

constexpr int kMaxActions = 1 << 24;
constexpr int kNarrow = 16;            // actions of rows that a thread takes
constexpr int kMaxSlices = 64;         // parts that a row is cut into where there are few rows
constexpr int kRowsPerBlock = 256;     // rows of a workgroup of the per-row kernels
constexpr int kMiddleRows = 32768;     // rows, and sequences, whose sums and pairs one workgroup does
constexpr int kPairSeqs = 64;
constexpr int kMiddleSeqs = 1024;      // sequences whose rows one workgroup counts
constexpr int kMaxSumBlocks = 2048;    // workgroups of the kernels that go over several rows
constexpr int kMaxSeqParts = 128;      // parts that the rows of a sequence are cut into

struct LogitsView {
    const void *data = nullptr;
    int64_t n = 0, stride = 0;
    int V = 1, dtype = PL_F32;
};

// Which sequence a row belongs to, and whether it counts (pl_rows).
struct RowsView {
    const int32_t *bounds = nullptr;
    const uint8_t *mask = nullptr;
    int64_t n = 0;
    int S = 1, L = 0, order = PL_ROWS_BY_SEQ;
    uint32_t magic = 0;                // n / (S or L) = high word of n * magic, shifted right (for n < 2^31; 0: that is 1 or none)
    int shift = 0;
    bool all = true;                   // every row counts, known on the host
};

// Maximum m and sums over a slice of a row: of 2^x and of 2^x x, x = (z - m) log2 e.
struct RowPart {
    float m, s, t;
};

// The gradient of a row: 2^x (A + B x) + C [j = a], x = (z_j - m) log2 e; all three zero: zeros.  Between the passes of a
// preference, A is 1 / s (0: the row adds nothing).
struct RowGrad {
    float m, A, B, C;
};

struct PolicyArgs {
    const int32_t *actions;
    const float *advantages, *old_logp, *ref_logp;
    float *out_logp, *out_entropy, *out_coeff, *out_entropy_coeff;
    float clip_low, clip_high, kl_coeff, entropy_coeff, grad_scale;
    int advantage_per_seq;
    float weight;                      // of a row, unless
    const float *weights;              // there is one for each sequence, or
    const float *weight_at;            // it is found on the device
};

struct PrefArgs {
    const int32_t *actions;
    const float *ref_logp;
    float *out_logp, *out_seq_logp, *out_margins, *out_coeff;
    const int32_t *pairs;
    float beta, smoothing, grad_scale;
    int average, n_pairs;
};

// One call's workspace, carved by carve_loss_workspace.
struct LossWorkspace {
    RowPart *parts = nullptr;          // [n, slices]
    RowGrad *grad = nullptr;           // [n]
    double *logp = nullptr;            // [n]
    double *seq_part = nullptr;        // [parts of a sequence, S, 2] sums of l, of l - ref
    int32_t *seq_part_n = nullptr;     // [parts of a sequence, S] rows that count
    double *seq_sum = nullptr;         // [S, 2]
    int32_t *seq_n = nullptr;          // [S]
    float *seq_coeff = nullptr;        // [S]
    float *weights = nullptr;          // [S], for PL_REDUCE_SEQS
    float *weight = nullptr;           // [1], for PL_REDUCE_ROWS
    double *sums = nullptr;            // [workgroups, 4]
    int slices = 1, seq_parts = 1;
    size_t bytes = 0;
};

LossWorkspace carve_loss_workspace(void *base, const LogitsView &x, const RowsView &rows);

// Weight of every row by a reduction: a number known on the host, or (counted on the device) one of all rows or one for each sequence.
struct RowWeights {
    float weight = 1.0f;
    const float *weights = nullptr, *weight_at = nullptr;
};

// csrc/kernels_losses.hip
RowWeights launch_row_weights(const LogitsView &x, const RowsView &rows, int reduction, const LossWorkspace &ws, hipStream_t s);
void launch_action_logp(const LogitsView &x, const RowsView &rows, const int32_t *actions, float *out_logp, float *out_entropy,
                        const LossWorkspace &ws, hipStream_t s);
void launch_policy_loss(const LogitsView &x, const RowsView &rows, const PolicyArgs &a, int reduction, float *out_stats,
                        void *out_grad, int64_t grad_stride, const LossWorkspace &ws, hipStream_t s);
void launch_preference_loss(const LogitsView &x, const RowsView &rows, const PrefArgs &a, float *out_stats, void *out_grad,
                            int64_t grad_stride, const LossWorkspace &ws, hipStream_t s);

// ---- learning from another policy (csrc/kernels_top.hip, csrc/kernels_distill.hip)
constexpr int kLaneRow = 128;          // actions of the widest rows that a lane takes
constexpr int kTopKept = 2048;         // candidates of a workgroup's row, and of a round that joins the slices of one

struct TopArgs {
    LogitsView x;
    const int32_t *actions;
    int32_t *out_top;
    float *out_top_logp, *out_logp, *out_entropy;
    int top;
    float per, per2;                   // 1 / T, log2 e / T
    uint32_t magic;                    // of the rows' width, for narrow rows
    RowPart *parts;                    // [n, slices], and
    uint64_t *lists;                   // [n, slices, top]: rows in slices
    int slices;
};

struct TopWorkspace {
    RowPart *parts = nullptr;
    uint64_t *lists = nullptr;
    int slices = 1;
    size_t bytes = 0;
};
TopWorkspace carve_top_workspace(void *base, const LogitsView &x, int top);
void launch_top(TopArgs a, const TopWorkspace &ws, hipStream_t s);

// A part of a row: its largest logit; of its actions outside the list the sum s of e^{(z - base) / T}, and the number of those at the lowest
// value that are not in it.
struct DistillPart {
    float m, base, s, lowest;
};

struct DistillArgs {
    LogitsView x;
    RowsView rows;
    RowWeights w;
    const int32_t *top;
    const float *top_logp;
    int k, tail;
    double per;                        // 1 / T
    float per2, grad_scale;
    float least;                       // sums over the unlisted actions below it are taken again relative to their own maximum; 0 without tail
    void *out_grad;
    int64_t grad_stride;
    float *out_values, *out_coeff;
    double *sums;                      // [workgroups, 4]
    float *out_stats;
    uint32_t magic;
    DistillPart *parts;                // [n, slices], rows in slices
    int slices;
    RowGrad *row_grad;                 // [n] (B: whether actions at the lowest value are masked), and what the gradients at the listed actions are
    int32_t *at;                       // [n, k] action, or -1
    float *inside;                     // [n, k]
};

struct DistillWorkspace {
    LossWorkspace loss;
    DistillPart *parts = nullptr;
    int32_t *at = nullptr;
    float *inside = nullptr;
    double *sums = nullptr;            // [workgroups, 4]
    size_t bytes = 0;
};
DistillWorkspace carve_distill_workspace(void *base, const LogitsView &x, const RowsView &rows, int k);
void launch_distill(DistillArgs a, int reduction, const DistillWorkspace &ws, hipStream_t s);

// csrc/kernels_clip.hip: the tensors of a call in chunks.  Up to kClipTensors of them go to the kernels by value (a kernel's
// arguments end at 4 KiB), more through a list in the workspace that is written from such tables.
constexpr int kClipTensors = 128;
constexpr int kClipBlocks = 1024;      // workgroups, and partial sums, at most
constexpr int kClipChunk = 16384;      // elements of a chunk, at most
// Elements of a call (of four tensors at most) that one workgroup does alone.  A call, one launch against two: 32768 floats 8.1 us
// against 10.9 (kernels 6.5 and 5.9), in three tensors 9.8 against 12.2 (9.2 and 6.0); 131072 floats 16.4 against 10.9.
constexpr int64_t kClipSmall = 32768;

struct ClipTensor {
    const void *src;
    void *dst;
    int64_t numel;
    int64_t dtype;
};
struct ClipTable {
    const void *src[kClipTensors];
    void *dst[kClipTensors];
    int64_t numel[kClipTensors];
    int32_t first[kClipTensors + 1];   // chunks in front of each tensor
    uint8_t dtype[kClipTensors];
    int32_t n, chunk;                  // tensors; elements of a chunk
};
struct ClipList {
    ClipTensor *tensors;
    int32_t *first;                    // [n + 1]
    int32_t n, chunk, chunks;
};

// The tensors of a table, from number `at` of the list on; the last call's table ends the list.
void launch_clip_list(const ClipTable &t, const ClipList &list, int at, hipStream_t s);
template <typename Tensors>            // ClipTable or ClipList
void launch_clip(const Tensors &t, int64_t chunks, double *sums, float max_norm, bool scales, float *out_norm, hipStream_t s);
void launch_clip_small(const ClipTable &t, float max_norm, float *out_norm, hipStream_t s);

}  // namespace pl

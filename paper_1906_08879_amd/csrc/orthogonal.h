// Internal declarations of the orthogonalised update (include/placeto.h): what its entry point hands to the kernels.
#pragma once
#include <cstddef>
#include <cstdint>

#include "internal.h"

namespace pl {

constexpr int kOrthBlock = 32;         // elements of a row whose two halves lie side by side
constexpr int kOrthLayout = 64;        // rows and columns of a workgroup's part where matrices are laid out
constexpr int kOrthMaxSteps = 32;
constexpr int kOrthMaxParts = 512;     // workgroups that share a matrix's norm
constexpr int kOrthListed = 12;        // matrices that one launch writes to the list

// A matrix as the kernels see it.  k is its shorter side, n its longer one; x lies as k rows of n, xt as n rows of k, in two halves:
// row r, column c at r * 2 * pad + (c / 32) * 64 + c % 32, the remainders 32 further, zeros from the last column to pad.
struct OrthMatrix {
    const void *grad, *weight;
    const float *momentum;
    float *new_momentum;
    void *new_weight, *out;
    int64_t grad_stride, momentum_stride, new_momentum_stride, weight_stride, new_weight_stride, out_stride;
    _Float16 *x, *xt[2], *a, *b;
    double *sums;                      // [sum_parts] of squares
    float *parts;                      // [tiles of X X', n_parts, a tile], where its long axis is shared by workgroups
    int32_t rows, cols, k, n, k_pad, n_pad;
    int32_t grad_dtype, weight_dtype, out_dtype;
    int32_t sum_parts;
    int32_t n_parts, part_blocks;      // blocks of 32 of the long axis that a workgroup sums
    int32_t first_sum, first_layout, first_join, first[3];     // workgroups of the matrices in front of it; the last ones: X X', A A, B X
    float scale;
    int32_t tall;                      // rows > cols: x is the transposed matrix
    int32_t run;                       // matrices of the same sides right in front of it in the list
};

struct OrthTable {
    OrthMatrix m[kOrthListed];
    int32_t n;
};

struct OrthCfg {
    float lr_decay, lr, beta, eps;     // lr_decay: 1 - lr decay
    int32_t nesterov;
};

// One iteration on scaled operands (sx X, sa A, sb B with powers of two): sa A = gram (sx X) (sx X)',
// sb B = unit I + linear (sa A) + square (sa A) (sa A), and the next X in its own scale = next (sb B) (sx X).
struct OrthStep {
    float gram, unit, linear, square, next;
};

// The tiles of a product over all matrices, and their kind.  A block of 32 takes a workgroup the longer the fewer are at work beside it:
// `alone`, or `full` where the matrix cores (and the card's power) are shared by all.  Larger tiles read less and multiply faster, smaller
// ones spread further.  Five iterations with all products in tiles of 64, and what other tiles add to the Gram matrices, us: 512 x 512 185
// and 47, 96, 191 (128, 192, 256); 32 of them 820 and -61, -54, 33; 2048 x 2048 twice 1553 and -23, 5, 236; 1024 x 1024 ten times 1197 and
// -55, -46, 79.  Over 34 such sets the choice by these figures was within 4% of the best one.
struct OrthKind {
    int32_t tile, at_once;               // rows and columns; workgroups that the card has room for
    double alone, full;                  // us
};
constexpr OrthKind kOrthKinds[] = {{64, 512, 0.38, 0.7}, {128, 512, 0.9, 1.37}, {192, 256, 1.3, 1.35}, {256, 256, 1.7, 2.35}};

constexpr int kOrthSplitTile = kOrthKinds[0].tile;   // tiles whose sums may be shared: the long axis of X X'

struct OrthWork {
    int64_t tiles;
    int32_t kind, part_blocks;           // (blocks of a workgroup's sum, at most)
};

struct OrthGrid {
    int32_t n_matrices;
    int64_t sums, layouts, joins;        // workgroups
    int32_t last_k, last_n, last_run;    // of the matrix placed last
    OrthWork work[3];
};

// Matrices of few rows (kernels_orthogonal_small.hip).  Up to 16 x 4096, 32 x 2048 or 64 x 1024, or the other way round, a workgroup does
// alone; longer ones of up to 32 rows are cut into parts.
constexpr int kOrthSmall = 65536;
constexpr int kOrthThin = 32;          // rows of matrices whose iteration goes over X X' alone, in float64
inline int orth_small_k(int k) { return k <= 16 ? 16 : k <= 32 ? 32 : 64; }
inline int orth_small_n(int n) { return n <= 128 ? 128 : n <= 512 ? 512 : 1024; }      // (of more than 32 rows)
inline bool orth_small(int k, int n) { return k <= 64 && n <= kOrthSmall / orth_small_k(k); }
inline bool orth_long(int k, int n) { return k <= kOrthThin && !orth_small(k, n); }
constexpr int kOrthSmallListed = 24;   // matrices that go to a launch by value (a kernel's arguments end at 4 KiB); more through a list

struct OrthSmall {
    const void *grad, *weight;
    const float *momentum;
    float *new_momentum;
    void *new_weight, *out;
    void *room;                        // orth_room() bytes
    uint32_t grad_stride, momentum_stride, new_momentum_stride, weight_stride, new_weight_stride, out_stride;
    int32_t rows, cols;
    int32_t first;                     // of long ones: parts of the matrices in front of it
    uint8_t grad_dtype, weight_dtype, out_dtype;
    float scale;
};

struct OrthSmallTable {
    OrthSmall m[kOrthSmallListed];
    OrthStep step[kOrthMaxSteps];
    float iteration[kOrthMaxSteps][3];
    OrthCfg cfg;
    float x_scale, per_last;           // of the first step's X; 1 over that of the result
    int32_t n, n_steps;
};
static_assert(sizeof(OrthSmallTable) <= 4000, "passed by value");

// Columns (of the longer side) of a part of a long matrix, 256 of them at most, and how many parts it has.
__host__ __device__ inline int orth_part(int n) { return n <= 256 * 1024 ? 1024 : ((n + 255) / 256 + 63) / 64 * 64; }
inline int orth_parts(int n) { return (n + orth_part(n) - 1) / orth_part(n); }

// Bytes of a matrix: of X by columns (more than 32 rows), or of the parts' X X' and the result's factor.
inline size_t orth_room(int rows, int cols)
{
    const int k = rows < cols ? rows : cols, n = rows < cols ? cols : rows, kb = k <= 16 ? 1 : 2;
    if (k > kOrthThin) return static_cast<size_t>(64) * orth_small_n(n) * sizeof(float);
    if (orth_small(k, n)) return 0;
    return (static_cast<size_t>(orth_parts(n)) * (kb * (kb + 1) / 2) + kb * kb) * 256 * sizeof(double);
}

// The table's matrices to list[at ..]; `count` matrices by value or from a list: a workgroup each, or long ones of `parts` parts together.
void launch_orth_small_list(const OrthSmallTable &t, OrthSmall *list, int at, hipStream_t s);
void launch_orth_small(const OrthSmallTable &t, const OrthSmall *list, int count, hipStream_t s);
void launch_orth_long(const OrthSmallTable &t, const OrthSmall *list, int count, int parts, hipStream_t s);
void launch_orth_list(const OrthTable &t, OrthMatrix *list, int at, hipStream_t s);
void launch_orth_start(const OrthMatrix *list, const OrthGrid &grid, const OrthCfg &cfg, float x_scale, hipStream_t s);
void launch_orth_step(const OrthMatrix *list, const OrthGrid &grid, const OrthCfg &cfg, const OrthStep &step, int number, bool last,
                      hipStream_t s);

}  // namespace pl

// C ABI of the orthogonalised update of matrices (include/placeto.h): checks of the arguments, the iteration's ranges and the
// workspace.
#include <algorithm>
#include <cmath>
#include <iterator>

#include "orthogonal.h"

namespace pl {
namespace {

size_t element_size(int dtype) { return dtype == PL_F32 ? 4 : 2; }
bool dtype_ok(int dtype) { return dtype == PL_F32 || dtype == PL_BF16 || dtype == PL_F16; }
bool aligned_to(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

constexpr int32_t kMaxMatrices = 1 << 16;
constexpr int32_t kMaxSide = 1 << 21;
constexpr int64_t kMaxStride = int64_t{1} << 31;

int check_size(const pl_matrix &m)
{
    if (m.rows < 1 || m.cols < 1 || m.rows > kMaxSide || m.cols > kMaxSide ||
        static_cast<int64_t>(m.rows) * m.cols > std::numeric_limits<int32_t>::max())
        return fail(PL_ERR_SHAPE, "a matrix must have 1 .. 2^21 rows and columns and less than 2^31 elements");
    return PL_OK;
}

int check_matrix(const pl_matrix &m)
{
    if (int rc = check_size(m)) return rc;
    if (!dtype_ok(m.grad_dtype) || (m.weight && !dtype_ok(m.weight_dtype)) || (m.out && !dtype_ok(m.out_dtype)))
        return fail(PL_ERR_SHAPE, "unknown type of a matrix");
    if (!m.grad) return fail(PL_ERR_NULL, "grad is required");
    if (!m.out && !m.new_weight) return fail(PL_ERR_NULL, "a matrix has neither out nor new_weight");
    if (!m.weight != !m.new_weight) return fail(PL_ERR_NULL, "weight and new_weight go together");
    if (m.new_momentum && !m.momentum) return fail(PL_ERR_NULL, "new_momentum needs momentum");
    if (!std::isfinite(m.scale)) return fail(PL_ERR_SHAPE, "scale must be finite");
    const struct { const void *p; int64_t stride; size_t size; } views[] = {
        {m.grad, m.grad_stride, element_size(m.grad_dtype)}, {m.momentum, m.momentum_stride, 4},
        {m.new_momentum, m.new_momentum_stride, 4}, {m.weight, m.weight_stride, element_size(m.weight_dtype)},
        {m.new_weight, m.new_weight_stride, element_size(m.weight_dtype)}, {m.out, m.out_stride, element_size(m.out_dtype)}};
    for (const auto &v : views) {
        if (!v.p) continue;
        if (v.stride < m.cols || v.stride > kMaxStride) return fail(PL_ERR_SHAPE, "row strides must be cols .. 2^31");
        if (!aligned_to(v.p, v.size)) return fail(PL_ERR_SHAPE, "matrices must be aligned to their elements");
    }
    if (m.momentum == m.new_momentum && m.momentum && m.momentum_stride != m.new_momentum_stride)
        return fail(PL_ERR_SHAPE, "in place, new_momentum_stride must be momentum_stride");
    if (m.weight == m.new_weight && m.weight && m.weight_stride != m.new_weight_stride)
        return fail(PL_ERR_SHAPE, "in place, new_weight_stride must be weight_stride");
    return PL_OK;
}

// The largest |a s + b s^3 + c s^5| over [0, m], and the largest |a + b t + c t^2| over [0, m^2].
void largest_values(double a, double b, double c, double m, double *of_x, double *of_b)
{
    const auto p = [&](double t) { return std::fabs(std::sqrt(t) * (a + t * (b + t * c))); };
    const auto q = [&](double t) { return std::fabs(a + t * (b + t * c)); };
    const double end = m * m;
    *of_x = p(end);
    *of_b = std::max(q(0.0), q(end));
    const auto at = [&](double t, const auto &f, double *most) {
        if (t > 0.0 && t < end) *most = std::max(*most, f(t));
    };
    if (c != 0.0) {
        at(-b / (2.0 * c), q, of_b);
        const double root = 9.0 * b * b - 20.0 * a * c;
        if (root >= 0.0) {
            at((-3.0 * b + std::sqrt(root)) / (10.0 * c), p, of_x);
            at((-3.0 * b - std::sqrt(root)) / (10.0 * c), p, of_x);
        }
    } else if (b != 0.0) {
        at(-a / (3.0 * b), p, of_x);
    }
}

// The power of two that takes values up to `most` to 2^13 .. 2^14 (1 where there are none).
float scale_of(double most)
{
    if (most == 0.0) return 1.0f;
    int e;
    std::frexp(most, &e);
    return static_cast<float>(std::ldexp(1.0, 14 - e));
}

// Every iteration's factors and scales.
int plan_steps(const pl_orthogonal_cfg &cfg, OrthStep *steps, float *x_scale, float *last_scale)
{
    constexpr double kLeast = 1.0 / (1 << 20), kMost = 1 << 20;
    double m = 1.0;
    for (int i = 0; i < cfg.n_steps; ++i) {
        const float *f = cfg.iteration + 3 * i;
        if (!std::isfinite(f[0]) || !std::isfinite(f[1]) || !std::isfinite(f[2])) return fail(PL_ERR_SHAPE, "factors of the iteration must be finite");
        double next, b;
        largest_values(f[0], f[1], f[2], m, &next, &b);
        if (!(next <= kMost) || !(b <= kMost) || next < kLeast || b < kLeast)
            return fail(PL_ERR_SHAPE, "the iteration must keep the largest singular value, and its own terms, in 2^-20 .. 2^20");
        const float sx = scale_of(m), sa = scale_of(m * m), sb = scale_of(b), to = scale_of(next);
        if (i == 0) *x_scale = sx;
        *last_scale = to;
        steps[i] = {sa / (sx * sx), f[0] * sb, f[1] * (sb / sa), f[2] * (sb / (sa * sa)), to / (sb * sx)};
        m = next;
    }
    return PL_OK;
}

struct Carver {
    char *base;
    size_t pos = 0;
    template <typename T>
    T *take(size_t count)
    {
        T *p = base ? reinterpret_cast<T *>(base + pos) : nullptr;
        pos += (count * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

int padded(int n) { return (n + kOrthBlock - 1) / kOrthBlock * kOrthBlock; }
int tiles(int n, int of) { return (n + of - 1) / of; }

// Tiles of a matrix in X X', A A (those on one side of the diagonal) and B X.
int64_t product_tiles(int k, int n, int product, int tile)
{
    const int64_t across = tiles(k, tile);
    return product < 2 ? across * (across + 1) / 2 : across * tiles(n, tile);
}

// A matrix' room in the workspace and its share of the launches.
OrthMatrix place_matrix(const pl_matrix &m, Carver *c, OrthGrid *g)
{
    OrthMatrix o{};
    o.rows = m.rows;
    o.cols = m.cols;
    o.tall = m.rows > m.cols;
    o.k = std::min(m.rows, m.cols);
    o.n = std::max(m.rows, m.cols);
    o.k_pad = padded(o.k);
    o.n_pad = padded(o.n);
    if (o.k == g->last_k && o.n == g->last_n) ++g->last_run;
    else g->last_run = 0;
    g->last_k = o.k;
    g->last_n = o.n;
    o.run = g->last_run;
    o.sum_parts = static_cast<int32_t>(std::min<int64_t>(kOrthMaxParts, (static_cast<int64_t>(m.rows) * m.cols + 8191) / 8192));
    const size_t k = o.k, n = o.n;
    o.x = c->take<_Float16>(k * 2 * o.n_pad);
    for (auto &xt : o.xt) xt = c->take<_Float16>(n * 2 * o.k_pad);
    o.a = c->take<_Float16>(k * 2 * o.k_pad);
    o.b = c->take<_Float16>(k * 2 * o.k_pad);
    o.sums = c->take<double>(o.sum_parts);
    o.first_sum = static_cast<int32_t>(g->sums);
    o.first_layout = static_cast<int32_t>(g->layouts);
    g->sums += o.sum_parts;
    g->layouts += static_cast<int64_t>(tiles(m.rows, kOrthLayout)) * tiles(m.cols, kOrthLayout);
    for (int p = 0; p < 3; ++p) {
        OrthWork &w = g->work[p];
        o.first[p] = static_cast<int32_t>(w.tiles);
        const int64_t of_it = product_tiles(o.k, o.n, p, kOrthKinds[w.kind].tile);
        if (p == 0) {
            o.part_blocks = w.part_blocks;
            o.n_parts = tiles(o.n_pad / kOrthBlock, w.part_blocks);
            o.first_join = static_cast<int32_t>(g->joins);
            if (o.n_parts > 1) {
                o.parts = c->take<float>(of_it * o.n_parts * kOrthSplitTile * kOrthSplitTile);
                g->joins += of_it;
            }
            w.tiles += of_it * o.n_parts;
        } else {
            w.tiles += of_it;
        }
    }
    return o;
}

int shorter(const pl_matrix &m) { return std::min(m.rows, m.cols); }
int longer(const pl_matrix &m) { return std::max(m.rows, m.cols); }

enum Class { SMALL, LONG, LARGE };     // a workgroup each; of few rows, in parts; in tiles

Class class_of(const pl_matrix &m)
{
    return orth_small(shorter(m), longer(m)) ? SMALL : orth_long(shorter(m), longer(m)) ? LONG : LARGE;
}

int32_t count_of(int32_t n_matrices, const pl_matrix *matrices, Class what)
{
    return static_cast<int32_t>(std::count_if(matrices, matrices + n_matrices, [&](const pl_matrix &m) { return class_of(m) == what; }));
}

// The large matrices, those with the longest sums first (workgroups begin in that order): f(matrix).
template <typename F>
void each_large(int32_t n_matrices, const pl_matrix *matrices, F f)
{
    for (int bit = 31; bit >= 0; --bit)
        for (int32_t i = 0; i < n_matrices; ++i)
            if (class_of(matrices[i]) == LARGE && longer(matrices[i]) >> bit == 1) f(matrices[i]);
}

constexpr int64_t kMostWorkgroups = 1 << 22;     // (of 512 threads, 2^32 together at most)

bool fits(const OrthGrid &g)
{
    const int64_t most = kMostWorkgroups;
    return g.sums <= most && g.layouts <= most && g.work[0].tiles <= most && g.work[2].tiles <= most;
}

// Which tiles a product takes, and how many blocks of X X' a workgroup sums where the long axis is shared: those whose workgroups are
// expected to be done first.
void choose_work(int32_t n_matrices, const pl_matrix *matrices, int product, OrthWork *best)
{
    constexpr int kWhole = 1 << 30;
    constexpr double kBegin = 12.0, kJoin = 6.0; // blocks that beginning and end of a tile take as long as; us
    double least = INFINITY;
    const auto consider = [&](int kind, int part_blocks) {
        const OrthKind &t = kOrthKinds[kind];
        double count = 0.0, work = 0.0, longest = 0.0;
        for (int32_t i = 0; i < n_matrices; ++i) {
            if (class_of(matrices[i]) != LARGE) continue;
            const int k = shorter(matrices[i]), n = longer(matrices[i]);
            const int blocks = tiles(product == 0 ? n : k, kOrthBlock), parts = tiles(blocks, part_blocks);
            const double depth = std::min(blocks, part_blocks) + kBegin, of_it = static_cast<double>(product_tiles(k, n, product, t.tile)) * parts;
            count += of_it;
            work += of_it * depth;
            longest = std::max(longest, depth);
        }
        const double later = std::ceil(count / t.at_once) - 1.0;             // rounds, which begin with the longest sums
        const double time = std::max(work / t.at_once * t.full, t.alone * (longest + later * work / count)) + (part_blocks < kWhole ? kJoin : 0.0);
        if (time < least) {
            least = time;
            best->kind = kind;
            best->part_blocks = part_blocks;
        }
    };
    for (int kind = 0; kind < static_cast<int>(std::size(kOrthKinds)); ++kind) consider(kind, kWhole);
    if (product == 0)
        for (int blocks = 8; blocks <= 64; blocks += blocks < 16 ? 4 : blocks < 32 ? 8 : 16) consider(0, blocks);
}

// The room and the launches of the large matrices; false: too many of them.
bool plan_large(int32_t n_matrices, const pl_matrix *matrices, Carver *c, OrthGrid *g, OrthMatrix **list)
{
    for (int p = 0; p < 3; ++p) choose_work(n_matrices, matrices, p, &g->work[p]);
    *list = c->take<OrthMatrix>(std::max(1, n_matrices));
    bool fit = true;
    each_large(n_matrices, matrices, [&](const pl_matrix &m) {
        if (!fit) return;
        place_matrix(m, c, g);
        ++g->n_matrices;
        fit = fits(*g);
    });
    return fit;
}

}  // namespace
}  // namespace pl

using namespace pl;

extern "C" {

size_t pl_orthogonal_workspace(int32_t n_matrices, const pl_matrix *matrices)
{
    if (n_matrices < 0 || n_matrices > kMaxMatrices || (n_matrices > 0 && !matrices)) return 0;
    Carver c{nullptr};
    OrthGrid g{};
    OrthMatrix *list;
    int64_t parts = 0;
    for (int32_t i = 0; i < n_matrices; ++i) {
        if (check_size(matrices[i])) return 0;
        const Class what = class_of(matrices[i]);
        if (what != LARGE) c.take<char>(orth_room(matrices[i].rows, matrices[i].cols));
        if (what == LONG) parts += orth_parts(longer(matrices[i]));
    }
    if (parts > kMostWorkgroups) return 0;
    for (const Class what : {SMALL, LONG}) {
        const int32_t n = count_of(n_matrices, matrices, what);
        if (n > kOrthSmallListed) c.take<OrthSmall>(n);
    }
    return plan_large(n_matrices, matrices, &c, &g, &list) ? c.pos : 0;
}

int pl_orthogonal_update(int32_t n_matrices, const pl_matrix *matrices, const pl_orthogonal_cfg *cfg, void *workspace,
                         size_t workspace_bytes, void *stream)
{
    if (n_matrices < 0 || n_matrices > kMaxMatrices) return fail(PL_ERR_SHAPE, "n_matrices must be 0 .. 2^16");
    if (!cfg || (n_matrices > 0 && !matrices)) return fail(PL_ERR_NULL, "matrices and cfg are required");
    if (cfg->n_steps < 1 || cfg->n_steps > kOrthMaxSteps) return fail(PL_ERR_SHAPE, "n_steps must be 1 .. 32");
    if (!cfg->iteration) return fail(PL_ERR_NULL, "iteration is NULL");
    if (!std::isfinite(cfg->lr) || !std::isfinite(cfg->decay) || !std::isfinite(cfg->beta)) return fail(PL_ERR_SHAPE, "lr, decay and beta must be finite");
    if (!(cfg->eps >= 0.0f) || !std::isfinite(cfg->eps)) return fail(PL_ERR_SHAPE, "eps must be finite and not negative");
    if (cfg->nesterov != 0 && cfg->nesterov != 1) return fail(PL_ERR_SHAPE, "nesterov must be 0 or 1");
    OrthStep steps[kOrthMaxSteps];
    float x_scale, last_scale;
    if (int rc = plan_steps(*cfg, steps, &x_scale, &last_scale)) return rc;
    for (int32_t i = 0; i < n_matrices; ++i)
        if (int rc = check_matrix(matrices[i])) return rc;
    if (n_matrices == 0) return PL_OK;
    if (!workspace) return fail(PL_ERR_NULL, "workspace is NULL");
    if (!aligned_to(workspace, 16)) return fail(PL_ERR_SHAPE, "workspace must be aligned to 16 bytes");
    const size_t need = pl_orthogonal_workspace(n_matrices, matrices);
    if (need == 0) return fail(PL_ERR_SHAPE, "too many matrices for one call");
    if (workspace_bytes < need) return fail(PL_ERR_SHAPE, "workspace holds fewer bytes than pl_orthogonal_workspace names");

    const hipStream_t s = static_cast<hipStream_t>(stream);
    const OrthCfg c{static_cast<float>(1.0 - static_cast<double>(cfg->lr) * cfg->decay), cfg->lr, cfg->beta, cfg->eps, cfg->nesterov};
    // those of few rows
    OrthSmallTable small;
    std::copy(steps, steps + cfg->n_steps, small.step);
    std::copy(cfg->iteration, cfg->iteration + 3 * cfg->n_steps, &small.iteration[0][0]);
    small.cfg = c;
    small.x_scale = x_scale;
    small.per_last = 1.0f / last_scale;
    small.n_steps = cfg->n_steps;
    Carver carver{static_cast<char *>(workspace)};
    for (const Class what : {SMALL, LONG}) {
        const int32_t count = count_of(n_matrices, matrices, what);
        if (count == 0) continue;
        OrthSmall *small_list = count > kOrthSmallListed ? carver.take<OrthSmall>(count) : nullptr;
        int32_t listed = 0, parts = 0;
        small.n = 0;
        for (int32_t i = 0; i < n_matrices; ++i) {
            const pl_matrix &m = matrices[i];
            if (class_of(m) != what) continue;
            const auto u32 = [](int64_t v) { return static_cast<uint32_t>(v); };
            const auto u8 = [](int32_t v) { return static_cast<uint8_t>(v); };
            small.m[small.n++] = {m.grad, m.weight, m.momentum, m.new_momentum, m.new_weight, m.out,
                                  carver.take<char>(orth_room(m.rows, m.cols)),
                                  u32(m.grad_stride), u32(m.momentum_stride), u32(m.new_momentum_stride), u32(m.weight_stride),
                                  u32(m.new_weight_stride), u32(m.out_stride), m.rows, m.cols, parts,
                                  u8(m.grad_dtype), u8(m.weight_dtype), u8(m.out_dtype), m.scale};
            if (what == LONG) parts += orth_parts(longer(m));
            if (small_list && (small.n == kOrthSmallListed || listed + small.n == count)) {
                launch_orth_small_list(small, small_list, listed, s);
                listed += small.n;
                small.n = 0;
            }
        }
        if (what == SMALL) launch_orth_small(small, small_list, count, s);
        else launch_orth_long(small, small_list, count, parts, s);
    }
    OrthGrid grid{};
    OrthMatrix *list;
    const Carver from = carver;
    plan_large(n_matrices, matrices, &carver, &grid, &list);
    if (grid.n_matrices == 0) {
        PL_HIP(hipGetLastError());
        return PL_OK;
    }
    steps[cfg->n_steps - 1].next /= last_scale;  // the result itself
    carver = from;
    carver.take<OrthMatrix>(n_matrices);
    OrthGrid at{};                               // as plan_large has placed them
    for (int p = 0; p < 3; ++p) {
        at.work[p].kind = grid.work[p].kind;
        at.work[p].part_blocks = grid.work[p].part_blocks;
    }
    OrthTable table;
    table.n = 0;
    int32_t listed = 0;
    each_large(n_matrices, matrices, [&](const pl_matrix &m) {
        OrthMatrix o = place_matrix(m, &carver, &at);
        o.grad = m.grad;
        o.grad_stride = m.grad_stride;
        o.grad_dtype = m.grad_dtype;
        o.momentum = m.momentum;
        o.momentum_stride = m.momentum_stride;
        o.new_momentum = m.new_momentum;
        o.new_momentum_stride = m.new_momentum_stride;
        o.weight = m.weight;
        o.weight_stride = m.weight_stride;
        o.weight_dtype = m.weight_dtype;
        o.new_weight = m.new_weight;
        o.new_weight_stride = m.new_weight_stride;
        o.out = m.out;
        o.out_stride = m.out_stride;
        o.out_dtype = m.out_dtype;
        o.scale = m.scale;
        table.m[table.n++] = o;
        if (table.n == kOrthListed || listed + table.n == grid.n_matrices) {
            launch_orth_list(table, list, listed, s);
            listed += table.n;
            table.n = 0;
        }
    });
    launch_orth_start(list, grid, c, x_scale, s);
    for (int i = 0; i < cfg->n_steps; ++i) launch_orth_step(list, grid, c, steps[i], i, i + 1 == cfg->n_steps, s);
    PL_HIP(hipGetLastError());
    return PL_OK;
}

}  // extern "C"

"""The losses on rows of logits and gradient clipping against their float64 oracle, through the public calls:
types, widths from one action to a large vocabulary, orders of rows, masks, strides, values at the ends of
the types, streams and graphs.

Bounds.  U = 2^-24.  A row's log probability is a difference z_a - m (exact to U |z_a - m|), minus log s; s has
terms off by a few U (and U times their exponent, which the terms' own size weighs down) and sums of at most
V / 64 terms one behind another.  EPS(V, l) = U (64 + V / 64 + 4 |l|) covers it with the entropy's
sums.  A gradient's element is p_j times a row's factor: off by EPS relative to the factor's parts, plus its rounding
to the logits' type.  Losses are sums of row values in float64, off by EPS relative to the sum of magnitudes."""
import numpy as np
import pytest

from oracle import losses as ol

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_ULP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"fp32": 1e-37, "bf16": 1e-37, "fp16": 2.0 ** -24}


def _t(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def _dev(a, dtype=None):
    import torch
    t = torch.as_tensor(np.ascontiguousarray(a))
    return t.to("cuda:0") if dtype is None else t.to(dtype).to("cuda:0")


def _logits(z, dtype, pad=0, offset=0, fill=float("nan")):
    """z on the device as rows `pad` elements apart, `offset` elements behind an aligned address."""
    import torch
    n, V = z.shape
    buf = torch.full((offset + n * (V + pad),), fill, dtype=_t(dtype), device="cuda:0")
    view = buf[offset:].view(n, V + pad)[:, :V]
    view.copy_(torch.from_numpy(z))
    return view


def _host(t):
    return t.double().cpu().numpy()


def eps(V, l):
    return U * (64.0 + V / 64.0 + 4.0 * np.abs(l))


def check_rows(got, ref, V, what):
    ok = np.where(np.isnan(ref), np.isnan(got), (got == ref) | (np.abs(got - ref) <= eps(V, ref) * np.maximum(1.0, np.abs(ref))))
    assert ok.all(), (what, np.flatnonzero(~ok)[:4], got[~ok][:4], ref[~ok][:4])


def check_grad(got, out, factor, dtype, what):
    """factor [n]: the magnitudes that make up a row's derivatives, with their own uncertainty in EPS."""
    every, ref = out["every"], out["grad"]
    V = ref.shape[1]
    p = np.exp(every)
    size = p * (1.0 + np.abs(np.where(p > 0, every, 0.0)))
    size[np.arange(len(ref)), np.clip(out["actions"], 0, V - 1)] += 1.0
    lmax = np.where(np.isfinite(out["logp"]), np.abs(out["logp"]), 0.0)
    tol = 4.0 * (eps(V, lmax) * factor)[:, None] * size + HALF_ULP[dtype] * np.abs(ref) + TINY[dtype]
    ok = np.where(np.isnan(ref), np.isnan(got), np.abs(got - ref) <= tol)
    assert ok.all(), (what, np.argwhere(~ok)[:4], got[~ok][:4], ref[~ok][:4], tol[~ok][:4])


def _state(rng, n, V, dtype, scale=3.0):
    import torch
    z = torch.from_numpy(rng.normal(0, scale, (n, V))).to(_t(dtype)).double().numpy()
    return z, rng.integers(0, V, n).astype(np.int32)


SHAPES = [(1, 1), (5, 1), (33, 2), (300, 3), (70, 8), (64, 15), (9, 16), (129, 17), (31, 63), (10, 64), (11, 65), (7, 130), (6, 257),
          (5, 1000), (3, 2049), (4, 4096), (3, 4100), (2, 16385), (3, 32768), (1, 50001), (1, 70000), (1, 131072), (1, 140001)]


# --------------------------------------------------------------------------- log probabilities
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,V", SHAPES)
def test_log_probabilities(n, V, dtype):
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(n * 1000003 + V)
    z, a = _state(rng, n, V, dtype)
    a[rng.random(n) < 0.1] = -1 if V % 2 else V
    for pad, offset in ((0, 0), (3, 1)):
        x = _logits(z, dtype, pad, offset)
        logp, ent = (torch.full((n,), -7.0, device="cuda:0") for _ in range(2))
        pl.action_logp(x, _dev(a), logp, ent)
        _, l, H, _ = ol.softmax_rows(z, a)
        check_rows(_host(logp), l, V, (n, V, dtype, pad, "logp"))
        check_rows(_host(ent), H, V, (n, V, dtype, pad, "entropy"))
        alone = torch.empty_like(logp)
        pl.action_logp(x, _dev(a), alone)
        check_rows(_host(alone), l, V, (n, V, dtype, pad, "logp alone"))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [4, 37, 700, 9000, 150001])
def test_values_at_the_ends_of_the_types(V, dtype):
    """Masked actions (-inf, the type's lowest value), rows of nothing else, infinities and NaN, rows far from zero."""
    import torch
    import paper_1906_08879_amd as pl
    low = float(torch.finfo(_t(dtype)).min)
    rng = np.random.default_rng(V)
    z, a = _state(rng, 12, V, dtype)
    a[:] = V // 2
    z[0, 1:] = -np.inf; z[0, a[0]] = 1.0                  # one action is left
    z[1, ::2] = low; z[1, a[1]] = 0.5
    z[2] = low                                            # all equally lowest: uniform
    z[3] = -np.inf                                        # nothing is allowed
    z[4, a[4]] = -np.inf                                  # the action taken is not allowed
    z[5, 0] = np.nan
    z[6, 0] = np.inf
    z[7] = torch.from_numpy(z[7] + 3e4).to(_t(dtype)).double().numpy()   # far from zero
    z[8] = -low                                           # all equally largest: uniform
    z[9, :] = low; z[9, a[9]] = -low
    z[10, 1:] = -np.inf; z[10, 0] = np.nan; z[10, a[10]] = -np.inf
    z[11, V - 1] = np.nan
    x = _logits(z, dtype)
    logp, ent = (torch.empty(12, device="cuda:0") for _ in range(2))
    pl.action_logp(x, _dev(a), logp, ent)
    _, l, H, live = ol.softmax_rows(z, a)
    check_rows(_host(logp), l, V, "logp")
    check_rows(_host(ent), H, V, "entropy")
    # the loss of the rows that have numbers; then one NaN row makes the loss NaN and no other row's gradient
    keep = np.array([1, 1, 1, 1, 1, 0, 0, 1, 1, 1, 0, 0], np.uint8)
    adv = rng.normal(0, 1, 12).astype(np.float32)
    for mask in (keep, np.ones(12, np.uint8)):
        rows = pl.DecisionRows(12, 1, mask=_dev(mask))
        stats, grad = torch.empty(5, device="cuda:0"), torch.full_like(x, 7.0)
        pl.clipped_policy_loss(x, _dev(a), _dev(adv), stats, rows=rows, entropy_coeff=0.1, out_grad=grad)
        out = ol.policy_loss(z, a, adv, rows=ol.rows_of(12, mask=mask), entropy_coeff=0.1)
        check_rows(_host(stats), out["stats"], V, "stats")
        check_grad(_host(grad), dict(out, actions=a), np.abs(adv) + 1.0, dtype, "grad")


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [1, 2, 8, 16, 40, 65, 500, 3000, 12345, 70001, 140001])
def test_certain_actions_and_rows_below_zero(V, dtype):
    """One action as good as certain: log probability and entropy 0 and no gradient, to the last bit.  Logits that are all
    negative, near zero (log probabilities themselves) and far below it."""
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(V)
    z, a = _state(rng, 6, V, dtype)
    z[0] = -300.0; z[0, a[0]] = 37.3
    z[1] = -np.inf; z[1, a[1]] = -41.7
    z[2] -= np.log(np.exp(z[2] - z[2].max()).sum()) + z[2].max() + 1e-3
    z[3] -= 60.0
    z[4] = -1000.0 - np.abs(z[4])
    z[5] = -0.0
    z = torch.from_numpy(z).to(_t(dtype)).double().numpy()
    x = _logits(z, dtype)
    logp, ent, stats = torch.empty(6, device="cuda:0"), torch.empty(6, device="cuda:0"), torch.empty(5, device="cuda:0")
    pl.action_logp(x, _dev(a), logp, ent)
    _, l, H, _ = ol.softmax_rows(z, a)
    check_rows(_host(logp), l, V, "logp")
    check_rows(_host(ent), H, V, "entropy")
    assert (_host(logp)[:2] == 0).all() and (_host(ent)[:2] == 0).all()
    grad, adv = torch.full_like(x, 7.0), np.ones(6, np.float32)
    pl.clipped_policy_loss(x, _dev(a), _dev(adv), stats, entropy_coeff=0.1, out_grad=grad)
    out = ol.policy_loss(z, a, adv, entropy_coeff=0.1)
    check_grad(_host(grad), dict(out, actions=a), adv + 1.0, dtype, "grad")
    assert (_host(grad)[:2] == 0).all()


def test_no_rows_and_masked_rows():
    import torch
    import paper_1906_08879_amd as pl
    x, i32 = torch.empty((0, 5), device="cuda:0"), torch.empty(0, dtype=torch.int32, device="cuda:0")
    f = torch.empty(0, device="cuda:0")
    stats = torch.full((5,), 7.0, device="cuda:0")
    pl.action_logp(x, i32, f)
    pl.clipped_policy_loss(x, i32, f, stats, out_grad=torch.empty_like(x))
    assert (_host(stats) == 0).all()
    two = torch.full((2,), 7.0, device="cuda:0")
    seq = torch.full((4,), 7.0, device="cuda:0")
    off = torch.zeros(5, dtype=torch.int32, device="cuda:0")
    pl.preference_loss(x, i32, pl.DecisionRows(0, 4, "packed", bounds=off), two, out_seq_logp=seq)
    assert np.allclose(_host(two), [np.log(2.0), 0.0]) and (_host(seq) == 0).all()
    pl.preference_loss(x, i32, pl.DecisionRows(0, 4, "packed", bounds=off), two,
                       pairs=torch.empty((0, 2), dtype=torch.int32, device="cuda:0"))
    assert (_host(two) == 0).all()
    for V in (3, 100, 9001):                              # every row masked, what lies in them is not read
        n = 40
        x = torch.full((n, V), float("nan"), device="cuda:0")
        a = torch.full((n,), 1 << 30, dtype=torch.int32, device="cuda:0")
        nan = torch.full((n,), float("nan"), device="cuda:0")
        rows = pl.DecisionRows(n, 4, mask=torch.zeros(n, dtype=torch.bool, device="cuda:0"))
        outs = [torch.full((n,), 7.0, device="cuda:0") for _ in range(4)]
        grad = torch.full_like(x, 7.0)
        for reduction in ("rows", "seqs", "sum"):
            pl.clipped_policy_loss(x, a, nan, stats, rows=rows, old_logp=nan, ref_logp=nan, kl_coeff=1.0, entropy_coeff=1.0,
                                   reduction=reduction, out_grad=grad, out_logp=outs[0], out_entropy=outs[1], out_coeff=outs[2],
                                   out_entropy_coeff=outs[3])
            for t in (stats, grad, *outs):
                assert (_host(t) == 0).all(), (V, reduction)
                t.fill_(7.0)
        pl.preference_loss(x, a, rows, two, ref_logp=nan, out_grad=grad, out_logp=outs[0], out_coeff=outs[1], out_seq_logp=seq)
        assert np.allclose(_host(two), [np.log(2.0), 0.0])
        for t in (grad, *outs[:2], seq):
            assert (_host(t) == 0).all(), V


# --------------------------------------------------------------------------- the clipped policy loss
def _rows(rng, n, S, order, kind):
    """Bounds and mask of a test, on the host."""
    bounds = mask = None
    if order == "packed":
        bounds = np.concatenate([[0], np.sort(rng.integers(0, n + 1, S - 1)), [n - (kind == "mask")]]).astype(np.int32)
        bounds = np.minimum(bounds, bounds[-1])
    elif kind != "all":
        bounds = rng.integers(0, n // S + 1, S).astype(np.int32)
    if kind == "mask":
        mask = (rng.random(n) < 0.7).astype(np.uint8)
    return bounds, mask


def _decision_rows(n, S, order, bounds, mask):
    import paper_1906_08879_amd as pl
    return pl.DecisionRows(n, S, order, bounds=None if bounds is None else _dev(bounds), mask=None if mask is None else _dev(mask))


def _poison(arrays, counts):
    """Entries of rows that do not count hold NaN."""
    for a in arrays:
        a[~counts] = np.nan


def _policy_case(seed, n, V, dtype, S, order, kind, reduction, per_seq=False, ref=True, old=True, ent=0.02, kl=0.1, pad=0, offset=0,
                 inplace=False, grad_scale=1.0):
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(seed)
    bounds, mask = _rows(rng, n, S, order, kind)
    z, a = _state(rng, n, V, dtype, 1.5)
    where = ol.rows_of(n, S, order, bounds, mask)
    l = ol.softmax_rows(z, a)[1]
    shift = rng.normal(0, 0.2, n)                         # (no ratio at the edges, where the gradient jumps)
    for edge in (np.log(0.8), np.log(1.3)):
        shift = np.where(np.abs(shift - edge) < 1e-2, shift + 3e-2, shift)
    old_l = (l - shift).astype(np.float32) if old else None
    ref_l = (l + rng.normal(0, 0.5, n)).astype(np.float32) if ref else None
    adv = rng.normal(0, 1, S if per_seq else n).astype(np.float32)
    z[~where[1]] = np.nan
    a[~where[1]] = 1 << 30
    if V > 1 and n > 20:
        a[np.flatnonzero(where[1])[:1]] = -5              # a row without an action
    _poison([t for t in (old_l, ref_l, None if per_seq else adv) if t is not None], where[1])
    x = _logits(z, dtype, pad, offset)
    kw = dict(clip_low=0.2, clip_high=0.3, kl_coeff=kl if ref else 0.0, entropy_coeff=ent, reduction=reduction, grad_scale=grad_scale)
    ref_out = ol.policy_loss(z, a, adv, rows=where, old=old_l, ref=ref_l, per_seq=per_seq, n_seqs=S, **kw)
    stats = torch.full((5,), 7.0, device="cuda:0")
    outs = {k: torch.full((n,), 7.0, device="cuda:0") for k in ("out_logp", "out_entropy", "out_coeff", "out_entropy_coeff")}
    grad = x if inplace else _logits(np.full((n, V), 7.0), dtype, pad, offset if pad else 0)
    pl.clipped_policy_loss(x, _dev(a), _dev(adv), stats, rows=_decision_rows(n, S, order, bounds, mask),
                           old_logp=None if old_l is None else _dev(old_l), ref_logp=None if ref_l is None else _dev(ref_l),
                           advantage_per_sequence=per_seq, out_grad=grad, **outs, **kw)
    what = (n, V, dtype, S, order, kind, reduction)
    check_rows(_host(outs["out_logp"]), ref_out["logp"], V, (what, "logp"))
    check_rows(_host(outs["out_entropy"]), ref_out["entropy"], V, (what, "entropy"))
    A = np.nan_to_num(np.abs(adv[where[0]] if per_seq else adv))
    e_d = np.exp(np.nan_to_num(np.abs(ref_l - ref_out["logp"]))) if ref else 0.0
    ratio = np.exp(np.nan_to_num(np.abs(old_l - ref_out["logp"]))) if old else 1.0
    size = A * ratio + kl * (1.0 + e_d)
    row_eps = eps(V, np.nan_to_num(ref_out["logp"]))
    w = ref_out["w"] * grad_scale
    assert (np.abs(_host(outs["out_coeff"]) - ref_out["coeff"]) <= 2 * row_eps * w * size + 1e-30).all(), (what, "coeff")
    assert (np.abs(_host(outs["out_entropy_coeff"]) - ref_out["entropy_coeff"]) <= 4 * U * np.abs(ref_out["entropy_coeff"])).all(), what
    tol = (row_eps * ref_out["w"] * (size + 1.0 + np.abs(ref_out["entropy"]))).sum(where=where[1]) * 2 + 1e-30
    assert (np.abs(_host(stats) - ref_out["stats"]) <= tol + U * np.abs(ref_out["stats"])).all(), (what, _host(stats), ref_out["stats"])
    check_grad(_host(grad), dict(ref_out, actions=a), w * (size + ent * (1 + np.abs(np.nan_to_num(ref_out["entropy"])))), dtype, what)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,V", [s for s in SHAPES if s[0] > 0])
def test_policy_loss_over_widths(n, V, dtype):
    _policy_case(n + V, n, V, dtype, 1, "by_seq", "all", "rows", grad_scale=64.0)
    _policy_case(n + V + 1, n, V, dtype, 1, "by_seq", "all", "sum", ref=False, ent=0.0, pad=5, offset=3, inplace=True)


@pytest.mark.parametrize("order", ["by_seq", "by_step", "packed"])
@pytest.mark.parametrize("kind", ["all", "bounds", "mask"])
@pytest.mark.parametrize("reduction", ["rows", "seqs", "sum"])
@pytest.mark.parametrize("n,V,S", [(24, 3, 6), (420, 5, 7), (1000, 2, 200), (60, 70, 4), (36, 5000, 3), (6, 20000, 6), (5000, 4, 1)])
def test_policy_loss_over_orders(order, kind, reduction, n, V, S):
    _policy_case(n + V, n, V, "fp32" if V < 100 else "bf16", S, order, kind, reduction, per_seq=S > 5, old=S != 7, ref=S != 4)


def test_rows_of_many_workgroups():
    """More rows than any launch has threads side by side; long sequences that are counted in parts."""
    _policy_case(5, 300000, 2, "fp32", 3, "by_step", "mask", "seqs")
    _policy_case(6, 70001, 5, "bf16", 1, "by_seq", "mask", "rows")
    _policy_case(7, 50000, 3, "fp32", 25000, "by_seq", "mask", "seqs")
    _policy_case(8, 3000, 300, "bf16", 5, "packed", "mask", "seqs")


# --------------------------------------------------------------------------- the preference loss
def _preference_case(seed, n, V, dtype, S, order, kind, pairs=None, average=False, smoothing=0.0, ref=True, pad=0, inplace=False,
                     beta=0.5):
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(seed)
    bounds, mask = _rows(rng, n, S, order, kind)
    z, a = _state(rng, n, V, dtype, 1.5)
    where = ol.rows_of(n, S, order, bounds, mask)
    l = ol.softmax_rows(z, a)[1]
    ref_l = (l + rng.normal(0, 0.3, n)).astype(np.float32) if ref else None
    z[~where[1]] = np.nan
    a[~where[1]] = -(1 << 30)
    if ref:
        _poison([ref_l], where[1])
    p = None
    if pairs:
        p = rng.integers(0, S, (pairs, 2)).astype(np.int32)
        p[: pairs // 10] = [S, 0]                         # out of range: left out
    x = _logits(z, dtype, pad)
    out = ol.preference_loss(z, a, where, S, pairs=p, ref=ref_l, beta=beta, smoothing=smoothing, average=average, grad_scale=8.0)
    n_pairs = len(out["margins"])
    stats = torch.full((2,), 7.0, device="cuda:0")
    logp, coeff = (torch.full((n,), 7.0, device="cuda:0") for _ in range(2))
    seq_logp, margins = torch.full((S,), 7.0, device="cuda:0"), torch.full((n_pairs,), 7.0, device="cuda:0")
    grad = x if inplace else torch.full_like(x, 7.0)
    pl.preference_loss(x, _dev(a), _decision_rows(n, S, order, bounds, mask), stats, pairs=None if p is None else _dev(p),
                       ref_logp=None if ref_l is None else _dev(ref_l), beta=beta, label_smoothing=smoothing, average=average,
                       grad_scale=8.0, out_grad=grad, out_logp=logp, out_seq_logp=seq_logp, out_margins=margins, out_coeff=coeff)
    what = (n, V, dtype, S, order, kind, pairs, average)
    check_rows(_host(logp), out["logp"], V, (what, "logp"))
    row_eps = eps(V, out["logp"])
    per_row = row_eps * np.maximum(1.0, np.abs(out["logp"]))
    length = np.bincount(where[0][where[1]], minlength=S)
    seq_tol = np.bincount(where[0][where[1]], weights=per_row[where[1]], minlength=S) / np.where(average, np.maximum(length, 1), 1)
    assert (np.abs(_host(seq_logp) - out["seq_logp"]) <= seq_tol + 2 * U * np.abs(out["seq_logp"])).all(), (what, "seq_logp")
    pp = p if p is not None else np.arange(S).reshape(-1, 2)
    good = ((pp >= 0) & (pp < S)).all(1)
    m_tol = np.zeros(n_pairs)
    m_tol[good] = beta * seq_tol[pp[good]].sum(1) + 2 * U * np.abs(out["margins"][good])
    got = _host(margins)
    assert (np.isnan(got) == ~good).all() and (np.abs(got - out["margins"])[good] <= m_tol[good]).all(), (what, "margins")
    clear = (np.abs(out["margins"][good]) > m_tol[good]).all()
    assert abs(_host(stats)[0] - out["stats"][0]) <= m_tol.max(initial=0) + 4 * U * max(1.0, out["stats"][0]), (what, _host(stats), out["stats"])
    assert not clear or abs(_host(stats)[1] - out["stats"][1]) <= 2 * U, (what, "order")
    # a sequence's derivative: its pairs' sigmas, each off by the margin's error (slope at most 1/4) and roundings
    mean = 8.0 * beta / max(1, good.sum())
    c_tol = np.zeros(S)
    for k in np.flatnonzero(good):
        for q in pp[k]:
            c_tol[q] += mean * (0.25 * m_tol[k] + 16 * U)
    c_tol /= np.where(average, np.maximum(length, 1), 1)
    assert (np.abs(_host(coeff) - out["coeff"]) <= c_tol[where[0]] + 4 * U * np.abs(out["coeff"])).all(), (what, "coeff")
    every_eps = eps(V, out["logp"])
    check_grad(_host(grad), dict(out, actions=a), np.abs(out["coeff"]) + c_tol[where[0]] / every_eps, dtype, what)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [1, 2, 4, 13, 16, 20, 64, 65, 300, 1025, 5000, 33000, 140001])
def test_preference_loss_over_widths(V, dtype):
    n = 32 if V < 2000 else 8
    _preference_case(V, n, V, dtype, 4, "packed", "all")
    _preference_case(V + 1, n, V, dtype, 2, "by_seq", "bounds", average=True, smoothing=0.2, pad=3, inplace=True)


@pytest.mark.parametrize("order", ["by_seq", "by_step", "packed"])
@pytest.mark.parametrize("kind", ["all", "bounds", "mask"])
@pytest.mark.parametrize("n,V,S,pairs", [(24, 3, 6, 0), (700, 4, 14, 300), (64, 70, 4, 9), (16, 9000, 2, 0), (1200, 2, 300, 1000), (4, 5, 4, 1)])
def test_preference_loss_over_orders(order, kind, n, V, S, pairs):
    _preference_case(n + V, n, V, "fp32" if V < 100 else "bf16", S, order, kind, pairs=pairs, average=S == 14, ref=S != 300,
                     smoothing=0.1 if pairs else 0.0)


def test_long_sequences_and_one_sequence():
    _preference_case(3, 120000, 2, "fp32", 2, "by_step", "mask")
    _preference_case(4, 60000, 3, "fp32", 2, "by_seq", "bounds", average=True)
    _preference_case(5, 40, 3, "fp32", 1, "by_seq", "all", pairs=1)


# --------------------------------------------------------------------------- memory, streams, graphs
def test_offsets_past_32_bits():
    """Rows whose first logit lies more than 2^31 elements into the buffer."""
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(0)
    n, stride = 5, (1 << 29) + 8
    for V in (7, 1000, 9000):
        z, a = _state(rng, n, V, "bf16")
        buf = torch.empty((n - 1) * stride + V, dtype=torch.bfloat16, device="cuda:0")
        x = buf.as_strided((n, V), (stride, 1))
        x.copy_(torch.from_numpy(z))
        adv, stats = rng.normal(0, 1, n).astype(np.float32), torch.empty(5, device="cuda:0")
        pl.clipped_policy_loss(x, _dev(a), _dev(adv), stats, out_grad=x)
        out = ol.policy_loss(z, a, adv)
        check_rows(_host(stats), out["stats"], V, "stats")
        check_grad(_host(x), dict(out, actions=a), np.abs(adv), "bf16", V)
        del buf, x


def test_what_lies_beside_the_rows_is_left_alone():
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(1)
    for V, dtype in ((3, "fp32"), (5, "bf16"), (67, "fp16"), (1003, "bf16"), (9001, "fp32")):
        z, a = _state(rng, 6, V, dtype)
        x = _logits(z, dtype, pad=2)
        buf = torch.full((6 * (V + 4) + 9,), 7.0, dtype=_t(dtype), device="cuda:0")
        grad = buf[5:5 + 6 * (V + 4)].view(6, V + 4)[:, :V]
        adv, stats = rng.normal(0, 1, 6).astype(np.float32), torch.empty(5, device="cuda:0")
        pl.clipped_policy_loss(x, _dev(a), _dev(adv), stats, out_grad=grad)
        check_grad(_host(grad), dict(ol.policy_loss(z, a, adv), actions=a), np.abs(adv), dtype, V)
        grad.fill_(7.0)
        assert (_host(buf) == 7.0).all(), (V, dtype)


def test_three_dimensional_logits_of_an_episode():
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(2)
    T, B, D = 9, 6, 4
    z, a = _state(rng, T * B, D, "fp32")
    x, logp = _logits(z, "fp32").view(T, B, D), torch.empty((T, B), device="cuda:0")
    pl.action_logp(x, _dev(a.reshape(T, B)), logp)
    check_rows(_host(logp).ravel(), ol.softmax_rows(z, a)[1], D, "episode")
    with pytest.raises(pl.PlacetoError):
        pl.action_logp(x.transpose(0, 1), _dev(a), logp)             # rows do not lie at one distance
    with pytest.raises(pl.PlacetoError):
        pl.action_logp(x.transpose(0, 2), _dev(a), logp)
    with pytest.raises(pl.PlacetoError):
        pl.action_logp(x[:1].expand(T, B, D), _dev(a), logp)


def _calls(rng, n, V, dtype):
    """Closures over one set of buffers: the calls, and what they write."""
    import torch
    import paper_1906_08879_amd as pl
    z, a = _state(rng, n, V, dtype)
    x, act, adv = _logits(z, dtype), _dev(a), _dev(rng.normal(0, 1, n).astype(np.float32))
    mask = _dev((rng.random(n) < 0.8).astype(np.uint8))
    rows = pl.DecisionRows(n, 2, mask=mask)
    logp, stats, pstats = torch.empty(n, device="cuda:0"), torch.empty(5, device="cuda:0"), torch.empty(2, device="cuda:0")
    grad, pgrad = torch.empty_like(x), torch.empty_like(x)
    ws = torch.empty(pl.loss_workspace_bytes(x, rows, 1), dtype=torch.uint8, device="cuda:0")
    tensors = [torch.randn(k, device="cuda:0").to(t) for k, t in ((5, torch.float32), (70001, torch.bfloat16), (4099, torch.float16))]
    clipped, norm = [torch.empty_like(t) for t in tensors], torch.empty(1, device="cuda:0")
    cws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda:0")

    def call(stream=None):
        pl.action_logp(x, act, logp, workspace=ws, stream=stream)
        pl.clipped_policy_loss(x, act, adv, stats, rows=rows, old_logp=logp, reduction="seqs", entropy_coeff=0.1, out_grad=grad,
                               workspace=ws, stream=stream)
        pl.preference_loss(x, act, rows, pstats, out_grad=pgrad, workspace=ws, stream=stream)
        pl.clip_gradients(tensors, 1.0, norm, out=clipped, workspace=cws, stream=stream)

    return call, [logp, stats, pstats, grad, pgrad, norm, *clipped], [x, act, adv, mask, rows, ws, tensors, cws]


@pytest.mark.parametrize("n,V,dtype", [(40, 4, "fp32"), (600, 8, "fp32"), (64, 900, "bf16"), (10, 40000, "bf16")])
def test_graph_replays_equal_the_eager_calls_bit_for_bit(n, V, dtype):
    import torch
    rng = np.random.default_rng(n)
    call, outs, keep = _calls(rng, n, V, dtype)
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        for t in outs:
            t.fill_(3.0 + i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, u in zip(outs, want):
            assert torch.equal(t.view(torch.uint8), u.view(torch.uint8)), i
        call()
        torch.cuda.synchronize()
    del keep


def test_calls_on_another_stream():
    """Workspaces that a call takes for itself belong to the stream it runs on."""
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(9)
    n, V = 2000, 1000
    z, a = _state(rng, n, V, "fp32")
    x, act = _logits(z, "fp32"), _dev(a)
    want = torch.empty(n, device="cuda:0")
    pl.action_logp(x, act, want)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [torch.empty(n, device="cuda:0") for _ in range(8)]
    for g in got:
        pl.action_logp(x, act, g, stream=s)
        torch.full((1 << 20,), 9, dtype=torch.uint8, device="cuda:0")    # would reuse a workspace freed too early
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


# --------------------------------------------------------------------------- clipping
def _clip_case(seed, sizes, dtypes, max_norm, offset=0, out=True, scale=1.0):
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(seed)
    grads = []
    for i, k in enumerate(sizes):
        buf = torch.zeros(k + offset, dtype=_t(dtypes[i % len(dtypes)]), device="cuda:0")
        buf[offset:] = torch.from_numpy(rng.normal(0, scale, k)).to(buf.dtype)
        grads.append(buf[offset:])
    host = [_host(g) for g in grads]
    norm = torch.full((1,), 7.0, device="cuda:0")
    res = [torch.full_like(g, 7.0) for g in grads] if out else grads
    pl.clip_gradients(grads, max_norm, norm, out=res if out else None)
    ref_norm, ref = ol.clip(host, max_norm)
    # the norm is float64 rounded once, the factor and the product are fp32, each rounded once
    assert abs(float(norm) - ref_norm) <= 2 * U * ref_norm, (sizes, float(norm), ref_norm)
    for i, (r, o, g) in enumerate(zip(ref, res, host)):
        d = dtypes[i % len(dtypes)]
        assert (np.abs(_host(o) - r) <= (HALF_ULP[d] + 3 * U) * np.abs(r) + TINY[d]).all(), (sizes[i], d)
        if ref_norm <= max_norm:
            assert (_host(o) == g).all()


@pytest.mark.parametrize("out", [True, False])
@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e9, float("inf")])
@pytest.mark.parametrize("sizes", [[1], [3], [4096], [65536], [65537], [100003], [1 << 20], [0, 5, 0, 0, 16385, 1], [7] * 300,
                                   [1, 300001, 2, 16384, 16383]])
def test_clipping(sizes, max_norm, out):
    for dtypes in (["fp32"], ["bf16"], ["fp32", "bf16", "fp16"]):
        _clip_case(len(sizes), sizes, dtypes, max_norm, out=out)
        _clip_case(len(sizes), sizes, dtypes, max_norm, offset=3, out=out)


def test_clipping_of_large_tensors_and_of_none():
    import torch
    import paper_1906_08879_amd as pl
    _clip_case(1, [30000001, 17, 5000000], ["bf16", "fp32"], 1.0)
    norm = torch.full((1,), 7.0, device="cuda:0")
    pl.clip_gradients([], 1.0, norm)
    assert float(norm) == 0.0
    pl.clip_gradients([torch.empty(0, device="cuda:0")], 1.0, norm)
    assert float(norm) == 0.0


@pytest.mark.parametrize("size", [40, 100000, 3000000])
def test_norms_that_are_not_finite_leave_the_gradients(size):
    import torch
    import paper_1906_08879_amd as pl
    for bad in (float("nan"), float("inf"), -float("inf")):
        for dtype in (torch.float32, torch.bfloat16):
            g = torch.randn(size, device="cuda:0").to(dtype)
            g[size // 2] = bad
            before, norm, out = g.clone(), torch.empty(1, device="cuda:0"), torch.empty_like(g)
            pl.clip_gradients([g], 1.0, norm, out=[out])
            pl.clip_gradients([g], 1.0, norm)
            assert not np.isfinite(float(norm))
            for t in (g, out):
                assert torch.equal(t.nan_to_num(5.0, 6.0, 8.0), before.nan_to_num(5.0, 6.0, 8.0))


def test_gradients_whose_squares_leave_fp32():
    import torch
    import paper_1906_08879_amd as pl
    for v in (1e30, 1e-30):
        g = torch.full((1000,), v, device="cuda:0")
        norm, out = torch.empty(1, device="cuda:0"), torch.empty_like(g)
        pl.clip_gradients([g], 1e-31, norm, out=[out])
        assert abs(float(norm) / (v * np.sqrt(1000.0)) - 1.0) < 1e-6
        assert abs(float(_host(out).astype(np.float64) @ _host(out)) ** 0.5 / 1e-31 - 1.0) < 1e-5


def test_clipping_is_the_same_bits_every_time():
    import torch
    import paper_1906_08879_amd as pl
    tensors = [torch.randn(k, device="cuda:0") for k in (1000003, 12, 777777)]
    norms = torch.empty(6, device="cuda:0")
    for i in range(6):
        pl.clip_gradients(tensors, float("inf"), norms[i:i + 1])
    assert (norms == norms[0]).all()

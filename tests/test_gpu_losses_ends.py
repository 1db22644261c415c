"""The losses on rows of logits and gradient clipping where a term leaves fp32, an action has no probability or a sum is
long, against their float64 oracle."""
import numpy as np
import pytest

from oracle import losses as ol
from tests.test_gpu_losses import U, _dev, _host, _logits, _state, _t, check_grad, check_rows, eps

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- masked by the lowest value
def _lowest(dtype):
    import torch
    return float(torch.finfo(_t(dtype)).min)


def _rows_with_masked_actions(rng, n, V, dtype):
    """The first half of the rows take an action whose logit is the type's lowest value or -inf; and the next one takes
    the lowest where nothing is larger."""
    z, a = _state(rng, n, V, dtype)
    a[:] = V // 2
    low = _lowest(dtype)
    z[0, V // 2] = low
    z[1, V // 2] = -np.inf
    z[2, V // 4:] = low                                   # as a padded vocabulary, the action among it
    z[3] = low; z[3, 0] = -low
    z[4] = low                                            # nothing larger: all equally likely
    z[5] = -np.inf; z[5, V // 2] = low                    # the only action there is
    return z, a, low


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [4, 5, 37, 700, 9000, 70001, 140001])
def test_an_action_masked_by_the_lowest_value_has_no_probability(V, dtype):
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(V)
    n = 12
    z, a, low = _rows_with_masked_actions(rng, n, V, dtype)
    x, act = _logits(z, dtype), _dev(a)
    _, l, H, live = ol.softmax_rows(z, a, lowest=low)
    assert (l[:4] == -np.inf).all() and live[4:].all() and not live[:4].any()
    logp, ent = torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0")
    pl.action_logp(x, act, logp, ent)
    check_rows(_host(logp), l, V, "logp")
    check_rows(_host(ent), H, V, "entropy")
    finite = np.where(np.isfinite(l), l, 0.0)
    old, ref = (finite + rng.normal(0, 0.1, n)).astype(np.float32), (finite + rng.normal(0, 0.3, n)).astype(np.float32)
    adv = rng.normal(0, 1, n).astype(np.float32)
    for o in (None, old):
        stats, grad = torch.empty(5, device="cuda:0"), torch.full_like(x, 7.0)
        kw = dict(kl_coeff=0.3, entropy_coeff=0.1, clip_low=1.0, clip_high=9.0)
        pl.clipped_policy_loss(x, act, _dev(adv), stats, old_logp=None if o is None else _dev(o), ref_logp=_dev(ref), out_grad=grad,
                               out_logp=logp, **kw)
        out = ol.policy_loss(z, a, adv, old=o, ref=ref, lowest=low, **kw)
        assert np.isfinite(out["stats"]).all() and (out["grad"][:4] == 0).all()
        check_rows(_host(logp), out["logp"], V, "logp of the loss")
        # per row: the surrogate and the KL estimate with e^d up to e^1, the entropy with its own size
        tol = (eps(V, finite) * (4.0 * np.abs(adv) + 2.0 + H)).sum() * 2.0 / n
        assert (np.abs(_host(stats) - out["stats"]) <= tol).all(), (_host(stats), out["stats"])
        check_grad(_host(grad), dict(out, actions=a), (4.0 * np.abs(adv) + 2.0 + H) / n, dtype, "grad")
    stats, grad, coeff = torch.empty(2, device="cuda:0"), torch.full_like(x, 7.0), torch.empty(n, device="cuda:0")
    pl.preference_loss(x, act, pl.DecisionRows(n, 4), stats, ref_logp=_dev(ref), beta=0.5, out_grad=grad, out_logp=logp, out_coeff=coeff)
    out = ol.preference_loss(z, a, ol.rows_of(n, 4), 4, ref=ref, beta=0.5, lowest=low)
    check_rows(_host(logp), out["logp"], V, "logp of the preference")
    tol = 0.5 * (eps(V, finite) * np.maximum(1.0, np.abs(finite))).sum() + 16 * U
    assert (np.abs(_host(stats) - out["stats"]) <= tol).all() and (np.abs(_host(coeff) - out["coeff"]) <= tol).all()
    assert (_host(grad)[:4] == 0).all() and (_host(coeff)[:4] == 0).all()
    check_grad(_host(grad), dict(out, actions=a), np.abs(out["coeff"]) + tol / eps(V, finite), dtype, "grad of the preference")


def test_the_lowest_half_precision_value_close_to_the_others_has_a_probability():
    import torch
    import paper_1906_08879_amd as pl
    low = _lowest("fp16")
    z = np.full((3, 20), low)
    z[0, 3] = low + 32.0                                  # the next number: 32 nats
    z[1, 3] = low + 96.0
    z[2, 3] = low + 128.0                                 # e^-128 is no fp32 number
    a, logp = np.zeros(3, np.int32), torch.empty(3, device="cuda:0")
    pl.action_logp(_logits(z, "fp16"), _dev(a), logp)
    check_rows(_host(logp), ol.softmax_rows(z, a, lowest=low)[1], 20, "logp")
    assert _host(logp)[1] == -96.0 and _host(logp)[2] == -np.inf


# --------------------------------------------------------------------------- terms that are multiplied by nothing
def _far_rows(V, dtype, row, shift):
    """Rows, and log probabilities of another policy that are `shift` off in one row."""
    rng = np.random.default_rng(V)
    z, a = _state(rng, 12, V, dtype, 1.0)
    other = (ol.softmax_rows(z, a)[1] + rng.normal(0, 0.1, 12)).astype(np.float32)
    other[row] += np.float32(shift)
    return rng, z, a, other


@pytest.mark.parametrize("V", [4, 5, 37, 700, 9000, 70001, 140001])
def test_a_reference_that_is_only_watched_adds_nothing(V):
    """kl_coeff 0: the loss and the gradient are those without a reference, however far it lies; its estimate is reported."""
    import torch
    import paper_1906_08879_amd as pl
    for shift in (100.0, 1000.0, -np.inf, np.nan):
        rng, z, a, ref = _far_rows(V, "bf16", 3, shift)
        x, act, adv = _logits(z, "bf16"), _dev(a), _dev(rng.normal(0, 1, 12).astype(np.float32))
        got = []
        for r in (None, _dev(ref)):
            stats, grad, coeff = torch.empty(5, device="cuda:0"), torch.full_like(x, 7.0), torch.empty(12, device="cuda:0")
            pl.clipped_policy_loss(x, act, adv, stats, ref_logp=r, entropy_coeff=0.1, out_grad=grad, out_coeff=coeff)
            got.append((_host(stats), _host(grad), _host(coeff)))
        (s0, g0, c0), (s1, g1, c1) = got
        assert np.isfinite(s1[[0, 1, 3, 4]]).all() and (s0[[0, 1, 3, 4]] == s1[[0, 1, 3, 4]]).all(), (shift, s0, s1)
        assert (g0 == g1).all() and (c0 == c1).all(), shift
        assert np.isnan(s1[2]) if np.isnan(shift) else s1[2] == np.inf       # (e^100 is no fp32 number)


@pytest.mark.parametrize("V", [4, 5, 37, 700, 9000, 70001, 140001])
def test_no_advantage_whatever_the_ratio(V):
    import torch
    import paper_1906_08879_amd as pl
    for shift in (-100.0, -np.inf):
        rng, z, a, old = _far_rows(V, "bf16", 3, shift)
        adv = rng.normal(0, 1, 12).astype(np.float32)
        adv[3] = 0.0
        x = _logits(z, "bf16")
        stats, grad, coeff = torch.empty(5, device="cuda:0"), torch.full_like(x, 7.0), torch.empty(12, device="cuda:0")
        pl.clipped_policy_loss(x, _dev(a), _dev(adv), stats, old_logp=_dev(old), out_grad=grad, out_coeff=coeff)
        # (the ratio of row 3 in 64 bits is a number, or not: its product with 0 is 0)
        old[3] = ol.softmax_rows(z, a)[1][3]
        out = ol.policy_loss(z, a, adv, old=old)
        size = np.abs(adv) * 2.0                          # ratios are e^(a few tenths), and held
        tol = (eps(V, out["logp"]) * size).sum() * 2.0 / 12 + 8 * U * np.abs(out["stats"])
        assert (np.abs(_host(stats) - out["stats"]) <= tol).all(), (_host(stats), out["stats"])
        assert _host(coeff)[3] == 0 and (_host(grad)[3] == 0).all()
        check_grad(_host(grad), dict(out, actions=a), size / 12, "bf16", (V, shift))


@pytest.mark.parametrize("V", [4, 37, 9000])
@pytest.mark.parametrize("smoothing,side", [(0.0, 0), (1.0, 1)])
@pytest.mark.parametrize("S", [4, 3000])
def test_a_pair_that_is_certain_costs_nothing(V, smoothing, side, S):
    """A reference of -inf makes a margin infinite; the term of the other order has no weight."""
    import torch
    import paper_1906_08879_amd as pl
    if V * S > 200000:
        V = 40
    rng = np.random.default_rng(V + S)
    n = 2 * S
    z, a = _state(rng, n, V, "fp32", 1.0)
    ref = (ol.softmax_rows(z, a)[1] + rng.normal(0, 0.1, n)).astype(np.float32)
    ref[2 * side] = -np.inf                               # of the first or of the second sequence
    for pairs in (None, np.array([[0, 1], [2, 3], [3, 2]], np.int32)):
        stats, margins, coeff = torch.empty(2, device="cuda:0"), torch.empty(S // 2 if pairs is None else 3, device="cuda:0"), torch.empty(n, device="cuda:0")
        grad = torch.empty((n, V), device="cuda:0")
        pl.preference_loss(_logits(z, "fp32"), _dev(a), pl.DecisionRows(n, S), stats, pairs=None if pairs is None else _dev(pairs),
                           ref_logp=_dev(ref), label_smoothing=smoothing, out_margins=margins, out_coeff=coeff, out_grad=grad)
        out = ol.preference_loss(z, a, ol.rows_of(n, S), S, pairs=pairs, ref=ref, smoothing=smoothing)
        assert out["margins"][0] == (-np.inf if side else np.inf) and np.isfinite(out["stats"]).all()
        assert _host(margins)[0] == out["margins"][0]
        # margins are beta = 0.1 times sums of four rows; the loss has a slope of at most 1 in them
        tol = 0.1 * 4.0 * (eps(V, out["logp"]) * np.maximum(1.0, np.abs(out["logp"]))).max() + 16 * U
        assert (np.abs(_host(stats) - out["stats"]) <= tol).all(), (_host(stats), out["stats"])
        assert (_host(coeff)[:4] == 0).all() and np.isfinite(_host(coeff)).all() and (_host(grad)[:4] == 0).all()


# --------------------------------------------------------------------------- long rows
@pytest.mark.parametrize("V", [1 << 18, 1 << 22])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_many_equal_logits_do_not_add_up_to_an_error(V, dtype):
    """Rows whose probabilities are equal but for the first ones (so many that every thread has met the largest logit): their
    roundings all go the same way.  From the formulas: s = first + (V - first) e^-c.  A term is off by the roundings of x and of its exponent (4 U), a sum by those of a few dozen additions one
    behind another, of lanes, waves and the logarithm: the 64 U of EPS without a share that grows with V."""
    import torch
    import paper_1906_08879_amd as pl
    n, first, c = 64, 2048, np.array([0.40625, 1.3125, 2.71875, 5.15625])        # (numbers of bf16)
    c = np.tile(c, n // 4)
    x = torch.empty((n, V), dtype=_t(dtype), device="cuda:0")
    x.copy_(-_dev(c).to(_t(dtype))[:, None].expand(n, V))
    x[:, :first] = 0.0
    logp, ent = torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0")
    pl.action_logp(x, _dev(np.full(n, 17, np.int32)), logp, ent)
    s = first + (V - first) * np.exp(-c)
    l, H = -np.log(s), np.log(s) + (V - first) * np.exp(-c) / s * c
    tol = U * (64.0 + 4.0 * np.abs(l))
    assert (np.abs(_host(logp) - l) <= tol).all(), (np.abs(_host(logp) - l) / tol).max()
    assert (np.abs(_host(ent) - H) <= 2.0 * tol + 64.0 * U * c).all(), (np.abs(_host(ent) - H) / tol).max()


# --------------------------------------------------------------------------- clipping
def test_a_norm_above_fp32_is_reported_and_leaves_the_gradients():
    import torch
    import paper_1906_08879_amd as pl
    for size in (4, 40000, 3000000):
        g = torch.full((size,), 3e38, device="cuda:0")
        before, out, norm = g.clone(), torch.full_like(g, 7.0), torch.empty(1, device="cuda:0")
        pl.clip_gradients([g], 1.0, norm, out=[out])
        assert float(norm) == float("inf") and torch.equal(out, before)
        pl.clip_gradients([g], 1.0, norm)
        assert float(norm) == float("inf") and torch.equal(g, before)


@pytest.mark.parametrize("dtype,value,size", [("fp16", 1.7998046875, 1310720), ("fp32", 1.1563552618026733, 786432),
                                              ("fp32", 1.0286269187927246, 1000000), ("bf16", 1.375, 2345672)])
def test_the_norm_of_equal_gradients_is_float64_rounded_once(dtype, value, size):
    """Squares whose partial sums in fp32 would all round the same way."""
    import torch
    import paper_1906_08879_amd as pl
    g = torch.full((size,), value, dtype=_t(dtype), device="cuda:0")
    v, norm = float(g[0]), torch.empty(1, device="cuda:0")
    pl.clip_gradients([g], float("inf"), norm)
    assert abs(float(norm) / (v * np.sqrt(size)) - 1.0) <= 1.001 * U, (float(norm) / (v * np.sqrt(size)) - 1.0) / U


@pytest.mark.parametrize("dtype,V", [("fp32", 1 << 18), ("fp32", 1 << 22), ("bf16", 1 << 22)])
def test_slowly_rising_logits_do_not_add_up_to_an_error(dtype, V):
    """Every step of a thread meets a logit that is a little larger than all before, so that what it has is scaled again and
    again by a factor close to 1.  The bound is that of equal logits."""
    import torch
    import paper_1906_08879_amd as pl
    n, a = 64, V // 3
    x = torch.empty((n, V), dtype=_t(dtype), device="cuda:0")
    ramp = torch.arange(V, dtype=torch.float64, device="cuda:0") / V
    l, H = np.zeros(n), np.zeros(n)
    rises = (0.03, 0.2, 0.7, 1.0, 3.0, 9.0, 30.0, 100.0)
    for k, rise in enumerate(rises):
        x[k::len(rises)] = (rise * ramp).to(_t(dtype))
        z = x[k].double()
        every = z - torch.logsumexp(z, 0)
        l[k::len(rises)], H[k::len(rises)] = float(every[a]), float(-(every.exp() * every).sum())
    logp, ent = torch.empty(n, device="cuda:0"), torch.empty(n, device="cuda:0")
    pl.action_logp(x, _dev(np.full(n, a, np.int32)), logp, ent)
    tol = U * (64.0 + 4.0 * np.abs(l))
    assert (np.abs(_host(logp) - l) <= tol).all(), (np.abs(_host(logp) - l) / tol)[:8]
    # t is a sum of terms of up to a few units' size beside s
    assert (np.abs(_host(ent) - H) <= 4.0 * tol).all(), (np.abs(_host(ent) - H) / tol)[:8]

"""The loss against a teacher's list where the policy has given up the actions outside it: far below the row's largest logit, at low
temperatures, with scaled gradients, masked by the type's lowest value.  Against the definition in logarithms (float64), whose terms
neither vanish nor overflow.

Bounds.  U = 2^-24.  With o_j the softmax over the unlisted actions, a value is sum q (ln q - ln p) + r (ln r - ln p_rest) and the unlisted
gradient scale (F p_j - r o_j).  Only the sum over the unlisted actions is fp32, RHO(V) of it as in test_gpu_distill; ln p_rest is off by RHO, o_j by RHO
and U (8 + 4 |x_j|) of itself, x_j its exponent relative to the largest unlisted one or, where p_rest is above 2^-40, to the row's
largest: up to 28 more.  Where p_rest is not below 2^-40, terms below 2^-126 of the row's largest are zero: 2^-86 of scale.  Then the roundings of
the results."""
import numpy as np
import pytest

from tests.test_gpu_distill import _round, rho
from tests.test_gpu_losses import HALF_ULP, TINY, U, _dev, _host, _logits, _t

pytestmark = pytest.mark.gpu


def _log_sum(x):
    m = x.max(-1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    with np.errstate(divide="ignore"):
        return np.log(np.exp(x - m).sum(-1)) + m[..., 0]


def expected(z, ids, lq, T, low):
    """Values and gradients (without weights) of rows whose listed actions are allowed, no two alike."""
    n, V = z.shape
    x = z / T
    masked = np.isneginf(z) | ((z == low) & ((z - z.max(1, keepdims=True)) / T < -150.0 * np.log(2.0)))
    x = np.where(masked, -np.inf, x)
    lp = x - _log_sum(x)[:, None]
    listed = np.zeros((n, V), bool)
    np.put_along_axis(listed, ids.astype(np.int64), True, 1)
    lq = lq.astype(np.float64)
    q, of_list = np.exp(lq), np.take_along_axis(lp, ids.astype(np.int64), 1)
    others = np.where(listed, -np.inf, lp)
    log_rest = _log_sum(others)
    left = np.isfinite(log_rest)
    mass = q.sum(1)
    r = np.where(left, np.maximum(0.0, 1.0 - mass), 0.0)
    values = (q * (lq - of_list)).sum(1) + np.where(r > 0, r * (np.log(np.where(r > 0, r, 1.0)) - np.where(left, log_rest, 0.0)), 0.0)
    F = mass + r
    o = np.exp(others - np.where(left, log_rest, 0.0)[:, None])
    grad = F[:, None] * np.exp(lp) - r[:, None] * o
    np.put_along_axis(grad, ids.astype(np.int64), F[:, None] * np.exp(of_list) - q, 1)
    with np.errstate(invalid="ignore"):
        depth = np.where(np.isfinite(others), others.max(1, keepdims=True) - others, 0.0)
    share = np.exp(_log_sum(of_list))
    return values, grad, dict(r=r, F=F, o=o, p=np.exp(lp), depth=depth, mass=mass, share=share)


def run(z, ids, lq, dtype, T=1.0, grad_scale=1.0, reduction="sum", pad=0, offset=0, empty=0):
    """`empty`: entries without an action in front of the list."""
    import torch
    import paper_1906_08879_amd as pl
    n, V = z.shape
    ref, g, of = expected(z, ids, lq, T, float(torch.finfo(_t(dtype)).min))
    if empty:
        ids = np.concatenate([np.full((n, empty), -1, np.int32), ids], 1)
        lq = np.concatenate([np.full((n, empty), -1.0, np.float32), lq], 1)
    x = _logits(z, dtype, pad, offset)
    stats, values = torch.full((3,), -7.0, device="cuda:0"), torch.full((n,), -7.0, device="cuda:0")
    grad = torch.full((n, V), 7.0, dtype=x.dtype, device="cuda:0")
    kw = dict(temperature=T, grad_scale=grad_scale, reduction=reduction)
    pl.distill_loss(x, _dev(ids), _dev(lq), stats, out_grad=grad, out_values=values, **kw)
    alone = torch.empty_like(values)
    pl.distill_loss(x, _dev(ids), _dev(lq), torch.empty_like(stats), out_values=alone, **kw)
    assert torch.equal(alone, values)
    w = 1.0 / n if reduction == "rows" else 1.0
    scale = w * grad_scale / T
    got = _host(values)
    tol = rho(V) * np.maximum(of["r"], of["mass"]) + 4 * U * np.abs(ref) + 1e-12
    assert (np.abs(got - ref) <= tol).all(), ("values", got, ref, tol)
    total = np.array([(w * ref).sum(), (w * of["mass"]).sum(), (w * of["share"]).sum()])
    bound = np.array([(w * tol).sum(), 0.0, rho(V) * w * n]) + 4 * U * np.abs(total) + 1e-12
    assert (np.abs(_host(stats) - total) <= bound).all(), ("stats", _host(stats), total, bound)
    got, want = _host(grad), scale * g
    size = of["F"][:, None] * of["p"] + of["r"][:, None] * of["o"]
    tol = scale * (size * (3 * rho(V) + U * (8 + 4 * (of["depth"] + 28))) + 2.0 ** -86) + (HALF_ULP[dtype] + 2 * U) * np.abs(want) + TINY[dtype]
    ok = np.abs(got - want) <= tol
    assert ok.all(), ("grad", np.argwhere(~ok)[:4], got[~ok][:4], want[~ok][:4], tol[~ok][:4])
    return _host(values), got


# narrow (whole slots and not), a row to a lane, to a wave and a workgroup of every size, in slices
WIDTHS = [(12, 8), (12, 5), (15000, 33), (12, 200), (12, 900), (12, 5000), (12, 13000), (3, 70001), (70, 60001), (65, 140001)]


def _given_up(rng, n, V, dtype, gaps, T):
    """Four listed actions, the others by `gaps` (in nats) below them and from one another."""
    z = rng.normal(0, 1, (n, V)) * T
    ids = np.stack([rng.permutation(V)[:4] for _ in range(n)]).astype(np.int32)
    for i in range(n):
        z[i, ids[i]] += gaps[i % len(gaps)] * T
    return _round(z, dtype), ids, np.log(np.tile([0.3, 0.2, 0.1, 0.1], (n, 1))).astype(np.float32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n,V", WIDTHS)
@pytest.mark.parametrize("T,grad_scale", [(1.0, 65536.0), (0.1, 1024.0), (0.5, 1.0)])
def test_gradients_of_actions_that_are_given_up_stay_finite(n, V, dtype, T, grad_scale):
    """75 to 87 nats: r / p_rest leaves fp32, the gradient does not."""
    z, ids, lq = _given_up(np.random.default_rng(V), n, V, dtype, (75.0, 79.0, 82.0, 84.0, 86.0, 87.0, 20.0, 27.0, 28.0, 40.0), T)
    run(z, ids, lq, dtype, T, grad_scale)


@pytest.mark.parametrize("n,V", WIDTHS)
@pytest.mark.parametrize("T", [1.0, 0.01, 2.0 ** -20])
def test_the_rest_counts_however_far_it_is_given_up(n, V, T):
    """88 nats and more: the value goes on with the gap, its gradient stays."""
    z, ids, lq = _given_up(np.random.default_rng(V + 1), n, V, "fp32", (86.0, 88.0, 90.0, 104.0, 200.0, 700.0, 800.0, 1e3, 1e5), T)
    run(z, ids, lq, "fp32", T, reduction="rows", pad=3, offset=1)


@pytest.mark.parametrize("grad_scale", [1e30, 3e-30])
@pytest.mark.parametrize("n,V", WIDTHS + [(12, 33001), (12, 70001)])
def test_scales_at_the_ends_of_fp32(n, V, grad_scale):
    z, ids, lq = _given_up(np.random.default_rng(V + 2), n, V, "fp32", (0.0, 10.0, 25.0, 60.0, 87.0, 120.0, 30.0, 33.0, 36.0), 1.0)
    run(z, ids, lq, "fp32", grad_scale=grad_scale)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,V", WIDTHS)
def test_masked_actions_outside_the_list(n, V, dtype):
    """Actions at -inf and at the lowest value have no share of the rest; where all others are such, there is none."""
    import torch
    low = float(torch.finfo(_t(dtype)).min)
    rng = np.random.default_rng(V + 3)
    z, ids, lq = _given_up(rng, n, V, dtype, (0.0, 10.0, 60.0, 90.0), 1.0)
    keep = np.take_along_axis(z, ids.astype(np.int64), 1)
    z = np.where(rng.random(z.shape) < 0.5, low, z)
    z = np.where(rng.random(z.shape) < 0.2, -np.inf, z)
    z[1] = low                                            # none of the others is allowed
    z[2] = -np.inf
    np.put_along_axis(z, ids.astype(np.int64), keep, 1)
    _, grad = run(z, ids, lq, dtype)
    listed = np.zeros(z.shape, bool)
    np.put_along_axis(listed, ids.astype(np.int64), True, 1)
    none = ~listed & (np.isneginf(z) | (z == low))
    assert (grad[none] == 0).all() and (grad[1:3][~listed[1:3]] == 0).all()


@pytest.mark.parametrize("n,V", WIDTHS)
@pytest.mark.parametrize("T", [20.0, 100.0, 2000.0])
def test_others_next_to_the_lowest_value(n, V, T):
    """fp16, others a step or two above -65504 and at it, by less than the mask's 2^-150 from one another: those at it are masked where the list
    lies far above, and count where it does not."""
    low = -65504.0
    rng = np.random.default_rng(V + 4)
    ids = np.stack([rng.permutation(V)[:4] for _ in range(n)]).astype(np.int32)
    z = low + 32.0 * rng.integers(0, 3, (n, V))
    z[::3] = low
    for i in range(n):
        z[i, ids[i]] = _round(np.array([low + (400.0, 60000.0)[i % 2]]), "fp16") + 32.0 * np.arange(4)
    lq = np.log(np.tile([0.3, 0.2, 0.1, 0.1], (n, 1))).astype(np.float32)
    run(_round(z, "fp16"), ids, lq, "fp16", T)


@pytest.mark.parametrize("given_up", [0, 1, 3])
@pytest.mark.parametrize("n,V", [(12, 4), (12, 7), (12, 16), (50000, 24), (12, 24), (12, 100), (12, 128)])
def test_lists_as_long_as_the_rows(n, V, given_up):
    """All actions listed, or all but a few that the policy has given up; with entries without an action in front of them."""
    rng = np.random.default_rng(V + 6)
    z = _round(rng.normal(0, 1, (n, V)), "fp32")
    ids = np.stack([rng.permutation(V) for _ in range(n)]).astype(np.int32)[:, given_up:]
    left = np.ones(z.shape, bool)
    np.put_along_axis(left, ids.astype(np.int64), False, 1)
    z[left] -= 100.0 + np.arange(n)[:, None].repeat(V, 1)[left] % 7
    lq = np.log(np.full(ids.shape, 0.9 / ids.shape[1])).astype(np.float32)
    run(_round(z, "fp32"), ids, lq, "fp32")
    run(_round(z, "fp32"), ids, lq, "fp32", empty=given_up)


@pytest.mark.parametrize("n,V", WIDTHS)
def test_in_place_where_the_rest_is_given_up(n, V):
    import torch
    import paper_1906_08879_amd as pl
    z, ids, lq = _given_up(np.random.default_rng(V + 5), n, V, "bf16", (0.0, 30.0, 86.0, 200.0), 1.0)
    x = _logits(z, "bf16", 5)
    out = torch.full((n, V + 5), 7.0, dtype=x.dtype, device="cuda:0")[:, :V]
    stats = [torch.empty(3, device="cuda:0") for _ in range(2)]
    pl.distill_loss(x, _dev(ids), _dev(lq), stats[0], out_grad=out)
    pl.distill_loss(x, _dev(ids), _dev(lq), stats[1], out_grad=x)
    assert torch.equal(x, out) and torch.equal(stats[0], stats[1])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("gap", [0.0, 120.0])
def test_the_largest_number_of_actions(gap, dtype):
    rng = np.random.default_rng(24)
    z, ids, lq = _given_up(rng, 1, 1 << 24, dtype, (gap,), 1.0)
    z[0, ids[0]] = 0.0
    ids[0, :2] = [(1 << 24) - 1, 0]
    z[0, ids[0]] = 3.0 + gap
    run(_round(z, dtype), ids, lq, dtype, grad_scale=1024.0)
    run(_round(z, dtype), ids, lq, dtype, grad_scale=1024.0, offset=1)

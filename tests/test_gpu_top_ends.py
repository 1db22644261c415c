"""Lists of likely actions in rows that are no numbers, together with what such rows seldom hold: actions masked by the type's lowest
value, a NaN of the largest bits.  By every width's kernel."""
import numpy as np
import pytest

from tests.test_gpu_losses import _dev, _host, _logits, _t
from tests.test_gpu_top import _run

pytestmark = pytest.mark.gpu

# narrow (whole slots and not), a row to a lane, to a wave, to a workgroup, streamed, in slices
WIDTHS = [(20, 4, 4), (20, 5, 5), (20000, 24, 24), (20, 300, 40), (20, 3000, 40), (20, 20001, 40), (3, 150001, 40)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n,V,k", WIDTHS)
def test_masked_actions_of_rows_that_are_no_numbers(n, V, k, dtype):
    """All their probabilities are NaN, as pl_action_logp has them; their actions in the order of the logits."""
    import torch
    import paper_1906_08879_amd as pl
    low = float(torch.finfo(_t(dtype)).min)
    rng = np.random.default_rng(V)
    z = rng.normal(0, 3, (n, V))
    z[:, 1:] = np.where(rng.random((n, V - 1)) < 0.9, low, z[:, 1:])
    z[:, 1] = low
    z[:, V - 1] = -np.inf
    for r in range(3):
        z[r, 0] = (np.nan, np.inf, 1.0)[r]
    a = np.ones(n, np.int32)
    top, lp, logp, ent = _run(z, k, dtype, a)
    assert np.isnan(lp[:2]).all() and np.isnan(logp[:2]).all() and np.isnan(ent[:2]).all()
    want = torch.empty(n, device="cuda:0")
    pl.action_logp(_logits(z, dtype), _dev(a), want)
    assert np.array_equal(_host(want), logp, equal_nan=True) and np.isneginf(logp[2])
    x = _logits(z, dtype)[:3]
    sign = x[0, 0].view(torch.int32 if dtype == "fp32" else torch.int16) < 0     # (torch's conversions of a NaN give either)
    order = np.maximum(np.where(np.isnan(z[:3]), 0.0, _host(x)), -1e300)
    order[0, 0] = -np.inf if sign else np.inf             # a NaN below -inf, or above all; +inf first
    assert (top[:3] == np.argsort(-order, axis=1, kind="stable")[:, :k]).all()


@pytest.mark.parametrize("n,V,k", WIDTHS + [(20, 16, 3), (20, 16, 16)])
@pytest.mark.parametrize("bits", [0x7fffffff, 0x7fc00000, -1, -0x400000])
def test_not_a_number_of_any_bits(n, V, k, bits):
    """A NaN is listed once, above all others or (with its sign) below them, wherever it lies."""
    import torch
    import paper_1906_08879_amd as pl
    gen = torch.Generator("cuda").manual_seed(V)
    x = torch.randn(n, V, device="cuda:0", generator=gen)
    at = [0, V // 2, V - 1]
    for r, j in enumerate(at):
        x.view(torch.int32)[r, j] = bits
    top, lp = torch.full((n, k), -7, dtype=torch.int32, device="cuda:0"), torch.empty(n, k, device="cuda:0")
    pl.top_actions(x, top, lp)
    order = x.double().cpu().numpy()
    for r, j in enumerate(at):
        order[r, j] = np.inf if bits > 0 else -np.inf
    assert (top.cpu().numpy() == np.argsort(-order, axis=1, kind="stable")[:, :k]).all()
    assert torch.isnan(lp[:3]).all() and torch.isfinite(lp[3:]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_the_largest_number_of_actions(dtype):
    """2^24 actions: hundreds of slices, indexes of 24 bits, equal logits at both ends."""
    from tests.test_gpu_top import _check, _round
    rng = np.random.default_rng(24)
    z = _round(rng.normal(0, 3, (1, 1 << 24)), dtype)
    _check(z, 128, dtype, rng)
    z[0, [0, 1, 77, (1 << 24) - 2, (1 << 24) - 1]] = 40.0
    _check(z, 20, dtype, rng, pad=1, offset=1)

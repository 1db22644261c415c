"""The oracle of the losses on rows of logits: its gradients against differences of its loss, and its values
against closed forms."""
import numpy as np
import pytest

from oracle import losses as ol


def _problem(seed, n=12, V=5):
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 1.5, (n, V))
    a = rng.integers(0, V, n)
    l = ol.softmax_rows(z, a)[1]
    return rng, z, a, l


def _differences(f, z, h=1e-5):
    g = np.zeros_like(z)
    for i in np.ndindex(*z.shape):
        up, down = z.copy(), z.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


@pytest.mark.parametrize("reduction", ["rows", "seqs", "sum"])
@pytest.mark.parametrize("order,bounds", [("by_seq", [3, 0, 4]), ("by_step", [4, 2, 1]), ("packed", [0, 5, 5, 11]), ("by_seq", None)])
def test_policy_gradient_of_logits_against_differences(reduction, order, bounds):
    rng, z, a, l = _problem(1)
    mask = (rng.random(12) < 0.8).astype(np.uint8)
    rows = ol.rows_of(12, 3, order, bounds, mask)
    old, ref, adv = l + rng.normal(0, 0.2, 12), l + rng.normal(0, 0.3, 12), rng.normal(0, 1, 3)
    kw = dict(rows=rows, old=old, ref=ref, kl_coeff=0.3, entropy_coeff=0.2, reduction=reduction, per_seq=True, n_seqs=3)
    out = ol.policy_loss(z, a, adv, **kw)
    g = _differences(lambda x: ol.policy_loss(x, a, adv, **kw)["stats"][0], z)
    assert np.abs(out["grad"] - g).max() <= 1e-8 * max(1.0, np.abs(g).max())
    assert np.abs(out["grad"]).max() > 1e-3
    assert bounds is not None or out["stats"][4] > 0          # (some arrangements have clipped rows, some none)


@pytest.mark.parametrize("average", [False, True])
@pytest.mark.parametrize("pairs", [None, [[0, 1], [0, 2], [3, 0], [1, 7], [2, 2]]])
def test_preference_gradient_of_logits_against_differences(average, pairs):
    rng, z, a, l = _problem(2)
    rows = ol.rows_of(12, 4, "packed", [0, 2, 2, 7, 11])
    kw = dict(rows=rows, n_seqs=4, pairs=pairs, ref=l + rng.normal(0, 0.5, 12), beta=0.7, smoothing=0.1, average=average)
    out = ol.preference_loss(z, a, **kw)
    g = _differences(lambda x: ol.preference_loss(x, a, **kw)["stats"][0], z)
    assert np.abs(out["grad"] - g).max() <= 1e-8 * max(1.0, np.abs(g).max())
    assert np.abs(out["grad"]).max() > 1e-3


def test_closed_forms():
    z = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.9, 0.0 + 1e-300]]))
    _, l, H, live = ol.softmax_rows(z, [0, 1])
    assert np.allclose(l, np.log([0.5, 0.9])) and live.all()
    assert np.allclose(H, [1.5 * np.log(2.0), -0.1 * np.log(0.1) - 0.9 * np.log(0.9)])
    # no reference, no old policy: the loss is minus the mean advantage, its gradient - A (e_a - p) / n
    out = ol.policy_loss(z, [0, 1], [1.0, -3.0])
    assert np.allclose(out["stats"][:2], 1.0) and np.allclose(out["grad"][0], -0.5 * np.array([0.5, -0.25, -0.25]))
    # equal sequences: log 2, and nothing to the right
    out = ol.preference_loss(np.zeros((2, 3)), [0, 1], ol.rows_of(2, 2), 2)
    assert np.allclose(out["stats"], [np.log(2.0), 0.0])
    norm, (c,) = ol.clip([np.array([3.0, 4.0])], 1.0)
    assert norm == 5.0 and np.allclose(c, [0.6, 0.8])

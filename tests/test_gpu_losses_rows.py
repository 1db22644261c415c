"""Losses on rows without a description of them: one sequence of all rows, against the float64 oracle."""
import numpy as np
import pytest

from oracle import losses as ol
from tests.test_gpu_losses import U, _dev, _host, _logits, _state, check_grad, eps

pytestmark = pytest.mark.gpu
SHAPES = [(1, 5), (2, 5), (300, 2), (257, 7), (600, 40), (70, 300), (40, 3000), (5, 20000), (3, 140001), (70, 140001)]


@pytest.mark.parametrize("n,V", SHAPES)
@pytest.mark.parametrize("reduction", ["rows", "seqs", "sum"])
def test_one_advantage_for_all_rows(n, V, reduction):
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(n + V)
    z, a = _state(rng, n, V, "bf16", 1.5)
    x, act = _logits(z, "bf16"), _dev(a)
    # what lies behind the one advantage is not to be used
    buf = torch.full((n + 1,), float("nan"), device="cuda:0")
    adv = np.array([-1.25], np.float32)
    buf[0] = float(adv[0])
    stats, grad, coeff = torch.empty(5, device="cuda:0"), torch.full_like(x, 7.0), torch.empty(n, device="cuda:0")
    pl.clipped_policy_loss(x, act, buf[:1], stats, reduction=reduction, advantage_per_sequence=True, entropy_coeff=0.02, out_grad=grad,
                           out_coeff=coeff)
    out = ol.policy_loss(z, a, adv, reduction=reduction, per_seq=True, entropy_coeff=0.02)
    size = 1.25 + 0.02 * (1.0 + out["entropy"])
    tol = (eps(V, out["logp"]) * out["w"] * (1.25 + 1.0 + out["entropy"])).sum() * 2.0
    assert (np.abs(_host(stats) - out["stats"]) <= tol + U * np.abs(out["stats"])).all(), (_host(stats), out["stats"])
    assert (np.abs(_host(coeff) - out["coeff"]) <= 4 * U * np.abs(out["coeff"])).all()
    check_grad(_host(grad), dict(out, actions=a), out["w"] * size, "bf16", (n, V, reduction))


@pytest.mark.parametrize("n,V", SHAPES)
def test_a_sequence_compared_with_itself(n, V):
    """The margin is zero and its two derivatives cancel, whichever kernel has the rows."""
    import torch
    import paper_1906_08879_amd as pl
    rng = np.random.default_rng(n + V)
    z, a = _state(rng, n, V, "bf16", 1.5)
    x, pairs = _logits(z, "bf16"), torch.zeros((1, 2), dtype=torch.int32, device="cuda:0")
    stats, grad, coeff = torch.empty(2, device="cuda:0"), torch.full_like(x, 7.0), torch.full((n,), 7.0, device="cuda:0")
    seq = torch.empty(1, device="cuda:0")
    pl.preference_loss(x, _dev(a), None, stats, pairs=pairs, out_grad=grad, out_coeff=coeff, out_seq_logp=seq)
    l = ol.softmax_rows(z, a)[1]
    assert abs(float(stats[0]) - np.log(2.0)) <= 4 * U and float(stats[1]) == 0.0
    assert abs(float(seq) - l.sum()) <= (eps(V, l) * np.maximum(1.0, np.abs(l))).sum() + 2 * U * np.abs(l.sum())
    assert (_host(grad) == 0).all() and (_host(coeff) == 0).all()


def test_pairs_that_are_no_list_of_pairs_are_refused():
    import torch
    import paper_1906_08879_amd as pl
    x, a, stats = torch.zeros((4, 3), device="cuda:0"), _dev(np.zeros(4, np.int32)), torch.empty(2, device="cuda:0")
    for pairs in (_dev(np.int32(1)), _dev(np.zeros(2, np.int32)), _dev(np.zeros((1, 3), np.int32)), _dev(np.zeros((1, 2), np.int64)),
                  torch.zeros((1, 2), dtype=torch.int32), [[0, 1]]):
        with pytest.raises(pl.PlacetoError):
            pl.preference_loss(x, a, pl.DecisionRows(4, 2), stats, pairs=pairs)

"""The losses in the training loop they are for (examples/tune_policy.py): decisions' weights into the gradient by
replay, against differences of the loss over the parameters; and the loop finds the placement that is known to be best."""
import os
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_gradient_by_replay_against_differences_of_the_loss(loss):
    """Directional derivatives.  The logits are fp32 sums of up to a thousand terms, the loss is good to about 1e-6: with
    steps of 2e-2 of unit length the quotient is good to 1e-4 and to the curvature's share (ReLU kinks among it),
    which a tenth of the gradient's length covers: another sign, scale or a missing term does not."""
    import torch
    import paper_1906_08879_amd as pl
    from examples.tune_policy import Problem
    p, rng = Problem(10, 3, 24, 2.0, 3), np.random.default_rng(5)
    w = p.weights(p.theta)
    start, actions, logits, old, runtime = p.rollouts(w, rng)
    noise = torch.from_numpy(rng.normal(0, 0.05, (p.n, p.B)).astype(np.float32)).to(p.dev)
    adv = torch.from_numpy(rng.normal(0.5, 1, (p.n, p.B)).astype(np.float32)).to(p.dev)
    old, ref = old + noise, old - noise
    rank = runtime.argsort().int()
    pairs = torch.stack([rank[:12], rank[12:]], 1).contiguous()

    def value(theta, **outs):
        w = p.weights(theta)
        z = p.replay_logits(w, start, actions)
        if loss == "policy":
            stats = p.f32(5)
            pl.clipped_policy_loss(z, actions, adv, stats, rows=p.rows, old_logp=old, ref_logp=ref, kl_coeff=0.5, entropy_coeff=0.2,
                                   **outs)
        else:
            stats = p.f32(2)
            pl.preference_loss(z, actions, p.rows, stats, pairs=pairs, ref_logp=ref, beta=0.3, **outs)
        w.close()
        return float(stats[0])

    coeff, ecoeff = p.f32(p.n, p.B), p.f32(p.n, p.B)
    value(p.theta, out_coeff=coeff, **({"out_entropy_coeff": ecoeff} if loss == "policy" else {}))
    grad = -p.policy_gradient(w, start, actions, coeff, ecoeff if loss == "policy" else None).cpu().numpy().astype(np.float64)
    length = np.linalg.norm(grad)
    assert float((p.replay_logits(w, start, actions) - logits).abs().max()) < 1e-4      # the same states as the rollouts'
    h = 2e-2
    for d in (grad / length, *(v / np.linalg.norm(v) for v in rng.normal(0, 1, (3, p.n_par)))):
        up, down = value((p.theta + h * d).astype(np.float32)), value((p.theta - h * d).astype(np.float32))
        slope = (up - down) / (2 * h)
        print(f"[tuning] {loss}: slope {slope:.5f}, by the gradient {grad @ d:.5f}", flush=True)
        assert abs(slope - grad @ d) <= 0.1 * length


def test_example_learns():
    from examples.tune_policy import train
    lines = []
    history = train(nodes=14, devices=3, rollouts=64, rounds=12, preference_rounds=4, say=lambda s: (lines.append(s), print(s, flush=True)))
    assert np.mean(history[:2]) > 1.5 * 14               # a random policy scatters the graph over the devices
    assert np.mean(history[-3:]) <= 1.2 * 14             # the tuned one keeps it together
    assert all(np.isfinite(history)) and len(lines) == 16

"""The gradient of examples/distil_policy.py, weight matrix by weight matrix: of 10020 parameters a random direction sees a hundredth of
the gradient, its own direction little of a single layer."""
import os
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

pytestmark = pytest.mark.gpu


def test_gradient_of_the_example_in_every_layer():
    """Slopes along the gradient of one matrix, or of one layer's biases, alone.  The loss is good to about 1e-6: a quotient over 2 h with h = 1e-2 to 1e-4,
    and the difference of two quotients to 2e-4.  The step's own share in the quotient of h is a third of what it differs by from that of 2 h where the
    loss is smooth; the whole difference is allowed, and a tenth of the layer's gradient for its kinks."""
    import paper_1906_08879_amd as pl
    from examples.distil_policy import Problem, Student, lists, loss_gradient
    from workloads import weight_layout
    p, rng = Problem(10, 4, 24, 2.0, 3), np.random.default_rng(5)
    teacher = p.weights(rng.normal(0.0, 0.4, p.n_par).astype(np.float32))
    w = p.weights(p.theta)
    start, actions, logits, _, _ = p.rollouts(w, rng)
    top, logp = lists(p, teacher, start, actions, 3)
    student, stats = Student(p, p.theta), p.f32(3)
    grad = loss_gradient(p, w, start, actions, logits, top, logp, stats, student.grad).cpu().numpy().astype(np.float64)

    def value(theta):
        w = p.weights(theta.astype(np.float32))
        pl.distill_loss(p.replay_logits(w, start, actions), top, logp, stats, rows=p.rows, tail=False)
        w.close()
        return float(stats[0])

    pos, seen, h = 0, 0, 1e-2
    for name, i, o in weight_layout(p.D, p.H, 2, True):
        for what, begin, end in (("weights", pos, pos + i * o), ("biases", pos + i * o, pos + i * o + o)):
            length = np.linalg.norm(grad[begin:end])
            if length == 0.0:
                continue
            d = np.zeros(p.n_par)
            d[begin:end] = grad[begin:end] / length
            slope, wide = ((value(p.theta + s * d) - value(p.theta - s * d)) / (2 * s) for s in (h, 2 * h))
            print(f"[teaching] {name} {what}: slope {slope:.5f}, over twice the step {wide:.5f}, by the gradient {length:.5f}", flush=True)
            assert abs(slope - length) <= 0.1 * length + abs(slope - wide) + 2e-4, (name, what)
            seen += length > 1e-3
        pos += i * o + o
    assert pos == p.n_par and seen >= 12

"""Fine-tunes a placement policy from recorded rollouts: several updates of the clipped policy loss with a KL term to the
policy it started from, then updates from pairs of rollouts, the faster one preferred.

Everything but the optimiser's step runs on the device: rollouts, simulated run times, the losses over all decisions of
all rollouts at once, the gradient by replay with the decisions' weights that a loss hands out, and its clipping.

    python examples/tune_policy.py [--nodes 14] [--devices 3] [--rollouts 64] [--rounds 12]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1906_08879_amd as pl  # noqa: E402
from workloads import tiny_random_dag, weight_count  # noqa: E402


class Problem:
    """Rollouts of one graph side by side: every operation costs 1, a transfer `transfer` times as much."""

    def __init__(self, nodes, devices, rollouts, transfer, seed, width=16):
        rng = np.random.default_rng(seed)
        src, dst = tiny_random_dag(rng, nodes, 0.25)
        self.n, self.D, self.B, self.H, self.transfer = nodes, devices, rollouts, width, transfer
        self.g = pl.GraphBatch(nodes, len(src), src, dst, replicate=rollouts)
        self.dev = torch.device("cuda")
        self.feats = torch.tensor([[1.0, 1.0, 0.0]], device=self.dev).repeat(rollouts * nodes, 1)
        self.order = torch.arange(nodes, dtype=torch.int32, device=self.dev).repeat(rollouts)
        self.n_par = weight_count(devices, width, 2, True)
        self.theta = rng.normal(0.0, 0.1, self.n_par).astype(np.float32)
        self.rows = pl.DecisionRows(nodes * rollouts, rollouts, "by_step")

    def weights(self, theta):
        return pl.Weights(theta, self.D, self.H, 2, 1, 1, "fp32")

    def f32(self, *shape):
        return torch.empty(shape, dtype=torch.float32, device=self.dev)

    def rollouts(self, w, rng):
        """One episode of every rollout from random placements: the start, every decision and the run times."""
        start = torch.from_numpy(rng.integers(0, self.D, self.B * self.n).astype(np.int32)).to(self.dev)
        feats, place, cur = self.feats.clone(), start.clone(), torch.zeros(self.B, dtype=torch.int32, device=self.dev)
        uniforms = torch.from_numpy(rng.random((self.n, self.B), dtype=np.float32)).to(self.dev)
        actions = torch.empty((self.n, self.B), dtype=torch.int32, device=self.dev)
        logits, logp, runtime = self.f32(self.n, self.B, self.D), self.f32(self.n, self.B), self.f32(self.B)
        pl.episode_run(self.g, w, feats, place, cur, self.order, uniforms, 0, self.n, logits, True, actions, logp)
        pl.simulate_runtime(self.g, self.D, feats, place, self.transfer, runtime)
        return start, actions, logits, logp, runtime

    def replay_logits(self, w, start, actions):
        """Logits [T, B, D] of a policy in the states of recorded rollouts."""
        feats, place = self.feats.clone(), start.clone()
        logits = self.f32(self.n, self.B, self.D)
        base = torch.arange(self.B, device=self.dev) * self.n
        for t in range(self.n):
            cur = self.order.view(self.B, self.n)[:, t].contiguous()
            pl.embed_forward(self.g, feats, place, cur, w, logits[t])
            place[base + cur] = actions[t]
            feats[base + cur, 2] = 1.0
        return logits

    def policy_gradient(self, w, start, actions, coeff, entropy_coeff=None):
        """Minus the gradient of a loss with respect to the parameters, from its decisions' weights."""
        grad, cur = self.f32(self.n_par), torch.zeros(self.B, dtype=torch.int32, device=self.dev)
        pl.episode_gradient(self.g, w, self.feats.clone(), start.clone(), cur, self.order, actions, coeff, 0, self.n, grad,
                            self.f32(self.B, self.D), entropy_coeff=entropy_coeff)
        return grad


class Adam:
    """On the host; parameters ascend along `grad`."""

    def __init__(self, lr, n):
        self.lr, self.t, self.m, self.v = lr, 0, np.zeros(n), np.zeros(n)

    def step(self, theta, grad):
        self.t += 1
        self.m = 0.9 * self.m + 0.1 * grad
        self.v = 0.999 * self.v + 0.001 * grad * grad
        step = self.m / (1 - 0.9 ** self.t) / (np.sqrt(self.v / (1 - 0.999 ** self.t)) + 1e-8)
        return (theta + self.lr * step).astype(np.float32)


def clipped_update(p, theta, adam, reference, rollout, epochs=4, max_norm=1.0):
    """`epochs` updates from one set of rollouts."""
    start, actions, logits, old, runtime = rollout
    reward = torch.zeros((p.n, p.B), device=p.dev)
    reward[-1] = -runtime                                    # the run time is known at the end
    group = torch.zeros(p.B, dtype=torch.int32, device=p.dev)
    advantage, baseline = p.f32(p.n, p.B), p.f32(p.n, 1)
    pl.reinforce_coeff(reward, group, 1, advantage, baseline)
    advantage /= advantage.std() + 1e-6
    ref = p.f32(p.n, p.B)
    pl.action_logp(p.replay_logits(reference, start, actions), actions, ref)
    stats, norm, coeff, entropy_coeff = p.f32(5), p.f32(1), p.f32(p.n, p.B), p.f32(p.n, p.B)
    for epoch in range(epochs):
        w = p.weights(theta)
        if epoch:                                            # the rollouts' own logits are those of the first update
            logits = p.replay_logits(w, start, actions)
        pl.clipped_policy_loss(logits, actions, advantage, stats, rows=p.rows, old_logp=old, ref_logp=ref, kl_coeff=0.02,
                               entropy_coeff=0.01, out_coeff=coeff, out_entropy_coeff=entropy_coeff)
        grad = p.policy_gradient(w, start, actions, coeff, entropy_coeff)
        pl.clip_gradients([grad], max_norm, norm)
        theta = adam.step(theta, grad.cpu().numpy())
        w.close()
    return theta, stats, norm


def preference_update(p, theta, adam, reference, rollout, max_norm=1.0):
    """One update: the faster half of the rollouts against the slower half."""
    start, actions, logits, _, runtime = rollout
    rank = runtime.argsort().int()
    pairs = torch.stack([rank[:p.B // 2], rank[p.B // 2:2 * (p.B // 2)]], 1).contiguous()
    ref = p.f32(p.n, p.B)
    pl.action_logp(p.replay_logits(reference, start, actions), actions, ref)
    stats, norm, coeff = p.f32(2), p.f32(1), p.f32(p.n, p.B)
    pl.preference_loss(logits, actions, p.rows, stats, pairs=pairs, ref_logp=ref, beta=0.2, out_coeff=coeff)
    w = p.weights(theta)
    grad = p.policy_gradient(w, start, actions, coeff)
    pl.clip_gradients([grad], max_norm, norm)
    theta = adam.step(theta, grad.cpu().numpy())
    w.close()
    return theta, stats, norm


def train(nodes=14, devices=3, rollouts=64, rounds=12, preference_rounds=4, transfer=5.0, seed=0, say=print):
    """Mean run times of the rounds' rollouts."""
    p, rng = Problem(nodes, devices, rollouts, transfer, seed), np.random.default_rng(seed + 1)
    theta, reference, history = p.theta, p.weights(p.theta), []
    adam = Adam(0.02, p.n_par)
    for i in range(rounds + preference_rounds):
        w = p.weights(theta)
        rollout = p.rollouts(w, rng)
        w.close()
        if i < rounds:
            theta, stats, norm = clipped_update(p, theta, adam, reference, rollout)
            what = "clipped policy loss {:.4f}, KL {:.4f}, clipped {:.0%}".format(*stats[[0, 2, 4]].tolist())
        else:
            theta, stats, norm = preference_update(p, theta, adam, reference, rollout)
            what = "preference loss {:.4f}, in order {:.0%}".format(*stats.tolist())
        history.append(float(rollout[4].mean()))
        say(f"round {i}: mean run time {history[-1]:.2f} (one device: {nodes}), {what}, gradient norm {float(norm):.3f}")
    return history


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--nodes", type=int, default=14)
    ap.add_argument("--devices", type=int, default=3)
    ap.add_argument("--rollouts", type=int, default=64)
    ap.add_argument("--rounds", type=int, default=12)
    a = ap.parse_args()
    train(a.nodes, a.devices, a.rollouts, a.rounds)

"""Timed cases of the operators on rows of logits and on gradients: what a program that scores,
trains or fine-tunes a policy asks of them, from one 32-step episode on two devices to batches of
tokens over a large vocabulary.

Operators (`op` of a case):
  logp        log probabilities of given actions (tokens) under rows of logits, with the entropies
  policy      clipped policy loss with a KL and an entropy term: its value and the gradient of the logits
  preference  loss of paired log ratios over sequences: value, margins and the gradient of the logits
  clip        norm over all gradients of a model and the clipped gradients

Rows are decisions.  `order` says how the rows of `seqs` sequences lie: "by_step" [steps, seqs] as an
episode over a batch of graphs records them, "by_seq" [seqs, steps] as a padded batch of texts,
"packed" one sequence behind the other with offsets.  `ragged`: the sequences end at different steps;
`prompt`: the first rows of every sequence are not scored (a mask).
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
CLIP_LOW, CLIP_HIGH, KL, ENTROPY = 0.2, 0.25, 0.05, 0.01
BETA = 0.1
GRAD_SCALE = {"fp32": 1.0, "bf16": 1.0, "fp16": 1024.0}      # half precision trains with scaled gradients


# --------------------------------------------------------------------------- cases
def _logp(name, rows, actions, dtype, entropy=False, pad=0):
    return dict(name=name, op="logp", rows=rows, actions=actions, dtype=dtype, entropy=entropy, pad=pad)


def _policy(name, order, seqs, steps, actions, dtype, ragged=False, prompt=False, kl=False, entropy=False,
            reduction="rows", by_seq_advantage=False):
    return dict(name=name, op="policy", order=order, seqs=seqs, steps=steps, actions=actions, dtype=dtype, ragged=ragged,
                prompt=prompt, kl=kl, entropy=entropy, reduction=reduction, by_seq_advantage=by_seq_advantage, pad=0)


def _preference(name, order, seqs, steps, actions, dtype, pairs=0, ragged=False, prompt=False, average=False,
                smoothing=0.0):
    return dict(name=name, op="preference", order=order, seqs=seqs, steps=steps, actions=actions, dtype=dtype, pairs=pairs,
                ragged=ragged, prompt=prompt, average=average, smoothing=smoothing, pad=0)


def _clip(name, tensors, width, numel, dtype, exceeds=True):
    return dict(name=name, op="clip", tensors=tensors, width=width, numel=numel, dtype=dtype, exceeds=exceeds)


def listed():
    return [
        # one token of one running request over a large vocabulary: the time of a call is all there is
        _logp("logp_token_131072", 1, 131072, "bf16"),
        # one step of a batch of requests, odd vocabulary, rows of a buffer that is padded behind them
        _logp("logp_requests_37x50001", 37, 50001, "fp16", entropy=True, pad=15),
        # scoring recorded tokens under a frozen reference policy
        _logp("logp_score_8192x32768", 8192, 32768, "bf16"),
        # the smallest training call: the 32 decisions of one episode on two devices
        _policy("policy_random_32x2", "by_step", 1, 32, 2, "fp32", entropy=True),
        # 256 rollouts of three-thousand-node graphs on eight devices, all steps at once, graphs of unequal size
        _policy("policy_nasnet_800000x8", "by_step", 256, 3124, 8, "fp32", ragged=True, kl=True, entropy=True),
        # fine-tuning on sampled texts of unequal length behind one another, odd vocabulary, KL to the reference,
        # one advantage per text, every text with equal weight
        _policy("policy_texts_4096x50001", "packed", 24, 171, 50001, "bf16", prompt=True, kl=True, reduction="seqs",
                by_seq_advantage=True),
        # the largest: a padded batch over a large vocabulary, with the entropy term
        _policy("policy_batch_8192x65536", "by_seq", 16, 512, 65536, "bf16", ragged=True, prompt=True, entropy=True),
        # a better and a worse placement of a 200-node graph on four devices, 32 such pairs
        _preference("preference_layered_64x200x4", "by_step", 64, 200, 4, "fp32"),
        # eight rollouts of every graph, compared with one another by their run times: a rollout is in many pairs
        _preference("preference_rollouts_128x600x4", "by_step", 128, 600, 4, "fp32", pairs=448, ragged=True, smoothing=0.1),
        # pairs of texts behind one another over a vocabulary, prompts not scored
        _preference("preference_texts_6144x32768", "packed", 24, 256, 32768, "bf16", prompt=True),
        # the gradient of a whole policy network is one block of floats (four devices, 64 columns)
        _clip("clip_blob_153732", 1, 0, 153732, "fp32"),
        # the gradients of a model of many tensors, matrices in bf16 and vectors in fp32
        _clip("clip_model_291", 291, 4097, 240000000, "mixed"),
    ]


def draw(rng):
    def over(lo, hi):                                    # spread over the logarithm, odd sizes among them
        return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))

    op = rng.choice(("logp", "policy", "policy", "preference", "clip"))
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    if op == "logp":
        actions = over(2, 131072)
        return _drop_name(_logp(None, over(1, max(1, min(1000000, 2 ** 27 // actions))), actions, dtype,
                                entropy=rng.random() < 0.5, pad=rng.choice((0, 0, 1, 16))))
    if op == "clip":
        tensors = rng.choice((1, over(2, 400)))
        width = over(1, 8192) if tensors > 1 else 0
        return _drop_name(_clip(None, tensors, width, over(max(64, tensors * (width + 1)), 200000000),
                                rng.choice(("fp32", "bf16", "mixed")), exceeds=rng.random() < 0.7))
    order = rng.choice(("by_step", "by_seq", "packed"))
    wide = rng.random() < 0.6
    actions = over(17, 131072) if wide else rng.randint(1, 16)
    if not wide:
        dtype = rng.choice(("fp32", dtype))
    seqs = over(2, 256)
    seqs += seqs % 2
    rows = max(seqs, over(seqs, max(seqs, min(600000, 2 ** 27 // actions))))
    common = dict(order=order, seqs=seqs, steps=max(1, rows // seqs), actions=actions, dtype=dtype,
                  ragged=rng.random() < 0.5, prompt=rng.random() < 0.4)
    if op == "preference":
        case = _preference(None, pairs=rng.choice((0, over(1, 1000))), average=rng.random() < 0.3,
                           smoothing=rng.choice((0.0, 0.1)), **common)
    else:
        case = _policy(None, kl=rng.random() < 0.5, entropy=rng.random() < 0.5, reduction=rng.choice(("rows", "seqs")),
                       by_seq_advantage=rng.random() < 0.3, **common)
    case["pad"] = rng.choice((0, 0, 8))
    return _drop_name(case)


def _drop_name(case):
    del case["name"]
    return case


def _numels(case):
    """Sizes of a model's tensors: every third a vector, the rest matrices of three sizes."""
    n, width, total = case["tensors"], case["width"], case["numel"]
    if n == 1:
        return [total]
    vectors = n // 3
    rest, parts = total - vectors * width, [1 + i % 3 for i in range(n - vectors)]
    unit, matrices = rest // sum(parts), []
    for p in parts:
        matrices.append(max(1, unit * p))
    matrices[0] = max(1, rest - sum(matrices[1:]))
    out = []
    for i in range(n):
        out.append(width if i % 3 == 2 and vectors else matrices.pop())
        vectors -= i % 3 == 2 and vectors > 0
    return out


# --------------------------------------------------------------------------- inputs
def _chunks(n_rows, n_actions, elements=2 ** 25):
    step = max(1, elements // n_actions)
    return [(i, min(n_rows, i + step)) for i in range(0, n_rows, step)]


def _scored(x, actions):
    """log probabilities of the actions, a chunk of rows at a time."""
    out = torch.empty(len(actions), device=x.device)
    for i, j in _chunks(*x.shape):
        z = x[i:j].double()
        out[i:j] = (z.gather(1, actions[i:j, None].long())[:, 0] - torch.logsumexp(z, 1)).float()
    return out


def _decisions(case, rows, gen):
    """Logits with one favoured action a row, and actions of which most are the favoured one."""
    dev, V = torch.device("cuda"), case["actions"]
    logits = torch.empty((rows, V + case["pad"]), dtype=DTYPE[case["dtype"]], device=dev)[:, :V]
    favoured = torch.randint(V, (rows,), generator=gen, device=dev)
    other = torch.randint(V, (rows,), generator=gen, device=dev)
    lift = math.log(V) * torch.rand(rows, generator=gen, device=dev) * 1.2
    for i, j in _chunks(rows, V):
        z = torch.randn((j - i, V), generator=gen, device=dev)
        z.scatter_add_(1, favoured[i:j, None], lift[i:j, None])
        logits[i:j] = z
    take = torch.rand(rows, generator=gen, device=dev) < 0.7
    return logits, torch.where(take, favoured, other).int()


def _bucket(grads, fill=None):
    """One flat buffer for the gradients of each type, as reductions over ranks take them, every tensor at a multiple of
    64 elements; the views of the tensors in it, with values where `fill` gives them."""
    flat, views = {}, []
    for t in dict.fromkeys(g.dtype for g in grads):
        flat[str(t)] = torch.zeros(sum(-(-g.numel() // 64) * 64 for g in grads if g.dtype == t), dtype=t, device=grads[0].device)
    at = dict.fromkeys(flat, 0)
    for i, g in enumerate(grads):
        k = str(g.dtype)
        views.append(flat[k][at[k]:at[k] + g.numel()])
        at[k] += -(-g.numel() // 64) * 64
        if fill is not None:
            views[-1].copy_(fill(g))
    return flat, views


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    if case["op"] == "clip":
        numels = _numels(case)
        kind = [case["dtype"] if case["dtype"] != "mixed" else ("fp32" if n == case["width"] else "bf16") for n in numels]
        size = torch.exp(torch.randn(len(numels), generator=gen, device=dev)).tolist()
        grads = [(torch.randn(n, generator=gen, device=dev) * (s * 1e-3)).to(DTYPE[k]) for n, s, k in zip(numels, size, kind)]
        norm = 1e-3 * math.sqrt(sum(n * s * s for n, s in zip(numels, size)))
        flat, clipped = _bucket(grads)
        # gradients some four times as long as allowed, or shorter than that
        return dict(case=case, grads=grads, max_norm=norm * (0.25 if case["exceeds"] else 2.0), flat=flat, clipped=clipped,
                    norm=torch.empty(1, device=dev))
    if case["op"] == "logp":
        logits, actions = _decisions(case, case["rows"], gen)
        return dict(case=case, logits=logits, actions=actions, logp=torch.empty(case["rows"], device=dev),
                    entropy=torch.empty(case["rows"], device=dev))
    S, steps = case["seqs"], case["steps"]
    N = S * steps
    bounds = mask = None
    if case["order"] == "packed":
        cuts = torch.randint(N + 1, (S - 1,), generator=gen, device=dev).sort().values
        even = torch.arange(1, S, device=dev) * steps
        cuts = cuts if case["ragged"] else (cuts + 3 * even) // 4           # lengths within a factor of about two, or any
        bounds = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), N)]).int()
        first = bounds[:-1].repeat_interleave(bounds.diff())
        step = torch.arange(N, device=dev) - first
        length = bounds.diff().repeat_interleave(bounds.diff())
    else:
        length = torch.full((S,), steps, device=dev)
        if case["ragged"]:
            length = steps - (torch.rand(S, generator=gen, device=dev) * (0.5 * steps)).long()
            bounds = length.int()
        n = torch.arange(N, device=dev)
        step = n // S if case["order"] == "by_step" else n % steps
        length = length[n % S if case["order"] == "by_step" else n // steps]
    if case["prompt"]:
        mask = (step >= length // 4).to(torch.uint8)
    logits, actions = _decisions(case, N, gen)
    logp = _scored(logits, actions)
    s = dict(case=case, logits=logits, actions=actions, bounds=bounds, mask=mask, grad=torch.empty_like(logits),
             logp=torch.empty(N, device=dev), coeff=torch.empty(N, device=dev))
    # the rows that each of these says something about are the scored ones; the rest stays as a buffer may be
    ref = logp - 0.2 * torch.randn(N, generator=gen, device=dev)
    if case["op"] == "preference":
        s.update(ref=ref, stats=torch.empty(2, device=dev), seq_logp=torch.empty(S, device=dev), pairs=None,
                 margins=torch.empty(case["pairs"] or S // 2, device=dev))
        if case["pairs"]:
            a = torch.randint(S, (case["pairs"],), generator=gen, device=dev)
            b = (a + torch.randint(1, max(2, S), (case["pairs"],), generator=gen, device=dev)) % S
            s["pairs"] = torch.stack([a, b], 1).int().contiguous()
        return s
    # ratios of the updated policy to the one that sampled; none within a thousandth of the edges, where the gradient jumps
    shift = 0.15 * torch.randn(N, generator=gen, device=dev)
    for edge in (math.log(1.0 - CLIP_LOW), math.log(1.0 + CLIP_HIGH)):
        shift = torch.where((shift - edge).abs() < 1e-3, shift + 4e-3, shift)
    s.update(old=logp - shift, ref=ref if case["kl"] else None, stats=torch.empty(5, device=dev),
             advantage=torch.randn(S if case["by_seq_advantage"] else N, generator=gen, device=dev),
             entropy_coeff=torch.empty(N, device=dev))
    return s


# --------------------------------------------------------------------------- plain forms
def _layout(s):
    """(sequence of every row, truth value: the row counts)"""
    case, N = s["case"], len(s["actions"])
    S, n = case["seqs"], torch.arange(N, device=s["actions"].device)
    if case["order"] == "packed":
        seq = torch.searchsorted(s["bounds"][1:].contiguous(), n.int(), right=True).clamp(max=S - 1)
        counts = n < s["bounds"][-1]
    else:
        seq, step = (n % S, n // S) if case["order"] == "by_step" else (n // case["steps"], n % case["steps"])
        counts = step < s["bounds"][seq] if s["bounds"] is not None else torch.ones_like(n, dtype=torch.bool)
    if s["mask"] is not None:
        counts = counts & (s["mask"] != 0)
    return seq, counts


def _softmax_parts(logits, actions):
    """log probabilities [N, V] and those of the actions, in 32 bits."""
    x = logits.float()
    x = x - x.amax(1, keepdim=True)
    logp = x - x.exp().sum(1, keepdim=True).log()
    return logp, logp.gather(1, actions.long()[:, None])[:, 0]


def _entropy(logp):
    return -(logp.exp() * logp).sum(1)


def _gradient(logits, logp_all, actions, d_logp, d_entropy=None, entropy=None):
    p = logp_all.exp()
    g = -p * d_logp[:, None]
    if d_entropy is not None:
        g -= d_entropy[:, None] * p * (logp_all + entropy[:, None])
    g.scatter_add_(1, actions.long()[:, None], d_logp[:, None])
    return g.to(logits.dtype)


def _plain_logp(s):
    every, logp = _softmax_parts(s["logits"], s["actions"])
    return {"logp": logp, "entropy": _entropy(every)} if s["case"]["entropy"] else {"logp": logp}


def _plain_policy(s):
    case = s["case"]
    seq, counts = _layout(s)
    if case["reduction"] == "seqs":
        length = torch.zeros(case["seqs"], device=seq.device).index_add_(0, seq, counts.float())
        w = 1.0 / (length[seq].clamp(min=1.0) * (length > 0).sum().clamp(min=1))
    else:
        w = 1.0 / counts.sum().clamp(min=1).float()
    w = torch.where(counts, w, 0.0)
    every, logp = _softmax_parts(s["logits"], s["actions"])
    adv = s["advantage"][seq] if case["by_seq_advantage"] else s["advantage"]
    ratio = (logp - s["old"]).exp()
    cut = torch.where(adv > 0, ratio > 1.0 + CLIP_HIGH, ratio < 1.0 - CLIP_LOW) & (adv != 0)
    surrogate = -adv * torch.where(cut, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH), ratio)
    d_logp = torch.where(cut, 0.0, -adv * ratio)
    kl = torch.zeros_like(logp)
    if case["kl"]:
        d = s["ref"] - logp
        kl = d.exp() - d - 1.0
        d_logp = d_logp + KL * (1.0 - d.exp())
    scale = GRAD_SCALE[case["dtype"]]
    d_logp = torch.where(counts, scale * w * d_logp, 0.0)
    entropy = _entropy(every)
    gamma = ENTROPY if case["entropy"] else 0.0
    d_entropy = -scale * gamma * w
    mean = [torch.where(counts, w * v, 0.0).sum() for v in (surrogate, kl, entropy, cut.float())]
    grad = _gradient(s["logits"], every, s["actions"], d_logp, d_entropy if case["entropy"] else None, entropy)
    out = {"stats": torch.stack([mean[0] + (KL if case["kl"] else 0.0) * mean[1] - gamma * mean[2], *mean]),
           "grad": grad, "logp": torch.where(counts, logp, 0.0)}
    if case["order"] == "by_step":
        out.update(coeff=-d_logp, entropy_coeff=-d_entropy)
    return out


def _pairs(s):
    if s["pairs"] is not None:
        return s["pairs"][:, 0].long(), s["pairs"][:, 1].long()
    even = torch.arange(0, s["case"]["seqs"], 2, device=s["actions"].device)
    return even, even + 1


def _plain_preference(s):
    case = s["case"]
    S, eps = case["seqs"], case["smoothing"]
    seq, counts = _layout(s)
    every, logp = _softmax_parts(s["logits"], s["actions"])
    add = lambda v: torch.zeros(S, device=seq.device).index_add_(0, seq, torch.where(counts, v, 0.0))  # noqa: E731
    total, ratio, weight = add(logp), add(logp - s["ref"]), torch.ones(S, device=seq.device)
    if case["average"]:
        weight = 1.0 / add(torch.ones_like(logp)).clamp(min=1.0)
    better, worse = _pairs(s)
    ratio = weight * ratio
    margin = BETA * (ratio[better] - ratio[worse])
    soft = lambda x: x.clamp(min=0.0) + (-x.abs()).exp().log1p()  # noqa: E731
    loss = ((1.0 - eps) * soft(-margin) + eps * soft(margin)).mean()
    d_margin = (eps / (1.0 + (-margin).exp()) - (1.0 - eps) / (1.0 + margin.exp())) / len(margin)
    d_ratio = torch.zeros(S, device=seq.device).index_add_(0, better, BETA * d_margin).index_add_(0, worse, -BETA * d_margin)
    d_logp = torch.where(counts, GRAD_SCALE[case["dtype"]] * (d_ratio * weight)[seq], 0.0)
    out = {"stats": torch.stack([loss, (margin > 0).float().mean()]), "margins": margin, "seq_logp": weight * total,
           "grad": _gradient(s["logits"], every, s["actions"], d_logp)}
    if case["order"] == "by_step":
        out.update(coeff=-d_logp)
    return out


def _plain_clip(s):
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    return {"norm": norm.reshape(1), **_bucket(s["grads"], lambda g: g.float() * scale)[0]}


# --------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if not own:
        return {"logp": _plain_logp, "policy": _plain_policy, "preference": _plain_preference, "clip": _plain_clip}[case["op"]](s)
    import paper_1906_08879_amd as pl
    if case["op"] == "logp":
        pl.action_logp(s["logits"], s["actions"], s["logp"], s["entropy"] if case["entropy"] else None)
        return {"logp": s["logp"], "entropy": s["entropy"]} if case["entropy"] else {"logp": s["logp"]}
    if case["op"] == "clip":
        pl.clip_gradients(s["grads"], s["max_norm"], s["norm"], out=s["clipped"])
        return {"norm": s["norm"], **s["flat"]}
    rows = pl.DecisionRows(len(s["actions"]), case["seqs"], case["order"], bounds=s["bounds"], mask=s["mask"])
    episodes = case["order"] == "by_step"                    # the weights that episode_gradient takes
    out = {"stats": s["stats"], "grad": s["grad"]}
    if case["op"] == "policy":
        pl.clipped_policy_loss(s["logits"], s["actions"], s["advantage"], s["stats"], rows=rows, old_logp=s["old"],
                               ref_logp=s["ref"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coeff=KL if case["kl"] else 0.0,
                               entropy_coeff=ENTROPY if case["entropy"] else 0.0, reduction=case["reduction"],
                               advantage_per_sequence=case["by_seq_advantage"], grad_scale=GRAD_SCALE[case["dtype"]], out_grad=s["grad"], out_logp=s["logp"],
                               out_coeff=s["coeff"] if episodes else None,
                               out_entropy_coeff=s["entropy_coeff"] if episodes else None)
        out["logp"] = s["logp"]
        if episodes:
            out.update(coeff=s["coeff"], entropy_coeff=s["entropy_coeff"])
        return out
    pl.preference_loss(s["logits"], s["actions"], rows, s["stats"], pairs=s["pairs"], ref_logp=s["ref"], beta=BETA,
                       label_smoothing=case["smoothing"], average=case["average"],
                       grad_scale=GRAD_SCALE[case["dtype"]], out_grad=s["grad"], out_margins=s["margins"], out_seq_logp=s["seq_logp"], out_coeff=s["coeff"] if episodes else None)
    out.update(margins=s["margins"], seq_logp=s["seq_logp"])
    if episodes:
        out["coeff"] = s["coeff"]
    return out


def work(case):
    """Every input read once, every output written once.  Operations of a logit: its share of the maximum, the exponent
    and the sum (and of the entropy), and of the gradient the exponent and a product."""
    if case["op"] == "clip":
        numels = _numels(case)
        wide = sum(n for n in numels if n == case["width"])
        per = {"fp32": 4.0, "bf16": 2.0, "fp16": 2.0}
        size = per[case["dtype"]] * sum(numels) if case["dtype"] != "mixed" else 4.0 * wide + 2.0 * (sum(numels) - wide)
        return {"bytes": 2.0 * size + 4.0, "flops": 3.0 * sum(numels)}
    elem = 4.0 if case["dtype"] == "fp32" else 2.0
    V = case["actions"]
    if case["op"] == "logp":
        N = case["rows"]
        return {"bytes": N * (elem * V + 8.0 + 4.0 * case["entropy"]), "flops": N * V * (4.0 + 2.0 * case["entropy"])}
    N, S = case["seqs"] * case["steps"], case["seqs"]
    rows = 4.0 + 1.0 * case["prompt"] + 4.0 * (case["order"] == "by_step")         # actions, mask, weights of the decisions
    if case["op"] == "policy":
        rows += 4.0 + 4.0 * (not case["by_seq_advantage"]) + 4.0 * case["kl"] + 4.0 + 4.0 * (case["order"] == "by_step")
        return {"bytes": N * (2.0 * elem * V + rows) + 4.0 * S + 20.0, "flops": N * V * (8.0 + 4.0 * case["entropy"])}
    pairs = case["pairs"] or S // 2
    return {"bytes": N * (2.0 * elem * V + rows + 4.0) + 8.0 * S + 12.0 * pairs, "flops": N * V * 8.0 + 20.0 * pairs}


# --------------------------------------------------------------------------- from the definitions, in 64 bits
def _row_weights(s):
    """Sequence and weight of every row, from the lists of the sequences' rows."""
    case, dev = s["case"], s["actions"].device
    S, steps, N = case["seqs"], case["steps"], len(s["actions"])
    ends = s["bounds"].tolist() if s["bounds"] is not None else None
    seq = torch.zeros(N, dtype=torch.long, device=dev)
    keep = torch.zeros(N, dtype=torch.float64, device=dev)
    for q in range(S):
        if case["order"] == "packed":
            at = slice(ends[q], ends[q + 1])
            seq[at], keep[at] = q, 1.0
        else:
            n = steps if ends is None else ends[q]
            a, b, d = (q, N, S) if case["order"] == "by_step" else (q * steps, (q + 1) * steps, 1)
            seq[a:b:d] = q
            keep[a:a + n * d:d] = 1.0
    if s["mask"] is not None:
        keep *= s["mask"].double()
    return seq, keep


def _by_autograd(s, value, d_rows=None):
    """Values of all rows by `value(log-softmax of a chunk, slice)`, and the gradient of their sum
    (or of the given multiples of them) with respect to the logits."""
    x, vals = s["logits"], []
    grad = torch.empty(x.shape, dtype=torch.float64 if x.numel() < 2 ** 27 else torch.float32, device=x.device)
    for i, j in _chunks(*x.shape, elements=2 ** 24):
        z = x[i:j].double().requires_grad_(True)
        v = value(torch.log_softmax(z, 1), slice(i, j))
        (v[0] if d_rows is None else (v[0] * d_rows[i:j]).sum()).backward()
        grad[i:j] = z.grad.to(grad.dtype)
        vals.append([t.detach() for t in v])
    return [torch.stack(c).sum(0) if c[0].dim() == 0 else torch.cat(c) for c in zip(*vals)], grad


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s["grads"]))
        f = min(1.0, s["max_norm"] / norm)
        flat = {k: v.to(torch.float32 if v.numel() > 2 ** 24 else torch.float64) for k, v in s["flat"].items()}
        for k, v in flat.items():
            at = 0
            for g in s["grads"]:
                if str(g.dtype) == k:
                    v[at:at + g.numel()] = g.double() * f
                    at += -(-g.numel() // 64) * 64
        return {"norm": torch.tensor([norm], dtype=torch.float64), **flat}
    pick = lambda lp, at: lp.gather(1, s["actions"][at].long()[:, None])[:, 0]  # noqa: E731
    if case["op"] == "logp":
        logp, ent = [], []
        for i, j in _chunks(*s["logits"].shape, elements=2 ** 24):
            lp = torch.log_softmax(s["logits"][i:j].double(), 1)
            logp.append(pick(lp, slice(i, j)))
            ent.append(torch.special.entr(lp.exp()).sum(1))
        out = {"logp": torch.cat(logp)}
        return dict(out, entropy=torch.cat(ent)) if case["entropy"] else out
    seq, keep = _row_weights(s)
    count = torch.zeros(case["seqs"], dtype=torch.float64, device=seq.device).index_add(0, seq, keep)
    up = GRAD_SCALE[case["dtype"]]
    if case["op"] == "policy":
        if case["reduction"] == "seqs":
            w = keep / count[seq].clamp(min=1.0) / max(1, int((count > 0).sum()))
        else:
            w = keep / max(1.0, float(keep.sum()))
        adv = (s["advantage"][seq] if case["by_seq_advantage"] else s["advantage"]).double()
        beta, gamma = (KL if case["kl"] else 0.0), (ENTROPY if case["entropy"] else 0.0)
        d_logp = torch.empty_like(w)

        def value(lp, at):
            mine = pick(lp, at)
            leaf = mine.detach().requires_grad_(True)

            def parts(l):
                r = torch.exp(l - s["old"][at].double())
                held = torch.clamp(r, 1.0 - CLIP_LOW, 1.0 + CLIP_HIGH)
                sur = -torch.minimum(r * adv[at], held * adv[at])
                kl = torch.zeros_like(l)
                if case["kl"]:
                    d = s["ref"][at].double() - l
                    kl = torch.expm1(d) - d
                return sur, kl, (held * adv[at] < r * adv[at]).double()

            sur, kl, _ = parts(leaf)
            (w[at] * (sur + beta * kl)).sum().backward()
            d_logp[at] = leaf.grad
            sur, kl, cut = parts(mine)
            ent = -(lp.exp() * lp).sum(1)
            mean = [(w[at] * t).sum() for t in (sur, kl, ent, cut)]
            return [mean[0] + beta * mean[1] - gamma * mean[2], *mean, mine * (keep[at] > 0)]

        (loss, sur, kl, ent, cut, logp), grad = _by_autograd(s, value)
        grad *= up
        out = {"stats": torch.stack([loss, sur, kl, ent, cut]), "grad": grad, "logp": logp}
        return dict(out, coeff=-up * d_logp, entropy_coeff=up * gamma * w) if case["order"] == "by_step" else out
    per = 1.0 / count.clamp(min=1.0) if case["average"] else torch.ones_like(count)
    logp = torch.cat([pick(torch.log_softmax(s["logits"][i:j].double(), 1), slice(i, j))
                      for i, j in _chunks(*s["logits"].shape, elements=2 ** 24)])
    total = torch.zeros_like(count).index_add(0, seq, keep * logp).requires_grad_(True)
    ref = torch.zeros_like(count).index_add(0, seq, keep * s["ref"].double())
    a, b = (s["pairs"][:, 0].long(), s["pairs"][:, 1].long()) if s["pairs"] is not None else (
        torch.arange(0, case["seqs"], 2, device=seq.device), torch.arange(1, case["seqs"], 2, device=seq.device))
    ratio = (total - ref) * per
    margin = BETA * (ratio[a] - ratio[b])
    loss = -((1.0 - case["smoothing"]) * torch.nn.functional.logsigmoid(margin)
             + case["smoothing"] * torch.nn.functional.logsigmoid(-margin)).mean()
    loss.backward()
    d_logp = up * total.grad[seq] * keep
    _, grad = _by_autograd(s, lambda lp, at: [pick(lp, at)], d_logp)
    out = {"stats": torch.stack([loss.detach(), (margin > 0).double().mean()]), "margins": margin.detach(),
           "seq_logp": (total * per).detach(), "grad": grad}
    return dict(out, coeff=-d_logp) if case["order"] == "by_step" else out

"""Timed cases of the trainer's operators, through the Python entry points.

The gate and the advantages say which rollouts a step learns from and how much; these operators are what the
trainer then does with them on the GPU.  Each case is one of five things:

``logprob``  log-probabilities of the tokens that were taken, from logits (``sr_token_logprob``): the scoring pass
             under the old or the reference policy, or of the tokens of one decoding step.
``grad``     its backward pass (``sr_token_logprob_backward``).
``policy``   per-rollout weights and the clipped policy loss with its KL term and gradient, from log-probabilities
             (``sr_loss_weights``, ``sr_policy_loss``).
``step``     the same loss from logits, with the gradient of the logits (``sr_policy_loss_logits``).
``clip``     the global norm of all gradients, and their clipping (``sr_grad_norm``, ``sr_clip_grads``).

Vocabularies are those of the repository's workloads (4096 actions, 151 936 tokens) or generic.  Logits are those of
a trained model: a broad floor with a few likely tokens a row, of which the taken one usually is one.  Old
log-probabilities are those of a policy a few updates older, the reference's of one further away.
"""
import math

import torch

own = False             # set from outside: the plain forms, or the framework's entry points

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
MODES = {"sum": 0, "token": 1, "rollout": 2}
MOST_LOGITS = {"logprob": 4096 * 151936 * 2, "grad": 2048 * 151936 * 2, "step": 4096 * 151936 * 2}   # bytes of logits
MOST_TOKENS = 1024 * 8 * 640
MOST_GRADS = 1 << 31    # bytes of gradients


def listed():
    return [
        # the tokens that the eight rollouts of one group have just sampled, with the entropies a log shows
        {"name": "score-step", "kind": "logprob", "T": 8, "V": 151936, "pad": 0, "dtype": "bf16", "tau": 0.7, "masked": 0.0, "banned": 0, "entropy": True},
        # a chunk of rollouts under the reference policy; a quarter of the tokens are observations, not actions
        {"name": "score-rollouts", "kind": "logprob", "T": 4096, "V": 151936, "pad": 0, "dtype": "bf16", "tau": 1.0, "masked": 0.25, "banned": 0, "entropy": False},
        # an odd vocabulary in a padded buffer, its last tokens banned
        {"name": "score-odd", "kind": "logprob", "T": 601, "V": 50021, "pad": 3, "dtype": "f16", "tau": 1.0, "masked": 0.1, "banned": 500, "entropy": True},
        # action-level policy head
        {"name": "grad-actions", "kind": "grad", "T": 240, "V": 4096, "pad": 0, "dtype": "f32", "tau": 1.0, "masked": 0.0, "banned": 0, "entropy": False},
        # a chunk of rollouts with an entropy bonus
        {"name": "grad-rollouts", "kind": "grad", "T": 2048, "V": 151936, "pad": 0, "dtype": "bf16", "tau": 1.0, "masked": 0.25, "banned": 0, "entropy": True},
        # the paper's iteration at action level: 10 prompts x 8 rollouts of up to 30 actions
        {"name": "policy-actions", "kind": "policy", "groups": 10, "N": 8, "shortest": 1, "longest": 30, "masked": 0.0, "cut": 0.2, "ref": True, "mode": "rollout", "beta": 0.02},
        # odd sizes, no reference policy
        {"name": "policy-odd", "kind": "policy", "groups": 301, "N": 5, "shortest": 0, "longest": 1023, "masked": 0.3, "cut": 0.2, "ref": False, "mode": "token", "beta": 0.0},
        # the rollouts of the repository's benchmark batch
        {"name": "policy-tokens", "kind": "policy", "groups": 1024, "N": 8, "shortest": 256, "longest": 1024, "masked": 0.25, "cut": 0.2, "ref": True, "mode": "token", "beta": 0.02},
        # the paper's iteration at action level, from the policy head's logits
        {"name": "step-actions", "kind": "step", "T": 1200, "V": 4096, "pad": 0, "dtype": "f32", "tau": 1.0, "masked": 0.0, "banned": 0, "groups": 10, "N": 8, "cut": 0.2, "ref": True, "beta": 0.02},
        # a chunk of rollouts of a language model
        {"name": "step-rollouts", "kind": "step", "T": 4096, "V": 151936, "pad": 0, "dtype": "bf16", "tau": 1.0, "masked": 0.25, "banned": 0, "groups": 1, "N": 8, "cut": 0.0, "ref": True, "beta": 0.02},
        # gradients of low-rank adapters, 14 matrices a layer
        {"name": "clip-adapters", "kind": "clip", "layers": 28, "width": 2048, "rank": 16, "vocab": 0, "dtype": "f32", "clipped": True},
        # gradients of a whole model
        {"name": "clip-weights", "kind": "clip", "layers": 14, "width": 2048, "rank": 0, "vocab": 151936, "dtype": "bf16", "clipped": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["logprob", "grad", "policy", "step", "clip"])
    if kind == "policy":
        N = rng.choice([8, 16, 4, rng.randint(2, 32)])
        longest = _log_int(rng, 8, 4000)
        shortest = rng.choice([0, 1, longest // 4, longest])
        groups = _log_int(rng, 2, max(4, min(4096, 2 * MOST_TOKENS // (N * (shortest + longest)))))
        return {"kind": kind, "groups": groups, "N": N, "shortest": shortest, "longest": longest, "masked": rng.choice([0.0, 0.25, 0.6]),
                "cut": rng.choice([0.0, 0.2]), "ref": rng.random() < 0.6, "mode": rng.choice(["sum", "token", "rollout"]), "beta": 0.02 if rng.random() < 0.8 else 0.0}
    if kind == "clip":
        rank = rng.choice([0, 0, 8, 16, 33])
        width = rng.choice([_log_int(rng, 64, 2560), 256 * rng.randint(1, 10)])
        dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
        a_layer = sum(a * b for a, b in _layer(width, rank)) * BYTES[dtype]
        layers = rng.randint(1, max(1, min(40, MOST_GRADS // a_layer)))
        return {"kind": kind, "layers": layers, "width": width, "rank": rank, "vocab": 0, "dtype": dtype, "clipped": rng.random() < 0.8}
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    V = rng.choice([151936, 4096, _log_int(rng, 500, 151936), _log_int(rng, 500, 151936) | 1])
    pad = rng.choice([0, 0, rng.randint(1, 64), -V % 64])
    T = _log_int(rng, 1 if kind == "logprob" else 16, max(32, min(16384, MOST_LOGITS[kind] // ((V + pad) * BYTES[dtype]))))
    case = {"kind": kind, "T": T, "V": V, "pad": pad, "dtype": dtype, "tau": rng.choice([1.0, 1.0, 0.7, 1.3]), "masked": rng.choice([0.0, 0.25, 0.6]) if T >= 16 else 0.0,
            "banned": rng.choice([0, 0, V // 100])}
    if kind == "step":
        N = rng.choice([8, 4, rng.randint(2, 16)])
        return {**case, "groups": max(1, min(64, T // (2 * N))), "N": N, "cut": rng.choice([0.0, 0.2]), "ref": rng.random() < 0.6, "beta": 0.02}
    return {**case, "entropy": rng.random() < 0.5}


# ------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _logits(case, g):
    """Logits [T, V] (a view of [T, V + pad]) and the tokens taken, -1 at the share that is masked."""
    T, V, B = case["T"], case["V"], case["banned"]
    dev = g.device
    x = torch.randn(T, V + case["pad"], generator=g, device=dev).mul_(2.0)
    likely = torch.randint(0, V - B, (T, 8), generator=g, device=dev)
    x.scatter_(1, likely, 4.0 + 8.0 * torch.rand(T, 8, generator=g, device=dev))
    if B:
        x[:, V - B:V] = -math.inf
    x = x.to(DTYPES[case["dtype"]])[:, :V]
    top = likely.gather(1, x.gather(1, likely).argmax(1, keepdim=True))
    other = likely.gather(1, torch.randint(0, 8, (T, 1), generator=g, device=dev))
    y = torch.where(torch.rand(T, 1, generator=g, device=dev) < 0.6, top, other)[:, 0].to(torch.int32)
    masked = int(case["masked"] * T)
    if masked:
        y[torch.randperm(T, generator=g, device=dev)[:masked]] = -1
    return x, y


def _row_stats(x, y, tau):
    """What the forward pass leaves for the backward one: [T, 2] maximum and sum of exponentials, entropies."""
    f = x.float()
    M = f.amax(1, keepdim=True)
    z = (f - M) / tau
    e = z.exp()
    S = e.sum(1, keepdim=True, dtype=torch.float64)
    U = torch.where(e > 0, e * z, 0.0).sum(1, keepdim=True, dtype=torch.float64)
    live = (y >= 0)[:, None]
    stats = torch.where(live, torch.cat([M, S.float()], 1), 0.0)
    return stats, torch.where(live, (S.log() - U / S).float(), 0.0)[:, 0], z, e, S


def _cut(groups, share, g):
    """Gate decisions: 1 for that share of the groups."""
    cut = torch.zeros(groups, dtype=torch.uint8, device=g.device)
    cut[torch.randperm(groups, generator=g, device=g.device)[:int(share * groups)]] = 1
    return cut


def _spread(T, rows, g):
    """Starts of `rows` rollouts that share T tokens."""
    cuts = torch.randint(0, T + 1, (rows - 1,), generator=g, device=g.device).sort().values
    return torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), T)])


def _advantages(groups, N, g):
    r = (torch.rand(groups, N, generator=g, device=g.device) < 0.5).float()
    return ((r - r.mean(1, keepdim=True)) / (r.std(1, unbiased=False, keepdim=True) + 1e-6)).contiguous()


def _layer(width, rank):
    """Shapes of the gradients of one layer: its seven matrices and two norms, or two factors of each matrix."""
    inner = width * 11 // 4
    full = [(width, width), (width // 4, width), (width // 4, width), (width, width), (inner, width), (inner, width), (width, inner)]
    if not rank:
        return full + [(1, width), (1, width)]
    return [f for a, b in full for f in ((rank, b), (a, rank))]


def _gradients(case):
    shapes = _layer(case["width"], case["rank"]) * case["layers"]
    return shapes + [(case["vocab"], case["width"])] * (case["vocab"] > 0)


def prepare(case, seed):
    g = _generator(seed)
    dev, kind = g.device, case["kind"]
    f32 = dict(dtype=torch.float32, device=dev)
    if kind == "clip":
        sizes = [a * b for a, b in _gradients(case)]
        dtype = DTYPES[case["dtype"]]
        starts, at = [], 0
        for n in sizes:                       # one flat buffer, each gradient on a boundary of 16 bytes
            starts.append(at)
            at += (n + 7) // 8 * 8
        flat, out = torch.zeros(at, dtype=dtype, device=dev), torch.zeros(at, dtype=dtype, device=dev)
        noise = torch.randn(1 << 22, generator=g, device=dev)
        for k, (b, n) in enumerate(zip(starts, sizes)):      # other magnitudes from tensor to tensor
            size = 1e-3 * 4.0 ** (k % 5 - 2)
            for c in range(0, n, 1 << 22):
                m = min(1 << 22, n - c)
                flat[b + c:b + c + m] = noise[:m] * size
            noise = noise.roll(k + 1)
        total = float(flat.double().square().sum().sqrt()) if at < 1 << 24 else float(torch.linalg.vector_norm(flat, dtype=torch.float32))
        return {"kind": kind, "flat": flat, "flat_out": out, "grads": [flat[b:b + n] for b, n in zip(starts, sizes)], "out": [out[b:b + n] for b, n in zip(starts, sizes)],
                "norm": torch.zeros(1, **f32), "max_norm": total / 7 if case["clipped"] else 4 * total}
    if kind == "policy":
        G, N = case["groups"], case["N"]
        lens = torch.linspace(case["shortest"], case["longest"], G * N, dtype=torch.float64).round().long().to(dev)
        lens = lens[torch.randperm(G * N, generator=g, device=dev)]
        start = torch.cat([lens.new_zeros(1), lens.cumsum(0)])
        T = int(start[-1])
        lp = -1.5 * torch.rand(T, generator=g, device=dev).square() * torch.randn(T, generator=g, device=dev).abs()
        return {"kind": kind, "N": N, "mode": MODES[case["mode"]], "beta": case["beta"], "clip": (0.2, 0.28), "row_start": start, "adv": _advantages(G, N, g),
                "drop": _cut(G, case["cut"], g), "scale": 1.0 / (G * N) if case["mode"] == "sum" else 1.0,
                "mask": (torch.rand(T, generator=g, device=dev) >= case["masked"]).to(torch.uint8) if case["masked"] else None,
                "lp": lp, "old": lp + 0.12 * torch.randn(T, generator=g, device=dev), "ref": lp + 0.2 * torch.randn(T, generator=g, device=dev) if case["ref"] else None,
                "weight": torch.empty(G * N, **f32), "counts": torch.empty(2, dtype=torch.int64, device=dev), "loss": torch.empty(1, **f32), "stats": torch.empty(4, **f32), "d_lp": torch.empty(T, **f32)}
    x, y = _logits(case, g)
    T, V, tau = case["T"], case["V"], case["tau"]
    s = {"kind": kind, "x": x, "y": y, "tau": tau, "lp": torch.empty(T, **f32)}
    if kind == "logprob":
        s.update(row_stats=torch.empty(T, 2, **f32), entropy=torch.empty(T, **f32) if case["entropy"] else None)
        return s
    s["dx"] = torch.empty(T, V + case["pad"], dtype=x.dtype, device=dev)[:, :V]
    if kind == "grad":
        stats, ent = _row_stats(x, y, tau)[:2]
        s.update(row_stats=stats, entropy=ent if case["entropy"] else None, d_lp=torch.randn(T, generator=g, device=dev) / T,
                 d_ent=0.01 * torch.randn(T, generator=g, device=dev) / T if case["entropy"] else None)
        return s
    G, N = case["groups"], case["N"]
    lp = _logprob(x, y, tau)[0]
    start = _spread(T, G * N, g)
    kept = (_cut(G, case["cut"], g) == 0).repeat_interleave(N)
    row = (torch.searchsorted(start, torch.arange(T, device=dev), right=True) - 1).clamp(0, G * N - 1)
    tokens = ((y >= 0) & kept[row]).sum().clamp(min=1)
    s.update(row_start=start, adv=_advantages(G, N, g), weight=torch.where(kept, 1.0 / tokens, 0.0).float(), beta=case["beta"], clip=(0.2, 0.28), mask=None,
             old=lp + 0.12 * torch.randn(T, generator=g, device=dev), ref=lp + 0.2 * torch.randn(T, generator=g, device=dev) if case["ref"] else None,
             loss=torch.empty(1, **f32), stats=torch.empty(4, **f32))
    return s


# ------------------------------------------------------------------------- plain forms
def _logprob(x, y, tau):
    stats, ent, z, e, S = _row_stats(x, y, tau)
    z_y = z.gather(1, y.clamp(min=0)[:, None].long())[:, 0].double()
    return torch.where(y >= 0, z_y - S[:, 0].log(), 0.0).float(), stats, ent


def _logits_gradient(x, y, tau, stats, d_lp, entropy, d_ent):
    d = torch.where(y >= 0, d_lp, 0.0)[:, None]
    z = (x.float() - stats[:, :1]) / tau
    live = (y >= 0)[:, None]
    p = torch.where(live, z.exp() / stats[:, 1:], 0.0)
    dx = -d * p
    dx.scatter_add_(1, y.clamp(min=0)[:, None].long(), d)
    if d_ent is not None:
        log_p = torch.where(p > 0, z - stats[:, 1:].log(), 0.0)
        dx -= torch.where(p > 0, d_ent[:, None] * p * (log_p + entropy[:, None]), 0.0)
    return (dx / tau).to(x.dtype)


def _policy(lp, old, ref, adv, weight, row_start, mask, clip, beta):
    """Loss, gradient of lp and figures.  In 64 bits: whether a ratio is clipped, and the KL term of two policies that
    nearly agree, are lost in 32."""
    rows = row_start.numel() - 1
    t = torch.arange(lp.numel(), device=lp.device)
    row = (torch.searchsorted(row_start, t, right=True) - 1).clamp(0, rows - 1)
    w = weight[row].double() * ((t >= row_start[0]) & (t < row_start[-1]))
    if mask is not None:
        w = w * (mask != 0)
    A, lp, old = adv.reshape(-1)[row].double(), lp.double(), old.double()
    rho = (lp - old).exp()
    clipped = ((A > 0) & (rho > 1 + clip[1])) | ((A < 0) & (rho < 1 - clip[0]))
    gain = torch.minimum(rho * A, rho.clamp(1 - clip[0], 1 + clip[1]) * A)
    d_lp = -torch.where(clipped, 0.0, A * rho)
    kl = torch.zeros_like(lp)
    if ref is not None:
        d = ref.double() - lp
        kl = torch.expm1(d) - d
        d_lp = d_lp - beta * torch.expm1(d)
    loss = (w * (beta * kl - gain)).sum().reshape(1)
    stats = torch.stack([(w * gain).sum(), (w * kl).sum(), (w * clipped).sum(), (w * rho).sum()])
    return loss.float(), (w * d_lp).float(), stats.float()


def _weights(s):
    start, rows = s["row_start"], s["row_start"].numel() - 1
    if s["mask"] is None:
        tokens = start[1:] - start[:-1]
    else:
        before = torch.cat([start.new_zeros(1), (s["mask"] != 0).long().cumsum(0)])
        tokens = before[start[1:]] - before[start[:-1]]
    tokens = tokens * (s["drop"] == 0).repeat_interleave(s["N"])
    counts = torch.stack([tokens.sum(), (tokens > 0).sum()])
    per = {0: torch.ones_like(tokens), 1: counts[0], 2: counts[1] * tokens}[s["mode"]]
    return torch.where(tokens > 0, s["scale"] / per.clamp(min=1).double(), 0.0).float().reshape(rows), counts


def _sr():
    import paper_2605_05802_b200 as sr
    return sr


def _scratch(s, name, bytes_of):
    """A workspace that the program allocates once."""
    if name not in s:
        s[name] = torch.empty(max(bytes_of(), 1), dtype=torch.uint8, device="cuda")
    return s[name]


def run(s):
    kind = s["kind"]
    if kind == "logprob":
        if not own:
            lp, stats, ent = _logprob(s["x"], s["y"], s["tau"])
            return {"lp": lp, "row_stats": stats, "entropy": ent if s["entropy"] is not None else None}
        _sr().sr_token_logprob(s["x"], s["y"], s["tau"], logp=s["lp"], row_stats=s["row_stats"], entropy=s["entropy"])
        return {"lp": s["lp"], "row_stats": s["row_stats"], "entropy": s["entropy"]}
    if kind == "grad":
        if not own:
            return _logits_gradient(s["x"], s["y"], s["tau"], s["row_stats"], s["d_lp"], s["entropy"], s["d_ent"])
        _sr().sr_token_logprob_backward(s["x"], s["y"], s["row_stats"], s["entropy"], s["d_lp"], s["d_ent"], s["tau"], d_logits=s["dx"])
        return s["dx"]
    if kind == "policy":
        if not own:
            weight, counts = _weights(s)
            loss, d_lp, stats = _policy(s["lp"], s["old"], s["ref"], s["adv"], weight, s["row_start"], s["mask"], s["clip"], s["beta"])
            return {"weight": weight, "counts": counts, "loss": loss, "d_lp": d_lp, "stats": stats}
        sr, rows, T = _sr(), s["weight"].numel(), s["lp"].numel()
        sr.sr_loss_weights(s["row_start"], s["mask"], s["drop"], s["N"], s["mode"], s["scale"], weight=s["weight"], counts=s["counts"],
                           workspace=_scratch(s, "weights_ws", lambda: sr.sr_loss_weights_workspace_bytes(rows)))
        sr.sr_policy_loss(s["lp"], s["old"], s["ref"], s["adv"], s["weight"], s["row_start"], s["mask"], s["clip"][0], s["clip"][1], s["beta"],
                          loss=s["loss"], d_logp=s["d_lp"], stats=s["stats"], workspace=_scratch(s, "loss_ws", lambda: sr.sr_policy_loss_workspace_bytes(T)))
        return {"weight": s["weight"], "counts": s["counts"], "loss": s["loss"], "d_lp": s["d_lp"], "stats": s["stats"]}
    if kind == "step":
        if not own:
            t = torch.arange(s["y"].numel(), device=s["y"].device)
            row = torch.searchsorted(s["row_start"], t, right=True) - 1
            y = torch.where(s["weight"][row] != 0, s["y"], -1)          # a rollout without weight is left out
            lp, row_stats = _logprob(s["x"], y, s["tau"])[:2]
            loss, d_lp, stats = _policy(lp, s["old"], s["ref"], s["adv"], s["weight"], s["row_start"], y >= 0, s["clip"], s["beta"])
            return {"loss": loss, "lp": lp, "stats": stats, "dx": _logits_gradient(s["x"], y, s["tau"], row_stats, d_lp, None, None)}
        sr, T = _sr(), s["lp"].numel()
        sr.sr_policy_loss_logits(s["x"], s["y"], s["old"], s["ref"], s["adv"], s["weight"], s["row_start"], s["mask"], s["clip"][0], s["clip"][1], s["beta"], s["tau"],
                                 loss=s["loss"], logp=s["lp"], d_logits=s["dx"], stats=s["stats"], workspace=_scratch(s, "loss_ws", lambda: sr.sr_policy_loss_logits_workspace_bytes(T)))
        return {"loss": s["loss"], "lp": s["lp"], "stats": s["stats"], "dx": s["dx"]}
    if not own:
        norm = s["flat"].float().square().sum(dtype=torch.float64).sqrt().float().reshape(1)
        scale = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
        return {"norm": norm, "grads": (s["flat"].float() * scale).to(s["flat"].dtype)}
    sr = _sr()
    sr.sr_grad_norm(s["grads"], norm=s["norm"], workspace=_scratch(s, "norm_ws", lambda: sr.sr_grad_norm_workspace_bytes(len(s["grads"]))))
    sr.sr_clip_grads(s["grads"], s["norm"], s["max_norm"], out=s["out"])
    return {"norm": s["norm"], "grads": s["flat_out"]}


def work(case):
    kind = case["kind"]
    if kind == "clip":
        n = sum(a * b for a, b in _gradients(case))      # the norm has to be known before anything is written: two reads
        return {"bytes": 3.0 * n * BYTES[case["dtype"]] + 4, "flops": 3.0 * n}
    if kind == "policy":
        rows = case["groups"] * case["N"]
        T = rows * (case["shortest"] + case["longest"]) / 2         # lengths are spread evenly
        return {"bytes": T * (4 + 4 + 4 + 4 * case["ref"] + (case["masked"] > 0)) + rows * 16 + case["groups"], "flops": 20.0 * T}
    e, T = BYTES[case["dtype"]], case["T"]
    live = T - int(case["masked"] * T)
    if kind == "step":
        live *= 1 - int(case["cut"] * case["groups"]) / case["groups"]      # rollouts that were cut are left out
    if kind == "logprob":
        return {"bytes": live * case["V"] * e + T * 16.0, "flops": (6.0 if case["entropy"] else 4.0) * live * case["V"]}
    return {"bytes": (live + T) * case["V"] * e + T * 20.0, "flops": (8.0 if kind == "step" or case["entropy"] else 5.0) * live * case["V"]}


# ------------------------------------------------------------- the definition, 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "clip":
        g = s["flat"].double()
        norm = torch.linalg.vector_norm(g)
        return {"norm": norm.reshape(1), "grads": g * min(1.0, s["max_norm"] / (float(norm) + 1e-6))}
    if kind == "policy":
        start, keep = s["row_start"].tolist(), s["drop"].tolist()
        counted = s["mask"].bool() if s["mask"] is not None else torch.ones_like(s["lp"], dtype=torch.bool)
        rows = len(start) - 1
        row = torch.repeat_interleave(torch.arange(rows, device="cuda"), s["row_start"][1:] - s["row_start"][:-1])
        counted &= torch.tensor(keep, device="cuda")[row // s["N"]] == 0
        tokens = torch.bincount(row[counted], minlength=rows)
        total, live = int(tokens.sum()), int((tokens > 0).sum())
        weight = {0: torch.full((rows,), s["scale"], dtype=torch.float64, device="cuda"), 1: torch.full((rows,), s["scale"] / max(total, 1), dtype=torch.float64, device="cuda"),
                  2: s["scale"] / (live * tokens.double()).clamp(min=1)}[s["mode"]] * (tokens > 0)
        loss, d_lp, stats = _exact_policy(s["lp"].double(), s, weight[row] * counted, row)
        return {"weight": weight, "counts": None, "loss": loss, "d_lp": d_lp, "stats": stats}
    V = case["V"] - case["banned"]                       # a banned token has probability 0: the rest is the distribution
    y = s["y"].clamp(min=0).long()
    live = s["y"] >= 0
    parts = {"lp": [], "entropy": [], "row_stats": [], "dx": []}
    loss = stats = d_all = None
    chunks = [slice(a, min(a + 256, case["T"])) for a in range(0, case["T"], 256)]
    if kind == "step":
        row = torch.repeat_interleave(torch.arange(s["weight"].numel(), device="cuda"), s["row_start"][1:] - s["row_start"][:-1])
        live &= s["weight"][row] != 0
        lp = torch.cat([torch.log_softmax(s["x"][c, :V].double() / s["tau"], 1).gather(1, y[c, None])[:, 0] for c in chunks]) * live
        loss, d_all, stats = _exact_policy(lp, s, s["weight"].double()[row] * live, row)
        parts["lp"].append(lp)
    for c in chunks:
        x = s["x"][c, :V].double().requires_grad_(kind != "logprob")
        log_p = torch.log_softmax(x / s["tau"], 1)
        taken = log_p.gather(1, y[c, None])[:, 0]
        ent = -(log_p.exp() * log_p).sum(1) if case.get("entropy") else None
        if kind == "logprob":
            M = x.amax(1)
            parts["lp"].append(taken * live[c])
            parts["row_stats"].append(torch.stack([M, (torch.logsumexp(x / s["tau"], 1) - M / s["tau"]).exp()], 1) * live[c, None])
            if ent is not None:
                parts["entropy"].append(ent * live[c])
            continue
        value = (taken * (s["d_lp"].double() if kind == "grad" else d_all)[c])[live[c]].sum()
        if ent is not None:
            value = value + (ent * s["d_ent"][c].double())[live[c]].sum()
        grad, = torch.autograd.grad(value, x)
        parts["dx"].append(torch.nn.functional.pad(grad, (0, case["banned"])))
    done = {k: torch.cat(v) if v else None for k, v in parts.items()}
    if kind == "logprob":
        return {"lp": done["lp"], "row_stats": done["row_stats"], "entropy": done["entropy"]}
    return done["dx"] if kind == "grad" else {"loss": loss, "lp": done["lp"], "stats": stats, "dx": done["dx"]}


def _exact_policy(lp, s, w, row):
    """By differentiation of the loss itself."""
    lo, hi = s["clip"]
    lp = lp.detach().requires_grad_(True)
    A = s["adv"].reshape(-1).double()[row]
    rho = torch.exp(lp - s["old"].double())
    gain = torch.where(A >= 0, A * torch.clamp(rho, max=1 + hi), A * torch.clamp(rho, min=1 - lo))
    kl = torch.zeros_like(rho)
    if s["ref"] is not None:
        far = s["ref"].double() - lp
        kl = torch.exp(far) - far - 1
    loss = (w * (s["beta"] * kl - gain)).sum()
    d_lp, = torch.autograd.grad(loss, lp)
    clipped = ((A > 0) & (rho > 1 + hi)) | ((A < 0) & (rho < 1 - lo))
    return loss.detach().reshape(1), d_lp, torch.stack([(w * v).sum() for v in (gain, kl, clipped, rho)]).detach()

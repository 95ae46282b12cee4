"""One training step: gate, advantages, weights, scoring, loss from logits, gradient norm and clipping, as a trainer calls them one
after the other, against differentiation in 64 bits."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_05802_b200 as sr
from train_ref import DTYPES, assert_near, logits_gradient, logprob, policy, weights

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
LO, HI, BETA = 0.2, 0.28, 0.05
G, N, K, WIDTH = 6, 4, 8, 32


def empty(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEV)


class Step:
    """The calls of a step on buffers that stay: rollouts, then everything up to the clipped gradients."""

    def __init__(self, T, row_start):
        self.rows = len(row_start) - 1
        self.row_start = torch.from_numpy(row_start).to(DEV)
        self.stop, self.mean = empty(G, dtype=torch.uint8), empty(G, dtype=torch.float64)
        self.adv, self.weight = empty(G, N), empty(self.rows)
        self.counts = empty(2, dtype=torch.int64)
        self.loss, self.stats, self.logp, self.norm = empty(1), empty(4), empty(T), empty(1)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.ws = [empty(n, dtype=torch.uint8) for n in (max(sr.sr_gate_workspace_bytes(G, N, 8, K), 1), sr.sr_loss_weights_workspace_bytes(self.rows),
                                                         sr.sr_policy_loss_logits_workspace_bytes(T), sr.sr_grad_norm_workspace_bytes(8))]

    def share_out(self, seqs, lens, rewards, mask, mode):
        sr.sr_gate(seqs, lens, K, 0.12, mean=self.mean, stop=self.stop, workspace=self.ws[0])
        sr.sr_grpo_advantage(rewards, self.stop, 1e-6, adv=self.adv)
        sr.sr_loss_weights(self.row_start, mask, self.stop, N, mode, 1.0, weight=self.weight, counts=self.counts, workspace=self.ws[1])

    def learn(self, x, y, old, ref, mask, tau, dx):
        sr.sr_policy_loss_logits(x, y, old, ref, self.adv, self.weight, self.row_start, mask, LO, HI, BETA, tau, loss=self.loss, logp=self.logp, d_logits=dx,
                                 stats=self.stats, status=self.status, workspace=self.ws[2])

    def clip(self, grads, max_norm):
        sr.sr_grad_norm(grads, norm=self.norm, workspace=self.ws[3])
        sr.sr_clip_grads(grads, self.norm, max_norm, status=self.status)


def rollouts(seed, padded):
    """Actions, rewards, token counts and the mask of action tokens; group 2 repeats itself (it is cut), group 4 has one reward."""
    rng = np.random.default_rng(seed)
    seqs = rng.integers(0, 50, (G, N, 8)).astype(np.int32)
    seqs[2] = seqs[2, :1]
    rewards = (rng.random((G, N)) < 0.5).astype(np.float32)
    rewards[:, 0], rewards[:, 1], rewards[4] = 1.0, 0.0, 1.0
    tokens = rng.integers(0, 41, G * N)
    tokens[3] = 0
    if padded:
        start = 40 * np.arange(G * N + 1, dtype=np.int64)
        real = (np.arange(40)[None] < tokens[:, None]).reshape(-1)
    else:
        start = np.concatenate([[0], np.cumsum(tokens)]).astype(np.int64)
        real = np.ones(start[-1], dtype=bool)
    mask = (real & (rng.random(real.size) < 0.7)).astype(np.uint8)
    return torch.from_numpy(seqs).to(DEV), torch.full((G, N), 8, dtype=torch.int32, device=DEV), torch.from_numpy(rewards).to(DEV), start, real, mask


@pytest.mark.parametrize("dtype,V,tau", [("f32", 501, 1.0), ("f16", 4096, 0.8), ("bf16", 21001, 1.0), ("f32", 21001, 1.0)])
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("mode", [sr.SR_LOSS_TOKEN_MEAN, sr.SR_LOSS_ROLLOUT_MEAN])
def test_step(dtype, V, tau, padded, mode):
    seqs, lens, rewards, start, real, mask = rollouts(V + padded, padded)
    T = real.size
    g = torch.Generator().manual_seed(V)
    h = torch.randn(T, WIDTH, generator=g).to(DEV)
    W = 0.3 * torch.randn(V, WIDTH, generator=g).to(DEV)
    moved = [W + 0.01 * torch.randn(V, WIDTH, generator=g).to(DEV) for _ in range(2)]
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).to(DEV)
    y[~torch.from_numpy(real).to(DEV)] = -1
    x = (h @ W.T).to(DTYPES[dtype])
    x[~torch.from_numpy(real).to(DEV)] = float("nan")              # nobody looks at padding

    scores = []
    for M in moved:                                                # of the policy that acted and of the reference
        z = (h @ M.T).to(DTYPES[dtype])
        scores.append(empty(T))
        sr.sr_token_logprob(z, y, tau, logp=scores[-1])
        want, bound = logprob(z, y, tau)
        assert_near(scores[-1], want[0], bound["lp"], "scores")
    old, ref = scores
    (lp64, _, _, _), lp_bound = logprob(torch.nan_to_num(x), y, tau)
    rho = torch.exp(lp64 - old.double()).cpu().numpy()
    mask[(np.abs(rho - 1 - HI) < 1e-4) | (np.abs(rho - 1 + LO) < 1e-4)] = 0       # a ratio on a border: either side is right
    m = torch.from_numpy(mask).to(DEV)

    s = Step(T, start)
    s.share_out(seqs, lens, rewards, m, mode)
    stop = s.stop.cpu().numpy()
    assert stop[2] == 1 and not stop[:2].any()
    adv64, _ = oracle.advantage(rewards.cpu().numpy(), stop, 1e-6)
    assert np.allclose(s.adv.cpu().numpy(), adv64, rtol=1e-6, atol=0)
    w64, total, live = weights(start, mask, stop, N, mode, 1.0, T)
    weight, adv = s.weight.cpu().numpy(), s.adv.cpu().numpy().reshape(-1)
    assert s.counts.tolist() == [total, live] and np.all(np.abs(weight - w64) <= 2.0 ** -24 * w64)

    logits = x.clone()
    s.learn(x, y, old, ref, m, tau, x)                             # over the logits
    row = np.searchsorted(start, np.arange(T), side="right") - 1
    counts = (mask != 0) & (y.cpu().numpy() >= 0) & (weight[row] != 0)
    c = torch.from_numpy(counts).to(DEV)

    # by differentiation, in 64 bits
    z = torch.nan_to_num(logits).double().requires_grad_(True)
    lp = torch.log_softmax(z / tau, 1).gather(1, y.clamp(min=0).long()[:, None])[:, 0]
    A, w = torch.from_numpy(adv[row]).to(DEV).double(), torch.from_numpy(weight[row] * counts).to(DEV).double()
    ratio, d = torch.exp(lp - old.double()), ref.double() - lp
    gain = torch.minimum(ratio * A, ratio.clamp(1 - LO, 1 + HI) * A)
    loss = (w * (BETA * (torch.exp(d) - 1 - d) - gain)).sum()
    dz, = torch.autograd.grad(loss, z)

    base = lp64.cpu().numpy()
    want, want_d, want_stats, d_bound, loss_bound, stats_bound = policy(base, old.cpu().numpy(), ref.cpu().numpy(), adv, weight, start, counts.astype(np.uint8), LO, HI, BETA)
    yy = torch.where(c, y, -1)
    formula, bound = logits_gradient(torch.nan_to_num(logits), yy, tau, torch.from_numpy(want_d).to(DEV), None, x.dtype)
    assert float((formula - dz).abs().max()) <= 1e-12 and abs(float(loss.detach()) - want) <= 1e-12
    err = lp_bound["lp"].cpu().numpy()
    slope = weight[row] * (np.abs(adv[row]) * 2 + BETA * 4) * counts                # second derivative by logp, ratios below 2
    d_err = torch.from_numpy(d_bound + slope * err).to(DEV)[:, None]
    bound = bound + d_err / tau * torch.softmax(torch.nan_to_num(logits).double() / tau, 1)
    bound = bound.scatter_add(1, yy.clamp(min=0).long()[:, None], d_err / tau)
    assert_near(s.logp, torch.where(c, lp64, 0.0), lp_bound["lp"], "logp")
    assert_near(x, dz, bound, "d_logits")
    assert abs(float(s.loss) - want) <= loss_bound + (slope * err).sum()
    assert bool((x[~c] == 0).all()) and int(s.status) == 0

    # the batch in two chunks: the same weights, starts moved by the chunk's first token
    sums, cut = 0.0, T // 2 + 1
    for a, b in ((0, cut), (cut, T)):
        part = Step(b - a, start - a)
        part.adv, part.weight = s.adv, s.weight
        dx = torch.full((b - a, V), 7.0, dtype=x.dtype, device=DEV)
        part.learn(logits[a:b], y[a:b], old[a:b], ref[a:b], m[a:b], tau, dx)
        assert_near(dx, dz[a:b], bound[a:b], "d_logits of a chunk")
        sums += float(part.loss)
    assert abs(sums - want) <= loss_bound + (slope * err).sum() + 2.0 ** -23 * abs(want)

    # gradients of the head, their norm, and clipping in place
    grads = [x.float().T @ h, x.float().sum(0)]
    exact = [dz.T @ h.double(), dz.sum(0)]
    bounds = [bound.T @ h.abs().double() + T * 2.0 ** -23 * (dz.abs().T @ h.abs().double()), bound.sum(0) + T * 2.0 ** -23 * dz.abs().sum(0)]
    norm = float(torch.sqrt(sum(e.square().sum() for e in exact)))
    norm_err = float(torch.sqrt(sum(b.square().sum() for b in bounds))) + 2.0 ** -22 * norm
    s.clip(grads, norm / 3)
    assert abs(float(s.norm) - norm) <= norm_err
    for got, e, b in zip(grads, exact, bounds):
        assert_near(got, e / 3, b / 3 + e.abs() / 3 * ((norm_err + 2e-6) / norm + 2.0 ** -21), "clipped gradient")
    assert int(s.status) == 0


@pytest.mark.parametrize("dtype,V", [("f32", 300), ("bf16", 21000)])
def test_a_captured_step_is_replayed_on_other_rollouts(dtype, V):
    """The whole step in a graph: other rollouts, rewards and logits in the same buffers give what separate calls give."""
    batches = []
    for seed in range(3):
        seqs, lens, rewards, start, real, mask = rollouts(seed, True)
        g = torch.Generator().manual_seed(seed)
        x = torch.randn(real.size, V, generator=g).to(DEV, DTYPES[dtype])
        y = torch.where(torch.from_numpy(real), torch.randint(0, V, (real.size,), generator=g), -1).to(torch.int32).to(DEV)
        old = empty(real.size)
        sr.sr_token_logprob(x, y, logp=old)
        batches.append((seqs, lens, rewards, torch.from_numpy(mask).to(DEV), x, y, old + 0.1 * torch.randn(real.size, generator=g).to(DEV), old + 0.1))
    T = batches[0][4].shape[0]

    def run(s, b, dx):
        seqs, lens, rewards, mask, x, y, old, ref = b
        s.share_out(seqs, lens, rewards, mask, sr.SR_LOSS_TOKEN_MEAN)
        s.learn(x, y, old, ref, mask, 1.0, dx)
        s.clip([dx], 0.01)

    static, s, dx = [t.clone() for t in batches[0]], Step(T, start), empty(T, V, dtype=DTYPES[dtype])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(s, static, dx)
    for b in batches[1:] + batches[:1]:
        for t, v in zip(static, b):
            t.copy_(v)
        graph.replay()
        e, e_dx = Step(T, start), empty(T, V, dtype=DTYPES[dtype])
        run(e, b, e_dx)
        torch.cuda.synchronize()
        assert float(s.loss) != 0.0 and float(s.norm) > 0.01
        for name in ("stop", "adv", "weight", "counts", "loss", "stats", "logp", "norm", "status"):
            assert torch.equal(getattr(s, name), getattr(e, name)), name
        assert torch.equal(dx, e_dx)


def test_a_step_without_a_kept_group():
    """Everything is cut: no token counts, the loss and all gradients are 0 and clipping leaves them so."""
    seqs, lens, rewards, start, real, mask = rollouts(5, False)
    seqs.copy_(seqs[:, :1].expand_as(seqs).clone())
    T, V = real.size, 21000
    x = torch.full((T, V), float("nan"), dtype=torch.bfloat16, device=DEV)
    y = torch.zeros(T, dtype=torch.int32, device=DEV)
    s, nothing = Step(T, start), torch.full((T,), float("nan"), device=DEV)
    s.share_out(seqs, lens, rewards, torch.from_numpy(mask).to(DEV), sr.SR_LOSS_ROLLOUT_MEAN)
    s.learn(x, y, nothing, nothing, torch.from_numpy(mask).to(DEV), 1.0, x)
    s.clip([x], 1.0)
    assert bool((s.stop == 1).all()) and s.counts.tolist() == [0, 0] and not bool(s.weight.any())
    assert float(s.loss) == 0.0 and not bool(s.stats.any()) and not bool(s.logp.any()) and float(s.norm) == 0.0 and not bool(x.any()) and int(s.status) == 0

"""The operators on token ids as a program uses them together: rollouts that are sampled from adjusted logits into the gate's own array, and a
training step of a policy whose table is its output projection too, from tokens to clipped gradients."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_05802_b200 as sr
from tokens_ref import adjust, embed, embed_gradient, pack
from train_ref import assert_near

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def empty(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device=DEV)


def test_rollouts_sampled_into_the_gates_array():
    """Greedy steps: embed the last tokens, the caller's products, adjust by each rollout's own history and by what the environment allows,
    append, gate.  The histories are the rows of the array that the gate reads."""
    G, N, stride, V, D, steps = 5, 4, 16, 203, 24, 12
    g = torch.Generator().manual_seed(3)
    W = torch.randn(V, D, generator=g).to(DEV)
    A = (0.3 * torch.randn(D, D, generator=g)).to(DEV)
    R = G * N
    seqs = torch.zeros(G, N, stride, dtype=torch.int32, device=DEV)
    seqs[:, :, 0] = torch.randint(0, V, (G, N), generator=g, dtype=torch.int32).to(DEV)
    seqs[2] = seqs[2, :1].clone()                                 # a group that repeats itself
    lens = torch.ones(G, N, dtype=torch.int32, device=DEV)
    start = stride * torch.arange(R, device=DEV)
    settings = {"repetition": torch.full((R,), 1.3, device=DEV), "presence": torch.full((R,), 0.4, device=DEV), "frequency": torch.full((R,), 0.2, device=DEV)}
    allowed = torch.rand(3, V, generator=g) < 0.6
    words = pack(allowed.numpy()).to(DEV)
    h, x, y = empty(R, D), empty(R, V), empty(R, V)
    mean, stop = empty(G, dtype=torch.float64), empty(G, dtype=torch.uint8)
    ws = empty(max(sr.sr_gate_workspace_bytes(G, N, stride, stride), 1), dtype=torch.uint8)
    for step in range(steps):
        last = seqs.view(R, stride).gather(1, (lens.view(R, 1) - 1).long())[:, 0].contiguous()
        sr.sr_embed_tokens(W, last, D ** 0.5, out=h)
        want, bound = embed(W, last, float(np.float32(D ** 0.5)), h.dtype)
        assert_near(h, want, bound, "embedded")
        torch.matmul(torch.tanh(h @ A), W.T, out=x)
        state = torch.full((R,), step % 3, dtype=torch.int32, device=DEV)
        sr.sr_adjust_logits(x, history=seqs, history_start=start, history_len=lens, **settings, allowed=words, mask_row=state, out=y)
        want, bound = adjust(x, seqs.cpu().numpy().reshape(-1), start.cpu().numpy(), lens.cpu().numpy().reshape(-1), None, *(settings[k].cpu().numpy() for k in ("repetition", "presence", "frequency")),
                             allowed=allowed.numpy(), mask_row=state.cpu().numpy())
        assert_near(y.cpu(), want, bound, "adjusted")
        token = y.argmax(1).to(torch.int32)
        assert bool(allowed[step % 3][token.cpu().long()].all())
        seqs.view(R, stride).scatter_(1, lens.view(R, 1).long(), token[:, None])
        lens += 1
        sr.sr_gate(seqs, lens, stride, 0.12, mean=mean, stop=stop, workspace=ws)
        _, _, omean, ostop = oracle.gate(seqs.cpu().numpy(), lens.cpu().numpy(), stride, 0.12, 0)
        assert np.array_equal(mean.cpu().numpy(), omean) and np.array_equal(stop.cpu().numpy(), ostop)
    assert int(stop[2]) == 1


class Policy:
    """Tied table W [V, D], one layer A [D, D]: logits of position p from the token there."""

    def __init__(self, V, D, seed):
        g = torch.Generator().manual_seed(seed)
        self.V, self.D, self.scale = V, D, 4.0
        self.W = (0.5 * torch.randn(V, D, generator=g)).to(DEV)
        self.A = (0.2 * torch.randn(D, D, generator=g)).to(DEV)


def batch(V, seed, G=3, N=4):
    """Prompts and responses back to back; every position but a rollout's last predicts the token behind it."""
    rng = np.random.default_rng(seed)
    prompt, length = rng.integers(1, 9, G * N), rng.integers(1, 30, G * N)
    ids, first = [], np.concatenate([[0], np.cumsum(prompt + length)])
    for p, n in zip(prompt, length):
        ids.append((np.exp(rng.random(p + n) * np.log(V + 1)) - 1).astype(np.int64).clip(0, V - 1))
    ids = np.concatenate(ids).astype(np.int32)
    T = ids.size
    row = np.searchsorted(first, np.arange(T), side="right") - 1
    target = np.full(T, -1, dtype=np.int32)
    for r in range(G * N):                                        # positions prompt - 1 .. end - 2 of the rollout predict its response
        a, b = first[r] + prompt[r] - 1, first[r + 1] - 1
        target[a:b] = ids[a + 1:b + 1]
    return {"ids": ids, "target": target, "row_start": first.astype(np.int64), "start": first[row].astype(np.int64), "length": (np.arange(T) - first[row] + 1).astype(np.int32),
            "prompt": prompt[row].astype(np.int32), "adv": rng.normal(size=G * N).astype(np.float32), "rng": rng}


class Step:
    def __init__(self, policy, b, mask):
        p, T = policy, b["ids"].size
        self.p, self.b, self.T = p, {k: torch.from_numpy(v).to(DEV) for k, v in b.items() if k != "rng"}, T
        self.words = pack(mask).to(DEV)
        self.state = torch.from_numpy((np.arange(T) % mask.shape[0]).astype(np.int32)).to(DEV)
        self.repetition, self.presence = torch.full((T,), 1.25, device=DEV), torch.full((T,), 0.5, device=DEV)
        self.h, self.x, self.y = empty(T, p.D), empty(T, p.V), empty(T, p.V)
        self.loss, self.logp, self.norm = empty(1), empty(T), empty(1)
        self.weight = torch.full((self.b["adv"].numel(),), 1.0 / T, device=DEV)
        self.dW, self.dA, self.dh = empty(p.V, p.D), empty(p.D, p.D), empty(T, p.D)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.ws = [empty(n, dtype=torch.uint8) for n in (sr.sr_policy_loss_logits_workspace_bytes(T), sr.sr_embed_tokens_backward_workspace_bytes(T, p.V, p.D), sr.sr_grad_norm_workspace_bytes(2))]
        self.history = dict(history=self.b["ids"], history_start=self.b["start"], history_len=self.b["length"])
        self.rules = dict(allowed=self.words, mask_row=self.state, status=self.status)

    def run(self, old, clip):
        p, b = self.p, self.b
        sr.sr_embed_tokens(p.W, b["ids"], p.scale, out=self.h, status=self.status)
        a = torch.tanh(self.h @ p.A)
        torch.matmul(a, p.W.T, out=self.x)
        sr.sr_adjust_logits(self.x, **self.history, prompt_len=b["prompt"], repetition=self.repetition, presence=self.presence, **self.rules, out=self.y)
        sr.sr_policy_loss_logits(self.y, b["target"], old, None, b["adv"], self.weight, b["row_start"], None, 0.2, 0.28, 0.0, loss=self.loss, logp=self.logp, d_logits=self.y, workspace=self.ws[0])
        sr.sr_adjust_logits_backward(self.y, self.x, **self.history, repetition=self.repetition, **self.rules, d_logits=self.y)
        torch.matmul(self.y.T, a, out=self.dW)                    # of the projection,
        back = (self.y @ p.W) * (1 - a * a)
        torch.matmul(self.h.T, back, out=self.dA)
        torch.matmul(back, p.A.T, out=self.dh)
        sr.sr_embed_tokens_backward(self.dh, b["ids"], p.scale, d_table=self.dW, accumulate=True, workspace=self.ws[1], status=self.status)      # and of the lookup
        sr.sr_grad_norm([self.dW, self.dA], norm=self.norm, workspace=self.ws[2])
        sr.sr_clip_grads([self.dW, self.dA], self.norm, clip, status=self.status)


@pytest.mark.parametrize("V,D", [(300, 32), (21001, 40)])
def test_a_training_step_of_a_tied_policy(V, D):
    """Against differentiation in 64 bits.  Roundings of logits below 30 to 2^-24 of themselves move probabilities and ratios by 4e-6 of themselves, the
    products of up to 64 fp32 terms their results by as much: 2e-5 of the parts together, and the parts of a gradient whose advantages have both
    signs may cancel to a fiftieth: 1e-3 of its norm."""
    p, b = Policy(V, D, V), batch(V, V)
    T = b["ids"].size
    mask = b["rng"].random((4, V)) < 0.7
    mask[:, b["ids"]] = True                                      # what was sampled had been allowed
    s = Step(p, b, mask)
    old = torch.full((T,), float("nan"), device=DEV)
    live = b["target"] >= 0

    W, A = p.W.double().requires_grad_(True), p.A.double().requires_grad_(True)
    h = W[s.b["ids"].long()] * p.scale
    x = torch.tanh(h @ A) @ W.T
    seen = torch.zeros(T, V, dtype=torch.bool)
    again = torch.zeros(T, V, dtype=torch.bool)
    for t in range(T):
        a, n, q = int(b["start"][t]), int(b["length"][t]), int(b["prompt"][t])
        seen[t, b["ids"][a:a + n]] = True
        again[t, b["ids"][a + min(q, n):a + n]] = True
    seen, again = seen.to(DEV), again.to(DEV)
    y = torch.where(seen, torch.where(x > 0, x / 1.25, x * 1.25), x) - 0.5 * again
    y = torch.where(torch.from_numpy(mask).to(DEV)[s.state.long()], y, -float("inf"))
    lp = torch.log_softmax(y, 1).gather(1, s.b["target"].clamp(min=0).long()[:, None])[:, 0]
    at = torch.from_numpy(live).to(DEV)
    old[at] = (lp.detach() + 0.05 * torch.randn(T, generator=torch.Generator().manual_seed(1)).to(DEV))[at].float()       # ratios well inside the clip range
    row = torch.from_numpy(np.searchsorted(b["row_start"], np.arange(T), side="right") - 1).to(DEV)
    ratio = torch.exp(lp[at] - old[at].double())
    assert 0.81 < float(ratio.detach().min()) and float(ratio.detach().max()) < 1.27
    loss = -(s.b["adv"].double()[row][at] * ratio).sum() / T
    dW, dA = torch.autograd.grad(loss, (W, A))
    norm = float(torch.sqrt(dW.square().sum() + dA.square().sum()))

    s.run(old, norm / 3)
    assert int(s.status) == 0
    assert abs(float(s.loss) - float(loss.detach())) <= 1e-4 * float((s.b["adv"].double()[row][at].abs() * ratio.detach()).sum() / T)
    assert abs(float(s.norm) - norm) <= 1e-3 * norm
    for got, want in ((s.dW, dW), (s.dA, dA)):
        assert float((got.double() * 3 - want).norm()) <= 2e-3 * norm
    assert not bool(torch.isnan(s.dW).any())

    # captured, and replayed on another batch of the same sizes
    graph = torch.cuda.CUDAGraph()
    s.run(old, norm / 3)
    with torch.cuda.graph(graph):
        s.run(old, norm / 3)
    other = torch.from_numpy(b["rng"].permutation(b["ids"])).to(DEV)
    s.b["ids"].copy_(other)
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (s.loss, s.norm, s.dW, s.dA)]
    s.run(old, norm / 3)
    for a, e in zip(got, (s.loss, s.norm, s.dW, s.dA)):
        assert torch.equal(a.nan_to_num(nan=7.0), e.nan_to_num(nan=7.0))


def test_lookups_gradient_beside_the_projections():
    """Added to a gradient that stands there in 32 bits, from rows in 16: what a program that keeps its gradients in fp32 does."""
    V, D, T = 1000, 72, 5000
    g = torch.Generator().manual_seed(0)
    ids = torch.randint(0, V // 2, (T,), generator=g, dtype=torch.int32).to(DEV)
    d = torch.randn(T, D, generator=g).to(DEV, torch.bfloat16)
    had = torch.randn(V, D, generator=g).to(DEV)
    dW = had.clone()
    ws = empty(sr.sr_embed_tokens_backward_workspace_bytes(T, V, D), dtype=torch.uint8)
    sr.sr_embed_tokens_backward(d, ids, 2.0, d_table=dW, accumulate=True, workspace=ws)
    want, bound = embed_gradient(d, ids, 2.0, V, dW.dtype, had)
    assert_near(dW, want, torch.where(bound > 0, bound, 0.0), "sum")
    assert torch.equal(dW[V // 2:], had[V // 2:])

"""sr_policy_loss_logits on rows that a cluster's shared memory holds: batches in which nothing counts, sizes of its helper kernels,
calls beside one another, replayed ones, large buffers."""
import numpy as np
import pytest
import torch

import paper_2605_05802_b200 as sr
from test_policy_loss_gpu import dev, logits, starts, step
from train_ref import DTYPES, assert_near, logits_gradient, logprob, policy

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def batch(T, rows, seed, lp=None):
    rng = np.random.default_rng(seed)
    return dict(old=None if lp is None else (lp + 0.05).astype(np.float32), ref=None if lp is None else (lp - 0.1).astype(np.float32),
                adv=rng.standard_normal(rows).astype(np.float32), weight=(rng.random(rows) + 0.5).astype(np.float32), row_start=starts(rng.multinomial(T, np.ones(rows) / rows)))


def check(x, y, b, mask, got, beta, rows):
    """Some rows of a step's outputs against 64 bits: gradient and logp (ratios here are clear of the clip range's borders)."""
    loss, lp, dx, stats, status = got
    rows = torch.as_tensor(rows, device=DEV)
    xx, yy = x[rows], y[rows]
    (lp64, _, _, _), bound = logprob(xx, yy, 1.0)
    at = rows.cpu().numpy()
    row = np.searchsorted(b["row_start"], at, side="right") - 1
    counts = (yy.cpu().numpy() >= 0) & (b["weight"][row] != 0) & (mask[at] != 0 if mask is not None else True)
    c = torch.from_numpy(counts).to(DEV)
    pick = lambda a: None if a is None else a[at]
    n = len(at)
    _, d, _, d_bound, _, _ = policy(lp64.cpu().numpy(), pick(b["old"]), pick(b["ref"]), b["adv"][row], b["weight"][row], np.arange(n + 1), counts.astype(np.uint8), 0.2, 0.28, beta)
    err = bound["lp"].cpu().numpy()
    d_err = torch.from_numpy(d_bound + b["weight"][row] * (np.abs(b["adv"][row]) * 2 + beta * 4) * counts * err).to(DEV)[:, None]
    yy = torch.where(c, yy, -1)
    g, g_bound = logits_gradient(xx, yy, 1.0, torch.from_numpy(d).to(DEV), None, x.dtype)
    g_bound = (g_bound + d_err * torch.softmax(xx.double(), 1)).scatter_add(1, yy.clamp(min=0).long()[:, None], d_err)
    assert_near(lp[rows], torch.where(c, lp64, 0.0), bound["lp"], "logp")
    assert_near(dx[rows], g, g_bound, "d_logits")
    assert status == 0


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T,V", [(400, 21000), (600, 21000), (300, 50021), (200, 151936)])
@pytest.mark.parametrize("counting", [0, 1, 3])
def test_hardly_anything_counts(T, V, counting, dtype):
    x, y = logits(T, V, dtype, T)
    b = batch(T, 5, T)
    keep = np.linspace(0, T - 1, counting).astype(int)
    mask = np.zeros(T, dtype=np.uint8)
    mask[keep] = 1
    safe = x.clone()
    x[torch.from_numpy(mask == 0).to(DEV)] = float("nan")
    got = step(x, y, b, mask, 1.0, 0.0)
    assert bool((got[2][torch.from_numpy(mask == 0).to(DEV)] == 0).all()) and int((got[1] != 0).sum()) == counting and got[4] == 0
    if counting:
        check(safe, y, b, mask, got, 0.0, list(range(0, T, 7)) + keep.tolist())
    else:
        assert float(got[0]) == 0.0 and not bool(got[3].any())


@pytest.mark.parametrize("T,V", [(4, 300), (50, 21000), (400, 21000), (600, 21000), (400, 50021)])
def test_no_rollouts(T, V):
    """Tokens, but no rollout that they could belong to."""
    x, y = logits(T, V, "bf16", T)
    b = dict(old=None, ref=None, adv=np.zeros(0, np.float32), weight=np.zeros(0, np.float32), row_start=np.zeros(1, np.int64))
    loss, lp, dx, stats, status = step(x, y, b, None, 1.0, 0.0)
    assert float(loss) == 0.0 and not bool(lp.any()) and not bool(dx.any()) and not bool(stats.any()) and status == 0


@pytest.mark.parametrize("T", [1025, 2049, 2500, 4100, 7000])
def test_batches_of_the_helper_kernels_sizes(T):
    """Lists and sums of clusters of two to eight CTAs, and a list of several sweeps."""
    x, y = logits(T, 10500, "f32", T)
    (lp, _, _, _), _ = logprob(x, y, 1.0)
    b = batch(T, 37, T, lp.cpu().numpy())
    rng = np.random.default_rng(T)
    mask = (rng.random(T) < 0.6).astype(np.uint8)
    got = step(x, y, b, mask, 1.0, 0.05)
    check(x, y, b, mask, got, 0.05, np.arange(0, T, 13))
    row = np.searchsorted(b["row_start"], np.arange(T), side="right") - 1
    m = torch.from_numpy(mask.astype(bool) & (row < 37)).to(DEV)
    want = policy(got[1].cpu().numpy(), b["old"], b["ref"], b["adv"], b["weight"], b["row_start"], m.cpu().numpy().astype(np.uint8), 0.2, 0.28, 0.05)
    # terms at logp as it was rounded to fp32: 2^-24 of |logp| < 32 off, times the slope of a term
    slope = (b["weight"][row] * (2 * np.abs(b["adv"][row]) + 0.05)).sum() * 2.0 ** -19
    assert abs(float(got[0]) - want[0]) <= want[4] + slope
    assert np.all(np.abs(got[3].cpu().numpy() - want[2]) <= want[5] + 2.0 ** -23 * np.abs(want[2]) + (b["weight"][row] * (2 * np.abs(b["adv"][row]) + 1)).sum() * 2.0 ** -19)


def test_calls_beside_one_another():
    """Three streams, a workspace each: every call's clusters take what room the others leave, and each gives the bits that it gives
    alone."""
    args = []
    for seed, (T, V, dtype) in enumerate([(700, 60000, "bf16"), (500, 50001, "f32"), (900, 21500, "f16")]):
        x, y = logits(T, V, dtype, seed)
        y[::5] = -1
        b = batch(T, 9, seed)
        args.append((x, y, [dev(b[k]) for k in ("old", "ref", "adv", "weight", "row_start")], step(x, y, b, None, 1.0, 0.0)))
    streams = [torch.cuda.Stream() for _ in args]
    outs = [dict(loss=torch.empty(1, device=DEV), logp=torch.empty(x.shape[0], device=DEV), d_logits=torch.empty_like(x),
                 workspace=torch.empty(sr.sr_policy_loss_logits_workspace_bytes(x.shape[0]), dtype=torch.uint8, device=DEV)) for x, *_ in args]
    torch.cuda.synchronize()
    for _ in range(10):
        for o in outs:
            o["d_logits"].fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(3):
            for (x, y, rest, _), o, s in zip(args, outs, streams):
                with torch.cuda.stream(s):
                    sr.sr_policy_loss_logits(x, y, *rest, None, 0.2, 0.28, 0.0, 1.0, **o)
        torch.cuda.synchronize()
        for (_, _, _, want), o in zip(args, outs):
            assert torch.equal(o["loss"], want[0]) and torch.equal(o["logp"], want[1]) and torch.equal(o["d_logits"], want[2])


def test_replayed_with_other_tokens_counting():
    T, V = 600, 50000
    x, y = logits(T, V, "bf16", 3)
    b = batch(T, 6, 3)
    rest = [dev(b[k]) for k in ("old", "ref", "adv", "weight", "row_start")]
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    o = dict(loss=torch.empty(1, device=DEV), logp=torch.empty(T, device=DEV), d_logits=torch.empty_like(x),
             workspace=torch.empty(sr.sr_policy_loss_logits_workspace_bytes(T), dtype=torch.uint8, device=DEV))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sr.sr_policy_loss_logits(x, y, *rest, mask, 0.2, 0.28, 0.0, 1.0, **o)
    rng = np.random.default_rng(3)
    for share in (1.0, 0.5, 0.0, 0.02, 0.9):
        m = (rng.random(T) < share).astype(np.uint8)
        mask.copy_(dev(m))
        o["workspace"].random_()                                   # nothing is left there from one replay to the next
        graph.replay()
        torch.cuda.synchronize()
        want = step(x, y, b, m, 1.0, 0.0)
        assert torch.equal(o["loss"], want[0]) and torch.equal(o["logp"], want[1]) and torch.equal(o["d_logits"], want[2])


def test_more_tokens_than_a_list_holds():
    """Above 65536 tokens rows are read twice: the same figures as in chunks that the ring takes."""
    T, V = 65600, 20600
    x = torch.empty(T, V, dtype=torch.bfloat16, device=DEV)
    for a in range(0, T, 4100):
        x[a:a + 4100] = 2 * torch.randn(min(4100, T - a), V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(a))
    y = torch.randint(0, V, (T,), dtype=torch.int32, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    y[::3] = -1
    b = batch(T, 50, 1)
    got = step(x, y, b, None, 1.0, 0.0)
    check(x, y, b, None, got, 0.0, [0, 1, 2, 40000, 65535, 65536, T - 2, T - 1])
    sums = 0.0
    for a in range(0, T, 32800):
        part = step(x[a:a + 32800], y[a:a + 32800], dict(b, row_start=b["row_start"] - a), None, 1.0, 0.0)
        assert bool(((part[1] - got[1][a:a + 32800]).abs() <= 2.0 ** -16).all())      # bound of logp: below, twice
        sums += float(part[0])
        del part
    (_, _, _, _), bound = logprob(x[:300], y[:300], 1.0)
    assert float(bound["lp"].max()) < 2.0 ** -17
    assert abs(sums - float(got[0])) <= 2.0 ** -20 * float(np.abs(b["adv"] * b["weight"]).max()) * T


def test_rows_behind_2_to_the_31_elements():
    T, V = 14400, 151936                                           # 2.19e9 logits
    x = torch.empty(T, V, dtype=torch.bfloat16, device=DEV)
    for a in range(0, T, 900):
        x[a:a + 900] = 2 * torch.randn(900, V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(a))
    y = torch.randint(0, V, (T,), dtype=torch.int32, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    y[1::2] = -1
    rows = [0, 1, 14130, 14135, 14136, 14137, 14398, T - 1]
    kept = x[rows].clone()
    b = batch(T, 20, 2)
    got = step(x, y, b, None, 1.0, 0.0, out=x)
    small = torch.empty(len(rows), V, dtype=torch.bfloat16, device=DEV)
    small.copy_(kept)
    row = np.searchsorted(b["row_start"], rows, side="right") - 1
    few = dict(old=None, ref=None, adv=b["adv"][row], weight=b["weight"][row], row_start=np.arange(len(rows) + 1))
    check(small, y[rows], few, None, (got[0], got[1][rows], got[2][rows], got[3], got[4]), 0.0, list(range(len(rows))))

"""sr_loss_weights, sr_policy_loss and sr_policy_loss_logits against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_05802_b200 as sr
from helpers import Guarded
from train_ref import DTYPES, assert_near, logits_gradient, logprob, policy, weights

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def dev(a, dtype=None):
    return None if a is None else torch.as_tensor(np.asarray(a), dtype=dtype).to(DEV)


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def run_weights(row_start, mask, drop, N, mode, scale, offset=0):
    rows, guard = len(row_start) - 1, Guarded(DEV)
    w, counts = guard.alloc((rows,), torch.float32, 7.0), guard.alloc((2,), torch.int64, -1)
    ws = guard.alloc((sr.sr_loss_weights_workspace_bytes(rows),), torch.uint8)
    m = None
    if mask is not None:
        m = torch.zeros(offset + len(mask), dtype=torch.uint8, device=DEV)[offset:]
        m.copy_(dev(mask))
    sr.sr_loss_weights(dev(row_start), m, dev(drop), N, mode, scale, weight=w, counts=counts, workspace=ws)
    guard.check("sr_loss_weights")
    return w.cpu().numpy(), counts.cpu().tolist()


def check_weights(row_start, mask, drop, N, mode, scale, offset=0):
    got, counts = run_weights(row_start, mask, drop, N, mode, scale, offset)
    want, total, live = weights(row_start, mask, drop, N, mode, scale, 0 if mask is None else len(mask))
    assert counts == [total, live]
    assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want)) and np.array_equal(got == 0, want == 0)


@pytest.mark.parametrize("mode", [sr.SR_LOSS_SUM, sr.SR_LOSS_TOKEN_MEAN, sr.SR_LOSS_ROLLOUT_MEAN])
@pytest.mark.parametrize("G,N,longest", [(1, 1, 1), (1, 2, 40), (3, 5, 0), (10, 8, 30), (40, 3, 700), (700, 16, 9), (9, 4, 20000), (1500, 8, 3)])
def test_weights(G, N, longest, mode):
    rng = np.random.default_rng(G * N + longest)
    lens = rng.integers(0, longest + 1, G * N)
    lens[rng.random(G * N) < 0.1] = 0
    rs = starts(lens)
    drop = (rng.random(G) < 0.3).astype(np.uint8) * rng.integers(1, 256, G).astype(np.uint8)
    mask = ((rng.random(rs[-1]) < 0.6) * rng.integers(1, 256, rs[-1])).astype(np.uint8)
    mask[:rs[-1] // 5] = 0
    for m in (None, mask):
        for d in (None, drop):
            check_weights(rs, m, d, N, mode, 0.37)
    check_weights(rs, mask, drop, N, mode, -2.5, offset=5)
    check_weights(rs, mask, np.ones(G, np.uint8), N, mode, 1.0)               # everything cut
    check_weights(rs, np.zeros_like(mask), None, N, mode, 1.0)                # nothing counts


def test_weights_of_chunks_and_long_rollouts():
    """Row starts outside the mask's tokens; one rollout over many tiles; tokens between the last rollout and the end."""
    rng = np.random.default_rng(1)
    mask = (rng.random(5000) < 0.5).astype(np.uint8)
    for rs in ([0, 5000], [-700, 3, 3, 4999, 9000], [100, 200, 1024, 1024, 2048, 2049, 4000], [0, 0, 0, 5000], [5000, 5000, 6000]):
        check_weights(np.array(rs, dtype=np.int64), mask, None, 1, sr.SR_LOSS_ROLLOUT_MEAN, 1.0)


def draw(rng, lens, n=None, ref=True, old=True, spread=0.15):
    rs = starts(lens)
    n = int(rs[-1]) if n is None else n
    lp = (-3 * rng.random(n) ** 2).astype(np.float32)
    return dict(lp=lp, old=(lp + spread * rng.standard_normal(n)).astype(np.float32) if old else None,
                ref=(lp + 2 * spread * rng.standard_normal(n)).astype(np.float32) if ref else None,
                adv=rng.standard_normal(len(lens)).astype(np.float32), weight=rng.random(len(lens)).astype(np.float32), row_start=rs)


def run_policy(b, mask, lo, hi, beta, offset=0, want_grad=True, in_place=False):
    n, guard = b["lp"].size, Guarded(DEV)

    def put(a):
        if a is None:
            return None
        t = torch.zeros(offset + len(a), dtype=torch.from_numpy(a).dtype, device=DEV)[offset:]
        t.copy_(dev(a))
        return t

    loss, stats = guard.alloc((1,), torch.float32, 7.0), guard.alloc((4,), torch.float32, 7.0)
    d = guard.alloc((offset + n,), torch.float32, 7.0)[offset:] if want_grad else None
    ws = guard.alloc((sr.sr_policy_loss_workspace_bytes(n),), torch.uint8)
    lp = put(b["lp"])
    if in_place:
        d = lp
    sr.sr_policy_loss(lp, put(b["old"]), put(b["ref"]), dev(b["adv"]), dev(b["weight"]), dev(b["row_start"]), put(mask), lo, hi, beta,
                      loss=loss, d_logp=d, stats=stats, workspace=ws)
    guard.check("sr_policy_loss")
    return float(loss), None if d is None else d.cpu().numpy(), stats.cpu().numpy()


def check_policy(b, mask, lo=0.2, hi=0.28, beta=0.05, **how):
    loss, d, stats = run_policy(b, mask, lo, hi, beta, **how)
    want, want_d, want_stats, d_bound, loss_bound, stats_bound = policy(b["lp"], b["old"], b["ref"], b["adv"], b["weight"], b["row_start"], mask, lo, hi, beta)
    assert abs(loss - want) <= loss_bound, (loss, want, loss_bound)
    assert np.all(np.abs(stats - want_stats) <= stats_bound + 2.0 ** -23 * np.abs(want_stats)), (stats, want_stats)
    if d is not None:
        off = np.abs(d - want_d) > d_bound
        assert not off.any(), (int(off.sum()), np.flatnonzero(off)[:3], d[off][:3], want_d[off][:3])
    return loss, d, stats


LENGTHS = {"one": [1], "two": [1, 2], "empty": [0, 3, 0, 0, 5, 0], "short": list(range(31)) * 3, "odd": [129, 1, 0, 1023, 2, 640] * 4, "long": [40000, 0, 3],
           "many": [7] * 6000}


@pytest.mark.parametrize("lens", list(LENGTHS))
@pytest.mark.parametrize("ref,old,masked", [(True, True, True), (False, True, False), (True, False, True), (False, False, False)])
def test_policy_loss(lens, ref, old, masked):
    rng = np.random.default_rng(len(lens))
    b = draw(rng, LENGTHS[lens], ref=ref, old=old)
    b["weight"][rng.random(b["weight"].size) < 0.2] = 0.0
    b["adv"][rng.random(b["adv"].size) < 0.2] = 0.0
    mask = (rng.random(b["lp"].size) < 0.7).astype(np.uint8) * 255 if masked else None
    first = check_policy(b, mask)
    check_policy(b, mask, beta=0.0)
    check_policy(b, mask, offset=1)
    assert check_policy(b, mask, want_grad=False)[0] == first[0]
    again = check_policy(b, mask, in_place=True)
    assert again[0] == first[0] and np.array_equal(again[1], first[1]) and np.array_equal(again[2], first[2])


def test_tokens_that_do_not_count_are_not_used():
    rng = np.random.default_rng(2)
    b = draw(rng, [50, 0, 70, 400, 80], n=700)                   # 100 tokens behind the last rollout
    b["row_start"] = b["row_start"] + 20                         # and 20 before the first
    b["weight"][2] = 0.0
    mask = (rng.random(700) < 0.5).astype(np.uint8)
    want = check_policy(b, mask)
    row = np.searchsorted(b["row_start"], np.arange(700), side="right") - 1
    out = (mask == 0) | (row < 0) | (row > 4) | (row == 2)
    for k in ("lp", "old", "ref"):
        b[k][out] = {"lp": np.nan, "old": np.inf, "ref": -np.inf}[k]
    b["adv"][2] = np.nan
    got = run_policy(b, mask, 0.2, 0.28, 0.05)
    assert got[0] == want[0] and np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
    assert np.all(got[1][out] == 0) and not np.signbit(got[1][out]).any()


def test_borders_of_the_clip_range():
    """Ratios within a few steps of 1 + high and 1 - low on either side, and large and small ones."""
    hi, lo = 0.28, 0.2
    near = []
    for border in (np.log(1 + hi), np.log(1 - lo)):
        x = np.float32(border)
        for k in range(-20, 21):
            near.append(np.float32(x + k * np.spacing(x)))
    near += [0.0, 5.0, -5.0, 80.0, -80.0, -110.0]
    lp = np.array(near * 2, dtype=np.float32)
    n = len(near)
    b = dict(lp=lp, old=np.zeros(2 * n, np.float32), ref=None, adv=np.array([1.5, -1.5], np.float32), weight=np.ones(2, np.float32), row_start=np.array([0, n, 2 * n], np.int64))
    check_policy(b, None, lo, hi, 0.0)
    b["adv"][:] = 0.0
    b["lp"][-1] = 200.0                                          # rho overflows, A = 0
    loss, d, stats = run_policy(b, None, lo, hi, 0.0)
    assert loss == 0.0 and not d.any()


@pytest.mark.parametrize("hi", [3.0, 2e5, 1e20])
def test_borders_of_wide_clip_ranges(hi):
    """Steps of log rho are steps of rho many times larger there, and so are errors."""
    x = np.float32(np.log1p(hi))
    lp = np.array([x + np.float32(k) * np.spacing(x) for k in range(-64, 65)], dtype=np.float32)
    n = lp.size
    b = dict(lp=lp, old=np.zeros(n, np.float32), ref=None, adv=np.full(1, 1.5, np.float32), weight=np.ones(1, np.float32), row_start=np.array([0, n], np.int64))
    check_policy(b, None, 0.2, hi, 0.0)
    far = dict(b, lp=lp - np.float32(20.0), old=np.full(n, -20.0, np.float32))          # the same ratios, rounded elsewhere
    check_policy(far, None, 0.2, hi, 0.0)


def test_kl_of_policies_that_nearly_agree_and_far_apart():
    d = np.concatenate([np.logspace(-7, 1.5, 400), -np.logspace(-7, 1.5, 400), [0.0, 0.5, -0.5, 0.49999997]]).astype(np.float32)
    lp = np.full(d.size, -1.0, np.float32)
    b = dict(lp=lp, old=None, ref=(lp + d).astype(np.float32), adv=np.zeros(1, np.float32), weight=np.ones(1, np.float32), row_start=np.array([0, d.size], np.int64))
    check_policy(b, None, beta=0.5)
    for k in range(0, d.size, 37):                               # each by itself: the sum hides small ones
        one = dict(b, lp=lp[k:k + 1], ref=b["ref"][k:k + 1], row_start=np.array([0, 1], np.int64))
        x = float(b["ref"][k]) - float(lp[k])
        kl = x * x * (0.5 + x / 6 + x * x / 24 + x ** 3 / 120 + x ** 4 / 720) if abs(x) < 0.01 else np.expm1(x) - x
        got = run_policy(one, None, 0.2, 0.2, 0.5)[2][1]
        assert abs(got - kl) <= 2.0 ** -20 * kl, (x, got, kl)


def test_gradient_against_differences():
    rng = np.random.default_rng(5)
    b = draw(rng, [4, 3], spread=0.02)                           # ratios well inside the clip range
    _, d, _ = run_policy(b, None, 0.2, 0.28, 0.3)
    h = 2.0 ** -7
    for t in range(7):
        f = []
        for s in (h, -h):
            c = dict(b, lp=b["lp"].copy())
            c["lp"][t] += s
            f.append(run_policy(c, None, 0.2, 0.28, 0.3)[0])
        # third order h^2 / 6 and rounding of the loss 2^-23 / h, for terms of order 2
        assert abs((f[0] - f[1]) / (2 * h) - d[t]) < 2e-4


def test_nothing_to_do():
    e = torch.empty(0, device=DEV)
    loss, stats = torch.full((1,), 7.0, device=DEV), torch.full((4,), 7.0, device=DEV)
    ws = torch.empty(sr.sr_policy_loss_workspace_bytes(0), dtype=torch.uint8, device=DEV)
    rs = torch.zeros(1, dtype=torch.int64, device=DEV)
    sr.sr_policy_loss(e, None, None, e, e, rs, None, 0.2, 0.2, 0.0, loss=loss, d_logp=e, stats=stats, workspace=ws)
    assert float(loss) == 0.0 and not bool(stats.any())
    d = torch.full((5,), 7.0, device=DEV)
    loss.fill_(7.0)
    sr.sr_policy_loss(torch.ones(5, device=DEV), None, None, e, e, rs, None, 0.2, 0.2, 0.0, loss=loss, d_logp=d, stats=None, workspace=ws)
    assert float(loss) == 0.0 and not bool(d.any())
    counts = torch.full((2,), 7, dtype=torch.int64, device=DEV)
    sr.sr_loss_weights(rs, None, None, 8, weight=e, counts=counts)
    assert counts.tolist() == [0, 0]
    loss.fill_(7.0)
    x = torch.empty(0, 50, device=DEV)
    ws = torch.empty(sr.sr_policy_loss_logits_workspace_bytes(0), dtype=torch.uint8, device=DEV)
    sr.sr_policy_loss_logits(x, torch.empty(0, dtype=torch.int32, device=DEV), None, None, e, e, rs, None, 0.2, 0.2, 0.0, loss=loss, logp=e, d_logits=x, workspace=ws)
    assert float(loss) == 0.0


# ------------------------------------------------------------------------------ from logits
def step(x, y, b, mask, tau, beta, out=None, lo=0.2, hi=0.28):
    T, guard = x.shape[0], Guarded(DEV)
    loss, stats, lp = guard.alloc((1,), torch.float32, 7.0), guard.alloc((4,), torch.float32, 7.0), guard.alloc((T,), torch.float32, 7.0)
    dx = guard.alloc(tuple(x.shape), x.dtype, 7.0) if out is None else out
    status = guard.alloc((1,), torch.int32, 0)
    ws = guard.alloc((sr.sr_policy_loss_logits_workspace_bytes(T),), torch.uint8)
    sr.sr_policy_loss_logits(x, y, dev(b["old"]), dev(b["ref"]), dev(b["adv"]), dev(b["weight"]), dev(b["row_start"]), dev(mask), lo, hi, beta, tau,
                             loss=loss, logp=lp, d_logits=dx, stats=stats, status=status, workspace=ws)
    guard.check("sr_policy_loss_logits")
    return loss, lp, dx, stats, int(status.item())


def logits(T, V, dtype, seed, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = (2 * torch.randn(T, V + pad, generator=g)).to(DEV, DTYPES[dtype])[:, :V]
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).to(DEV)
    x[torch.arange(T, device=DEV), y.long()] += 4
    return x, y


STEPS = [(1, 1), (4, 3), (7, 129), (60, 4096), (400, 4096), (3, 8200), (5, 50021), (2, 151936), (301, 1001), (3, 300000), (2, 999983), (700, 40),
         (1000, 21003), (160, 50021), (84, 151936)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T,V", STEPS)
@pytest.mark.parametrize("pad,tau", [(0, 1.0), (5, 0.8)])
def test_step_from_logits(T, V, pad, tau, dtype):
    x, y = logits(T, V, dtype, T + V, pad)
    rng = np.random.default_rng(T + V)
    lens = rng.multinomial(T, np.ones(6) / 6)
    (lp64, _, _, _), bound = logprob(x, y, tau)
    y[torch.from_numpy(rng.random(T) < 0.2).to(DEV)] = -1
    base = lp64.cpu().numpy()
    far = np.where(rng.random(T) < 0.3, rng.choice([-0.6, 0.6], T), 0.1 * rng.uniform(-1, 1, T))      # clear of the borders of the clip range
    b = dict(old=(base - far).astype(np.float32), ref=(base + 0.2 * rng.standard_normal(T)).astype(np.float32), adv=rng.standard_normal(6).astype(np.float32),
             weight=rng.random(6).astype(np.float32), row_start=starts(lens))
    b["weight"][1] = 0.0
    mask = (rng.random(T) < 0.9).astype(np.uint8)
    loss, lp, dx, stats, status = step(x, y, b, mask, tau, 0.05)
    row = np.searchsorted(b["row_start"], np.arange(T), side="right") - 1
    counts = torch.from_numpy((mask != 0) & (b["weight"][row] != 0)).to(DEV) & (y >= 0)
    yy = torch.where(counts, y, -1)
    assert_near(lp, torch.where(counts, lp64, 0.0), torch.where(counts, bound["lp"], 0.0), "logp")
    # the loss and its gradient at the exact log-probabilities; what logp's error does to them is first order: |d2 loss| <= w (|A| rho + beta e^d)
    c = counts.cpu().numpy().astype(np.uint8)
    want, want_d, want_stats, d_bound, loss_bound, stats_bound = policy(base, b["old"], b["ref"], b["adv"], b["weight"], b["row_start"], c, 0.2, 0.28, 0.05)
    err = bound["lp"].cpu().numpy()
    slope = b["weight"][row] * (np.abs(b["adv"][row]) * 2 + 0.05 * 4) * c
    assert abs(float(loss) - want) <= loss_bound + (slope * err).sum()
    assert np.all(np.abs(stats.cpu().numpy() - want_stats) <= stats_bound + 2.0 ** -23 * np.abs(want_stats) + 4 * ((np.abs(b["adv"][row]) + 1) * b["weight"][row] * err * c).sum())
    g, g_bound = logits_gradient(x, yy, tau, torch.from_numpy(want_d).to(DEV), None, x.dtype)
    d_err = torch.from_numpy(d_bound + slope * err).to(DEV)[:, None]
    g_bound = g_bound + d_err / tau * torch.softmax(x.double() / tau, 1)
    g_bound = g_bound.scatter_add(1, yy.clamp(min=0).long()[:, None], d_err / tau)
    assert_near(dx, g, g_bound, "d_logits")
    assert bool((dx[~counts] == 0).all())
    # over the logits, and the same bits again
    again = step(x, y, b, mask, tau, 0.05, out=x)
    same = x[:, :V].contiguous() if pad == 0 else None
    if same is not None:
        assert torch.equal(same, dx)
    else:                                       # another alignment may add up in another order
        assert_near(x, g, g_bound, "d_logits over the logits")
    if pad == 0:
        assert torch.equal(again[0], loss) and torch.equal(again[1], lp) and torch.equal(again[3], stats)
    assert status == 0


def test_step_rows_without_a_distribution_and_bad_targets():
    for V in (300, 40000):
        x, y = logits(8, V, "bf16", V)
        x[1] = -float("inf")
        x[2, 7] = float("nan")
        x[3] = torch.finfo(torch.bfloat16).min
        x[4, V // 2:] = -float("inf")
        x[5, 3] = float("inf")
        y[4], y[6], y[7] = 1, V, -5
        x[7] = float("nan")
        b = dict(old=None, ref=None, adv=np.ones(8, np.float32), weight=np.ones(8, np.float32), row_start=np.arange(9))
        loss, lp, dx, stats, status = step(x, y, b, None, 1.0, 0.0)
        assert status == sr.SR_STATUS_BAD_TARGET
        nan = torch.isnan(dx).all(1).tolist()
        assert nan == [False, True, True, False, False, True, False, False] and torch.isnan(lp).tolist() == nan
        assert bool((dx[6:] == 0).all()) and bool(torch.isfinite(dx[[0, 3, 4]]).all()) and bool((dx[4, V // 2:] == 0).all()) and bool(torch.isnan(loss).all())
        (want, _, _, _), bound = logprob(x[[0, 3, 4]], y[[0, 3, 4]], 1.0)
        assert_near(lp[[0, 3, 4]], want, bound["lp"], "logp")


def test_step_equals_the_three_calls():
    """What the separate entry points give one after the other, to rounding of logp to fp32 between them; and in a graph that is
    replayed on other inputs, beside another graph with a workspace of its own."""
    T, V = 120, 20000
    x, y = logits(T, V, "f32", 8)
    rng = np.random.default_rng(8)
    b = draw(rng, [30, 50, 40])
    b["lp"] = None
    args = [dev(b[k]) for k in ("old", "ref", "adv", "weight", "row_start")]
    lp, st, d = torch.empty(T, device=DEV), torch.empty(T, 2, device=DEV), torch.empty(T, device=DEV)
    dx, loss = torch.empty_like(x), torch.empty(1, device=DEV)
    ws = torch.empty(sr.sr_policy_loss_workspace_bytes(T), dtype=torch.uint8, device=DEV)
    sr.sr_token_logprob(x, y, logp=lp, row_stats=st)
    args[0].copy_(lp - 0.05)
    args[1].copy_(lp + 0.03)
    sr.sr_policy_loss(lp, *args, None, 0.2, 0.28, 0.05, loss=loss, d_logp=d, workspace=ws)
    sr.sr_token_logprob_backward(x, y, st, None, d, None, d_logits=dx)
    b["old"], b["ref"] = args[0].cpu().numpy(), args[1].cpu().numpy()
    got = step(x, y, b, None, 1.0, 0.05)
    # each way is within its bounds of the exact one (above): twice those, with logp here of at most 32
    (_, _, _, _), bound = logprob(x, y, 1.0)
    err = 2 * bound["lp"]
    assert bool(((got[1] - lp).abs() <= err).all())
    slope = 2 * d.double().abs() + 0.05 * args[3].double().max()
    assert abs(float(got[0] - loss)) <= float((slope * err).sum()) + 2.0 ** -19 * float(d.abs().sum() + loss.abs())
    assert bool(((got[2] - dx).abs().amax(1) <= slope * err + 2.0 ** -17 * d.abs()).all())
    graphs, outs = [], []
    for k in range(2):
        o = dict(loss=torch.empty(1, device=DEV), logp=torch.empty(T, device=DEV), d_logits=torch.empty_like(x), workspace=torch.empty(sr.sr_policy_loss_logits_workspace_bytes(T), dtype=torch.uint8, device=DEV))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sr.sr_policy_loss_logits(x, y, *args, None, 0.2, 0.28, 0.05 * (k + 1), 1.0, **o)
        graphs.append(g)
        outs.append(o)
    x.mul_(0.9)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    for k, o in enumerate(outs):
        want = step(x, y, b, None, 1.0, 0.05 * (k + 1))
        assert torch.equal(o["loss"], want[0]) and torch.equal(o["logp"], want[1]) and torch.equal(o["d_logits"], want[2])

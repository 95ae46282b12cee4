"""sr_policy_loss where the loss is a small difference of large terms: the advantages of a group add up to 0, and near the policy that
the rollouts came from every ratio is nearly 1.

The loss is -sum w A - sum w A (rho' - 1), rho' the ratio within the clip range.  The first sum needs no ratio: in fp64 it is exact to
2^-50 of its terms.  Terms of the second are A (rho' - 1), of which fp32 loses 2^-20 at most as it does of other terms."""
import numpy as np
import pytest

from test_policy_loss_gpu import logits, run_policy, starts, step

pytestmark = pytest.mark.gpu
LO, HI = 0.2, 0.28


def reference(b, mask, beta):
    """loss, figures and their bounds; vectorised, since cancelling takes many tokens."""
    n, rows = b["lp"].size, len(b["row_start"]) - 1
    row = np.clip(np.searchsorted(b["row_start"], np.arange(n), side="right") - 1, 0, rows - 1)
    w = b["weight"].astype(np.float64)[row] * (1 if mask is None else mask != 0)
    A = b["adv"].astype(np.float64)[row]
    delta = b["lp"].astype(np.float64) - b["old"].astype(np.float64)
    less = np.where(A > 0, np.minimum(np.expm1(delta), HI), np.where(A < 0, np.maximum(np.expm1(delta), -LO), 0.0))
    clipped = ((A > 0) & (np.expm1(delta) > HI)) | ((A < 0) & (np.expm1(delta) < -LO))
    d = 0 * delta if b["ref"] is None else b["ref"].astype(np.float64) - b["lp"]
    kl = np.expm1(d) - d
    kl = np.where(np.abs(d) < 1e-3, d * d * (0.5 + d / 6 + d * d / 24), kl)
    gain = (w * A).sum() + (w * A * less).sum()
    size = 2.0 ** -20 * (np.abs(w * A * less) * (1 + np.abs(delta))).sum() + 2.0 ** -45 * np.abs(w * A).sum()
    kl_sum, kl_size = (w * kl).sum(), 2.0 ** -20 * (w * (kl + np.abs(np.expm1(d) * d))).sum()
    loss = beta * kl_sum - gain
    return loss, size + beta * kl_size + 2.0 ** -23 * abs(loss), gain, size + 2.0 ** -23 * abs(gain), (w * clipped).sum()


def cancelling(groups, N, lens, seed, equal):
    """Advantages of each group that add up to 0, and equal lengths or others; weights of a token mean."""
    rng = np.random.default_rng(seed)
    half = rng.standard_normal((groups, N // 2)).astype(np.float32)
    adv = np.concatenate([half, -half], 1).reshape(-1)
    rows = groups * N
    lens = np.full(rows, lens) if equal else rng.integers(0, 2 * lens, rows)
    return dict(adv=adv, weight=np.full(rows, 1.0 / max(int(lens.sum()), 1), np.float32), row_start=starts(lens)), rng


@pytest.mark.parametrize("spread", [0.0, 1e-6, 1e-4, 1e-2, 0.1, 1.0])
@pytest.mark.parametrize("groups,N,lens", [(1, 2, 1), (1, 2, 2), (10, 8, 15), (40, 4, 64), (3, 6, 500), (128, 8, 640)])
@pytest.mark.parametrize("equal,masked,ref", [(True, False, False), (False, True, True)])
def test_loss(groups, N, lens, spread, equal, masked, ref):
    b, rng = cancelling(groups, N, lens, groups + lens, equal)
    n = int(b["row_start"][-1])
    b["lp"] = (-3 * rng.random(n) ** 2).astype(np.float32)
    b["old"] = (b["lp"] + spread * rng.standard_normal(n)).astype(np.float32)
    b["ref"] = (b["lp"] + 2 * spread * rng.standard_normal(n)).astype(np.float32) if ref else None
    mask = (rng.random(n) < 0.7).astype(np.uint8) if masked else None
    beta = 0.05 if ref else 0.0
    want, bound, gain, gain_bound, clipped = reference(b, mask, beta)
    for offset in (0, 1):                                     # vectors, and single loads
        loss, d, stats = run_policy(b, mask, LO, HI, beta, offset=offset)
        assert abs(loss - want) <= bound, (loss, want, bound)
        assert abs(stats[0] - gain) <= gain_bound, (stats[0], gain, gain_bound)
        assert abs(stats[2] - clipped) <= 2.0 ** -20 * clipped


@pytest.mark.parametrize("n,rows", [(30, 2), (5000, 10), (60000, 80)])
def test_without_an_older_policy_the_loss_is_the_weighted_sum_of_advantages(n, rows):
    """rho = 1: nothing but the first sum is left, to its rounding to fp32 at the end."""
    rng = np.random.default_rng(n)
    rs = np.arange(rows + 1) * n // rows
    adv, weight = rng.standard_normal(rows).astype(np.float32), (rng.random(rows) / n).astype(np.float32)
    adv[::2], weight[::2] = -adv[1::2], weight[1::2]          # rollouts of one length cancel exactly, others nearly
    b = dict(lp=(-rng.random(n)).astype(np.float32), old=None, ref=None, adv=adv, weight=weight, row_start=rs)
    loss, d, stats = run_policy(b, None, LO, HI, 0.0)
    terms = weight.astype(np.float64) * adv.astype(np.float64) * np.diff(rs)
    want = -terms.sum()
    assert abs(loss - want) <= 2.0 ** -23 * abs(want) + 2.0 ** -45 * np.abs(terms).sum()
    row = np.searchsorted(rs, np.arange(n), side="right") - 1
    assert np.all(np.abs(d + weight[row] * adv[row]) <= 2.0 ** -23 * np.abs(weight[row] * adv[row]))


@pytest.mark.parametrize("T,V,dtype", [(6, 300, "f32"), (60, 4096, "f32"), (1200, 1000, "bf16"), (60, 50021, "bf16"), (600, 21000, "bf16"), (300, 50021, "f32"), (132, 151936, "bf16")])
def test_from_logits(T, V, dtype):
    """Three advantages that add up to 0 exactly, over rollouts of one length: rho = 1, and nothing is left of the loss but what is lost on the way."""
    rng = np.random.default_rng(T)
    x, y = logits(T, V, dtype, T)
    rows = 6
    a = rng.integers(1, 1 << 20, rows // 3).astype(np.float32)
    c = rng.integers(1, 1 << 20, rows // 3).astype(np.float32)
    adv = np.stack([a, c, -(a + c)], 1).reshape(-1) * np.float32(1e-6)
    exact = adv.astype(np.float64).reshape(-1, 3).sum(1)        # what the rounding by 1e-6 has left
    weight = np.full(rows, 1 / 3, np.float32)
    b = dict(old=None, ref=None, adv=adv, weight=weight, row_start=np.arange(rows + 1) * T // rows)
    got = step(x, y, b, None, 1.0, 0.0)
    want = -(exact * float(weight[0])).sum() * (T // rows)
    size = (np.abs(adv).astype(np.float64) * float(weight[0])).sum() * (T // rows)
    bound = 2.0 ** -45 * size + 2.0 ** -23 * abs(want)
    assert abs(float(got[0]) - want) <= bound, (float(got[0]), want, bound)
    assert abs(float(got[3][0]) + want) <= bound


@pytest.mark.parametrize("delta", [-3.0, -8.0, -15.0, -40.0, -79.0, -81.0])
def test_small_ratios_keep_their_digits(delta):
    """rho far below 1 is a small number of its own in gradient and figures, not 1 less nearly 1."""
    n = 512
    lp = (delta + np.linspace(-0.9, 0.9, n)).astype(np.float32)
    b = dict(lp=lp, old=np.zeros(n, np.float32), ref=None, adv=np.array([1.5, 0.5], np.float32), weight=np.array([0.5, 2.0], np.float32), row_start=np.array([0, n // 2, n]))
    loss, d, stats = run_policy(b, None, LO, HI, 0.0)
    rho, wA, w = np.exp(lp.astype(np.float64)), np.repeat([0.75, 1.0], n // 2), np.repeat([0.5, 2.0], n // 2)
    # two ulp of the exponential and |delta| 2^-23 of its argument's rounding, with a product of three
    assert np.all(np.abs(d + wA * rho) <= wA * rho * 2.0 ** -21 * (1 + np.abs(lp)) + 2.0 ** -126)
    assert abs(stats[3] - (w * rho).sum()) <= (w * rho * 2.0 ** -21 * (2 + np.abs(lp))).sum() + 2.0 ** -126

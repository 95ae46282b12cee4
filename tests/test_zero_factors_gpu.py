"""sr_policy_loss where a factor is 0: a token of advantage 0 gains nothing whatever its ratio is, and beta = 0 leaves the KL term out
whatever the reference says, beside which tokens the odd one may stand."""
import math

import numpy as np
import pytest
import torch

from test_policy_loss_gpu import logits, run_policy, step
from train_ref import policy

pytestmark = pytest.mark.gpu
LO, HI = 0.2, 0.28
ODD = {"nan": np.nan, "inf": np.inf, "-inf": -np.inf}


def batch(n, rows):
    rng = np.random.default_rng(n)
    lp = (-3 * rng.random(n) ** 2).astype(np.float32)
    return dict(lp=lp, old=(lp + 0.1 * rng.uniform(-1, 1, n)).astype(np.float32), ref=(lp + 0.2 * rng.standard_normal(n)).astype(np.float32),
                adv=rng.choice([-1.5, 0.7, 1.1], rows).astype(np.float32), weight=(0.5 + rng.random(rows)).astype(np.float32), row_start=np.arange(rows + 1) * n // rows)


def check(got, b, beta, figures):
    """Against the formulas in 64 bits on a batch without odd values; of the figures only those named are looked at."""
    loss, d, stats = got
    want, want_d, want_stats, d_bound, loss_bound, stats_bound = policy(b["lp"], b["old"], b["ref"], b["adv"], b["weight"], b["row_start"], None, LO, HI, beta)
    assert np.all(np.abs(d - want_d) <= d_bound), np.flatnonzero(~(np.abs(d - want_d) <= d_bound))[:5]
    assert abs(loss - want) <= loss_bound
    for k in figures:
        assert abs(stats[k] - want_stats[k]) <= stats_bound[k] + 2.0 ** -23 * abs(want_stats[k])


@pytest.mark.parametrize("odd", list(ODD))
@pytest.mark.parametrize("where", ["lp", "old"])
@pytest.mark.parametrize("beside", ["alone", "border"])
@pytest.mark.parametrize("n,rows", [(4, 1), (12, 3), (300, 3), (300, 150), (5000, 7), (40000, 11)])
def test_advantage_zero(n, rows, beside, where, odd):
    """Rollouts of one token as of many, with a ratio at a border among the same four or not; no KL term."""
    b = batch(n, rows)
    b["ref"] = None
    row = np.searchsorted(b["row_start"], np.arange(n), side="right") - 1
    b["adv"][rows // 2] = 0.0
    zero = np.flatnonzero(row == rows // 2)
    if beside == "border":
        at = zero[0] // 4 * 4 + 3
        b["old"][at:at + 1] = b["lp"][at:at + 1] - np.float32(math.log1p(HI))
    sane = dict(b, lp=b["lp"].copy(), old=b["old"].copy())
    pick = zero[::3]
    pick = pick[pick % 4 != 3]
    b[where] = b[where].copy()
    b[where][pick] = ODD[odd]
    check(run_policy(b, None, LO, HI, 0.0), sane, 0.0, [0, 2] if odd == "nan" else [0])


@pytest.mark.parametrize("odd", list(ODD))
@pytest.mark.parametrize("beside", ["alone", "border"])
@pytest.mark.parametrize("n,rows", [(4, 1), (12, 3), (300, 3), (300, 150), (5000, 7), (40000, 11)])
def test_beta_zero(n, rows, beside, odd):
    b = batch(n, rows)
    if beside == "border":
        b["old"][3::8] = b["lp"][3::8] - np.float32(math.log1p(HI))
    sane = dict(b, ref=b["ref"].copy())
    b["ref"] = b["ref"].copy()
    b["ref"][::5] = ODD[odd]
    check(run_policy(b, None, LO, HI, 0.0), sane, 0.0, [0, 2, 3])


def test_both_zero():
    b = batch(2000, 4)
    b["adv"][:] = 0.0
    b["lp"][::3] = np.nan
    b["ref"][::7] = np.inf
    loss, d, stats = run_policy(b, None, LO, HI, 0.0)
    assert loss == 0.0 and not d.any() and stats[0] == 0.0 and stats[2] == 0.0 and np.isnan(stats[3])


def test_a_nan_that_has_a_factor_reaches_its_own_gradient_and_the_loss():
    b = batch(300, 3)
    b["lp"][[5, 17, 250]] = np.nan
    loss, d, stats = run_policy(b, None, LO, HI, 0.0)
    assert math.isnan(loss) and np.array_equal(np.flatnonzero(np.isnan(d)), [5, 17, 250]) and np.isnan(stats[0])
    b = batch(300, 3)
    b["ref"][[5, 17, 250]] = np.nan
    loss, d, stats = run_policy(b, None, LO, HI, 0.02)
    assert math.isnan(loss) and np.array_equal(np.flatnonzero(np.isnan(d)), [5, 17, 250]) and np.isnan(stats[1]) and not np.isnan(stats[0])


@pytest.mark.parametrize("T,V", [(60, 4096), (50, 21000), (600, 21000)])
def test_from_logits(T, V):
    """A row without a distribution, of advantage 0, leaves the loss alone here as from log-probabilities."""
    x, y = logits(T, V, "bf16", T)
    adv = np.ones(T, np.float32)
    adv[::5] = 0.0
    b = dict(old=None, ref=None, adv=adv, weight=np.ones(T, np.float32), row_start=np.arange(T + 1))
    x[::5, 7] = float("nan")
    loss, lp, dx, stats, status = step(x, y, b, None, 1.0, 0.0)
    assert float(loss) == -float((adv != 0).sum()) and bool(torch.isnan(lp[::5]).all()) and not bool(torch.isnan(dx).view(T, -1).any(1)[torch.arange(T) % 5 != 0].any())

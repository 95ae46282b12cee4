"""sr_policy_loss_logits on tokens whose ratio lies next to a border of the clip range: loss, figures and gradient take the same side,
and the right one wherever the log-probability's error leaves no doubt."""
import math

import numpy as np
import pytest
import torch

from test_policy_loss_gpu import DEV, logits, step
from train_ref import assert_near, logits_gradient, logprob

pytestmark = pytest.mark.gpu
LO, HI = 0.2, 0.28

# rows held in the shared memory of one CTA, two, four and eight; in registers; read twice
SHAPES = [(600, 21000, "bf16"), (500, 21000, "f16"), (600, 10500, "f32"), (300, 50021, "bf16"), (300, 50021, "f32"), (130, 151936, "bf16"), (120, 151936, "f32"),
          (400, 4096, "f32"), (60, 50021, "bf16")]


@pytest.mark.parametrize("tau", [1.0, 0.7, 0.02])
@pytest.mark.parametrize("T,V,dtype", SHAPES)
def test_gradient_and_figures_take_the_same_side(T, V, dtype, tau):
    x, y = logits(T, V, dtype, T + V)
    rng = np.random.default_rng(T)
    (lp64, _, _, _), bound = logprob(x, y, tau)
    lp64, err = lp64.cpu().numpy(), bound["lp"].cpu().numpy()
    adv = np.where(rng.random(T) < 0.5, 1.0, -1.0).astype(np.float32)
    border = np.where(adv > 0, math.log1p(HI), math.log1p(-LO))
    near = (2.0 ** -17 + np.abs(lp64) * 2.0 ** -21) * rng.uniform(-1, 1, T)        # a few roundings of logp to fp32 on either side
    old = (lp64 - border - near).astype(np.float32)
    b = dict(old=old, ref=None, adv=adv, weight=np.ones(T, np.float32), row_start=np.arange(T + 1))
    # Sides are read off the gradient d (1 - p) of the target.  Where p rounds to 1 that is 0 on either side, and the neighbours'
    # may round to 0 as well: such rows, which low temperatures have, are left out of the batch.
    telling = lp64 < -2.0 ** -10
    assert telling.sum() > T // 4
    loss, lp, dx, stats, status = step(x, y, b, telling.astype(np.uint8), tau, 0.0, lo=LO, hi=HI)
    assert status == 0
    x, y, dx = (a[torch.from_numpy(telling).to(DEV)] for a in (x, y, dx))
    lp64, err, adv, border, old = (a[telling] for a in (lp64, err, adv, border, old))
    T = len(y)
    clipped = (dx == 0).all(1)
    assert torch.equal(clipped, dx[torch.arange(T, device=DEV), y.long()] == 0)
    clipped = clipped.cpu().numpy()
    assert int(stats[2]) == int(clipped.sum()), "the gradient leaves out other tokens than the figures"
    over = (lp64 - old.astype(np.float64) - border) * adv                          # > 0: past the border
    sure = np.abs(over) > err
    assert sure.sum() > T // 8 and (~sure).sum() < T
    assert np.array_equal(clipped[sure], over[sure] > 0)
    # what is left of the gradient is that of the exact log-probability, to what its error makes of the ratio
    rho = np.exp(lp64 - old.astype(np.float64))
    d = torch.from_numpy(np.where(clipped, 0.0, -adv * rho)).to(DEV)
    g, g_bound = logits_gradient(x, y, tau, d, None, x.dtype)
    d_err = (d.abs() * torch.from_numpy(err + 2.0 ** -20).to(DEV))[:, None] / tau
    g_bound = (g_bound + d_err * torch.softmax(x.double() / tau, 1)).scatter_add(1, y.long()[:, None], d_err)
    assert_near(dx, g, g_bound, "d_logits")


@pytest.mark.parametrize("T,V,dtype", [(600, 21000, "bf16"), (300, 50021, "f32"), (130, 151936, "bf16")])
def test_chunks_take_the_sides_of_the_whole(T, V, dtype):
    """A chunk of a few rows is read another way than the whole batch: log-probabilities are the same to their rounding to fp32, and so
    are the sides of tokens farther than that from a border."""
    x, y = logits(T, V, dtype, T)
    rng = np.random.default_rng(V)
    (lp64, _, _, _), bound = logprob(x, y, 1.0)
    lp64, err = lp64.cpu().numpy(), bound["lp"].cpu().numpy()
    adv = np.where(rng.random(T) < 0.5, 1.0, -1.0).astype(np.float32)
    border = np.where(adv > 0, math.log1p(HI), math.log1p(-LO))
    off = rng.uniform(1.0, 3.0, T) * rng.choice([-1.0, 1.0], T) * (err + 2.0 ** -23 * np.abs(lp64))
    old = (lp64 - border - off).astype(np.float32)
    over = np.abs(lp64 - old.astype(np.float64) - border)
    b = dict(old=old, ref=None, adv=adv, weight=np.ones(T, np.float32), row_start=np.arange(T + 1))
    whole = step(x, y, b, None, 1.0, 0.0, lo=LO, hi=HI)[2]
    for a in range(0, T, 50):
        n = min(50, T - a)
        c = dict(old=old[a:a + n], ref=None, adv=adv[a:a + n], weight=np.ones(n, np.float32), row_start=np.arange(n + 1))
        part = step(x[a:a + n], y[a:a + n], c, None, 1.0, 0.0, lo=LO, hi=HI)[2]
        sure = torch.from_numpy(over[a:a + n] > err[a:a + n]).to(DEV)
        assert torch.equal((part == 0).all(1)[sure], (whole[a:a + n] == 0).all(1)[sure])

"""The trainer's operators in 64 bits, from their formulas, and how far a kernel may be from them.

Rounding to nearest is off by half a step: eps(type) / 2 of the value.  2^t of the kernels is within 2 ulp (2^-22 of the
value), and a relative error of 2^-23 in t = (x - M) log2(e) / temperature (two roundings, one of the constant) is one of
|t| 2^-23 ln 2 in 2^t.  Sums of up to 32 terms in fp32 add at most 11 roundings of 2^-24.  So the sum S of a row is within
rel_S = 2^-22 (6 + E|t|), E over the distribution of the row; the four beyond 2 + 11/4 cover rescaling when a thread's maximum
grows (each time 2 ulp, on what is then a fraction of the sum)."""
import math

import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SMALLEST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -24}


def distribution(x, tau):
    """log p, p, t (log2 units, from the maximum) of rows in float64; rows without a distribution are NaN."""
    z = x.double() / tau
    M = z.amax(1, keepdim=True)
    log_p = (z - M) - torch.exp(z - M).sum(1, keepdim=True).log()
    return log_p, log_p.exp(), torch.nan_to_num((z - M) / math.log(2.0), neginf=-1100.0)


def rel_S(p, t):
    return 2.0 ** -22 * (6 + (p * t.abs()).sum(1))


def logprob(x, y, tau):
    """(logp, entropy, M, S) and the bounds of their errors."""
    live = (y >= 0) & (y < x.shape[1])
    at = torch.where(live, y, 0).long()[:, None]
    log_p, p, t = distribution(x, tau)
    lp = log_p.gather(1, at)[:, 0]
    H = -torch.where(p > 0, p * log_p, 0.0).sum(1)
    H = torch.where(torch.isnan(lp) & torch.isnan(p).any(1), math.nan, H)
    M = x.double().amax(1)
    S = torch.exp((x.double() - M[:, None]) / tau).sum(1)
    err_S = rel_S(p, t)
    E1, E2 = (p * t.abs()).sum(1), (p * t * t).sum(1)
    bounds = {"lp": err_S + 2.0 ** -23 * lp.abs(), "S": S * (err_S + 2.0 ** -24), "H": 2 * err_S * (1 + E1) + 2.0 ** -22 * (E2 + 6 * E1) + 2.0 ** -23 * H.abs()}
    zero = torch.zeros_like(lp)
    return tuple(torch.where(live, v, zero) for v in (lp, H, M, S)), {k: torch.where(live, v, zero) for k, v in bounds.items()}


def logits_gradient(x, y, tau, d_lp, d_H, out_dtype):
    """Gradient of the logits by the formula, and the bound of its error element by element."""
    live = ((y >= 0) & (y < x.shape[1]))[:, None]
    at = torch.where(live[:, 0], y, 0).long()[:, None]
    log_p, p, t = distribution(x, tau)
    d = d_lp.double()[:, None]
    g = (-d * p).scatter_add(1, at, d)
    size = d.abs() * p
    if d_H is not None:
        H = -torch.where(p > 0, p * log_p, 0.0).sum(1, keepdim=True)
        part = torch.where(p > 0, p * (log_p + H), 0.0)
        g = g - d_H.double()[:, None] * part
        size = size + d_H.double()[:, None].abs() * torch.where(p > 0, p * (log_p.abs() + H + t.abs() + 1), 0.0)
    g = g / tau
    err_p = 2.0 ** -22 * (10 + t.abs()) + rel_S(p, t)[:, None]
    eps = torch.finfo(out_dtype).eps
    bound = size / tau * err_p + (eps / 2 + 2.0 ** -22) * g.abs() + SMALLEST[out_dtype] * (1 + d.abs() / tau)
    bound = bound.scatter_add(1, at, 2.0 ** -23 * d.abs() / tau)
    return torch.where(live, g, 0.0), torch.where(live, bound, 0.0)


def assert_near(got, want, bound, what=""):
    got, want = got.double(), want.double()
    nan = torch.isnan(want)
    assert bool((torch.isnan(got) == nan).all()), f"{what}: NaN elsewhere"
    inf = torch.isinf(want)
    assert bool((got[inf] == want[inf]).all()), f"{what}: infinities differ"
    off = ((got - want).abs() > bound) & ~nan & ~inf
    if bool(off.any()):
        k = torch.nonzero(off)[0].tolist()
        raise AssertionError(f"{what}: {int(off.sum())} of {off.numel()} off, first at {k}: got {got[tuple(k)].item()!r}, want {want[tuple(k)].item()!r} "
                             f"within {bound[tuple(k)].item():.3g}")


def weights(row_start, mask, drop, N, mode, scale, n_tokens):
    """(weight float64 [rows], tokens that count, rollouts with some) one rollout after the other."""
    rows = len(row_start) - 1
    tokens = np.zeros(rows, dtype=np.int64)
    for r in range(rows):
        if drop is not None and drop[r // N]:
            continue
        if mask is None:
            tokens[r] = max(0, row_start[r + 1] - row_start[r])
        else:
            a, e = max(0, row_start[r]), min(n_tokens, row_start[r + 1])
            tokens[r] = int((mask[a:e] != 0).sum()) if e > a else 0
    total, live = int(tokens.sum()), int((tokens > 0).sum())
    w = np.zeros(rows)
    for r in range(rows):
        if tokens[r]:
            w[r] = scale if mode == 0 else scale / total if mode == 1 else scale / (live * tokens[r])
    return w, total, live


def policy(lp, old, ref, adv, weight, row_start, mask, lo, hi, beta):
    """loss, d_logp, stats in float64 with the error bounds of fp32 terms; numpy arrays, one token after the other."""
    n, rows = lp.size, len(row_start) - 1
    d_lp, d_bound = np.zeros(n), np.zeros(n)
    sums, sizes = np.zeros(4), np.zeros(4)
    row = np.searchsorted(row_start, np.arange(n), side="right") - 1
    for t in range(n):
        r = row[t]
        if r < 0 or r >= rows or (mask is not None and mask[t] == 0) or weight[r] == 0:
            continue
        w, A, x = float(weight[r]), float(adv[r]), float(lp[t])
        delta = 0.0 if old is None else x - float(old[t])
        rho = math.exp(delta)
        clipped = (A > 0 and rho > 1 + hi) or (A < 0 and rho < 1 - lo)
        used = min(rho, 1 + hi) if A > 0 else max(rho, 1 - lo) if A < 0 else 0.0
        d = 0.0 if ref is None else float(ref[t]) - x
        kl, em1 = math.expm1(d) - d, math.expm1(d)
        if abs(d) < 1e-3:
            kl = d * d * (0.5 + d / 6 + d * d / 24 + d ** 3 / 120)
        d_lp[t] = w * ((0.0 if clipped else -A * rho) - beta * em1)
        # expf and expm1f within 2 ulp, their argument within 2^-24, four products: 2^-20 of the parts
        d_bound[t] = abs(w) * 2.0 ** -20 * ((0.0 if clipped else abs(A) * rho * (1 + abs(delta))) + beta * (abs(em1) + math.exp(d) * abs(d))) + 2.0 ** -126
        terms = np.array([w * A * used, w * kl, w if clipped else 0.0, w * rho])
        sums += terms
        sizes += np.abs(terms) * (1 + abs(delta)) + np.array([0, abs(w) * abs(em1 * d), 0, 0])
    loss = beta * sums[1] - sums[0]
    return loss, d_lp, sums, d_bound, 2.0 ** -20 * (beta * sizes[1] + sizes[0]) + 2.0 ** -23 * abs(loss), 2.0 ** -20 * sizes

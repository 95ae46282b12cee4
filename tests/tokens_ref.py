"""The operators on token ids in 64 bits, from their formulas, and how far a kernel may be from them.

A rounding to nearest is off by half a step: 2^-24 of the value in fp32, eps(type) / 2 at the end, where the smallest number of the type is the
least step.  Adjusted logits are at most four fp32 operations, each of them on numbers no larger than S = |x'| + |f c| + |p| + |b|, x' being
x / r or x r: 4 x 2^-24 S.  For 16-bit logits x / r may be x times the rounded 1 / r, a fifth rounding of x': 5 x 2^-24 S; and for
gradients two instead of one.  A sum of n fp32 terms in any order is within (n - 1) 2^-24 (1 + n 2^-24) of the sum of their sizes; scaling
it, and adding what stood there, is a rounding each."""
import numpy as np
import torch

from train_ref import DTYPES, SMALLEST  # noqa: F401


def adjust(x, hist=None, start=None, length=None, prompt=None, rep=None, pres=None, freq=None, bias_token=None, bias_value=None, bias_start=None, bias_len=None,
           allowed=None, mask_row=None):
    """(y, bound) for x [T, V] of any type; rules are numpy arrays, masks bool [M, V]."""
    T, V = x.shape
    out_dtype = x.dtype
    x = x.double().cpu().numpy()
    y, size = x.copy(), np.abs(np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0))
    touched = np.zeros((T, V), dtype=bool)
    for t in range(T):
        if rep is not None or pres is not None or freq is not None:
            a = np.arange(max(0, int(length[t])), dtype=np.int64)
            at = int(start[t]) + a
            ok = (at >= 0) & (at < len(hist))
            ids, late = hist[at[ok]], (a >= (0 if prompt is None else int(prompt[t])))[ok]
            real = (ids >= 0) & (ids < V)
            ids, late = ids[real], late[real]
            seen, c = np.zeros(V, dtype=bool), np.zeros(V)
            seen[ids] = True
            np.add.at(c, ids[late], 1.0)
            if rep is not None:
                r = float(rep[t])
                y[t] = np.where(seen, np.where(y[t] > 0, y[t] / r, y[t] * r), y[t])
                size[t] = np.where(seen, np.abs(np.nan_to_num(y[t], nan=0.0, posinf=0.0, neginf=0.0)), size[t])
            f, p = (0.0 if freq is None else float(freq[t])), (0.0 if pres is None else float(pres[t]))
            y[t] = np.where(c > 0, y[t] - f * c - p, y[t])
            size[t] += np.where(c > 0, abs(f) * c + abs(p), 0.0)
            touched[t] |= seen
        if bias_value is not None:
            mine = {}
            for i in range(int(bias_start[t]), int(bias_start[t]) + max(0, int(bias_len[t]))):
                if 0 <= i < len(bias_value) and 0 <= bias_token[i] < V:
                    mine[int(bias_token[i])] = float(bias_value[i])
            for v, b in mine.items():
                y[t, v] += b
                size[t, v] += abs(b)
                touched[t, v] = True
    eps = torch.finfo(out_dtype).eps
    bound = np.where(touched, (4 if out_dtype == torch.float32 else 5) * 2.0 ** -24 * size * (1 + eps) + eps / 2 * np.abs(np.nan_to_num(y, nan=0.0, posinf=0.0, neginf=0.0)) + SMALLEST.get(out_dtype, 0.0), 0.0)
    if allowed is not None:
        for t in range(T):
            m = t if mask_row is None else int(mask_row[t])
            if 0 <= m < len(allowed):
                y[t, ~allowed[m]] = -np.inf
    return torch.from_numpy(y), torch.from_numpy(bound)


def adjust_gradient(d, x, hist=None, start=None, length=None, rep=None, allowed=None, mask_row=None):
    T, V = d.shape
    dx, touched = d.double().cpu().numpy().copy(), np.zeros((T, V), dtype=bool)
    x = None if x is None else x.double().cpu().numpy()
    for t in range(T):
        if rep is not None:
            at = int(start[t]) + np.arange(max(0, int(length[t])), dtype=np.int64)
            ids = hist[at[(at >= 0) & (at < len(hist))]]
            seen = np.zeros(V, dtype=bool)
            seen[ids[(ids >= 0) & (ids < V)]] = True
            r = float(rep[t])
            dx[t] = np.where(seen, np.where(x[t] > 0, dx[t] / r, dx[t] * r), dx[t])
            touched[t] = seen
        if allowed is not None:
            m = t if mask_row is None else int(mask_row[t])
            if 0 <= m < len(allowed):
                dx[t, ~allowed[m]] = 0.0
    eps = torch.finfo(d.dtype).eps
    bound = np.where(touched, ((1 if d.dtype == torch.float32 else 2) * 2.0 ** -24 * (1 + eps) + eps / 2) * np.abs(dx) + SMALLEST[d.dtype], 0.0)
    return torch.from_numpy(dx), torch.from_numpy(bound)


def pack(allowed):
    """bool [M, V] -> int32 words [M, ceil(V / 32)]; the bits behind the vocabulary are set at random."""
    M, V = allowed.shape
    words = (V + 31) // 32
    bits = np.random.default_rng(V).random((M, words * 32)) < 0.5
    bits[:, :V] = allowed
    return torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view("<i4").copy())


def embed(table, tokens, scale, out_dtype):
    V = table.shape[0]
    ok = (tokens >= 0) & (tokens < V)
    want = torch.where(ok[:, None], scale * table.double()[torch.where(ok, tokens, 0).long()], 0.0)
    return want, torch.where(ok[:, None], (torch.finfo(out_dtype).eps / 2 + 2.0 ** -24) * want.abs() + SMALLEST.get(out_dtype, 0.0), 0.0)


def embed_gradient(d_out, tokens, scale, V, table_dtype, had=None):
    """Sums by token, in float64, and the bound of fp32 sums; `had`: what is added to."""
    ok = (tokens >= 0) & (tokens < V)
    at = torch.where(ok, tokens, V).long()
    D = d_out.shape[1]
    d = d_out.double()
    total, size = (torch.zeros(V + 1, D, dtype=torch.float64, device=d.device) for _ in range(2))
    for column in range(0, D, 512):                       # one term after the other in 64 bits
        total[:, column:column + 512].index_add_(0, at, d[:, column:column + 512])
        size[:, column:column + 512].index_add_(0, at, d[:, column:column + 512].abs())
    n = torch.bincount(at, minlength=V + 1)[:V].double()[:, None]
    total, size = scale * total[:V], abs(scale) * size[:V]
    if had is not None:
        total, size = total + had.double(), size + had.double().abs()
    eps = torch.finfo(table_dtype).eps
    bound = torch.where(n > 0, 2.0 ** -24 * (n + 3) * (1 + n * 2.0 ** -23) * size + (eps / 2) * total.abs() + SMALLEST[table_dtype], 0.0)
    return total, bound

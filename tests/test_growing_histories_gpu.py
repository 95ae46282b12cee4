"""Rows of rollouts whose histories grow token by token, many of them to a CTA, and histories that begin anew behind such rows.

Counts come from sums along the history in whole numbers, values and bounds from tokens_ref's roundings: four fp32 operations of numbers no larger than
S = |x'| + |f c| + |p| (five of 16-bit logits, whose x / r is x times a rounded 1 / r), and the last rounding to the logits' type."""
import numpy as np
import pytest
import torch

import paper_2605_05802_b200 as sr
from tokens_ref import DTYPES, pack
from train_ref import SMALLEST, assert_near

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def rollouts(V, T, seed):
    """Rollouts one after the other, each scored from its first position on (so that prompts end in mid-run); most rows see one id more than the one before."""
    rng = np.random.default_rng(seed)
    hist, start, length, prompt = [], [], [], []
    at = 0
    while len(start) < T:
        n = int(rng.integers(300, 1500))
        q = int(rng.integers(0, 200))
        step = rng.choice([1, 1, 1, 1, 1, 1, 1, 1, 0, 3], n)            # now and then none, or three
        seen = np.cumsum(step) - step[0]
        ids = (np.exp(rng.random(seen[-1] + 1) * np.log(V + 1)) - 1).astype(np.int64).clip(0, V - 1)
        ids[rng.random(ids.size) < 0.05] = -3
        ids[rng.random(ids.size) < 0.01] = V + 5
        hist.append(ids)
        start += [at] * n
        length += seen.tolist()
        prompt += [q] * n
        at += ids.size
    r = {"hist": np.concatenate(hist).astype(np.int32), "start": np.array(start[:T], np.int64), "length": np.array(length[:T], np.int32), "prompt": np.array(prompt[:T], np.int32)}
    grows = (r["start"][1:] == r["start"][:-1]) & (np.diff(r["length"]) == 1)
    assert grows.mean() > 0.7
    r["rep"] = rng.choice(np.array([1.0, 1.25, 1.7, 0.5], np.float32), T)
    r["pres"], r["freq"] = rng.choice(np.array([0.0, 0.5], np.float32), T), rng.choice(np.array([0.0, 0.125, 0.3], np.float32), T)
    return {k: torch.from_numpy(v).to(DEV) for k, v in r.items()}


def counts(r, V):
    """[T, V] whole numbers: how often a token stands in a row's history, and how often behind the prompt."""
    ids = r["hist"].long()
    real = (ids >= 0) & (ids < V)
    upto = torch.zeros(ids.numel() + 1, V, dtype=torch.int32, device=DEV)
    upto[1:][real, ids[real]] = 1
    upto = upto.cumsum(0, dtype=torch.int32)
    begin, end = r["start"], r["start"] + r["length"]
    return upto[end] - upto[begin], upto[end] - upto[torch.minimum(begin + r["prompt"], end)]


def column(v):
    return v.double()[:, None]


def expected(x, r, allowed):
    seen, c = counts(r, x.shape[1])
    x = x.double()
    y = torch.where(seen > 0, torch.where(x > 0, x / column(r["rep"]), x * column(r["rep"])), x)
    size = y.abs()
    y = torch.where(c > 0, y - column(r["freq"]) * c - column(r["pres"]), y)
    size = size + torch.where(c > 0, column(r["freq"]) * c + column(r["pres"]), 0.0)
    return torch.where(allowed, y, -float("inf")), torch.where((seen > 0) & allowed, size, 0.0), seen > 0


def in_rows(t, pad):
    """The same rows in a buffer whose rows begin `pad` elements apart from each other."""
    whole = torch.empty(t.shape[0], t.shape[1] + pad, dtype=t.dtype, device=DEV)[:, :t.shape[1]]
    whole.copy_(t)
    return whole


@pytest.mark.parametrize("dtype,V,T", [("f32", 700, 24000), ("bf16", 704, 24000), ("f16", 8200, 12000)])
def test_rows_that_grow_by_one_id(dtype, V, T):
    """Some 20 rows to a CTA and more (24000 of one slice are dealt out to 888 to 1184 CTAs, two slices of 12000 as well): records are read anew several times in
    a run, with tokens of the rows before still to be entered where rows lie off 16 bytes."""
    r = rollouts(V, T, V)
    g = torch.Generator().manual_seed(V)
    x, d = ((2.0 * torch.randn(T, V, generator=g)).to(DEV, DTYPES[dtype]) for _ in range(2))
    few = torch.rand(5, V, generator=g) < torch.tensor([0.02, 0.5, 0.98, 1.0, 0.7])[:, None]
    mask_row = torch.randint(-1, 5, (T,), generator=g, dtype=torch.int32).to(DEV)
    allowed = few.to(DEV)[mask_row.clamp(min=0).long()] | (mask_row < 0)[:, None]
    want, size, seen = expected(x, r, allowed)
    eps = torch.finfo(x.dtype).eps
    bound = (4 if dtype == "f32" else 5) * 2.0 ** -24 * size * (1 + eps) + torch.where(size > 0, eps / 2 * want.abs() + SMALLEST[x.dtype], 0.0)
    dw = torch.where(allowed, torch.where(seen, torch.where(x > 0, d.double() / column(r["rep"]), d.double() * column(r["rep"])), d.double()), 0.0)
    d_bound = torch.where(seen, ((1 if dtype == "f32" else 2) * 2.0 ** -24 * (1 + eps) + eps / 2) * dw.abs() + SMALLEST[x.dtype], 0.0)
    rules = dict(history=r["hist"], history_start=r["start"], history_len=r["length"], allowed=pack(few.numpy()).to(DEV), mask_row=mask_row)
    settings = dict(prompt_len=r["prompt"], repetition=r["rep"], presence=r["pres"], frequency=r["freq"])
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for pad in (0, 1):                                    # rows on 16 bytes, and off them
        apart = in_rows(torch.zeros_like(x), pad)
        sr.sr_adjust_logits(in_rows(x, pad), **rules, **settings, out=apart, status=st)
        assert_near(apart, want, bound, f"adjusted, {pad}")
        same = in_rows(x, pad)
        sr.sr_adjust_logits(same, **rules, **settings, out=same)
        assert torch.equal(same, apart)
        sr.sr_adjust_logits_backward(in_rows(d, pad), in_rows(x, pad), **rules, repetition=r["rep"], d_logits=apart)
        assert_near(apart, dw, d_bound, f"gradient, {pad}")
        for place in (0, 1):                              # of the gradient, and of the logits
            both = in_rows(d, pad), in_rows(x, pad)
            sr.sr_adjust_logits_backward(*both, **rules, repetition=r["rep"], d_logits=both[place])
            assert torch.equal(both[place], apart)
    assert int(st) == sr.SR_STATUS_BAD_TARGET


@pytest.mark.parametrize("unused", [0, 400_000])
def test_frequent_tokens_behind_frequent_tokens(unused):
    """Rows that begin anew one behind the other, some 20 to a CTA, with other tokens that occur more than 8192 times, or the same one on either side of that: what
    was counted for the row before must not stay.  (unused: ids that no row has.  With more than eight a row, a call takes rows to begin anew.)"""
    V, T = 500, 24000
    blocks = [{123: 9000}, {77: 8700, 123: 40}, {123: 8193, 77: 8300}, {123: 8190}, {9: 8600, 77: 8192}, {123: 12, 9: 1}]
    hist = np.concatenate([np.random.default_rng(k).permutation(np.repeat(list(b), list(b.values()))) for k, b in enumerate(blocks)])
    begin = np.concatenate([[0], np.cumsum([sum(b.values()) for b in blocks])])
    # rows of a turn: (block, length), each beginning anew or, with one id more, going on; 23 of them, so that CTAs begin in different places
    turn = [(0, 8500), (1, None), (0, 8999), (0, 9000), (3, None), (2, None), (5, None), (4, None), (4, 16792), (0, 8192), (3, 8189), (3, 8190), (1, 8000), (0, 8191), (0, 8192), (0, 8193), (2, 16000),
            (5, 3), (2, None), (1, 8740), (4, None), (0, 8600), (3, 20)]
    assert len(turn) == 23
    rows = [(int(begin[b]), int(begin[b + 1] - begin[b]) if n is None else n) for b, n in turn]
    times = np.stack([np.bincount(hist[a:a + n], minlength=V) for a, n in rows]).astype(np.float32)
    assert all(a + n <= hist.size for a, n in rows) and (times > 8192).sum() >= 8
    kind = np.arange(T) % len(rows)
    want = torch.from_numpy(-times[kind]).to(DEV)                       # exact: whole numbers below 2^24
    history = torch.from_numpy(np.concatenate([hist, np.full(unused, -1)]).astype(np.int32)).to(DEV)
    start = torch.from_numpy(np.array([a for a, _ in rows], np.int64)[kind]).to(DEV)
    length = torch.from_numpy(np.array([n for _, n in rows], np.int32)[kind]).to(DEV)
    assert (history.numel() > 8 * T) == (unused > 0)
    for pad in (0, 1):
        x = in_rows(torch.zeros(T, V, device=DEV), pad)
        out = in_rows(torch.ones(T, V, device=DEV), pad)
        rules = dict(history=history, history_start=start, history_len=length, frequency=torch.ones(T, device=DEV))
        sr.sr_adjust_logits(x, **rules, out=out)
        assert torch.equal(out, want), pad
        sr.sr_adjust_logits(x, **rules, out=x)
        assert torch.equal(x, want), pad

"""Adjusted logits and their gradient against the formulas in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_05802_b200 as sr
from helpers import Guarded
from tokens_ref import DTYPES, adjust, adjust_gradient, pack
from train_ref import assert_near

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def dev(a, dtype=None):
    t = None if a is None else torch.from_numpy(np.ascontiguousarray(a)) if isinstance(a, np.ndarray) else a
    return None if t is None else t.to(DEV) if dtype is None else t.to(DEV, dtype)


def logits(T, V, dtype, seed, pad=0, special=True):
    g = torch.Generator().manual_seed(seed)
    x = 3.0 * torch.randn(T, V + pad, generator=g)
    if special and V >= 16:
        x[:, 3], x[:, 5], x[:, 7], x[:, 11] = float("-inf"), float("nan"), float("inf"), 0.0
    return x.to(DEV, DTYPES[dtype])[:, :V]


def rules(T, V, seed, which, shared=False, most=40):
    """Numpy rules of T rows.  shared: rows of three rollouts, each going on where the one before it ended."""
    rng = np.random.default_rng(seed)
    r = {}
    if set(which) & set("rpf"):
        n = 3 if shared else T
        total = most * n
        r["hist"] = np.where(rng.random(total) < 0.7, np.exp(rng.random(total) * np.log(V + 1)) - 1, rng.integers(0, V, total)).astype(np.int32).clip(0, V - 1)
        r["hist"][rng.random(total) < 0.05] = -3
        if shared:
            owner = np.sort(rng.integers(0, 3, T))
            r["start"] = (owner * most).astype(np.int64)
            r["prompt"] = np.array([0, most // 3, most])[owner].astype(np.int32)
            r["length"] = np.minimum(most // 4 + np.array([np.sum(owner[:t] == owner[t]) for t in range(T)]) * rng.integers(0, 3), most).astype(np.int32)
        else:
            r["start"] = (np.arange(T) * most).astype(np.int64)
            r["length"] = rng.integers(0, most + 1, T).astype(np.int32)
            r["prompt"] = rng.integers(0, most + 1, T).astype(np.int32)
        if "r" in which:
            r["rep"] = rng.choice(np.array([1.0, 1.1, 1.7, 0.5], dtype=np.float32), T)
        if "p" in which:
            r["pres"] = rng.choice(np.array([0.0, 0.5, -0.25], dtype=np.float32), T)
        if "f" in which:
            r["freq"] = rng.choice(np.array([0.0, 0.125, 0.3], dtype=np.float32), T)
    if "b" in which:
        n = min(V, 13)
        r["bias_token"] = rng.integers(0, V, n * T).astype(np.int32)          # some twice: the last one counts
        r["bias_value"] = rng.normal(size=n * T).astype(np.float32)
        r["bias_start"] = (rng.permutation(T) * n).astype(np.int64)
        r["bias_len"] = rng.integers(0, n + 1, T).astype(np.int32)
        if shared:
            r["bias_start"][:], r["bias_len"][:] = 0, n
    if "m" in which:
        M = max(3, T // 2)
        r["allowed"] = rng.random((M, V)) < rng.choice([0.02, 0.5, 0.98], (M, 1))
        r["allowed"][0], r["allowed"][1] = False, True
        r["mask_row"] = rng.integers(-1, M, T).astype(np.int32)
    return r


NAMES = {"hist": "history", "start": "history_start", "length": "history_len", "prompt": "prompt_len", "rep": "repetition", "pres": "presence", "freq": "frequency"}


def on_device(r):
    return {NAMES.get(k, k): (pack(v).to(DEV) if k == "allowed" else dev(v)) for k, v in r.items()}


def backward_rules(r):
    return {k: v for k, v in r.items() if k in ("hist", "start", "length", "rep", "allowed", "mask_row")}


def check(x, r, out, status=0):
    want, bound = adjust(x, **r)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    sr.sr_adjust_logits(x, **on_device(r), out=out, status=st)
    torch.cuda.synchronize()
    assert_near(out.cpu(), want, bound, "adjusted")
    assert int(st) == status
    return want


def check_backward(d, x, r, dx, status=0):
    r = backward_rules(r)
    want, bound = adjust_gradient(d, x, **r)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    sr.sr_adjust_logits_backward(d, x, **on_device(r), d_logits=dx, status=st)
    torch.cuda.synchronize()
    assert_near(dx.cpu(), want, bound, "gradient")
    assert int(st) == status


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T,V,pad", [(1, 1, 0), (2, 7, 0), (5, 33, 6), (9, 1000, 0), (3, 8192, 0), (4, 8193, 0), (2, 16389, 3), (3, 50021, 0), (2, 151936, 64)])
@pytest.mark.parametrize("which", ["rpfbm", "r", "pf", "b", "m", "rm", ""])
def test_sizes_and_rules(dtype, T, V, pad, which):
    x = logits(T, V, dtype, T + V, pad)
    r = rules(T, V, V + len(which), which)
    guard = Guarded(DEV)
    whole = guard.alloc((T, V + pad), x.dtype, 7.0)
    check(x, r, whole[:, :V])
    guard.check("out")
    assert bool((whole[:, V:] == 7.0).all())
    d = logits(T, V, dtype, T + V + 1, pad)
    whole.fill_(7.0)
    check_backward(d, x, r, whole[:, :V])
    guard.check("d_logits")
    assert bool((whole[:, V:] == 7.0).all())


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [40, 9001, 24576])
@pytest.mark.parametrize("which", ["rpfbm", "rf", "pm"])
def test_in_place_is_the_same(dtype, V, which):
    T = 6
    x = logits(T, V, dtype, V, 5)
    r = rules(T, V, V, which)
    apart, same = torch.empty_like(x), logits(T, V, dtype, V, 5)
    check(x, r, apart)
    sr.sr_adjust_logits(same, **on_device(r), out=same)
    assert torch.equal(same.nan_to_num(nan=1e4), apart.nan_to_num(nan=1e4)) and torch.equal(same.isnan(), apart.isnan())
    d = logits(T, V, dtype, V + 1, 5)
    rb = on_device(backward_rules(r))
    sr.sr_adjust_logits_backward(d, x, **rb, d_logits=apart)
    over_logits = logits(T, V, dtype, V, 5)
    sr.sr_adjust_logits_backward(d, over_logits, **rb, d_logits=over_logits)
    sr.sr_adjust_logits_backward(d, x, **rb, d_logits=d)
    for got in (d, over_logits):
        assert torch.equal(got.nan_to_num(nan=1e4), apart.nan_to_num(nan=1e4)) and torch.equal(got.isnan(), apart.isnan())


@pytest.mark.parametrize("dtype,V,T", [("bf16", 8200, 700), ("f32", 700, 4000), ("f16", 30001, 300), ("bf16", 8203, 700), ("f32", 701, 4000)])
@pytest.mark.parametrize("which", ["rpf", "rpfbm"])
def test_rollouts_as_a_whole(dtype, V, T, which):
    """Many rows of a few histories that grow row by row: runs of rows in one CTA, one rollout after the other."""
    x = logits(T, V, dtype, V)
    r = rules(T, V, V, which, shared=True, most=90)
    out = torch.empty_like(x)
    check(x, r, out)
    check_backward(logits(T, V, dtype, 1), x, r, out)


def test_gradient_of_many_rows_that_come_from_memory():
    """Far more than L2 holds, masks that leave some rows nothing to change: copies ahead that a row has no use for must not reach the next
    one's.  Every element is d, d / r or d r, by the sign of its own logit."""
    T, V = 1024, 151936
    g = torch.Generator(device=DEV).manual_seed(1)
    x, d = (torch.randn(T, V, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    history = (torch.exp(torch.rand(1200, generator=g, device=DEV) * np.log(V)) - 1).to(torch.int32)
    start, length = torch.zeros(T, dtype=torch.int64, device=DEV), (torch.arange(T, device=DEV) // 2 + 400).to(torch.int32)
    few = torch.rand(64, V, generator=g, device=DEV) < torch.where(torch.arange(64, device=DEV)[:, None] % 2 == 0, 0.01, 0.98)
    mask_row = torch.randint(0, 64, (T,), generator=g, device=DEV, dtype=torch.int32)
    dx, rep = torch.empty_like(d), torch.full((T,), 2.0, device=DEV)                 # 2: no rounding
    rest = dict(history=history, history_start=start, history_len=length, repetition=rep, allowed=pack(few.cpu().numpy()).to(DEV), mask_row=mask_row)
    for _ in range(3):
        x, d = x.roll(1, 1), d.roll(3, 1)
        sr.sr_adjust_logits_backward(d, x, **rest, d_logits=dx)
        for a in range(0, T, 128):
            r = slice(a, a + 128)
            seen = torch.zeros(128, V, dtype=torch.bool, device=DEV)
            for t in range(128):
                seen[t, history[:int(length[a + t])].long()] = True
            want = torch.where(seen, torch.where(x[r] > 0, d[r] * 0.5, d[r] * 2), d[r])
            want = torch.where(few[mask_row[r].long()], want, torch.zeros_like(want))
            assert torch.equal(dx[r], want), a
    sr.sr_adjust_logits(x, **rest, out=dx)                                           # and the rows themselves
    for a in range(0, T, 128):
        r = slice(a, a + 128)
        seen = torch.zeros(128, V, dtype=torch.bool, device=DEV)
        for t in range(128):
            seen[t, history[:int(length[a + t])].long()] = True
        want = torch.where(seen, torch.where(x[r] > 0, x[r] * 0.5, x[r] * 2), x[r])
        assert torch.equal(dx[r], torch.where(few[mask_row[r].long()], want, torch.full_like(want, -float("inf")))), a


def test_rows_that_do_not_go_on():
    """Next to one another: a history that shrinks, one that stays, another prompt, another bias list, an earlier start."""
    V, T = 600, 4096 * 4                                  # many more rows than CTAs: runs
    rng = np.random.default_rng(1)
    hist = rng.integers(0, V, 64).astype(np.int32)
    r = {"hist": hist, "start": rng.integers(0, 2, T).astype(np.int64), "length": rng.integers(0, 4, T).astype(np.int32) * 9, "prompt": rng.integers(0, 2, T).astype(np.int32) * 5,
         "rep": np.full(T, 1.5, np.float32), "freq": np.full(T, 0.25, np.float32), "pres": np.full(T, 0.5, np.float32), "bias_token": rng.integers(0, V, 20).astype(np.int32),
         "bias_value": rng.normal(size=20).astype(np.float32), "bias_start": rng.integers(0, 2, T).astype(np.int64), "bias_len": rng.integers(0, 3, T).astype(np.int32) * 8}
    for pad in (0, 3):
        x = logits(T, V, "bf16", 2, pad)
        check(x, r, torch.empty(T, V + pad, dtype=x.dtype, device=DEV)[:, :V])


@pytest.mark.parametrize("shift_in,shift_out", [(0, 1), (3, 0), (1, 1), (5, 2)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rows_off_16_bytes(dtype, shift_in, shift_out):
    T, V = 4, 9000
    x = torch.empty(T, V + 8, dtype=DTYPES[dtype], device=DEV)[:, shift_in:shift_in + V]
    x.copy_(logits(T, V, dtype, 5))
    r = rules(T, V, 5, "rpfbm")
    whole = torch.full((T, V + 11), 3.0, dtype=x.dtype, device=DEV)
    out = whole[:, shift_out:shift_out + V]
    check(x, r, out)
    d = logits(T, V, dtype, 6, 2)
    check_backward(d, x, r, out)
    assert bool((whole[:, :shift_out] == 3.0).all()) and bool((whole[:, shift_out + V:] == 3.0).all())


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_gradient_whose_logits_lie_elsewhere(dtype):
    """Gradients on 16 bytes, the logits off them and with another pitch."""
    T, V = 300, 9000
    x = torch.empty(T, V + 13, dtype=DTYPES[dtype], device=DEV)[:, 3:3 + V]
    x.copy_(logits(T, V, dtype, 5))
    r = rules(T, V, 5, "rm", shared=True, most=200)
    d = logits(T, V, dtype, 6)
    check_backward(d, x, r, torch.empty_like(d))


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_what_a_mask_leaves(dtype):
    """Nothing, one token, all; NaN, infinities and the type's lowest value in masked places and in allowed ones."""
    V = 20000
    low = torch.finfo(DTYPES[dtype]).min
    x = torch.zeros(4, V, dtype=DTYPES[dtype], device=DEV)
    for k, v in enumerate([float("nan"), float("inf"), float("-inf"), low, -low, -0.0]):
        x[:, k::6] = v
    allowed = np.zeros((3, V), dtype=bool)
    allowed[1, 9973] = True
    allowed[2] = True
    row = np.array([0, 1, 2, 0], dtype=np.int32)
    out = torch.empty_like(x)
    check(x, {"allowed": allowed, "mask_row": row}, out)
    assert bool((out[0] == float("-inf")).all()) and int((out[1] != float("-inf")).sum()) == 1
    assert torch.equal(out[2].view(torch.int32 if dtype == "f32" else torch.int16), x[2].view(torch.int32 if dtype == "f32" else torch.int16))
    check_backward(x, None, {"allowed": allowed, "mask_row": row}, out)
    lp = torch.empty(4, device=DEV)                       # rows without a token: NaN in their own outputs
    sr.sr_adjust_logits(torch.ones_like(x), allowed=pack(allowed).to(DEV), mask_row=dev(row), out=out)
    sr.sr_token_logprob(out, torch.full((4,), 9973, dtype=torch.int32, device=DEV), logp=lp)
    assert lp.isnan().tolist() == [True, False, False, True] and float(lp[1]) == 0.0


def test_one_mask_a_row_without_an_index():
    x = logits(5, 777, "bf16", 1)
    r = rules(5, 777, 3, "m")
    allowed = np.concatenate([r["allowed"]] * 3)[:5]
    check(x, {"allowed": allowed}, torch.empty_like(x))


def test_positions_and_ids_that_do_not_count():
    V, T = 500, 8
    hist = np.array([1, 2, -1, 499, 2, 3, -2 ** 31, 7], dtype=np.int32)
    r = {"hist": hist, "start": np.array([-3, 0, 6, 100, -2 ** 62, 2 ** 62, 7, -2], dtype=np.int64), "length": np.array([5, 99, 9, 3, 7, 7, 2 ** 31 - 1, 2 ** 31 - 1], dtype=np.int32),
         "prompt": np.array([0, 3, -5, 0, 0, 0, 2 ** 31 - 1, 4], dtype=np.int32), "rep": np.full(T, 2.0, np.float32), "pres": np.ones(T, np.float32), "freq": np.ones(T, np.float32)}
    x = logits(T, V, "f32", 3)
    check(x, {**r, "length": np.minimum(r["length"], 1000)}, torch.empty_like(x))       # (the reference walks lengths)
    out, long = torch.empty_like(x), torch.empty_like(x)
    sr.sr_adjust_logits(x, **on_device(r), out=long)
    sr.sr_adjust_logits(x, **on_device({**r, "length": np.minimum(r["length"], 1000)}), out=out)
    assert torch.equal(out.nan_to_num(nan=1e4), long.nan_to_num(nan=1e4))


def test_status_bits():
    V, T = 100, 2
    x = logits(T, V, "f32", 3)
    out = torch.empty_like(x)
    one = {"start": np.zeros(T, np.int64), "rep": np.full(T, 2.0, np.float32)}
    check(x, {**one, "hist": np.array([5, 100], np.int32), "length": np.array([1, 2], np.int32)}, out, sr.SR_STATUS_BAD_TARGET)
    check(x, {**one, "hist": np.array([5, 100], np.int32), "length": np.array([1, 1], np.int32)}, out, 0)
    check(x, {**one, "hist": np.array([5, 9], np.int32), "length": np.array([1, -2], np.int32)}, out, sr.SR_STATUS_NEG_LEN)
    check_backward(x, x, {**one, "hist": np.array([5, 100], np.int32), "length": np.array([-1, 2], np.int32)}, out, sr.SR_STATUS_BAD_TARGET | sr.SR_STATUS_NEG_LEN)
    check(x, {"allowed": np.ones((1, V), bool), "mask_row": np.array([0, 1], np.int32)}, out, sr.SR_STATUS_BAD_INDEX)
    bias = {"bias_start": np.zeros(T, np.int64), "bias_value": np.ones(2, np.float32)}
    check(x, {**bias, "bias_token": np.array([3, 200], np.int32), "bias_len": np.array([2, 0], np.int32)}, out, sr.SR_STATUS_BAD_TARGET)
    check(x, {**bias, "bias_token": np.array([3, -200], np.int32), "bias_len": np.array([2, -1], np.int32)}, out, sr.SR_STATUS_NEG_LEN)


def test_a_bias_twice_and_lists_that_reach_out():
    V = 9000
    x = logits(3, V, "f32", 4)
    r = {"bias_token": np.array([8500, 1, 8500, 1, 8500, 2, -1], np.int32), "bias_value": np.array([1, 2, 4, 8, 16, 32, 64], np.float32), "bias_start": np.array([-2, 0, 4], np.int64),
         "bias_len": np.array([5, 7, 2 ** 31 - 1], np.int32)}
    check(x, {**r, "bias_len": np.minimum(r["bias_len"], 50)}, torch.empty_like(x))
    sr.sr_adjust_logits(x, **on_device(r), out=torch.empty_like(x))


@pytest.mark.parametrize("which", ["rpfbm", "rm"])
def test_a_list_of_its_own_for_hundreds_of_rows(which):
    """Rows that all begin anew, several to a CTA: tables emptied and filled again, ids copied ahead."""
    T, V = 900, 20000
    x = logits(T, V, "bf16", 9)
    r = rules(T, V, 9, which, most=70)
    out = torch.empty_like(x)
    check(x, r, out)
    check_backward(logits(T, V, "bf16", 10), x, r, out)


def test_lists_longer_than_what_is_copied_ahead():
    T, V = 700, 9000
    rng = np.random.default_rng(4)
    n = 3000
    r = {"hist": rng.integers(0, V, n).astype(np.int32), "start": rng.integers(0, 900, T).astype(np.int64), "length": rng.integers(900, 2100, T).astype(np.int32),
         "prompt": rng.integers(0, 2100, T).astype(np.int32), "rep": np.full(T, 1.5, np.float32), "freq": np.full(T, 0.125, np.float32), "bias_token": rng.integers(0, V, n).astype(np.int32),
         "bias_value": rng.normal(size=n).astype(np.float32), "bias_start": rng.integers(0, 900, T).astype(np.int64), "bias_len": rng.integers(200, 2100, T).astype(np.int32)}
    x = logits(T, V, "f32", 2)
    check(x, r, torch.empty_like(x))


def test_a_bias_list_that_is_cut():
    V = 70000
    x = logits(1, V, "f32", 2)
    r = {"bias_token": np.arange(V, dtype=np.int32), "bias_value": np.ones(V, np.float32), "bias_start": np.zeros(1, np.int64)}
    out, st = torch.empty_like(x), torch.zeros(1, dtype=torch.int32, device=DEV)
    sr.sr_adjust_logits(x, **on_device({**r, "bias_len": np.array([V], np.int32)}), out=out, status=st)
    assert int(st) == sr.SR_STATUS_BAD_INDEX
    want, bound = adjust(x, **{**r, "bias_len": np.array([65535], np.int32)})
    assert_near(out.cpu(), want, bound, "cut")


def test_more_frequent_tokens_than_the_table_holds():
    """Each of 80 tokens of one slice 8500 times: beyond the 14 bits of a count, and more of them than have a counter of their own."""
    V, n, each = 9000, 80, 8500
    hist = np.repeat(np.arange(n, dtype=np.int32), each)
    r = {"hist": hist, "start": np.zeros(2, np.int64), "length": np.array([n * each, n * each - 3], np.int32), "prompt": np.array([5, 5], np.int32), "freq": np.full(2, 2.0 ** -12, np.float32)}
    x = logits(2, V, "f32", 1)
    check(x, r, torch.empty_like(x))


@pytest.mark.parametrize("step", [1, 2])
def test_a_token_that_becomes_frequent(step):
    """Its count leaves 14 bits between two rows of one rollout, added by one thread or by all."""
    T, V = 40, 500
    hist = np.full(9000, 123, np.int32)
    r = {"hist": hist, "start": np.zeros(T, np.int64), "length": (8170 + step * np.arange(T)).astype(np.int32), "freq": np.full(T, 0.25, np.float32), "pres": np.ones(T, np.float32)}
    big = {k: np.concatenate([v] * 40) if k != "hist" else v for k, v in r.items()}              # many rows to a CTA
    for pad in (0, 1):                                    # rows on 16 bytes, and off them
        x = logits(40 * T, V, "f32", 1, pad)
        check(x, big, torch.empty(40 * T, V + pad, device=DEV)[:, :V])


def test_no_rows_and_empty_lists():
    e = lambda *s, **k: torch.empty(*s, device=DEV, **k)
    sr.sr_adjust_logits(e(0, 50), out=e(0, 50))
    sr.sr_adjust_logits_backward(e(0, 50), None, d_logits=e(0, 50))
    x = logits(2, 50, "f32", 1)
    out = torch.empty_like(x)
    none = dict(history=e(0, dtype=torch.int32), history_start=torch.zeros(2, dtype=torch.int64, device=DEV), history_len=torch.full((2,), 4, dtype=torch.int32, device=DEV))
    sr.sr_adjust_logits(x, **none, repetition=torch.full((2,), 2.0, device=DEV), bias_token=e(0, dtype=torch.int32), bias_value=e(0), out=out)
    assert torch.equal(out.nan_to_num(nan=9.0), x.nan_to_num(nan=9.0))


@pytest.mark.parametrize("n", [5000, 200_003])
def test_long_histories(n):
    """Thousands of times the same token, and histories longer than a CTA has threads many times over."""
    V = 20011
    rng = np.random.default_rng(n)
    hist = rng.integers(0, V, n).astype(np.int32)
    hist[rng.random(n) < 0.5] = 12345
    T = 3
    r = {"hist": hist, "start": np.array([0, 0, 1], np.int64), "length": np.array([n - 1, n, n - 1], np.int32), "prompt": np.array([n // 2, n // 2, 0], np.int32),
         "rep": np.full(T, 1.25, np.float32), "freq": np.full(T, 2.0 ** -10, np.float32)}
    x = logits(T, V, "f32", 1)
    check(x, r, torch.empty_like(x))
    check_backward(x, x, r, torch.empty_like(x))


def test_rows_behind_2_to_the_31_elements():
    V, pitch, T = 4000, (1 << 30) + 8, 4
    whole = torch.empty(T * pitch, dtype=torch.bfloat16, device=DEV)
    x = whole.as_strided((T, V), (pitch, 1))
    x.copy_(logits(T, V, "bf16", 8))
    r = rules(T, V, 8, "rpfbm")
    check(x, r, torch.empty(T, V, dtype=x.dtype, device=DEV))
    apart = x.clone()
    sr.sr_adjust_logits(apart, **on_device(r), out=apart)
    sr.sr_adjust_logits(x, **on_device(r), out=x)
    assert torch.equal(x.nan_to_num(nan=1e4), apart.nan_to_num(nan=1e4))


def test_captured_and_on_other_streams():
    """A graph replayed on other data gives what separate calls give, beside a call on another stream."""
    T, V = 16, 30000
    batches = [(logits(T, V, "bf16", s), on_device(rules(T, V, s, "rpfbm"))) for s in range(3)]
    x, r = batches[0][0].clone(), {k: v.clone() for k, v in batches[0][1].items()}
    out, dx = torch.empty_like(x), torch.empty_like(x)
    rb = {k: v for k, v in r.items() if k in ("history", "history_start", "history_len", "repetition", "allowed", "mask_row")}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sr.sr_adjust_logits(x, **r, out=out)
        sr.sr_adjust_logits_backward(out, x, **rb, d_logits=dx)
    side = torch.cuda.Stream()
    for bx, br in batches[1:] + batches[:1]:
        x.copy_(bx)
        for k, v in r.items():
            v.copy_(br[k])
        torch.cuda.synchronize()
        graph.replay()
        e, e_dx = torch.empty_like(x), torch.empty_like(x)
        sr.sr_adjust_logits(bx, **br, out=e, stream=side)
        with torch.cuda.stream(side):
            sr.sr_adjust_logits_backward(e, bx, **{k: br[k] for k in rb}, d_logits=e_dx)
        torch.cuda.synchronize()
        assert torch.equal(out.nan_to_num(nan=1e4), e.nan_to_num(nan=1e4)) and torch.equal(dx.nan_to_num(nan=1e4), e_dx.nan_to_num(nan=1e4))


def test_gradient_against_differences():
    """Central differences of the formula in 64 bits, away from x = 0."""
    T, V = 3, 200
    x = logits(T, V, "f32", 2, special=False)
    x = torch.where(x.abs() < 0.1, 0.5, x)
    r = rules(T, V, 2, "rpfbm")
    allowed, rows = r.pop("allowed"), r.pop("mask_row")
    d = logits(T, V, "f32", 3, special=False)
    dx = torch.empty_like(x)
    full = {**r, "allowed": allowed, "mask_row": rows}
    sr.sr_adjust_logits_backward(d, x, **on_device(backward_rules(full)), d_logits=dx)
    ok = np.stack([np.ones(V, bool) if m < 0 else allowed[m] for m in rows])
    up, down = (adjust(x.double() + h, **r)[0] for h in (1e-3, -1e-3))
    want = torch.from_numpy(ok) * d.cpu().double() * (up - down) / 2e-3
    assert float((dx.cpu().double() - want).abs().max()) <= 2.0 ** -22 * float(want.abs().max()) + 1e-9

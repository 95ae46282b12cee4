"""Embedding of tokens and the gradient of its table against sums in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2605_05802_b200 as sr
from helpers import Guarded
from tokens_ref import DTYPES, embed, embed_gradient
from train_ref import assert_near

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f16")]       # of the table, of the rows


def draw_tokens(T, V, seed, how="text", padding=0.1):
    rng = np.random.default_rng(seed)
    if how == "text":
        t = (np.exp(rng.random(T) * np.log(V + 1)) - 1).astype(np.int64).clip(0, V - 1)
    elif how == "all":
        t = rng.permutation(max(T, V))[:T] % V
    elif how == "one":
        t = np.full(T, V - 1)
    else:
        t = rng.integers(0, V, T)
    t[rng.random(T) < padding] = -1
    return torch.from_numpy(t.astype(np.int32)).to(DEV)


def rows(n, D, dtype, seed, pad=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    whole = torch.randn(n, D + pad + shift, generator=g).to(DEV, DTYPES[dtype])
    return whole[:, shift:shift + D]


def gradient(d, tokens, scale, V, table_dtype, had=None, pad=0, shift=0, guard=None):
    """d_table as the kernel leaves it, in a padded buffer whose rest is checked."""
    D = d.shape[1]
    guard = Guarded(DEV)
    whole = guard.alloc((V, D + pad + shift), DTYPES[table_dtype], 5.0)
    table = whole[:, shift:shift + D]
    if had is not None:
        table.copy_(had)
    ws = guard.alloc((sr.sr_embed_tokens_backward_workspace_bytes(tokens.numel(), V, D),), torch.uint8)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    sr.sr_embed_tokens_backward(d, tokens, scale, d_table=table, accumulate=had is not None, workspace=ws, status=st)
    guard.check("gradient")
    assert bool((whole[:, :shift] == 5.0).all()) and bool((whole[:, shift + D:] == 5.0).all())
    return table, int(st)


@pytest.mark.parametrize("table,out", TYPES)
@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (3, 7, 5), (70, 50, 64), (33, 1000, 1001), (1000, 300, 520), (257, 20000, 4096), (5, 3, 9000)])
def test_embedding(table, out, T, V, D):
    w = rows(V, D, table, T)
    tokens = draw_tokens(T, V, D)
    guard = Guarded(DEV)
    y = guard.alloc((T, D), DTYPES[out], 5.0)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    for scale in (1.0, D ** 0.5, -0.3):
        sr.sr_embed_tokens(w, tokens, scale, out=y, status=st)
        guard.check("out")
        want, bound = embed(w, tokens, float(np.float32(scale)), y.dtype)
        assert_near(y, want, bound, "embedded")
        assert bool((y[tokens < 0].view(torch.int32 if out == "f32" else torch.int16) == 0).all())
    if table == out:
        sr.sr_embed_tokens(w, tokens, out=y)
        assert torch.equal(y[tokens >= 0], w[tokens[tokens >= 0].long()])
    assert int(st) == 0


@pytest.mark.parametrize("table,out", TYPES)
@pytest.mark.parametrize("T,V,D,how", [(1, 1, 1, "text"), (2, 5, 3, "one"), (100, 50, 64, "text"), (1200, 4096, 256, "text"), (333, 70, 1001, "text"), (3000, 9, 40, "even"), (700, 700, 33, "all"),
                                       (9000, 151936, 72, "text"), (20001, 30, 128, "one"), (40000, 1500, 24, "even"), (8192, 100, 8, "text"), (8193, 100, 8, "text"), (500, 20000, 2056, "text")])
def test_gradient(table, out, T, V, D, how):
    d = rows(T, D, out, T + 1)
    tokens = draw_tokens(T, V, T + D, how)
    scale = 1.0 if D % 2 else D ** 0.5
    got, st = gradient(d, tokens, scale, V, table)
    want, bound = embed_gradient(d, tokens, float(np.float32(scale)), V, got.dtype)
    assert_near(got, want, bound, "gradient")
    untaken = torch.ones(V, dtype=torch.bool, device=DEV)
    untaken[tokens[tokens >= 0].long()] = False
    assert bool((got[untaken].view(torch.int32 if table == "f32" else torch.int16) == 0).all()) and st == 0
    again, _ = gradient(d, tokens, scale, V, table)
    assert torch.equal(got, again)


@pytest.mark.parametrize("table,out", TYPES)
@pytest.mark.parametrize("T,V,D,pad,shift", [(50, 40, 64, 0, 0), (900, 300, 100, 3, 1), (12000, 2000, 96, 8, 0), (400, 3, 1000, 0, 4)])
def test_added_to_what_stands_there(table, out, T, V, D, pad, shift):
    d = rows(T, D, out, 3, pad, shift)
    tokens = draw_tokens(T, V, 4)
    had = rows(V, D, table, 5)
    untaken = torch.ones(V, dtype=torch.bool, device=DEV)
    untaken[tokens[tokens >= 0].long()] = False
    had[untaken] = float("nan")                           # neither read nor written
    got, _ = gradient(d, tokens, 1.5, V, table, had, pad, shift)
    want, bound = embed_gradient(d, tokens, 1.5, V, got.dtype, had)
    assert_near(got, want, bound, "sum")
    assert bool(got[untaken].isnan().all())


@pytest.mark.parametrize("table,out", TYPES)
@pytest.mark.parametrize("pad,shift", [(1, 0), (2, 2), (8, 8), (5, 3), (4, 4)])
def test_rows_apart_and_off_16_bytes(table, out, pad, shift):
    T, V, D = 60, 50, 264
    w, d = rows(V, D, table, 1, pad, shift), rows(T, D, out, 2, pad, shift)
    tokens = draw_tokens(T, V, 3)
    whole = torch.full((T, D + pad + shift), 5.0, dtype=DTYPES[out], device=DEV)
    y = whole[:, shift:shift + D]
    sr.sr_embed_tokens(w, tokens, 2.0, out=y)
    want, bound = embed(w, tokens, 2.0, y.dtype)
    assert_near(y, want, bound, "embedded")
    assert bool((whole[:, :shift] == 5.0).all()) and bool((whole[:, shift + D:] == 5.0).all())
    got, _ = gradient(d, tokens, 2.0, V, table, None, pad, shift)
    want, bound = embed_gradient(d, tokens, 2.0, V, got.dtype)
    assert_near(got, want, bound, "gradient")


def test_tokens_outside_the_vocabulary():
    V, D = 100, 64
    tokens = torch.tensor([5, -1, 100, -2 ** 31, 2 ** 31 - 1, 99, 5, 0], dtype=torch.int32, device=DEV)
    w, d = rows(V, D, "bf16", 1), rows(8, D, "bf16", 2)
    d[1:5] = float("nan")                                 # rows of no token are not read
    y, st = torch.empty(8, D, dtype=torch.bfloat16, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    sr.sr_embed_tokens(w, tokens, out=y, status=st)
    assert int(st) == sr.SR_STATUS_BAD_TARGET and not bool(y[1:5].any()) and torch.equal(y[5], w[99])
    got, st = gradient(d, tokens, 1.0, V, "bf16")
    want, bound = embed_gradient(d.nan_to_num(), tokens, 1.0, V, got.dtype)
    assert_near(got, want, bound, "gradient")
    assert st == sr.SR_STATUS_BAD_TARGET
    tokens[2], tokens[4] = -7, -8
    sr.sr_embed_tokens(w, tokens, out=y)
    assert gradient(d, tokens, 1.0, V, "bf16")[1] == 0


def test_no_tokens_and_none_that_counts():
    V, D = 30, 16
    for T in (0, 5):
        tokens = torch.full((T,), -1, dtype=torch.int32, device=DEV)
        d = torch.full((T, D), float("nan"), device=DEV)
        got, _ = gradient(d, tokens, 1.0, V, "f32")
        assert not bool(got.any())
        had = rows(V, D, "f32", 1)
        assert torch.equal(gradient(d, tokens, 1.0, V, "f32", had)[0], had)
        y = torch.full((T, D), 3.0, device=DEV)
        sr.sr_embed_tokens(had, tokens, out=y)
        assert not bool(y.any())


def test_numbers_that_are_not_finite_stay_in_their_rows():
    V, D = 10, 24
    tokens = torch.tensor([1, 2, 1, 3, 2], dtype=torch.int32, device=DEV)
    d = rows(5, D, "f32", 1)
    d[2, 3], d[4, 5] = float("nan"), float("inf")
    got, _ = gradient(d, tokens, 1.0, V, "f32")
    bad = torch.zeros(V, D, dtype=torch.bool, device=DEV)
    bad[1, 3], bad[2, 5] = True, True
    assert torch.equal(~got.isfinite(), bad)


@pytest.mark.parametrize("V", [1, 2, 1023, 1024, 1 << 20, (1 << 20) + 1, 3_000_000])
def test_digits_of_the_sort(V):
    """One, two and three passes, the last token of the vocabulary among those that are taken."""
    T, D = 9000, 2
    tokens = draw_tokens(T, V, V, "even")
    tokens[7], tokens[8001] = V - 1, V - 1
    d = rows(T, D, "f32", 1)
    got, _ = gradient(d, tokens, 1.0, V, "f32")
    want, bound = embed_gradient(d, tokens, 1.0, V, got.dtype)
    assert_near(got, want, bound, "gradient")


@pytest.mark.parametrize("T", [300_000, 1_000_003])
def test_many_tokens(T):
    V, D = 50000, 16
    tokens = draw_tokens(T, V, T)
    d = rows(T, D, "bf16", 1)
    got, _ = gradient(d, tokens, 1.0, V, "f32")
    want, bound = embed_gradient(d, tokens, 1.0, V, got.dtype)
    assert_near(got, want, bound, "gradient")


def test_rows_behind_2_to_the_31_elements():
    pitch, V, D, T = (1 << 30) + 8, 4, 512, 9
    whole = torch.empty(V * pitch, dtype=torch.bfloat16, device=DEV)
    w = whole.as_strided((V, D), (pitch, 1))
    w.copy_(rows(V, D, "bf16", 1))
    tokens = draw_tokens(T, V, 1, "even", 0.0)
    tokens[0] = 3
    y = torch.empty(T, D, dtype=torch.bfloat16, device=DEV)
    sr.sr_embed_tokens(w, tokens, out=y)
    assert torch.equal(y, w[tokens.long()])
    d = rows(T, D, "bf16", 2)
    ws = torch.empty(sr.sr_embed_tokens_backward_workspace_bytes(T, V, D), dtype=torch.uint8, device=DEV)
    sr.sr_embed_tokens_backward(d, tokens, d_table=w, workspace=ws)
    want, bound = embed_gradient(d, tokens, 1.0, V, w.dtype)
    assert_near(w, want, bound, "table far apart")
    far = whole.as_strided((4, D), (pitch, 1))            # and the tokens' rows
    far.copy_(d[:4])
    got, _ = gradient(far, tokens[:4], 1.0, V, "f32")
    want, bound = embed_gradient(d[:4], tokens[:4], 1.0, V, got.dtype)
    assert_near(got, want, bound, "rows far apart")


def test_captured_and_on_other_streams():
    """A graph replayed on other tokens gives what separate calls give, beside a call on another stream with a workspace of its own."""
    T, V, D = 9500, 3000, 48
    batches = [(draw_tokens(T, V, s), rows(T, D, "bf16", s)) for s in range(3)]
    tokens, d = batches[0][0].clone(), batches[0][1].clone()
    n = sr.sr_embed_tokens_backward_workspace_bytes(T, V, D)
    ws, ws2 = (torch.empty(n, dtype=torch.uint8, device=DEV) for _ in range(2))
    table, y = torch.empty(V, D, dtype=torch.float32, device=DEV), torch.empty(T, D, dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sr.sr_embed_tokens_backward(d, tokens, d_table=table, workspace=ws)
        sr.sr_embed_tokens(table, tokens, out=y)
    side = torch.cuda.Stream()
    for bt, bd in batches[1:] + batches[:1]:
        tokens.copy_(bt)
        d.copy_(bd)
        torch.cuda.synchronize()
        graph.replay()
        e, ey = torch.empty_like(table), torch.empty_like(y)
        with torch.cuda.stream(side):
            sr.sr_embed_tokens_backward(bd, bt, d_table=e, workspace=ws2)
        sr.sr_embed_tokens(e, bt, out=ey, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(table, e) and torch.equal(y, ey)


def test_gradient_against_differences():
    """The gradient of <embed(table), d> by the table, from differences of the call itself: it is linear, so one of any size will do."""
    V, D, T = 7, 8, 30
    tokens = draw_tokens(T, V, 2)
    w, d = rows(V, D, "f32", 1), rows(T, D, "f32", 2)
    got, _ = gradient(d, tokens, 0.5, V, "f32")
    y, moved = torch.empty(T, D, device=DEV), torch.empty(T, D, device=DEV)
    sr.sr_embed_tokens(w, tokens, 0.5, out=y)
    for v, c in ((0, 0), (3, 5), (6, 7)):
        m = w.clone()
        m[v, c] += 1.0
        sr.sr_embed_tokens(m, tokens, 0.5, out=moved)
        by = float(((moved.double() - y.double()) * d.double()).sum())
        assert abs(by - float(got[v, c])) <= 2.0 ** -20 * float((d[:, c].abs().sum() + 1) * (w[v, c].abs() + 1))

"""sr_token_logprob and its backward pass against 64 bits: types, sizes, pitches, masks, rows without a distribution."""
import pytest
import torch

import paper_2605_05802_b200 as sr
from helpers import Guarded
from train_ref import DTYPES, assert_near, logits_gradient, logprob

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def make(T, V, dtype, seed, pad=0, offset=0, spread=2.0):
    """Logits [T, V] as a view of rows V + pad apart that begin `offset` elements into their buffer; targets with some masked."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.randn(offset + T * (V + pad), generator=g).mul_(spread)
    x = buf.to(DEV, DTYPES[dtype])[offset:].view(T, V + pad)[:, :V]
    for t in range(min(T, 4)):                                  # a likely token or two
        x[t, torch.randint(0, V, (2,), generator=g).to(DEV)] = 9.0 + t
    y = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    y[torch.rand(T, generator=g) < 0.2] = -1
    y[0] = min(V - 1, 3)
    return x, y.to(DEV)


def forward(x, y, tau, entropy=True):
    T, guard = x.shape[0], Guarded(DEV)
    lp, st = guard.alloc((T,), torch.float32, 7.0), guard.alloc((T, 2), torch.float32, 7.0)
    H, status = guard.alloc((T,), torch.float32, 7.0) if entropy else None, guard.alloc((1,), torch.int32, 0)
    sr.sr_token_logprob(x, y, tau, logp=lp, row_stats=st, entropy=H, status=status)
    guard.check("sr_token_logprob")
    return lp, st, H, int(status.item())


def check_forward(x, y, tau, what, entropy=True):
    lp, st, H, status = forward(x, y, tau, entropy)
    (want, want_H, M, S), bound = logprob(x, y, tau)
    assert_near(lp, want, bound["lp"], what + " logp")
    assert bool((st[:, 0].double() == M).all()), what
    assert_near(st[:, 1], S, bound["S"], what + " S")
    if entropy:
        assert_near(H, want_H, bound["H"], what + " entropy")
    return lp, st, H, status


def check_backward(x, y, tau, st, H, entropy, what, pad=0, offset=0):
    T, V = x.shape
    g = torch.Generator().manual_seed(T + V)
    d_lp = torch.randn(T, generator=g).to(DEV)
    d_H = (0.3 * torch.randn(T, generator=g)).to(DEV) if entropy else None
    guard = Guarded(DEV)
    buf = guard.alloc((offset + T * (V + pad),), x.dtype, 5.0)
    dx = buf[offset:].view(T, V + pad)
    sr.sr_token_logprob_backward(x, y, st, H if entropy else None, d_lp, d_H, tau, d_logits=dx[:, :V])
    guard.check("sr_token_logprob_backward")
    want, bound = logits_gradient(x, y, tau, d_lp, d_H, x.dtype)
    assert_near(dx[:, :V], want, bound, what + " d_logits")
    assert bool((dx[:, V:] == 5.0).all()) and bool((buf[:offset] == 5.0).all()), what + ": wrote between the rows"
    return dx[:, :V], d_lp, d_H


SIZES = [(1, 1), (3, 1), (2, 2), (5, 7), (4, 8), (3, 9), (2, 63), (7, 257), (1, 4096), (300, 4096), (2, 8191), (400, 1000), (3, 50021), (1, 151936), (9, 151936)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T,V", SIZES)
def test_sizes(T, V, dtype):
    x, y = make(T, V, dtype, seed=T * 7 + V)
    _, st, H, _ = check_forward(x, y, 1.0, f"{T}x{V} {dtype}")
    check_backward(x, y, 1.0, st, H, False, f"{T}x{V} {dtype}")
    check_backward(x, y, 1.0, st, H, True, f"{T}x{V} {dtype} entropy")
    plain = forward(x, y, 1.0, entropy=False)
    lp, _, _, _ = forward(x, y, 1.0)
    assert torch.equal(plain[0], lp) and torch.equal(plain[1], st)      # the entropy changes nothing else


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (5, 7), (8, 4), (0, 3)])
@pytest.mark.parametrize("T,V", [(11, 500), (5, 12345), (330, 77)])
def test_pitches_and_alignment(T, V, pad, offset, dtype):
    x, y = make(T, V, dtype, seed=V + pad, pad=pad, offset=offset)
    _, st, H, _ = check_forward(x, y, 0.7, "pitch")
    check_backward(x, y, 0.7, st, H, True, "same pitch", pad, offset)
    check_backward(x, y, 0.7, st, H, False, "other pitch", pad + 2, offset + 1)


@pytest.mark.parametrize("tau", [0.01, 0.7, 1.5, 40.0])
def test_temperatures(tau):
    x, y = make(6, 3001, "f32", seed=3, spread=4.0)
    _, st, H, _ = check_forward(x, y, tau, f"tau {tau}")
    check_backward(x, y, tau, st, H, True, f"tau {tau}")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [9, 640, 40000])
def test_banned_tokens_and_rows_without_a_distribution(V, dtype):
    x, y = make(12, V, dtype, seed=V)
    low = torch.finfo(DTYPES[dtype]).min
    y[:] = torch.arange(12, device=DEV, dtype=torch.int32) % V
    x[1, V // 2:] = -float("inf")                     # banned tail
    x[2, :] = -float("inf")
    x[2, 2] = 0.5                                     # one token left
    x[3, :] = -float("inf")                           # nothing left
    x[4, V // 3] = float("nan")
    x[5, 5 % V] = float("inf")
    x[6, :] = low                                     # masked with the lowest value throughout: uniform
    x[7, 1:] = low
    x[8, 8 % V] = -float("inf")                       # the taken token cannot occur
    x[9, :] = 60000.0
    x[10, :] = float("nan")
    y[11] = V + 5
    lp, st, H, status = forward(x, y, 1.0)
    assert status == sr.SR_STATUS_BAD_TARGET
    (want, want_H, M, S), bound = logprob(x, y, 1.0)
    fine = [0, 1, 2, 6, 7, 8, 9, 11]
    assert_near(lp[fine], want[fine], bound["lp"][fine], "logp")
    assert_near(H[fine], want_H[fine], bound["H"][fine], "entropy")
    none = [3, 4, 5, 10]
    assert bool(torch.isnan(lp[none]).all()) and bool(torch.isnan(H[none]).all()) and bool(torch.isnan(st[none, 1]).all())
    for entropy in (False, True):
        d_lp, d_H = torch.full((12,), 0.5, device=DEV), torch.full((12,), 0.25, device=DEV) if entropy else None
        dx = torch.empty_like(x)
        sr.sr_token_logprob_backward(x, y, st, H, d_lp, d_H, d_logits=dx)
        g, b = logits_gradient(x, y, 1.0, d_lp, d_H, x.dtype)
        assert_near(dx[fine], g[fine], b[fine], "d_logits")
        assert bool(torch.isnan(dx[none]).all())


def test_masked_rows_are_not_read():
    x, y = make(40, 2048, "bf16", seed=1)
    y[::2] = -1
    y[1] = -(2 ** 31)
    want = forward(x, y, 1.0)
    x[::2] = float("nan")
    x[1] = float("nan")
    got = forward(x, y, 1.0)
    for a, b in zip(got[:3], want[:3]):
        assert torch.equal(a, b)
    assert bool((got[0][::2] == 0).all()) and bool((got[1][::2] == 0).all()) and bool((got[2][::2] == 0).all()) and got[3] == 0
    dx = torch.full_like(x, 3.0)
    sr.sr_token_logprob_backward(x, y, got[1], None, torch.ones(40, device=DEV), None, d_logits=dx)
    assert bool((dx[::2] == 0).all()) and bool((dx[1] == 0).all()) and bool(torch.isfinite(dx).all())


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T,V,pad", [(3, 5001, 3), (500, 999, 0), (2, 100000, 0)])
def test_gradient_over_the_logits(T, V, pad, dtype):
    x, y = make(T, V, dtype, seed=V, pad=pad)
    _, st, H, _ = forward(x, y, 1.0)
    d = torch.linspace(-1, 1, T, device=DEV)
    dx = torch.empty_like(x)
    sr.sr_token_logprob_backward(x, y, st, H, d, d, d_logits=dx)
    sr.sr_token_logprob_backward(x, y, st, H, d, d, d_logits=x)
    assert torch.equal(x, dx)


def test_against_differences_and_autograd():
    """The gradient of sum a logp + b entropy, from differences of the forward pass and from torch's differentiation."""
    T, V, tau = 5, 37, 0.8
    x, y = make(T, V, "f32", seed=9)
    y[:] = torch.tensor([0, 5, 36, 7, 7])
    a, b = torch.tensor([1.0, -2.0, 0.5, 3.0, 1.0], device=DEV), torch.tensor([0.3, 0.1, -0.4, 0.0, 1.0], device=DEV)
    _, st, H, _ = forward(x, y, tau)
    dx = torch.empty_like(x)
    sr.sr_token_logprob_backward(x, y, st, H, a, b, tau, d_logits=dx)
    xd = x.double().requires_grad_(True)
    log_p = torch.log_softmax(xd / tau, 1)
    value = (a * log_p.gather(1, y[:, None].long())[:, 0]).sum() + (b * -(log_p.exp() * log_p).sum(1)).sum()
    auto, = torch.autograd.grad(value, xd)
    want, bound = logits_gradient(x, y, tau, a, b, torch.float32)
    assert float((want - auto).abs().max()) < 1e-12
    assert_near(dx, auto, bound, "against autograd")
    h = 2.0 ** -6                                     # third-order error h^2 |f'''| and 2^-22 |f| / h: well below 2e-3 for terms of order 1
    for j in (0, 5, 36):
        up, down = x.clone(), x.clone()
        up[:, j] += h
        down[:, j] -= h
        f = [a * r[0] + b * r[2] for r in (forward(up, y, tau), forward(down, y, tau))]
        assert float((((f[0] - f[1]) / (2 * h)) - dx[:, j]).abs().max()) < 2e-3


def test_far_rows_of_a_large_buffer():
    """Rows whose offsets pass 2^32 elements."""
    T, V, pitch = 300, 1000, 1 << 24
    buf = torch.empty((T - 1) * pitch + V, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((T, V), (pitch, 1))
    small, y = make(T, V, "bf16", seed=4)
    x.copy_(small)
    a, b = forward(x, y, 1.0), forward(small, y, 1.0)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
    d = torch.ones(T, device=DEV)
    dx = torch.empty_like(small)
    sr.sr_token_logprob_backward(small, y, b[1], None, d, None, d_logits=dx)
    sr.sr_token_logprob_backward(x, y, a[1], None, d, None, d_logits=x)
    assert torch.equal(x, dx)


def test_no_tokens():
    x, y = torch.empty((0, 100), device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    e = torch.empty(0, device=DEV)
    sr.sr_token_logprob(x, y, logp=e)
    sr.sr_token_logprob_backward(x, y, e, None, e, None, d_logits=x)
    torch.cuda.synchronize()


def test_same_bits_every_time_and_on_another_stream():
    for T, V in ((3, 151936), (500, 4096)):
        x, y = make(T, V, "bf16", seed=T)
        first = forward(x, y, 1.0)
        s = torch.cuda.Stream()
        lp, st = torch.empty(T, device=DEV), torch.empty(T, 2, device=DEV)
        s.wait_stream(torch.cuda.current_stream())
        sr.sr_token_logprob(x, y, logp=lp, row_stats=st, stream=s)
        s.synchronize()
        assert torch.equal(lp, first[0]) and torch.equal(st, first[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            sr.sr_token_logprob(x, y, logp=lp, row_stats=st)
        x.mul_(0.5)
        want = forward(x, y, 1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(lp, want[0]) and torch.equal(st, want[1])

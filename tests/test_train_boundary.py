"""Refusals of the trainer's operators, on the host: no call here gets as far as a launch."""
import ctypes

import pytest
import torch

import paper_2605_05802_b200 as sr
from paper_2605_05802_b200 import binding, build

FAKE = 1 << 20           # never dereferenced


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_logprob_refusals(lib):
    def call(x=FAKE, dtype=0, T=4, V=100, pitch=100, y=FAKE, tau=1.0, lp=FAKE):
        return lib.sr_token_logprob(x, dtype, T, V, pitch, y, tau, lp, None, None, None, None)

    assert call(T=-1) == sr.SR_ERR_BAD_SIZE and call(V=0) == sr.SR_ERR_BAD_SIZE and call(pitch=99) == sr.SR_ERR_BAD_SIZE
    assert call(pitch=1 << 40) == sr.SR_ERR_BAD_SIZE
    assert call(dtype=3) == sr.SR_ERR_BAD_DTYPE and call(dtype=-1) == sr.SR_ERR_BAD_DTYPE
    for tau in (0.0, -1.0, float("nan"), float("inf"), 1e-40, 1e40):
        assert call(tau=tau) == sr.SR_ERR_BAD_VALUE
    assert call(x=None) == sr.SR_ERR_NULL and call(y=None) == sr.SR_ERR_NULL and call(lp=None) == sr.SR_ERR_NULL
    assert call(x=FAKE + 2) == sr.SR_ERR_ALIGN and call(x=FAKE + 1, dtype=1) == sr.SR_ERR_ALIGN and call(y=FAKE + 2) == sr.SR_ERR_ALIGN
    assert call(T=0, x=None, y=None, lp=None) == sr.SR_OK


def test_backward_refusals(lib):
    def call(x=FAKE, T=4, V=100, pitch=100, stats=FAKE, H=FAKE, d=FAKE, dH=None, dx=2 * FAKE, d_pitch=100, dtype=0):
        return lib.sr_token_logprob_backward(x, dtype, T, V, pitch, FAKE, stats, H, d, dH, 1.0, dx, d_pitch, None)

    assert call(stats=None) == sr.SR_ERR_NULL and call(d=None) == sr.SR_ERR_NULL and call(dx=None) == sr.SR_ERR_NULL
    assert call(H=None, dH=FAKE) == sr.SR_ERR_NULL
    assert call(d_pitch=99) == sr.SR_ERR_BAD_SIZE and call(dx=2 * FAKE + 1) == sr.SR_ERR_ALIGN
    # neither the logits themselves nor apart from them
    assert call(dx=FAKE + 4) == sr.SR_ERR_OVERLAP and call(dx=FAKE + 1596) == sr.SR_ERR_OVERLAP and call(dx=FAKE - 4) == sr.SR_ERR_OVERLAP
    assert call(dx=FAKE, d_pitch=101) == sr.SR_ERR_OVERLAP
    assert call(pitch=250, d_pitch=250, dx=FAKE + 4 * 99) == sr.SR_ERR_OVERLAP
    assert call(pitch=250, d_pitch=250, dx=FAKE + 4 * 151) == sr.SR_ERR_OVERLAP
    assert call(T=0, x=None, stats=None, d=None, dx=None) == sr.SR_OK


def test_weights_refusals(lib):
    def call(rs=FAKE, T=10, G=2, N=3, mode=1, scale=1.0, w=FAKE, counts=None, ws=FAKE, wsb=256):
        return lib.sr_loss_weights(rs, None, T, None, G, N, mode, scale, w, counts, ws, wsb, None)

    assert call(G=-1) == sr.SR_ERR_BAD_N and call(N=0) == sr.SR_ERR_BAD_N and call(G=1 << 20, N=1 << 11) == sr.SR_ERR_BAD_N
    assert call(T=-1) == sr.SR_ERR_BAD_SIZE and call(mode=3) == sr.SR_ERR_BAD_MODE and call(mode=-1) == sr.SR_ERR_BAD_MODE
    assert call(scale=float("nan")) == sr.SR_ERR_BAD_VALUE and call(scale=float("inf")) == sr.SR_ERR_BAD_VALUE
    assert call(rs=None) == sr.SR_ERR_NULL and call(w=None) == sr.SR_ERR_NULL
    assert call(rs=FAKE + 4) == sr.SR_ERR_ALIGN and call(counts=FAKE + 4) == sr.SR_ERR_ALIGN
    assert call(ws=None) == sr.SR_ERR_WORKSPACE and call(wsb=8) == sr.SR_ERR_WORKSPACE and call(ws=FAKE + 8) == sr.SR_ERR_WORKSPACE
    assert lib.sr_loss_weights_workspace_bytes(-1) == 0 and lib.sr_loss_weights_workspace_bytes(1000) >= 4000


def test_policy_refusals(lib):
    big = 1 << 20

    def call(lp=FAKE, adv=FAKE, w=FAKE, rs=FAKE, R=3, T=10, lo=0.2, hi=0.2, beta=0.0, loss=FAKE, ws=FAKE, wsb=big):
        return lib.sr_policy_loss(lp, None, None, adv, w, rs, R, None, T, lo, hi, beta, loss, None, None, ws, wsb, None)

    def logits(x=FAKE, T=4, lp=FAKE, dx=2 * FAKE, loss=FAKE, ws=FAKE, wsb=big, tau=1.0, hi=0.2, R=3):
        return lib.sr_policy_loss_logits(x, 0, T, 100, 100, FAKE, None, None, FAKE, FAKE, FAKE, R, None, 0.2, hi, 0.0, tau, loss, lp, dx, 100, None, None, ws, wsb, None)

    assert call(T=-1) == sr.SR_ERR_BAD_SIZE and call(R=-1) == sr.SR_ERR_BAD_N and logits(R=-1) == sr.SR_ERR_BAD_N
    for bad in (-0.1, float("nan"), float("inf")):
        assert call(lo=bad) == sr.SR_ERR_BAD_VALUE and call(hi=bad) == sr.SR_ERR_BAD_VALUE and call(beta=bad) == sr.SR_ERR_BAD_VALUE and logits(hi=bad) == sr.SR_ERR_BAD_VALUE
    for name in ("lp", "adv", "w", "rs", "loss"):
        assert call(**{name: None}) == sr.SR_ERR_NULL, name
    assert call(rs=FAKE + 4) == sr.SR_ERR_ALIGN
    assert call(ws=None) == sr.SR_ERR_WORKSPACE and call(wsb=100) == sr.SR_ERR_WORKSPACE and call(ws=FAKE + 8) == sr.SR_ERR_WORKSPACE
    for name in ("x", "lp", "dx", "loss"):
        assert logits(**{name: None}) == sr.SR_ERR_NULL, name
    assert logits(tau=0.0) == sr.SR_ERR_BAD_VALUE and logits(dx=FAKE + 4) == sr.SR_ERR_OVERLAP
    need = lib.sr_policy_loss_logits_workspace_bytes(100000)
    assert logits(T=100000, dx=FAKE, wsb=need - 1) == sr.SR_ERR_WORKSPACE and need >= 100000 * 20
    assert lib.sr_policy_loss_workspace_bytes(-1) == 0 and lib.sr_policy_loss_logits_workspace_bytes(-1) == 0


def test_gradient_list_refusals(lib):
    def arrays(ptrs, counts, dtypes):
        n = len(ptrs)
        return (ctypes.c_void_p * n)(*ptrs), (ctypes.c_int64 * n)(*counts), (ctypes.c_int32 * n)(*dtypes), n

    def norm(ptrs=(FAKE, 2 * FAKE), counts=(10, 20), dtypes=(0, 1), out=FAKE, ws=FAKE, wsb=1 << 20, n=None):
        p, c, d, k = arrays(ptrs, counts, dtypes)
        return lib.sr_grad_norm(p, c, d, k if n is None else n, out, ws, wsb, None)

    def clip(ptrs=(FAKE, 2 * FAKE), counts=(10, 20), dtypes=(0, 1), out=None, at=FAKE * 3, most=1.0):
        p, c, d, k = arrays(ptrs, counts, dtypes)
        return lib.sr_clip_grads(p, c, d, k, at, most, None if out is None else (ctypes.c_void_p * k)(*out), None, None)

    assert norm(n=-1) == sr.SR_ERR_BAD_N and norm(counts=(10, -1)) == sr.SR_ERR_BAD_SIZE and norm(counts=(1 << 50, 1)) == sr.SR_ERR_BAD_SIZE
    assert norm(dtypes=(0, 3)) == sr.SR_ERR_BAD_DTYPE and norm(ptrs=(FAKE, None)) == sr.SR_ERR_NULL and norm(out=None) == sr.SR_ERR_NULL
    assert norm(ptrs=(FAKE + 2, 2 * FAKE)) == sr.SR_ERR_ALIGN and norm(ptrs=(FAKE, 2 * FAKE + 1)) == sr.SR_ERR_ALIGN
    assert norm(ws=None) == sr.SR_ERR_WORKSPACE and norm(wsb=8) == sr.SR_ERR_WORKSPACE
    assert lib.sr_grad_norm(None, None, None, 2, FAKE, FAKE, 1 << 20, None) == sr.SR_ERR_NULL
    for most in (-1.0, float("nan"), float("inf"), 1e39):
        assert clip(most=most) == sr.SR_ERR_BAD_VALUE
    assert clip(at=None) == sr.SR_ERR_NULL and clip(out=(FAKE, None)) == sr.SR_ERR_NULL and clip(out=(FAKE + 2, 2 * FAKE)) == sr.SR_ERR_ALIGN
    assert clip(ptrs=(FAKE, FAKE)) == sr.SR_ERR_OVERLAP and clip(ptrs=(FAKE, FAKE + 36)) == sr.SR_ERR_OVERLAP
    assert clip(out=(FAKE + 4, 2 * FAKE)) == sr.SR_ERR_OVERLAP and clip(out=(4 * FAKE, 4 * FAKE)) == sr.SR_ERR_OVERLAP and clip(out=(2 * FAKE, FAKE)) == sr.SR_ERR_OVERLAP
    assert clip(at=FAKE + 8) == sr.SR_ERR_OVERLAP
    assert clip(ptrs=(), counts=(), dtypes=()) == sr.SR_OK


def test_binding_refuses_what_the_library_cannot_see(lib):
    x, y, f = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    with pytest.raises(ValueError, match="CUDA tensor"):
        sr.sr_token_logprob(x, y, logp=f)
    with pytest.raises(ValueError, match="vocabulary"):
        sr.sr_token_logprob(f, y, logp=f)
    with pytest.raises(TypeError):
        sr.sr_token_logprob([1.0], y, logp=f)
    with pytest.raises(ValueError, match="CUDA tensor"):
        sr.sr_policy_loss(f, None, None, f, f, torch.zeros(2, dtype=torch.int64), None, 0.2, 0.2, 0.0, loss=f, workspace=f)
    with pytest.raises(ValueError, match="n_groups"):
        sr.sr_loss_weights(torch.zeros(10, dtype=torch.int64), None, None, 4, weight=f, workspace=f)
    with pytest.raises(ValueError, match="row_start"):
        sr.sr_loss_weights(None, None, None, 4, weight=f, workspace=f)
    with pytest.raises(ValueError, match="CUDA tensor"):
        sr.sr_grad_norm([f], norm=f, workspace=f)
    for bad in (f, None, "ab", [None], [1.0]):
        with pytest.raises(TypeError):
            sr.sr_grad_norm(bad, norm=f, workspace=f)


def test_numbers_that_fp32_does_not_hold_and_addresses_off_their_type(lib):
    """Weights, beta and factors are fp32 in the kernels; an address off a boundary of its type would fault there."""
    def weights(scale=1.0, w=FAKE):
        return lib.sr_loss_weights(FAKE, None, 10, None, 2, 3, 1, scale, w, None, FAKE, 1 << 20, None)

    def policy(lp=FAKE, old=None, ref=None, adv=FAKE, w=FAKE, beta=0.0, loss=FAKE, d=None, stats=None):
        return lib.sr_policy_loss(lp, old, ref, adv, w, FAKE, 3, None, 10, 0.2, 0.2, beta, loss, d, stats, FAKE, 1 << 20, None)

    def step(lp=FAKE, old=None, ref=None, beta=0.0, stats=None, status=None):
        return lib.sr_policy_loss_logits(FAKE, 0, 4, 100, 100, FAKE, old, ref, FAKE, FAKE, FAKE, 3, None, 0.2, 0.2, beta, 1.0, FAKE, lp, 2 * FAKE, 100, stats, status, FAKE, 1 << 20, None)

    def logprob(lp=FAKE, st=None, H=None, status=None):
        return lib.sr_token_logprob(FAKE, 0, 4, 100, 100, FAKE, 1.0, lp, st, H, status, None)

    def backward(st=FAKE, H=FAKE, d=FAKE, dH=None):
        return lib.sr_token_logprob_backward(FAKE, 0, 4, 100, 100, FAKE, st, H, d, dH, 1.0, 2 * FAKE, 100, None)

    for bad in (1e39, -1e39):
        assert weights(scale=bad) == sr.SR_ERR_BAD_VALUE
    assert policy(beta=1e39) == sr.SR_ERR_BAD_VALUE and step(beta=1e39) == sr.SR_ERR_BAD_VALUE
    odd = FAKE + 2
    assert weights(w=odd) == sr.SR_ERR_ALIGN
    for name in ("lp", "old", "ref", "adv", "w", "loss", "d", "stats"):
        assert policy(**{name: odd}) == sr.SR_ERR_ALIGN, name
    for name in ("lp", "old", "ref", "stats", "status"):
        assert step(**{name: odd}) == sr.SR_ERR_ALIGN, name
    for name in ("lp", "st", "H", "status"):
        assert logprob(**{name: odd}) == sr.SR_ERR_ALIGN, name
    for name in ("st", "H", "d", "dH"):
        assert backward(**{name: odd}) == sr.SR_ERR_ALIGN, name
    one = (ctypes.c_void_p * 1)(FAKE), (ctypes.c_int64 * 1)(10), (ctypes.c_int32 * 1)(0)
    assert lib.sr_grad_norm(*one, 1, odd, FAKE, 1 << 20, None) == sr.SR_ERR_ALIGN
    assert lib.sr_clip_grads(*one, 1, odd, 1.0, None, None, None) == sr.SR_ERR_ALIGN
    assert lib.sr_clip_grads(*one, 1, 3 * FAKE, 1.0, None, odd, None) == sr.SR_ERR_ALIGN


@pytest.mark.gpu
def test_binding_refuses_tensors_of_another_type_or_size():
    d = torch.device("cuda:0")
    x, y, f = torch.zeros(4, 10, device=d), torch.zeros(4, dtype=torch.int32, device=d), torch.zeros(4, device=d)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device=d)
    for args, kind in (((x.double(), y), TypeError), ((x, y.long()), TypeError), ((x, y[:3]), ValueError), ((x.t(), torch.zeros(10, dtype=torch.int32, device=d)), ValueError),
                       ((x[:, ::2], y), ValueError)):
        with pytest.raises(kind):
            sr.sr_token_logprob(*args, logp=torch.zeros(10, device=d))
    with pytest.raises(ValueError):
        sr.sr_token_logprob(x, y, logp=f[:3])
    with pytest.raises(ValueError):
        sr.sr_token_logprob(x, y, logp=f, row_stats=f)
    with pytest.raises(sr.SrError) as e:
        sr.sr_token_logprob(x[:1].expand(4, 10), y, logp=f)
    assert e.value.code == sr.SR_ERR_BAD_SIZE
    stats = torch.ones(4, 2, device=d)
    with pytest.raises(TypeError):
        sr.sr_token_logprob_backward(x, y, stats, None, f, None, d_logits=x.half())
    with pytest.raises(ValueError):
        sr.sr_token_logprob_backward(x, y, stats, None, f, None, d_logits=torch.zeros(4, 11, device=d))
    rs = torch.tensor([0, 4], device=d)
    for bad in (dict(loss=f.cpu()), dict(loss=f[:0]), dict(loss=f, d_logp=f[:2]), dict(loss=f, stats=f[:3]), dict(loss=f, workspace=ws[1:]), dict(loss=f, workspace=ws[:8])):
        with pytest.raises((ValueError, sr.SrError)):
            sr.sr_policy_loss(f, None, None, f, f, rs, None, 0.2, 0.2, 0.0, **{"workspace": ws, **bad})
    with pytest.raises(TypeError):
        sr.sr_policy_loss(f, None, None, f, f, rs.int(), None, 0.2, 0.2, 0.0, loss=f, workspace=ws)
    with pytest.raises(TypeError):
        sr.sr_policy_loss(f, None, None, f, f, rs, f, 0.2, 0.2, 0.0, loss=f, workspace=ws)
    with pytest.raises(TypeError):
        sr.sr_grad_norm([f.double()], norm=f, workspace=ws)
    with pytest.raises(ValueError):
        sr.sr_grad_norm([x[:, ::2]], norm=f, workspace=ws)
    with pytest.raises(ValueError):
        sr.sr_clip_grads([x], f, 1.0, out=[])
    with pytest.raises(TypeError):
        sr.sr_clip_grads([x], f, 1.0, out=[x.half()])
    with pytest.raises(ValueError):
        sr.sr_clip_grads([x], f, 1.0, out=[torch.zeros(10, 4, device=d)])

"""sr_grad_norm and sr_clip_grads against 64 bits."""
import math

import pytest
import torch

import paper_2605_05802_b200 as sr
from helpers import Guarded
from train_ref import DTYPES

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def norm_of(grads):
    guard = Guarded(DEV)
    out, ws = guard.alloc((1,), torch.float32, 7.0), guard.alloc((sr.sr_grad_norm_workspace_bytes(len(grads)),), torch.uint8)
    sr.sr_grad_norm(grads, norm=out, workspace=ws)
    guard.check("sr_grad_norm")
    return out


def exact_norm(grads):
    return math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


# a square and up to 32 additions in fp32 (half a step each), the square root halves their relative error, and the result is rounded
NORM = 2.0 ** -24 * (33 / 2 + 1)


def check(grads, max_norm, offsets=None):
    """Norm, clipping into other buffers and in place."""
    norm = norm_of(grads)
    want = exact_norm(grads)
    assert abs(float(norm) - want) <= NORM * want, (float(norm), want)
    factor = min(1.0, max_norm / (float(norm) + 1e-6))
    guard = Guarded(DEV)
    outs = [guard.alloc((g.numel() + (offsets[i] if offsets else 0),), g.dtype, 7.0)[offsets[i] if offsets else 0:].view(g.shape) for i, g in enumerate(grads)]
    status = guard.alloc((1,), torch.int32, 0)
    sr.sr_clip_grads(grads, norm, max_norm, out=outs, status=status)
    guard.check("sr_clip_grads")
    assert int(status) == 0
    for g, o in zip(grads, outs):
        w = g.double() * factor
        eps = torch.finfo(g.dtype).eps / 2
        # the factor: an addition and a division; the product: 2^-24; the rounding; below the type's normal range half its smallest step
        bound = w.abs() * (eps + 3 * 2.0 ** -24) + torch.finfo(g.dtype).smallest_normal * torch.finfo(g.dtype).eps
        assert bool(((o.double() - w).abs() <= bound).all())
        if factor == 1.0:
            assert torch.equal(o, g)
    copies = [g.clone() for g in grads]
    sr.sr_clip_grads(copies, norm, max_norm)
    for c, o in zip(copies, outs):
        assert torch.equal(c, o)
    return float(norm)


def tensors(sizes, dtype, seed, offset=0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(offset + n, generator=g) * 10.0 ** (k % 3 - 2)).to(DEV, DTYPES[dtype])[offset:] for k, n in enumerate(sizes)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("sizes", [[1], [0, 1, 0], [7, 8, 9], [3, 8191, 8192, 8193], [16384, 16385, 16383, 1], [1 << 20, 5, 0, 777777], [64] * 33, [1000 + k for k in range(900)]],
                         ids=["one", "none", "few", "piece", "pieces", "large", "33", "900"])
def test_sizes(sizes, dtype):
    grads = tensors(sizes, dtype, len(sizes))
    n = check(grads, 0.3)
    check(grads, 2 * n + 1)                        # not clipped
    check(grads, 0.0)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("offset,out_offset", [(1, 1), (3, 0), (0, 5), (7, 7)])
def test_off_their_alignment(offset, out_offset, dtype):
    grads = tensors([1, 6, 40001, 8200], dtype, 3, offset)
    check(grads, 0.5, [out_offset] * 4)


def test_types_together_and_any_dense_layout():
    grads = tensors([5000, 70], "f32", 1) + tensors([123457], "bf16", 2) + tensors([99, 0], "f16", 3)
    grads.append(torch.randn(8, 5, 7, device=DEV).permute(2, 0, 1))
    norm = norm_of(grads)
    want = exact_norm(grads)
    assert abs(float(norm) - want) <= NORM * want
    outs = [torch.empty_like(g) for g in grads]
    assert outs[-1].stride() == grads[-1].stride()
    sr.sr_clip_grads(tuple(grads), norm, 1.0, out=outs)
    for g, o in zip(grads, outs):
        assert float((o.double() - g.double() / float(norm)).abs().max() if g.numel() else 0.0) <= 2.0 ** -8 * (float(g.double().abs().max() if g.numel() else 0.0) / float(norm) + 1e-6)


@pytest.mark.parametrize("scale", [1e30, 1e19, 1e-19, 1e-30, 1e-38, 0.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_magnitudes_whose_squares_leave_fp32(scale, dtype):
    g = torch.Generator().manual_seed(5)
    big = (torch.randn(50000, generator=g).double() * scale).to(DEV, DTYPES[dtype])
    small = torch.full((33,), 1e-3, device=DEV) if scale > 1 else torch.zeros(33, device=DEV)
    want = exact_norm([big, small])
    assert abs(float(norm_of([big, small])) - want) <= NORM * want + 2.0 ** -150
    big[777] *= 100.0
    want = exact_norm([big])
    assert abs(float(norm_of([big])) - want) <= NORM * want + 2.0 ** -150


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_not_finite(bad, dtype):
    grads = tensors([1000, 20000], dtype, 7)
    grads[1][12345] = bad
    norm = norm_of(grads)
    assert not math.isfinite(float(norm)) and math.isnan(float(norm)) == math.isnan(bad)
    status, outs = torch.zeros(1, dtype=torch.int32, device=DEV), [torch.zeros_like(g) for g in grads]
    keep = [g.clone() for g in grads]
    sr.sr_clip_grads(grads, norm, 0.1, out=outs, status=status)
    assert int(status) == sr.SR_STATUS_NONFINITE
    sr.sr_clip_grads(grads, norm, 0.1)
    for g, o, k in zip(grads, outs, keep):
        assert torch.equal(torch.nan_to_num(o, nan=3.0), torch.nan_to_num(k, nan=3.0)) and torch.equal(torch.nan_to_num(g, nan=3.0), torch.nan_to_num(k, nan=3.0))


def test_no_tensors_and_the_same_tensor_twice():
    assert float(norm_of([])) == 0.0
    sr.sr_clip_grads([], torch.ones(1, device=DEV), 1.0)
    g = torch.randn(100, device=DEV)
    assert abs(float(norm_of([g, g])) - exact_norm([g, g])) < 1e-5
    norm = norm_of([g])
    for grads, out in (([g, g], None), ([g, g[50:]], None), ([g[:50]], [g[1:51]]), ([g[:10], g[10:20]], [g[20:30], g[29:39]]), ([g[:10]], [g[5:15]])):
        with pytest.raises(sr.SrError) as e:
            sr.sr_clip_grads(grads, norm, 1.0, out=out)
        assert e.value.code == sr.SR_ERR_OVERLAP
    with pytest.raises(sr.SrError):
        sr.sr_clip_grads([norm], norm, 1.0)
    sr.sr_clip_grads([g[:50], g[50:]], norm, 0.5)            # neighbours are fine


def test_far_elements_of_a_large_tensor():
    """Elements whose offsets pass 2^32."""
    n = (1 << 32) + 4099
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g[-1], g[1 << 31], g[0] = 3.0, 4.0, 12.0
    norm = norm_of([g])
    assert float(norm) == 13.0
    sr.sr_clip_grads([g], norm, 6.5)
    assert float(g[-1]) == 1.5 and float(g[1 << 31]) == 2.0 and float(g[0]) == 6.0 and int((g != 0).sum()) == 3


def test_same_bits_and_replayed_graphs():
    grads = tensors([100000, 3, 65536], "bf16", 1) + tensors([777], "f32", 2)
    a, norm = norm_of(grads), torch.empty(1, device=DEV)
    assert torch.equal(a, norm_of(grads))
    ws = torch.empty(sr.sr_grad_norm_workspace_bytes(4), dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(g) for g in grads]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sr.sr_grad_norm(grads, norm=norm, workspace=ws)
        sr.sr_clip_grads(grads, norm, 0.25, out=outs)
    for g in grads:
        g.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(norm, norm_of(grads)) and abs(exact_norm(outs) - 0.25) < 2.0 ** -9 * 0.25

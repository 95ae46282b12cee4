"""sr_token_logprob on many rows too long to be held: sizes, alignments, masks, rows without a
distribution, calls beside one another and replayed."""
import pytest
import torch

import paper_2605_05802_b200 as sr
from test_token_logprob_gpu import check_forward, forward, make
from train_ref import DTYPES, assert_near, logprob

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T,V,pad,offset", [(297, 20600, 0, 0), (300, 21001, 3, 1), (601, 50021, 0, 5), (400, 65536, 8, 4), (1000, 24577, 0, 0), (299, 151936, 0, 0)])
def test_sizes(T, V, pad, offset, dtype):
    x, y = make(T, V, dtype, T + V, pad, offset)
    for entropy in (True, False):
        check_forward(x, y, 0.9, f"{dtype} {T}x{V}", entropy)


@pytest.mark.parametrize("counting", [0, 1, 2, 600])
def test_masks(counting):
    """Rows that do not count are not read, however many of them there are."""
    T, V = 5000, 21000
    x, y = make(T, V, "bf16", counting)
    keep = torch.linspace(0, T - 1, max(counting, 1)).long()[:counting].to(DEV)
    mine = torch.full_like(y, -1)
    mine[keep] = y[keep].clamp(min=0)
    safe = x[keep].clone()
    out = torch.ones(T, dtype=torch.bool, device=DEV)
    out[keep] = False
    x[out] = float("nan")
    lp, st, H, status = forward(x, mine, 1.0)
    assert status == 0 and not bool(lp[out].any()) and not bool(st[out].any()) and not bool(H[out].any())
    if counting:
        (want, want_H, M, S), bound = logprob(safe, mine[keep], 1.0)
        assert_near(lp[keep], want, bound["lp"], "logp")
        assert_near(H[keep], want_H, bound["H"], "entropy")
        assert_near(st[keep, 1], S, bound["S"], "S")


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rows_without_a_distribution_among_others(dtype):
    T, V = 330, 30001
    x, y = make(T, V, dtype, 7)
    y[:12] = torch.arange(12, device=DEV, dtype=torch.int32)
    low = torch.finfo(DTYPES[dtype]).min
    x[1, V // 2:] = -float("inf")
    x[2, :] = -float("inf")
    x[2, 2] = 0.5
    x[3, :] = -float("inf")
    x[4, V // 3] = float("nan")
    x[5, 5] = float("inf")
    x[6, :] = low
    x[7, 1:] = low
    x[8, 8] = -float("inf")
    x[10, :] = float("nan")
    y[11] = V
    lp, st, H, status = forward(x, y, 1.0)
    assert status == sr.SR_STATUS_BAD_TARGET
    none = [3, 4, 5, 10]
    assert bool(torch.isnan(lp[none]).all()) and bool(torch.isnan(H[none]).all()) and bool(torch.isnan(st[none, 1]).all())
    fine = [t for t in range(T) if t not in none]
    (want, want_H, _, _), bound = logprob(x[fine], y[fine], 1.0)
    assert_near(lp[fine], want, bound["lp"], "logp")
    assert_near(H[fine], want_H, bound["H"], "entropy")


def test_calls_beside_one_another_and_replayed():
    """Each gives the bits that it gives alone."""
    args = []
    for seed, (T, V, dtype) in enumerate([(700, 60000, "bf16"), (500, 30001, "f32"), (900, 21500, "f16")]):
        x, y = make(T, V, dtype, seed)
        args.append((x, y, forward(x, y, 1.0)))
    streams = [torch.cuda.Stream() for _ in args]
    outs = [dict(logp=torch.empty(len(y), device=DEV), row_stats=torch.empty(len(y), 2, device=DEV), entropy=torch.empty(len(y), device=DEV)) for _, y, _ in args]
    graphs = []
    for (x, y, _), o in zip(args, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(2):
                sr.sr_token_logprob(x, y, **o)
        graphs.append(g)
    torch.cuda.synchronize()
    for turn in range(6):
        for o in outs:
            for v in o.values():
                v.fill_(7.0)
        torch.cuda.synchronize()
        for (x, y, _), o, s, g in zip(args, outs, streams, graphs):
            with torch.cuda.stream(s):
                if turn % 2:
                    g.replay()
                else:
                    for _ in range(3):
                        sr.sr_token_logprob(x, y, **o)
        torch.cuda.synchronize()
        for (_, _, want), o in zip(args, outs):
            for a, b in zip(o.values(), want[:3]):
                assert torch.equal(a, b)


def test_rows_behind_2_to_the_31_elements():
    T, V = 14400, 151936
    x = torch.empty(T, V, dtype=torch.bfloat16, device=DEV)
    for a in range(0, T, 900):
        x[a:a + 900] = 2 * torch.randn(900, V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(a))
    y = torch.randint(0, V, (T,), dtype=torch.int32, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    rows = [0, 1, 14130, 14135, 14136, 14137, 14398, T - 1]
    lp, st, H, status = forward(x, y, 1.0)
    (want, want_H, _, S), bound = logprob(x[rows], y[rows], 1.0)
    assert_near(lp[rows], want, bound["lp"], "logp")
    assert_near(H[rows], want_H, bound["H"], "entropy")
    assert_near(st[rows, 1], S, bound["S"], "S")
    assert status == 0 and bool((lp < 0).all())

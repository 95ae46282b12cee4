"""Tokens that are seen thousands of times, at the border where their counts leave 14 bits (8192 occurrences)."""
import pytest
import torch

import paper_2605_05802_b200 as sr

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def milliseconds(call):
    times = []
    for _ in range(4):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return min(times[1:])


@pytest.mark.parametrize("pad", [0, 1])
def test_a_count_that_is_whole_is_not_counted_again(pad):
    """8192 occurrences in the first part of a history of two million positions: the count has them all, so that the row takes what it takes with one less.
    (Counted again by the one thread that has the token, it took 40 to 55 times as long.)"""
    V, n = 500, 2_000_000
    x = torch.full((1, V + pad), 3.0, device=DEV)[:, pad:]
    out = torch.empty(1, V + pad, device=DEV)[:, pad:]
    rest = dict(history_start=torch.zeros(1, dtype=torch.int64, device=DEV), history_len=torch.full((1,), n, dtype=torch.int32, device=DEV), frequency=torch.full((1,), 2.0 ** -12, device=DEV))
    took = []
    for times in (8191, 8192):
        history = torch.full((n,), -1, dtype=torch.int32, device=DEV)
        history[:times] = 123
        took.append(milliseconds(lambda: sr.sr_adjust_logits(x, history=history, **rest, out=out)))
        want = x.clone()
        want[0, 123] -= times * 2.0 ** -12                # exact in fp32
        assert torch.equal(out, want)
    assert took[1] < 4 * took[0] + 1, took


@pytest.mark.parametrize("tokens", [63, 64, 65, 200])
@pytest.mark.parametrize("pad", [0, 1])
def test_a_table_that_is_nearly_full(tokens, pad):
    """Of one slice's tokens as many as the table holds, one less, one more and many more occur 8600 times, some others 8190 to 8194 times: all are counted."""
    V = 1000
    times = torch.zeros(V, dtype=torch.int64)
    chosen = torch.randperm(V, generator=torch.Generator().manual_seed(tokens))
    times[chosen[:tokens]] = 8600
    times[chosen[tokens:tokens + 5]] = torch.arange(8190, 8195)
    history = torch.repeat_interleave(torch.arange(V), times).to(torch.int32)
    history = history[torch.randperm(history.numel(), generator=torch.Generator().manual_seed(1))].to(DEV)
    x = torch.zeros(2, V + pad, device=DEV)[:, pad:]
    out = torch.empty(2, V + pad, device=DEV)[:, pad:]
    sr.sr_adjust_logits(x, history=history, history_start=torch.zeros(2, dtype=torch.int64, device=DEV), history_len=torch.full((2,), history.numel(), dtype=torch.int32, device=DEV),
                        frequency=torch.full((2,), 1.0, device=DEV), out=out)
    assert torch.equal(out, -times.to(DEV).float().expand(2, V))

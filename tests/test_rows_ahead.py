"""Rows of logits that are copied ahead, up to the last of 2^31 - 1: on the host by the function that decides, and on the GPU with as many rows as a
call may have."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2605_05802_b200 as sr

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_05802_b200", "csrc")
MOST = 2 ** 31 - 1


def test_rows_ahead_of_the_last_one(tmp_path):
    src, out = tmp_path / "rows.cpp", tmp_path / "rows.so"
    src.write_text('#include "rows_ahead.cuh"\nextern "C" int ahead(int row, int by, int end) { return sr::row_ahead(row, by, end); }\n')
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fsanitize=signed-integer-overflow", "-fno-sanitize-recover", "-I", CSRC, "-o", str(out), str(src)])
    lib = ctypes.CDLL(str(out))
    for end in (1, 2, 3, 64, 2 ** 30, MOST - 2, MOST - 1, MOST):
        for row in [-2, -1, 0, 1, 2] + [end - k for k in range(1, 6)]:
            for by in range(4):
                assert bool(lib.ahead(row, by, end)) == (row + by < end), (row, by, end)


def test_no_kernel_works_out_a_row_behind_the_next():
    """row < row_end holds in the loop, so that row + 1 is a number; row + 2 need not be."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "adjust.cu")).read())
    sums = re.findall(r"(?<!\(int64_t\))\brow \+ ([\w ]+?)(?: - \w+)?\s*<", text)
    assert sums and set(sums) == {"1"}, sums


@pytest.mark.gpu
@pytest.mark.parametrize("V", [1, 8])
def test_as_many_rows_as_a_call_may_have(V):
    """Rows of 2 bytes, most of them off 16 bytes, and of a vector each: every one keeps its bits, and what lies behind the last is left as it is.  Eight more
    lie in the buffers behind the rows of the call."""
    d = torch.device("cuda:0")
    x, y = (torch.empty(MOST + 8, V, dtype=torch.bfloat16, device=d) for _ in range(2))
    part = 1 << 26
    for a in range(0, MOST + 8, part):
        n = min(part, MOST + 8 - a)
        x[a:a + n] = ((torch.arange(a, a + n, device=d) % 251)[:, None] + torch.arange(V, device=d)).to(torch.bfloat16)
    y.fill_(-7.0)
    sr.sr_adjust_logits(x[:MOST], out=y[:MOST])
    torch.cuda.synchronize()
    assert bool((y[MOST:] == -7.0).all())
    for a in range(0, MOST, part):
        assert torch.equal(y[a:min(MOST, a + part)].view(torch.int16), x[a:min(MOST, a + part)].view(torch.int16)), a

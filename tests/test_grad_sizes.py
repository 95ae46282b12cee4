"""Lists of gradients that are too long for the kernels' numbers are refused, on the host: none is left out in silence."""
import ctypes

import pytest

import paper_2605_05802_b200 as sr
from paper_2605_05802_b200 import binding, build

FAKE = 1 << 20           # never dereferenced
MOST = (2 ** 31 - 1) * 16384     # bytes: pieces of 16 KB are numbered in 32 bits
SIZE = {sr.SR_DTYPE_F32: 4, sr.SR_DTYPE_BF16: 2, sr.SR_DTYPE_F16: 2}


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def lists(counts, dtypes):
    n = len(counts)
    at, ptrs = FAKE, []
    for c, d in zip(counts, dtypes):
        ptrs.append(at)
        at += (c * SIZE[d] + 15) // 16 * 16
    return (ctypes.c_void_p * n)(*ptrs), (ctypes.c_int64 * n)(*counts), (ctypes.c_int32 * n)(*dtypes), n


def norm(lib, counts, dtypes):
    return lib.sr_grad_norm(*lists(counts, dtypes), FAKE, None, 0, None)          # no workspace: refused before anything starts


def clip(lib, counts, dtypes):
    return lib.sr_clip_grads(*lists(counts, dtypes), FAKE - 64, -1.0, None, None, None)      # a max_norm that is refused behind the sizes


@pytest.mark.parametrize("dtype", list(SIZE))
def test_one_tensor(lib, dtype):
    most = MOST // SIZE[dtype]
    for call, after in ((norm, sr.SR_ERR_WORKSPACE), (clip, sr.SR_ERR_BAD_VALUE)):
        assert call(lib, [most + 1], [dtype]) == sr.SR_ERR_BAD_SIZE
        assert call(lib, [5, most + 1, 7], [dtype] * 3) == sr.SR_ERR_BAD_SIZE
        assert call(lib, [1 << 62], [dtype]) == sr.SR_ERR_BAD_SIZE
        assert call(lib, [most], [dtype]) == after


def test_all_of_them_together(lib):
    """Each would do; together they have more pieces than there are numbers, also where the last of a piece is not whole."""
    half = (2 ** 30) * 4096
    for call, after in ((norm, sr.SR_ERR_WORKSPACE), (clip, sr.SR_ERR_BAD_VALUE)):
        assert call(lib, [half, half], [0, 0]) == sr.SR_ERR_BAD_SIZE
        assert call(lib, [half, half - 4096], [0, 0]) == after
        assert call(lib, [half, half - 4096, 1], [0, 0, 1]) == sr.SR_ERR_BAD_SIZE
        assert call(lib, [half - 1, half - 4095], [0, 0]) == sr.SR_ERR_BAD_SIZE
        assert call(lib, [half, 0, half - 4096, 0], [0, 1, 0, 2]) == after
        assert call(lib, [half // 2] * 4, [1] * 4) == after                        # 16-bit: half the bytes


def test_a_list_that_was_left_out_in_silence(lib):
    """2^43 fp32 numbers are 2^31 pieces: clipping returned without a launch and without an error."""
    assert lib.sr_clip_grads(*lists([1 << 43], [0]), FAKE - 64, 1.0, None, None, None) == sr.SR_ERR_BAD_SIZE

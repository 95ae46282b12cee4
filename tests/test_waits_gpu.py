"""The waits of the kernel that holds long rows: they end, and what a wait that has ended makes of the loss.

Nothing makes a wait of that kernel last, so its parts are taken by themselves: a wait at a barrier where nobody arrives, with a limit
of its own, and the sum over the tokens after a CTA has said that it gave up."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_05802_b200", "csrc")
DEV = torch.device("cuda:0")

SOURCE = r"""
#include "policy.cu"
#include "ring.cuh"
namespace sr {
void note_cuda_error(cudaError_t, const char*) {}
__global__ void wait_kernel(unsigned long long limit, int arrives, int* out) {
    __shared__ uint64_t bar;
    __shared__ int gave_up;
    if (threadIdx.x == 0) {
        barrier_init(&bar, 1);
        gave_up = 0;
        barriers_ready();
    }
    __syncthreads();
    if (arrives && threadIdx.x == 0) barrier_arrive(&bar);
    const unsigned long long began = nanoseconds();
    barrier_wait(&bar, 0, &gave_up, limit);
    out[2 + threadIdx.x] = (int)((nanoseconds() - began) / 1000);
    __syncthreads();
    if (threadIdx.x == 0) out[0] = gave_up;
}
__global__ void ones_kernel(PolicyTerms* terms, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) terms[i] = PolicyTerms{1, 1, 1, 1};
}
}
extern "C" int terms_bytes(int n) { return n * (int)sizeof(sr::PolicyTerms); }
extern "C" int make_ones(void* terms, int n, void* s) {
    sr::ones_kernel<<<n / 256 + 1, 256, 0, (cudaStream_t)s>>>((sr::PolicyTerms*)terms, n);
    return (int)cudaGetLastError();
}
extern "C" int run_wait(long long limit, int arrives, int* out, void* s) {
    sr::wait_kernel<<<1, 64, 0, (cudaStream_t)s>>>((unsigned long long)limit, arrives, out);
    return (int)cudaGetLastError();
}
extern "C" int run_sum(const void* terms, int n, double beta, const int* gave_up, float* loss, float* stats, double* partial, void* s) {
    return sr::launch_sum_terms((const sr::PolicyTerms*)terms, n, beta, gave_up, loss, stats, partial, (cudaStream_t)s);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("waits")
    src, out = d / "waits.cu", d / "waits.so"
    src.write_text(SOURCE)
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17", "-Xcompiler", "-fPIC", "-shared",
                           "-cudart", "static", "-I", os.path.join(ROOT, "include"), "-I", CSRC, str(src), "-o", str(out)])
    return ctypes.CDLL(str(out))


def address(t):
    return ctypes.c_void_p(t.data_ptr())


def stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


@pytest.mark.gpu
def test_a_wait_ends_and_says_so(lib):
    out = torch.full((66,), -1, dtype=torch.int32, device=DEV)
    assert lib.run_wait(ctypes.c_longlong(10 ** 9), 1, address(out), stream()) == 0
    torch.cuda.synchronize()
    assert int(out[0]) == 0                                              # somebody arrived
    assert lib.run_wait(ctypes.c_longlong(200_000), 0, address(out), stream()) == 0
    torch.cuda.synchronize()
    assert int(out[0]) == 1
    assert int(out[2:].min()) >= 100 and int(out[2:].max()) < 200_000    # after the limit (us), long before a second


@pytest.mark.gpu
@pytest.mark.parametrize("n", [0, 1, 1000, 65536, 200_000])
def test_a_loss_with_rows_missing_is_nan(lib, n):
    terms = torch.empty(lib.terms_bytes(n + 1), dtype=torch.uint8, device=DEV)
    assert lib.make_ones(address(terms), n, stream()) == 0
    partial = torch.empty(1184 * 4, dtype=torch.float64, device=DEV)
    loss, stats = torch.full((1,), 7.0, device=DEV), torch.full((4,), 7.0, device=DEV)
    for flag, nan in ((None, False), (0, False), (1, True)):
        given = None if flag is None else torch.full((1,), flag, dtype=torch.int32, device=DEV)
        for beta in (0.0, 0.5):
            loss.fill_(7.0)
            stats.fill_(7.0)
            assert lib.run_sum(address(terms), n, ctypes.c_double(beta), None if given is None else address(given), address(loss), address(stats), address(partial), stream()) == 0
            torch.cuda.synchronize()
            if nan:
                assert bool(torch.isnan(loss).all()) and bool(torch.isnan(stats).all())
            else:
                assert float(loss) == (beta - 1) * n and stats.tolist() == [n] * 4


def test_it_compiles(lib):
    assert lib.run_wait and lib.run_sum

"""Workspaces of a token's step on the host: one that serves a number of rows serves any smaller one,
and the binding gives the same size whether or not the library was loaded before."""
import ctypes as C
import os
import subprocess
import sys

import pytest

import paper_2507_05228_amd as cas

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cas.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return cas.load_library()


@pytest.mark.parametrize("vocab", [1, 700, 8192, 8193, 32000, 50257, 128256, 1 << 20])
@pytest.mark.parametrize("dtype", [cas.BF16, cas.F32])
def test_a_workspace_of_tokens_serves_fewer_rows(lib, vocab, dtype):
    sizes = [lib.cascade_sample_workspace_bytes(C.byref(cas.SampleDesc(dtype, r, vocab, 0, 0))) for r in [*range(1, 1200), 4096, 65535, 65536]]
    assert sizes[0] > 0 and sizes == sorted(sizes)
    assert sizes[-1] <= 65536 * -(-vocab // 8192) * 9300   # (no more than the bins of every chunk)


@pytest.mark.parametrize("n,k,group", [(4096, 14336, 128), (14336, 4096, 64), (48, 1 << 17, 32), (17, 96, 32), (8192, 8192, 128), (100000, 512, 128)])
@pytest.mark.parametrize("dtype", [cas.BF16, cas.F32])
@pytest.mark.parametrize("x_format", [cas.Q8_NONE, cas.Q8_INT8, cas.Q8_E4M3])
@pytest.mark.parametrize("epilogue", [0, cas.EPI_SWIGLU])
def test_a_workspace_of_products_serves_fewer_rows(lib, n, k, group, dtype, x_format, epilogue):
    w = cas.W4Weights(dtype, n, k, group, 0, 0, None)
    sizes = [lib.cascade_w4_gemm_workspace_bytes(C.byref(w), C.byref(cas.W4GemmDesc(r, x_format, 0, epilogue, 0, 0, 0)))
             for r in [*range(1, 300), 1000, 5000, 40000, 1 << 20]]
    assert sizes == sorted(sizes)


def test_the_first_question_for_a_workspace_has_the_same_answer(lib):
    code = ("import torch, paper_2507_05228_amd as cas\n"
            "for dtype, n, k in ((cas.BF16, 4096, 14336), (cas.F32, 4096, 14336), (cas.F32, 8192, 8192)):\n"
            "    w = cas.W4Weights(dtype, n, k, 128, 0, 0, None)\n"
            "    for x in (torch.empty((rows, k), dtype=t) for rows in (32, 64) for t in (torch.int8, torch.float8_e4m3fn)):\n"
            "        cas._lib, cas._Q8 = None, {}\n"
            "        print(*(cas.cascade_w4_gemm_workspace_bytes(w, x) for _ in range(2)))\n")
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, check=True, capture_output=True, text=True, timeout=600).stdout
    pairs = [line.split() for line in out.splitlines() if line[:1].isdigit()]
    assert len(pairs) == 12 and all(a == b for a, b in pairs), out

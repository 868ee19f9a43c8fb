"""Products with 4-bit weights at the ends of what a call may bring: a workspace for more rows.  Bounds as in test_gpu_w4."""
import pytest

from test_gpu_w4 import make_weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cas():
    import torch
    assert torch.cuda.is_available()
    import paper_2507_05228_amd as cas
    cas.load_library()
    return cas


@pytest.mark.parametrize("dtype,swiglu,most,few", [("bfloat16", False, 65, 64), ("bfloat16", False, 200, 33), ("float32", True, 33, 32), ("float32", False, 100, 5)])
def test_a_workspace_for_many_rows_serves_fewer(cas, dtype, swiglu, most, few):
    import torch
    g = torch.Generator(device="cuda").manual_seed(most)
    dt, n, k = getattr(torch, dtype), 4096, 14336
    if swiglu:
        n, k = k, n
    w = cas.make_w4_weights(*make_weights(n, k, 128, dt, False, g))
    x = torch.randn((most, k), device="cuda", generator=g).to(dt)
    results = []
    for rows in (most, few):
        y = torch.empty((few, n), device="cuda", dtype=dt)
        ws = cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w, x[:rows], w if swiglu else None))
        cas.cascade_w4_gemm(w, x[:few], y, weights_up=w if swiglu else None, epilogue=cas.EPI_SWIGLU if swiglu else 0, workspace=ws)
        results.append(y)
    assert torch.equal(*results)

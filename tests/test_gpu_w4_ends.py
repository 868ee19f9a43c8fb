"""Products with 4-bit weights at the ends of what a call may bring: a workspace for more rows, infinities and NaN in any
place of X, sums beyond fp32.  Bounds as in test_gpu_w4; an output that is formed again term by term is a sum in 64 bits, rounded once."""
import pytest

from test_gpu_w4 import dense, make_weights, run

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


def same_as_formula(y, want, half):
    """NaN where the formula has it, infinities of its sign (and where a finite value is beyond the type), else half a step."""
    import torch
    nan, most = torch.isnan(want), torch.finfo(y.dtype).max
    assert torch.equal(torch.isnan(y), nan)
    inf = ~nan & (want.abs() > most * (1 + half))
    assert torch.equal(y[inf].double(), want[inf].sign() * float("inf"))
    fine = ~nan & (want.abs() <= most)
    assert ((y.double() - want).abs()[fine] <= 1.001 * half * want.abs()[fine] + 1e-38).all()


@pytest.mark.parametrize("dtype,x,rows,k,n,group,x_group", [
    ("bf16", "same", 1, 96, 17, 32, 0), ("bf16", "same", 16, 14336, 256, 128, 0), ("bf16", "same", 64, 2048, 4096, 64, 0), ("bf16", "same", 33, 1056, 200, 32, 0),
    ("f32", "same", 5, 160, 40, 32, 0), ("f32", "same", 40, 4096, 100, 128, 0), ("bf16", "e4m3", 20, 1152, 300, 128, 64), ("f32", "e4m3", 70, 512, 33, 64, 0)])
@pytest.mark.parametrize("act", ["none", "swiglu"])
@pytest.mark.parametrize("zeros", [False, True])
def test_infinities_and_nan_in_any_place(cas, dtype, x, rows, k, n, group, x_group, act, zeros):
    """A row each: an infinity in the first, a middle and the last place, two of either sign, NaN in the first and last, all of it NaN."""
    import torch
    inf, nan = float("inf"), float("nan")
    # (E4M3 knows no infinities)
    plants = [((0, nan),), ((k - 1, nan),), tuple((j, nan) for j in range(k))]
    if x == "same":
        plants += [((0, inf),), ((k // 2 + 5, -inf),), ((k - 1, inf),), ((3, inf), (k - 40, -inf)), ((1, inf), (k - 1, nan))]
    at = {(7 * i + 3) % rows: p for i, p in enumerate(plants)}

    def edit(t):
        f = t.float()
        for r, p in at.items():
            for j, v in p:
                f[r, j] = v
        t.copy_(f)

    y, want, slack, half = run(cas, rows, k, n, dtype=dtype, x=x, group=group, x_group=x_group, act=act, zeros=zeros, edit=edit, seed=k + n)
    keep = [r for r in range(rows) if r not in at]
    off = (y[keep].double() - want[keep]).abs() - slack[keep] - half * (want[keep].abs() + slack[keep])
    assert not keep or off.max().item() <= 0
    if act == "none":
        for r in at:
            same_as_formula(y[r], want[r], half)
    else:                                                  # (silu of -infinity is a limit)
        for r in at:
            assert not torch.isfinite(y[r]).any() or x == "same"
            assert torch.isnan(y[r][torch.isnan(want[r])]).all()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("rows,k", [(3, 256), (20, 14336)])
def test_scales_of_rows_that_are_no_numbers(cas, dtype, rows, k):
    """What the norm leaves of a row with a NaN: codes 0, scale NaN; for the row, and for one group of it."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    dt = getattr(torch, dtype)
    codes, scales, zeros = make_weights(70, k, 64, dt, True, g)
    w, d = cas.make_w4_weights(codes, scales, zeros), dense(codes, scales, zeros, 64)
    for groups in (1, k // 128):
        q = torch.randint(-127, 128, (rows, k), device="cuda", generator=g).to(torch.int8)
        s = torch.full((rows, groups), 0.01, device="cuda")
        s[1, groups - 1] = float("nan")
        q[1, k - k // groups:] = 0
        y = torch.empty((rows, 70), device="cuda", dtype=dt)
        cas.cascade_w4_gemm(w, q, y, x_scale=s, workspace=cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w, q)))
        assert torch.isnan(y[1]).all()
        keep = [r for r in range(rows) if r != 1]
        want = (q.double().view(rows, groups, -1) * s.double()[..., None]).view(rows, k)[keep] @ d.t()
        size = want.square().mean().sqrt()
        assert ((y[keep].double() - want).square().mean().sqrt() <= (torch.finfo(dt).eps / 2 + 2.0 ** -17) * size).all()


def test_sums_that_leave_the_range_on_their_way(cas):
    """Products of fp32 values next to the largest that cancel: 1.4e39 in 64 bits leaves 2^-53 of it, 1.6e23, of the others, 3e30 + 2 * 5e30."""
    import torch
    k, n = 256, 48
    codes = torch.full((n, k), 8, device="cuda", dtype=torch.uint8)
    codes[:, 10], codes[:, 20], codes[:, 30], codes[:, 200] = 15, 1, 9, 10       # 7, -7, 1, 2
    w = cas.make_w4_weights(codes, torch.ones((n, k // 32), device="cuda"))
    x = torch.zeros((12, k), device="cuda")
    x[:, 30], x[:, 200] = 3e30, 5e30
    x[11, 10], x[11, 20] = 2e38, 2e38
    y = torch.empty((12, n), device="cuda")
    cas.cascade_w4_gemm(w, x, y, workspace=cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w, x)))
    want = x[0, 30].double() + 2 * x[0, 200].double()
    assert ((y.double() - want).abs() <= 2.0 ** -22 * want).all()

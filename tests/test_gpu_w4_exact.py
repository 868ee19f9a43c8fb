"""fp32 rows in products with 4-bit weights: every bit of X counts.

X enters as three bf16 numbers that add up to it, over codes less their zero points: no sums of X, at most |code - zero| scale |x| an
element.  A row that picks one element gives x (code - zero) scale, which is exact where scale and code - zero are powers of two: the
parts are added from the largest on, and the sum of the first two, x less at most 2^-16 of it, is a multiple of x's last place.

Root mean square.  The 32 elements of a step meet in 3 * 32 additions, each off by at most 2^-23 of the sum so far (a matrix
instruction may cut off), which is no larger than the step's in the mean; signs mix, so sqrt(96) 2^-23 = 2^-19.7 of a step's sum, and the
steps' errors add up like the steps themselves.  The steps are added one to another, k / 32 roundings of 2^-24 in all: sqrt(k / 32) 2^-24,
below 2^-20.5 up to k = 4096.  Together below 2^-19.2, which is the bound; X without its third part would be off by 2^-18.6."""
import pytest

from test_gpu_w4 import dense, make_weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cas():
    import torch
    assert torch.cuda.is_available()
    import paper_2507_05228_amd as cas
    cas.load_library()
    return cas


@pytest.mark.parametrize("k,n,group", [(160, 48, 32), (1024, 33, 64), (4096, 20, 128)])
def test_rows_that_pick_an_element_keep_all_its_bits(cas, k, n, group):
    import torch
    g = torch.Generator(device="cuda").manual_seed(k)
    zeros = torch.where(torch.arange(k // group, device="cuda") % 2 == 0, 8, 7).to(torch.uint8).expand(n, -1).contiguous()
    zero = zeros.repeat_interleave(group, 1).int()
    choices = torch.tensor([0, 1, -1, 2, -2, 4, -4, 8], device="cuda", dtype=torch.int32)
    less = choices[torch.randint(0, len(choices), (n, k), device="cuda", generator=g)]
    codes = (zero + torch.where((less == 8) & (zero == 8), -8, less)).to(torch.uint8)
    assert int(codes.max()) == 15
    scales = 2.0 ** torch.randint(-3, 4, (n, k // group), device="cuda", generator=g).float()
    w = cas.make_w4_weights(codes, scales, zeros)
    want_w = dense(codes, scales, zeros, group)
    for rows in (7, 16, 31):                               # row tiles of 16 and of 32
        at = torch.randint(0, k, (rows,), device="cuda", generator=g)
        bits = torch.randint(0, 1 << 23, (rows,), device="cuda", generator=g, dtype=torch.int32) | 1
        bits[:4] = torch.tensor([0x7fffff, 0x7fff01, 0x008001, 0x018081], device="cuda", dtype=torch.int32)
        value = ((1 + bits.double() / (1 << 23)) * 2.0 ** torch.randint(-20, 21, (rows,), device="cuda", generator=g).double()).float()
        value[1::2] *= -1
        x = torch.zeros((rows, k), device="cuda")
        x[torch.arange(rows, device="cuda"), at] = value
        y = torch.empty((rows, n), device="cuda")
        cas.cascade_w4_gemm(w, x, y, workspace=cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w, x)))
        assert torch.equal(y.double(), value.double()[:, None] * want_w[:, at].t())


@pytest.mark.parametrize("rows", [3, 16, 20, 40])
@pytest.mark.parametrize("k,group,zeros", [(256, 64, True), (1024, 128, False), (4096, 32, True)])
def test_root_mean_square_of_fp32_rows(cas, rows, k, group, zeros):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows + k)
    codes, scales, z = make_weights(400, k, group, torch.float32, zeros, g)
    w = cas.make_w4_weights(codes, scales, z)
    x = torch.randn((rows, k), device="cuda", generator=g)
    y = torch.empty((rows, 400), device="cuda")
    cas.cascade_w4_gemm(w, x, y, workspace=cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w, x)))
    want = x.double() @ dense(codes, scales, z, group).t()
    size = want.square().mean().sqrt().item()
    off = (y.double() - want).square().mean().sqrt().item()
    print(f"{rows} x {k}: {off / size:.2e}")
    assert off <= 2.0 ** -19.2 * size

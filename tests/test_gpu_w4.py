"""Products with 4-bit weights against the formula in 64 bits.

Tolerances.  Codes, zeros and 8-bit rows enter the products exactly.  A group's sum takes (16 + code) x and -(16 + zero) x, in
magnitude at most 62 scale |x| an element, in at most 128 / 32 matrix steps of 2 products (6 in fp32) that each add at
most 32 terms: 4 (2 + 32) < 2^8 roundings of 2^-23 (a matrix instruction may cut off) of that magnitude at the very worst,
2^-15; the sums of the groups add less.  INT8 rows have no such sum.  The bound below takes S = 62 sum |x| scale times 2^-15, which never happens to be
reached; a second one holds the root mean square of all errors to 2^-17 of the results' (signs of roundings mix: 2^-23 * 62 / 4.6 *
a few, at most 2^-18).  Behind the sum: bias, activation (bf16: 2^-12 of the value by the fast forms), residual, half a step."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cas():
    import torch
    assert torch.cuda.is_available()
    import paper_2507_05228_amd as cas
    cas.load_library()
    return cas


def make_weights(n, k, group, dtype, zeros, g):
    import torch
    codes = torch.randint(0, 16, (n, k), device="cuda", generator=g, dtype=torch.uint8)
    scales = ((0.5 + torch.rand((n, k // group), device="cuda", generator=g)) / (4.6 * k ** 0.5)).to(dtype)
    z = torch.randint(0, 16, (n, k // group), device="cuda", generator=g, dtype=torch.uint8) if zeros else None
    return codes, scales, z


def dense(codes, scales, zeros, group):
    n, k = codes.shape
    w = codes.double().view(n, -1, group) - (8 if zeros is None else zeros.double()[..., None])
    return (w * scales.double()[..., None]).view(n, k)


def make_x(rows, k, kind, dtype, x_group, g):
    """x as given, its scales, and its values in 64 bits."""
    import torch
    x = torch.randn((rows, k), device="cuda", generator=g)
    if kind == "same":
        x = x.to(dtype)
        return x, None, x.double()
    scale = 0.5 + torch.rand((rows, k // (x_group or k)), device="cuda", generator=g)
    if kind == "int8":
        q = torch.randint(-128, 128, (rows, k), device="cuda", generator=g).to(torch.int8)
        scale = scale / 64
    else:
        q = (100 * x).clamp(-448, 448).to(torch.float8_e4m3fn)
        scale = scale / 100
    values = (q.double().view(rows, -1, x_group or k) * scale.double()[..., None]).view(rows, k)
    return q, scale, values


def activation(y, act):
    import torch
    return {"none": lambda: y, "gelu": lambda: y * torch.special.ndtr(y), "gelu_tanh": lambda: y * torch.sigmoid((8 / np.pi) ** 0.5 * (y + 0.044715 * y ** 3))}[act]()


def run(cas, rows, k, n, dtype="bf16", group=128, zeros=False, x="same", x_group=0, act="none", bias=False, residual=False, seed=0, edit=None, strides=False):
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(seed)
    xq, xs, x64 = make_x(rows, k, x, dt, x_group, g)
    if edit:
        edit(xq)
        x64 = xq.double() if xs is None else (xq.double().view(rows, -1, x_group or k) * xs.double()[..., None]).view(rows, k)
    if strides:                                            # rows further apart than they are long
        wide = torch.zeros((rows, k + 48), device="cuda", dtype=xq.dtype)
        wide[:, :k] = xq
        xq = wide[:, :k]
    mats = [make_weights(n, k, group, dt, zeros, g) for _ in range(2 if act == "swiglu" else 1)]
    w4 = [cas.make_w4_weights(*m) for m in mats]
    b = torch.randn(n, device="cuda", generator=g).to(dt) if bias else None
    res = torch.randn((rows, n + (5 if strides else 0)), device="cuda", generator=g).to(dt)[:, :n] if residual else None
    room = torch.full((rows + 1, n + (3 if strides else 0)), 7.0, device="cuda", dtype=dt)
    y = room[:rows, :n]
    flags = {"none": 0, "gelu": cas.EPI_GELU_ERF, "gelu_tanh": cas.EPI_GELU_TANH, "swiglu": cas.EPI_SWIGLU}[act]
    flags |= (cas.EPI_BIAS if bias else 0) | (cas.EPI_RESIDUAL if residual else 0)
    ws = cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w4[0], xq, w4[1] if len(w4) > 1 else None))
    cas.cascade_w4_gemm(w4[0], xq, y, x_scale=xs, weights_up=w4[1] if len(w4) > 1 else None, bias=b, residual=res, epilogue=flags, workspace=ws)
    torch.cuda.synchronize()
    assert (room[rows:] == 7).all() and (room[:, n:] == 7).all()
    sums = [x64 @ dense(*m, group).t() for m in mats]
    tops = [62 * (x64.abs() @ m[1].double().abs().repeat_interleave(group, 1).t()) for m in mats]
    want, slack = sums[0], 2.0 ** -15 * tops[0]
    if bias:
        want = want + b.double()
    soft = 2.0 ** -12 if dtype == "bf16" else 2.0 ** -20
    if act == "swiglu":
        gate = want * torch.sigmoid(want)
        slack = 1.1 * slack * sums[1].abs() + gate.abs() * 2.0 ** -15 * tops[1] + 1.1 * slack * 2.0 ** -15 * tops[1]
        want = gate * sums[1]
        slack = slack + soft * want.abs()
    elif act != "none":
        slack = 1.2 * slack + soft * want.abs()
        want = activation(want, act)
    if residual:
        want = want + res.double()
        slack = slack + 2.0 ** -23 * want.abs()
    half = torch.finfo(dt).eps / 2
    return y, want, slack, half


def check(y, want, slack, half, rms=True):
    import torch
    assert torch.isfinite(y).all()
    off = (y.double() - want).abs()
    over = off - slack - half * (want.abs() + slack)
    assert over.max().item() <= 0, f"{over.max().item()} over the bound"
    if rms:
        size = want.square().mean().sqrt().item()
        assert off.square().mean().sqrt().item() <= (half + 2.0 ** -17) * size


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 31, 33, 48, 64, 65, 130])
@pytest.mark.parametrize("x", ["same", "int8", "e4m3"])
def test_rows(cas, rows, x):
    check(*run(cas, rows, 1024, 144, x=x))
    check(*run(cas, rows, 512, 80, dtype="f32", x=x, group=64, zeros=True))


@pytest.mark.parametrize("k,group", [(32, 32), (64, 32), (64, 64), (96, 32), (128, 128), (160, 32), (192, 64), (384, 128), (1056, 32), (1088, 64), (1152, 128), (4096, 128), (14336, 64)])
@pytest.mark.parametrize("zeros", [False, True])
def test_reductions_and_groups(cas, k, group, zeros):
    for dtype, x in (("bf16", "same"), ("f32", "same"), ("bf16", "int8"), ("f32", "e4m3")):
        check(*run(cas, 5, k, 96, dtype=dtype, group=group, zeros=zeros, x=x, seed=k))


@pytest.mark.parametrize("n", [1, 7, 15, 16, 17, 33, 100, 8191, 8192 + 16, 8209])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_columns(cas, n, act):
    check(*run(cas, 3, 256, n, act=act))
    check(*run(cas, 18, 256, n, act=act, dtype="f32", x="int8", group=32))


@pytest.mark.parametrize("x", ["int8", "e4m3"])
@pytest.mark.parametrize("x_group", [32, 64, 128, 256])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_scales_of_8_bit_rows(cas, x, x_group, group):
    for rows in (1, 20, 40):
        check(*run(cas, rows, 768, 50, x=x, x_group=x_group, group=group, zeros=rows > 1))


@pytest.mark.parametrize("act", ["none", "gelu", "gelu_tanh", "swiglu"])
@pytest.mark.parametrize("residual", [False, True])
def test_epilogues(cas, act, residual):
    for dtype in ("bf16", "f32"):
        for rows in (4, 36):
            check(*run(cas, rows, 640, 210, dtype=dtype, act=act, residual=residual, bias=act != "swiglu", group=64, zeros=True))


def test_strides(cas):
    for x in ("same", "int8"):
        check(*run(cas, 19, 512, 203, x=x, residual=True, bias=True, strides=True))


@pytest.mark.parametrize("seed", range(12))
def test_drawn_calls(cas, seed):
    rng = np.random.default_rng(seed)

    def size(most):
        return int(round(np.exp(rng.uniform(0, np.log(most)))))

    for _ in range(5):
        dtype, x, act = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["same", "int8", "e4m3"]), rng.choice(["none", "none", "gelu", "swiglu"])
        group, x_group = int(rng.choice([32, 64, 128])), int(rng.choice([0, 32, 64, 128, 256])) if x != "same" else 0
        unit = max(group, x_group)
        call = dict(dtype=dtype, x=x, group=group, x_group=x_group, act=act, zeros=bool(rng.integers(2)), bias=act != "swiglu" and bool(rng.integers(2)),
                    residual=bool(rng.integers(2)), strides=bool(rng.integers(2)))
        rows, k, n = size(200), unit * size(8192 // unit), size(3000)
        print(rows, k, n, call, flush=True)
        check(*run(cas, rows, k, n, seed=seed, **call), rms=rows * n > 200)


def test_longest_reduction(cas):
    """8192 groups are added one to another: 2^13 roundings of 2^-24 of at most 15 scale |x| an element, 2^-11 * 15 / 62 of the magnitude
    that `slack` is 2^-15 of: less than four times `slack` on top of it."""
    for rows, x in ((3, "same"), (20, "int8"), (40, "same")):
        y, want, slack, half = run(cas, rows, 1 << 20, 16, x=x, zeros=True, seed=11)
        check(y, want, 5 * slack, half, rms=False)


def test_gate_and_up_of_the_same_weights(cas):
    import torch
    g = torch.Generator(device="cuda").manual_seed(12)
    codes, scales, _ = make_weights(200, 512, 64, torch.float32, False, g)
    w = cas.make_w4_weights(codes, scales)
    x = torch.randn((3, 512), device="cuda", generator=g)
    y, plain = torch.empty((3, 200), device="cuda"), torch.empty((3, 200), device="cuda")
    ws = cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w, x, w))
    cas.cascade_w4_gemm(w, x, y, weights_up=w, epilogue=cas.EPI_SWIGLU, workspace=ws)
    cas.cascade_w4_gemm(w, x, plain, workspace=cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w, x)))
    p = plain.double()
    # the two may be cut differently: 2^-18 of either factor's largest, and the fast exponential's 2^-20
    top = p.abs().max()
    assert ((y.double() - p * p * torch.sigmoid(p)).abs() <= 2.0 ** -16 * (top * top + 1)).all()


def test_offsets_beyond_32_bits(cas):
    """Codes of more than 4 GiB, a scale for 128 of them; the first, some inner and the last columns."""
    import torch
    n, k, rows = (1 << 20) + 24, 8320, 2
    g = torch.Generator(device="cuda").manual_seed(13)
    codes = torch.randint(0, 16, (n, k), device="cuda", generator=g, dtype=torch.uint8)
    scales = ((0.5 + torch.rand((n, k // 128), device="cuda", generator=g)) / (4.6 * k ** 0.5)).bfloat16()
    w = cas.make_w4_weights(codes, scales)
    assert cas.load_library().cascade_w4_bytes(w) > 1 << 32
    x = torch.randn((rows, k), device="cuda", generator=g).bfloat16()
    y = torch.empty((rows, n), device="cuda", dtype=torch.bfloat16)
    cas.cascade_w4_gemm(w, x, y, workspace=cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w, x)))
    for c in (slice(0, 64), slice(n // 2 - 32, n // 2 + 32), slice(n - 100, n)):
        want = x.double() @ dense(codes[c], scales[c], None, 128).t()
        top = 62 * (x.double().abs() @ scales[c].double().repeat_interleave(128, 1).t())
        check(y[:, c], want, 2.0 ** -15 * top, torch.finfo(torch.bfloat16).eps / 2)


def test_residual_in_place(cas):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    codes, scales, _ = make_weights(300, 512, 64, torch.bfloat16, False, g)
    w = cas.make_w4_weights(codes, scales)
    x = torch.randn((6, 512), device="cuda", generator=g).bfloat16()
    h = torch.randn((6, 300), device="cuda", generator=g).bfloat16()
    apart = torch.empty_like(h)
    cas.cascade_w4_gemm(w, x, apart, residual=h, epilogue=cas.EPI_RESIDUAL)
    cas.cascade_w4_gemm(w, x, h, residual=h, epilogue=cas.EPI_RESIDUAL)
    assert torch.equal(h, apart)


def test_high_bits_of_codes_and_zeros_do_not_count(cas):
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    codes, scales, zeros = make_weights(40, 256, 32, torch.bfloat16, True, g)
    x = torch.randn((2, 256), device="cuda", generator=g).bfloat16()
    a, b = torch.empty((2, 40), device="cuda", dtype=torch.bfloat16), torch.empty((2, 40), device="cuda", dtype=torch.bfloat16)
    cas.cascade_w4_gemm(cas.make_w4_weights(codes, scales, zeros), x, a)
    cas.cascade_w4_gemm(cas.make_w4_weights(codes | 0xf0, scales, zeros | 0x50), x, b)
    assert torch.equal(a, b)


def test_every_code_of_every_place(cas):
    """Rows that pick one reduction element each: the weights come back exactly."""
    import torch
    k, n = 160, 48
    g = torch.Generator(device="cuda").manual_seed(5)
    codes, _, zeros = make_weights(n, k, 32, torch.float32, True, g)
    scales = 2.0 ** torch.randint(-3, 4, (n, k // 32), device="cuda", generator=g).float()
    w = cas.make_w4_weights(codes, scales, zeros)
    want = dense(codes, scales, zeros, 32).t().float()
    one = torch.ones((k, 1), device="cuda")
    y = torch.empty((k, n), device="cuda")
    for x in (torch.eye(k, device="cuda"), torch.eye(k, device="cuda").to(torch.int8), torch.eye(k, device="cuda").to(torch.float8_e4m3fn)):
        cas.cascade_w4_gemm(w, x, y, x_scale=None if x.dtype == torch.float32 else one)
        assert torch.equal(y, want)


@pytest.mark.parametrize("dtype,x", [("bf16", "same"), ("f32", "same"), ("bf16", "e4m3")])
def test_infinities_and_nan_reach_their_row_alone(cas, dtype, x):
    import torch
    inf, nan = float("inf"), float("nan")

    def edit(t):
        f = t.float()
        if x == "same":
            f[1, 77] = inf
            f[4, 300] = -inf
        f[6, 5] = nan
        t.copy_(f)

    y, want, slack, half = run(cas, 20, 512, 70, dtype=dtype, x=x, edit=edit, seed=9, zeros=True)
    keep = [r for r in range(20) if r not in (1, 4, 6)]
    check(y[keep], want[keep], slack[keep], half, rms=False)
    for r in (1, 4, 6):
        assert torch.equal(torch.isnan(y[r]), torch.isnan(want[r]))
        fine = torch.isfinite(want[r])
        same = ~torch.isnan(want[r]) & ~fine
        assert torch.equal(y[r][same].double(), want[r][same])


def test_fp32_rows_next_to_the_largest(cas):
    import torch

    def edit(t):
        t[2, 10] = 3.4e38
        t[2, 11:] = 0

    y, want, _, _ = run(cas, 4, 128, 20, dtype="f32", edit=edit)
    fine = want[2].abs() < 3e38
    assert ((y[2].double() - want[2]).abs()[fine] <= 2.0 ** -18 * want[2].abs()[fine]).all()


def test_scale_of_infinity_or_nan_stays_in_its_columns(cas):
    import torch
    g = torch.Generator(device="cuda").manual_seed(6)
    codes, scales, _ = make_weights(64, 256, 64, torch.bfloat16, False, g)
    x = torch.randn((3, 256), device="cuda", generator=g).bfloat16()
    clean, hit = torch.empty((3, 64), device="cuda", dtype=torch.bfloat16), torch.empty((3, 64), device="cuda", dtype=torch.bfloat16)
    cas.cascade_w4_gemm(cas.make_w4_weights(codes, scales), x, clean)
    scales[7, 1], scales[33, 0] = float("nan"), float("inf")
    cas.cascade_w4_gemm(cas.make_w4_weights(codes, scales), x, hit)
    others = [c for c in range(64) if c not in (7, 33)]
    assert torch.equal(hit[:, others], clean[:, others]) and torch.isnan(hit[:, 7]).all() and not torch.isfinite(hit[:, 33]).any()


def test_no_rows_other_stream_same_bits(cas):
    import torch
    g = torch.Generator(device="cuda").manual_seed(7)
    codes, scales, zeros = make_weights(4096, 4096, 128, torch.bfloat16, True, g)
    w = cas.make_w4_weights(codes, scales, zeros)
    x = torch.randn((9, 4096), device="cuda", generator=g).bfloat16()
    cas.cascade_w4_gemm(w, x[:0], torch.empty((0, 4096), device="cuda", dtype=torch.bfloat16))
    s, outs = torch.cuda.Stream(), []
    ws = cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(w, x))
    for _ in range(3):
        y = torch.empty((9, 4096), device="cuda", dtype=torch.bfloat16)
        torch.cuda.synchronize()
        cas.cascade_w4_gemm(w, x, y, workspace=ws, stream=s)
        s.synchronize()
        outs.append(y)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_binding_refuses(cas):
    import torch
    g = torch.Generator(device="cuda").manual_seed(8)
    codes, scales, zeros = make_weights(64, 256, 64, torch.bfloat16, True, g)
    for bad in ((codes.int(), scales, zeros), (codes, scales[:10], zeros), (codes, scales, zeros[:, :2]), (codes, scales.half(), zeros), (codes.t(), scales, zeros),
                (codes, scales[:, :3].contiguous(), None), (codes.cpu(), scales, zeros)):
        with pytest.raises(cas.CascadeError):
            cas.make_w4_weights(*bad)
    w = cas.make_w4_weights(codes, scales, zeros)
    x, y = torch.zeros((4, 256), device="cuda", dtype=torch.bfloat16), torch.zeros((4, 64), device="cuda", dtype=torch.bfloat16)
    q = torch.zeros((4, 256), device="cuda", dtype=torch.int8)

    def refused(x=x, y=y, **kw):
        with pytest.raises(cas.CascadeError):
            cas.cascade_w4_gemm(w, x, y, **kw)

    refused(x=x.float())
    refused(x=x[:, :128])
    refused(x=x[:3])
    refused(y=y.float())
    refused(y=y[:, :32])
    refused(y=y[:1].expand(4, 64))
    refused(x=q)
    refused(x=q, x_scale=torch.ones(3, device="cuda"))
    refused(x=q, x_scale=torch.ones((4, 16), device="cuda"))
    refused(x_scale=torch.ones(4, device="cuda"))
    refused(bias=y[0])
    refused(bias=y[0].float(), epilogue=cas.EPI_BIAS)
    refused(residual=y[:2], epilogue=cas.EPI_RESIDUAL)
    refused(epilogue=cas.EPI_SWIGLU)
    refused(x=torch.zeros((4, 257), device="cuda", dtype=torch.bfloat16)[:, 1:])

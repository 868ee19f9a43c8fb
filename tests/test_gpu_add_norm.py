"""The residual's addition, the norm and its 8-bit output against the formula in 64 bits.

Tolerances.  One rounding to the result's type is half a step: eps / 2 of the value.  In fp32 before it: s has one rounding (2^-24); the
mean of D squares (or of D values) adds at most 32 terms a thread, 6 exchanges and 16 wavefronts, under 64 roundings, and the
root, division and products a few more: R = 2^-17 of the value covers them; the layer norm's distances from the mean err by R of the
row's largest |s| besides.  A value in 8 bits is off by half a step of its format and by R of the group's largest."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

R = 2.0 ** -17


@pytest.fixture(scope="module")
def cas():
    import torch
    assert torch.cuda.is_available()
    import paper_2507_05228_amd as cas
    cas.load_library()
    return cas


def make(rows, D, dtype, seed=0, pad=(0, 0), amp=2.0):
    """x, delta [rows, D] (views of wider rows if pad), gain, bias."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = [(amp * torch.randn((rows, D + p), device="cuda", generator=g)).to(dtype)[:, :D] for p in pad]
    v = [(c + 0.3 * torch.randn(D, device="cuda", generator=g)).to(dtype) for c in (1.0, 0.0)]
    return (*t, *v)


def reference(x, delta, gain, bias, layer, eps):
    s = x.double() + (0 if delta is None else delta.double())
    c = s - s.mean(-1, keepdim=True) if layer else s
    r = 1 / (c.square().mean(-1, keepdim=True) + eps).sqrt()
    y = c * r * gain.double() + (0 if bias is None else bias.double())
    slack = R * (y.abs() + (0 if bias is None else bias.double().abs()))
    if layer:
        slack = slack + R * s.abs().amax(-1, keepdim=True) * r * gain.double().abs()
    return s, y, slack


def check(name, got, want, slack, half_step):
    off = (got.double() - want).abs() - slack - half_step * (want.abs() + slack)
    assert off.max().item() <= 0, f"{name}: {off.max().item()} over the bound"


def check_8_bits(q, scale, y, slack, most, D):
    import torch
    groups = scale.numel() // len(y)
    y, slack, q = (t.double().view(len(y), groups, -1) for t in (y, slack, q.float()))
    scale = scale.double().view(len(y), groups, 1)
    largest = y.abs().amax(-1, keepdim=True)
    slack = slack.amax(-1, keepdim=True)
    want = (largest / most).clamp_min(2.0 ** -100)
    assert ((scale - want).abs() <= slack / most + 2.0 ** -22 * want).all()
    assert (q.abs() <= most).all()
    half = scale / 2 if most == 127 else torch.maximum(2.0 ** -4 * y.abs(), scale * 2.0 ** -10)
    off = (q * scale - y).abs() - 1.0001 * half - 3 * slack - 2.0 ** -20 * largest
    assert off.max().item() <= 0


def run(cas, rows, D, dtype, layer=False, delta=True, bias=False, q=None, group=0, y=True, pad=(0, 0), seed=0, amp=2.0, inplace="", eps=1e-5):
    import torch
    x, d, gain, b = make(rows, D, dtype, seed, pad, amp)
    d, b = d if delta else None, b if bias else None
    s64, y64, slack = reference(x, d, gain, b, layer, eps)
    out_sum = {"sum=x": x, "sum=delta": d}.get(inplace, torch.full((rows, D), 7.0, device="cuda", dtype=dtype) if delta else None)
    out_y = {"y=x": x, "y=delta": d}.get(inplace, torch.full((rows, D), 7.0, device="cuda", dtype=dtype) if y else None)
    out_q = torch.empty((rows, D), device="cuda", dtype=q) if q else None
    out_s = torch.full((rows, D // (group or D)), 7.0, device="cuda") if q else None
    cas.cascade_add_norm(x, gain, cas.NORM_LAYERNORM if layer else cas.NORM_RMSNORM, eps, delta=d, bias=b, sum=out_sum, y=out_y, q=out_q, q_scale=out_s)
    torch.cuda.synchronize()
    half = torch.finfo(dtype).eps / 2
    if out_sum is not None:
        check("sum", out_sum, s64, 2.0 ** -24 * s64.abs(), half)
    if out_y is not None:
        check("y", out_y, y64, slack, half)
    if q:
        check_8_bits(out_q, out_s, y64, slack, 127 if q == torch.int8 else 448, D)
    return out_sum, out_y, out_q, out_s


SIZES = [(1, 1), (3, 7), (2, 8), (5, 9), (4, 64), (3, 100), (7, 511), (2, 513), (64, 4096), (3, 4097), (33, 8192), (2, 8199), (3, 12288), (2, 16384), (3, 20000), (2, 32768)]


@pytest.mark.parametrize("rows,D", SIZES)
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_sizes(cas, rows, D, dtype):
    import torch
    dt = getattr(torch, dtype)
    run(cas, rows, D, dt, layer=False, q=torch.int8)
    run(cas, rows, D, dt, layer=True, bias=True, q=torch.float8_e4m3fn, seed=1)
    run(cas, rows, D, dt, delta=False, bias=True, seed=2)


@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("rows,D", [(1, 256), (5, 768), (3, 4096), (2, 8448), (2, 32768)])
def test_groups(cas, group, rows, D):
    import torch
    for dt in (torch.bfloat16, torch.float32):
        for q in (torch.int8, torch.float8_e4m3fn):
            run(cas, rows, D, dt, q=q, group=group, y=False)


@pytest.mark.parametrize("inplace", ["sum=x", "sum=delta", "y=x", "y=delta"])
def test_in_place(cas, inplace):
    import torch
    for dt, D in ((torch.bfloat16, 4096), (torch.float32, 1001), (torch.bfloat16, 20001)):
        run(cas, 9, D, dt, inplace=inplace, q=torch.int8)


@pytest.mark.parametrize("D", [100, 4096, 16390])
def test_strides_and_addresses_off_any_boundary(cas, D):
    import torch
    for dt in (torch.bfloat16, torch.float32):
        run(cas, 6, D, dt, pad=(3, 13), q=torch.int8)
        run(cas, 6, D, dt, pad=(1, 0), layer=True)
    big = torch.randn(6 * (D + 5) + 1, device="cuda").to(torch.bfloat16)
    x = big[1:].view(6, D + 5)[:, :D]
    gain = torch.ones(D + 1, device="cuda", dtype=torch.bfloat16)[1:]
    room = torch.full((6, D + 7), 9, device="cuda", dtype=torch.int8)
    q, scale = room[:, 3:3 + D], torch.empty(6, device="cuda")
    cas.cascade_add_norm(x, gain, cas.NORM_RMSNORM, 1e-5, q=q, q_scale=scale)
    _, y, slack = reference(x, None, gain, None, False, 1e-5)
    check_8_bits(q, scale, y, slack, 127, D)
    assert (room[:, :3] == 9).all() and (room[:, 3 + D:] == 9).all()


def test_many_rows(cas):
    import torch
    run(cas, 70000, 64, torch.bfloat16, q=torch.float8_e4m3fn)


def test_offsets_beyond_32_bits(cas):
    import torch
    stride = (1 << 31) + 40
    big = torch.zeros(2 * stride, device="cuda", dtype=torch.bfloat16)
    x = big.as_strided((2, 512), (stride, 1))
    x.copy_(torch.randn(2, 512, device="cuda"))
    gain = torch.ones(512, device="cuda", dtype=torch.bfloat16)
    y = torch.empty(2, 512, device="cuda", dtype=torch.bfloat16)
    cas.cascade_add_norm(x, gain, cas.NORM_RMSNORM, 1e-5, y=y)
    _, want, slack = reference(x, None, gain, None, False, 1e-5)
    check("y", y, want, slack, 2.0 ** -8)


@pytest.mark.parametrize("amp", [0.0, 1e-30, 1e-12, 1e15])
def test_values_from_zero_to_large(cas, amp):
    import torch
    for dt in (torch.bfloat16, torch.float32):
        for q in (torch.int8, torch.float8_e4m3fn):
            run(cas, 4, 512, dt, q=q, amp=amp, group=128)
            run(cas, 4, 512, dt, q=q, amp=amp, layer=amp < 1e10, bias=True)


def test_gain_of_zero_gives_the_least_scale(cas):
    import torch
    x, _, _, _ = make(3, 256, torch.float32)
    gain = torch.zeros(256, device="cuda")
    gain[128:] = 1e-35
    for q, most in ((torch.int8, 127), (torch.float8_e4m3fn, 448)):
        out, scale = torch.empty((3, 256), device="cuda", dtype=q), torch.empty((3, 2), device="cuda")
        cas.cascade_add_norm(x, gain, cas.NORM_RMSNORM, 1e-5, q=out, q_scale=scale)
        assert (scale == 2.0 ** -100).all() and (out[:, :128].float() == 0).all()
        _, y, slack = reference(x, None, gain, None, False, 1e-5)
        check_8_bits(out, scale, y, slack, most, 256)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_infinities_and_nan_stay_in_their_row_and_group(cas, bad):
    import torch
    for q in (torch.int8, torch.float8_e4m3fn):
        x, d, gain, _ = make(4, 512, torch.float32)
        bias = torch.zeros(512, device="cuda")
        bias[200] = bad                                    # one group of every row
        out, scale, y = torch.empty((4, 512), device="cuda", dtype=q), torch.empty((4, 4), device="cuda"), torch.empty((4, 512), device="cuda")
        cas.cascade_add_norm(x, gain, cas.NORM_RMSNORM, 1e-5, delta=d, bias=bias, y=y, q=out, q_scale=scale)
        hit = torch.zeros(512, dtype=torch.bool, device="cuda")
        hit[200] = True
        assert not torch.isfinite(y[:, hit]).any() and torch.isfinite(y[:, ~hit]).all()
        assert torch.isnan(scale[:, 1]).all() and (out[:, 128:256].float() == 0).all() and torch.isfinite(scale[:, [0, 2, 3]]).all()
        x[2, 300] = bad                                    # a row
        s = torch.empty_like(x)
        cas.cascade_add_norm(x, gain, cas.NORM_RMSNORM, 1e-5, sum=s, y=y, q=out, q_scale=torch.empty(4, device="cuda"))
        assert torch.isfinite(y[[0, 1, 3]]).all() and not torch.isfinite(y[2, 300]) and not torch.isfinite(s[2, 300])


def test_no_rows_and_outputs_alone(cas):
    import torch
    x, d, gain, _ = make(5, 96, torch.bfloat16)
    cas.cascade_add_norm(x[:0], gain, cas.NORM_RMSNORM, 1e-5, y=torch.empty_like(x[:0]))
    s = torch.empty_like(x)
    cas.cascade_add_norm(x, gain, cas.NORM_RMSNORM, 1e-5, delta=d, sum=s)
    assert torch.equal(s, x + d)


def test_same_result_as_cascade_norm_without_a_residual(cas):
    import torch
    x, _, gain, bias = make(17, 4096, torch.float32)
    for kind in (cas.NORM_RMSNORM, cas.NORM_LAYERNORM):
        a, b = torch.empty_like(x), torch.empty_like(x)
        cas.cascade_norm(x, gain, bias, a, kind, 1e-5)
        cas.cascade_add_norm(x, gain, kind, 1e-5, bias=bias, y=b)
        assert (a - b).abs().max().item() <= 2 * R * (a.abs().max().item() + bias.abs().max().item())


def test_other_stream_and_same_bits(cas):
    import torch
    s = torch.cuda.Stream()
    outs = []
    for _ in range(3):
        x, d, gain, _ = make(40, 4096, torch.bfloat16)
        y, q, sc = torch.empty_like(x), torch.empty(x.shape, device="cuda", dtype=torch.int8), torch.empty(40, device="cuda")
        torch.cuda.synchronize()
        cas.cascade_add_norm(x, gain, cas.NORM_RMSNORM, 1e-5, delta=d, y=y, q=q, q_scale=sc, stream=s)
        s.synchronize()
        outs.append((y, q, sc))
    assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(outs[0], o))


def test_binding_refuses(cas):
    import torch
    x, d, gain, bias = make(4, 128, torch.bfloat16)
    q, s = torch.empty((4, 128), device="cuda", dtype=torch.int8), torch.empty(4, device="cuda")

    def refused(**kw):
        with pytest.raises(cas.CascadeError):
            cas.cascade_add_norm(kw.pop("x", x), kw.pop("gain", gain), cas.NORM_RMSNORM, 1e-5, **kw)

    refused()
    refused(y=torch.empty_like(x).float())
    refused(y=torch.empty(4, 64, device="cuda", dtype=torch.bfloat16))
    refused(y=x.t())
    refused(y=x[:1].expand(4, 128))
    refused(y=torch.empty_like(x).cpu())
    refused(y=torch.empty_like(x), gain=gain[:64])
    refused(y=torch.empty_like(x), bias=bias.float())
    refused(y=torch.empty_like(x), delta=d.float())
    refused(q=q)
    refused(q_scale=s, y=torch.empty_like(x))
    refused(q=q, q_scale=torch.empty(7, device="cuda"))
    refused(q=q, q_scale=s.double())
    refused(q=q.to(torch.uint8), q_scale=s)
    refused(q=q, q_scale=torch.empty((4, 8), device="cuda"))
    refused(x=x.half(), y=torch.empty_like(x))

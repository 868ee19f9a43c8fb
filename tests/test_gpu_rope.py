"""Rotary positions against complex numbers in 64 bits: layouts, parts of a head, scaled frequencies, far positions, strides."""
import math

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


def turned(x, positions, rot, theta, layout="half", scaling="none", factor=1.0, low=1.0, high=4.0, original=0, amplitude=1.0):
    x = np.asarray(x, np.float64)
    i = np.arange(rot // 2)
    f = theta ** (-2.0 * i / rot)
    if scaling == "linear":
        f = f / factor
    elif scaling == "ramp":
        g = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0, 1)
        f = f * ((1 - g) / factor + g)
    e = amplitude * np.exp(1j * np.asarray(positions, np.float64)[:, None, None] * f)
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if layout == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    z = (a + 1j * b) * e
    y = x.copy()
    if layout == "half":
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    return y


def desc_of(cas, rot, theta, layout="half", scaling="none", factor=1.0, low=1.0, high=4.0, original=0, amplitude=1.0):
    return cas.make_rope_desc(rot, theta, layout=cas.ROPE_HALF if layout == "half" else cas.ROPE_INTERLEAVED,
                              scaling={"none": cas.ROPE_UNSCALED, "linear": cas.ROPE_LINEAR, "ramp": cas.ROPE_RAMP}[scaling],
                              factor=factor, low=low, high=high, original_len=original, amplitude=amplitude)


def check(got, x, want, dtype, amplitude=1.0, positions=()):
    """Cosine and sine are off by an fp32 rounding and the series' 2^-24 (of 1), products and sums by one each; the angle by its
    64-bit rounding, and by that of this test's own.  Then the result's rounding."""
    from paged_reference import HALF_STEP
    angle = 4 * float(np.abs(np.asarray(positions, np.float64)).max(initial=0)) * 2.0 ** -52
    pair = np.sqrt(2) * np.abs(x).max(-1, keepdims=True) * amplitude
    bound = pair * (5 * 2.0 ** -24 + angle) + np.abs(want) * HALF_STEP[dtype] * 1.01 + 1e-37
    err = np.abs(got.float().cpu().numpy().astype(np.float64) - want)
    assert (err <= bound).all(), (err / bound).max()


def draw(shape, dtype, seed):
    import torch
    from paged_reference import DT
    t = torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(DT[dtype])
    return t.cuda(), t.float().numpy().astype(np.float64)


SCALINGS = [dict(), dict(scaling="linear", factor=3.7), dict(scaling="ramp", factor=8.0, original=8192),
            dict(scaling="ramp", factor=40.0, low=1.0, high=32.0, original=4096, amplitude=1.37)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,d,rot", [(40, 128, 128), (3, 64, 16), (1, 128, 64), (5, 80, 32), (2, 96, 96), (4, 10, 6), (3, 7, 2), (1, 512, 512),
                                         (300, 8, 8)])
def test_layouts_and_parts_of_a_head(cas, dtype, layout, heads, d, rot):
    import torch
    for rows in (1, 37):
        x, xr = draw((rows, heads, d), dtype, rows)
        pos = np.random.default_rng(1).integers(0, 5000, rows).astype(np.int32)
        y = torch.full_like(x, 7.0)
        cas.cascade_rope(desc_of(cas, rot, 10000.0, layout), x, torch.from_numpy(pos).cuda(), y)
        want = turned(xr, pos, rot, 10000.0, layout)
        check(y, xr, want, dtype, positions=pos)
        assert torch.equal(y[..., rot:], x[..., rot:])
        cas.cascade_rope(desc_of(cas, rot, 10000.0, layout), x, torch.from_numpy(pos).cuda())      # in place
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", SCALINGS)
@pytest.mark.parametrize("theta", [10000.0, 500000.0, 1234.5678])
def test_scaled_frequencies(cas, dtype, kw, theta):
    import torch
    rows = 2100                                             # several rows of a workgroup
    x, xr = draw((rows, 6, 128), dtype, 2)
    pos = np.random.default_rng(3).integers(0, 131072, rows).astype(np.int32)
    y = torch.empty_like(x)
    cas.cascade_rope(desc_of(cas, 128, theta, **kw), x, torch.from_numpy(pos).cuda(), y)
    check(y, xr, turned(xr, pos, 128, theta, **kw), dtype, kw.get("amplitude", 1.0), pos)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_and_negative_positions(cas, layout):
    import torch
    pos = np.array([0, 1, -1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31, 123456789, -7], np.int32)
    x, xr = draw((8, 2, 64), "f32", 4)
    y = torch.empty_like(x)
    cas.cascade_rope(desc_of(cas, 64, 500000.0, layout), x, torch.from_numpy(pos).cuda(), y)
    check(y, xr, turned(xr, pos, 64, 500000.0, layout), "f32", positions=pos)
    # and back
    near = np.array([0, 1, 5, 100, 4096, 131071, 70000, 3], np.int32)
    z = torch.empty_like(x)
    cas.cascade_rope(desc_of(cas, 64, 500000.0, layout), x, torch.from_numpy(near).cuda(), z)
    cas.cascade_rope(desc_of(cas, 64, 500000.0, layout), z, torch.from_numpy(-near).cuda())
    assert (z - x).abs().max() <= 2 * 5 * 2.0 ** -24 * 1.5 * x.abs().max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("offset", [0, 1])
def test_strides_and_alignment(cas, dtype, layout, offset):
    """Heads of a wider row; rows that begin anywhere.  What lies between them stays."""
    import torch
    from paged_reference import DT
    rows, H, d = 9, 3, 32
    flat = torch.randn(rows * (H * d + 24) + 8, generator=torch.Generator().manual_seed(5)).to(DT[dtype]).cuda()
    x = flat[offset:offset + rows * (H * d + 24)].view(rows, H * d + 24)[:, 8:8 + H * d].unflatten(1, (H, d))
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") * 11
    before, xr = flat.clone(), x.float().cpu().numpy().astype(np.float64)
    want = turned(xr, pos.cpu().numpy(), 16, 10000.0, layout)
    cas.cascade_rope(desc_of(cas, 16, 10000.0, layout), x, pos)
    check(x, xr, want, dtype, positions=[99])
    after = flat.clone()
    after[offset:offset + rows * (H * d + 24)].view(rows, H * d + 24)[:, 8:8 + H * d] = 0
    before[offset:offset + rows * (H * d + 24)].view(rows, H * d + 24)[:, 8:8 + H * d] = 0
    assert torch.equal(after, before)


def test_it_is_the_rotation_of_the_projection(cas):
    """The shard GEMM with an identity as its weights and EPI_ROPE rotates as cascade_rope does, up to the roundings."""
    import torch
    rows, d = 50, 64
    x, xr = draw((rows, 2, d), "f32", 6)
    plan = cas.cascade_plan_create(1, rows, 1, np.zeros(rows, np.int32))
    y = torch.empty((rows, 2 * d), device="cuda")
    cas.cascade_shard_gemm(plan, x.view(rows, 2 * d), torch.eye(2 * d, device="cuda"), y, epilogue=cas.EPI_ROPE, rope_cols=2 * d, head_dim=d,
                           rope_theta=10000.0)
    z = torch.empty_like(x)
    cas.cascade_rope(desc_of(cas, d, 10000.0), x, torch.arange(rows, dtype=torch.int32, device="cuda"), z)
    assert (y.view_as(z) - z).abs().max() <= 1e-5 * x.abs().max()

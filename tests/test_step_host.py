"""The operators of a token's step around its attention on the host: layouts of the descriptors, sizes, and what the entry points
refuse before they touch the GPU (pointers here are addresses that nothing reads)."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2507_05228_amd as cas

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20                                                # an aligned address


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cas.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return cas.load_library()


def test_descriptors_have_the_layout_of_the_header(tmp_path):
    src = tmp_path / "layout.c"
    fields = {"cascade_add_norm_desc": (cas.AddNormDesc, "eps q_group x_stride q_stride"), "cascade_w4_weights": (cas.W4Weights, "group zero_points packed"),
              "cascade_w4_gemm_desc": (cas.W4GemmDesc, "epilogue x_stride y_stride"), "cascade_sample_desc": (cas.SampleDesc, "vocab stride")}
    lines = [f'printf("%zu\\n", sizeof({c}));' + "".join(f'printf("%zu\\n", offsetof({c}, {f}));' for f in names.split())
             for c, (_, names) in fields.items()]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "cascade.h"\nint main(void){' + "".join(lines) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(t) for t in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [n for t, names in fields.values() for n in [C.sizeof(t)] + [getattr(t, f).offset for f in names.split()]]


# ------------------------------------------------------------------ add_norm
def add_norm(lib, x=P, delta=2 * P, gain=3 * P, bias=None, sum=4 * P, y=5 * P, q=None, q_scale=None, **change):
    d = cas.AddNormDesc(cas.BF16, 4, 256, cas.NORM_RMSNORM, 1e-5, 0, 0, 0, 0, 0, 0, 0)
    for k, v in change.items():
        setattr(d, k, v)
    return lib.cascade_add_norm(C.byref(d), x, delta, gain, bias, sum, y, q, q_scale, None)


Q = dict(q=6 * P, q_scale=7 * P, q_format=1)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), cas.EINVAL), (dict(gain=None), cas.EINVAL), (dict(sum=None, y=None), cas.EINVAL), (dict(rows=-1), cas.EINVAL),
    (dict(d_model=0), cas.EINVAL), (dict(norm_kind=0), cas.EINVAL), (dict(norm_kind=3), cas.EINVAL), (dict(q_format=1), cas.EINVAL),
    (dict(q=P, q_scale=P), cas.EINVAL), (dict(Q, q_scale=None), cas.EINVAL), (dict(Q, q_format=3), cas.EINVAL), (dict(Q, q_format=-1), cas.EINVAL),
    (dict(Q, q_group=-32), cas.EINVAL), (dict(Q, q=P), cas.EINVAL), (dict(Q, q=5 * P), cas.EINVAL), (dict(sum=5 * P), cas.EINVAL),
    (dict(x_stride=-1), cas.EINVAL), (dict(dtype=2), cas.EUNSUPPORTED), (dict(d_model=32769), cas.EUNSUPPORTED),
    (dict(Q, q_group=48), cas.EUNSUPPORTED), (dict(Q, q_group=512), cas.EUNSUPPORTED), (dict(Q, q_group=64, d_model=96), cas.ESHAPE),
    (dict(x_stride=255), cas.ESHAPE), (dict(delta_stride=8), cas.ESHAPE), (dict(sum_stride=1), cas.ESHAPE), (dict(y_stride=1), cas.ESHAPE),
    (dict(Q, q_stride=255), cas.ESHAPE), (dict(sum=P, x_stride=512), cas.ESHAPE), (dict(y=2 * P, y_stride=512), cas.ESHAPE),
    (dict(rows=0), cas.OK), (dict(Q, rows=0, q_group=128, sum=P, y=2 * P), cas.OK)])
def test_add_norm_refuses(lib, change, status):
    assert add_norm(lib, **change) == status


def test_null_descriptors(lib):
    assert lib.cascade_add_norm(None, P, P, P, P, P, P, None, None, None) == cas.EINVAL
    assert lib.cascade_w4_pack(None, P, P, P, None) == cas.EINVAL and lib.cascade_w4_bytes(None) == 0
    assert lib.cascade_w4_gemm(C.byref(weights()), None, None, P, None, None, None, P, P, 0, None) == cas.EINVAL
    assert lib.cascade_sample(None, P, P, P, P, P, P, P, P, P, 1 << 40, None) == cas.EINVAL and lib.cascade_sample_workspace_bytes(None) == 0


# ------------------------------------------------------------------ 4-bit weights
def weights(**change):
    w = cas.W4Weights(cas.BF16, 100, 256, 64, 0, 0, P)
    for k, v in change.items():
        setattr(w, k, v)
    return w


BAD_WEIGHTS = [(dict(n_out=0), cas.EINVAL), (dict(k=0), cas.EINVAL), (dict(group=0), cas.EINVAL), (dict(reserved=1), cas.EINVAL),
               (dict(zero_points=2), cas.EINVAL), (dict(dtype=2), cas.EUNSUPPORTED), (dict(group=16), cas.EUNSUPPORTED),
               (dict(group=256), cas.EUNSUPPORTED), (dict(k=288), cas.ESHAPE), (dict(k=(1 << 20) + 64), cas.EUNSUPPORTED),
               (dict(n_out=(1 << 31) - 1), cas.EUNSUPPORTED), (dict(n_out=(1 << 26) + 1), cas.EUNSUPPORTED), (dict(packed=None), cas.EINVAL), (dict(packed=P + 128), cas.EUNSUPPORTED)]


@pytest.mark.parametrize("change,status", BAD_WEIGHTS)
def test_every_entry_point_checks_the_weights(lib, change, status):
    w = C.byref(weights(**change))
    d = cas.W4GemmDesc(4, 0, 0, 0, 0, 0, 0)
    assert lib.cascade_w4_pack(w, P, P, None, None) == status
    assert lib.cascade_w4_gemm(w, None, C.byref(d), P, None, None, None, 2 * P, P, 1 << 40, None) == status
    if "packed" not in change:
        assert lib.cascade_w4_bytes(w) == 0 and lib.cascade_w4_gemm_workspace_bytes(w, C.byref(d)) == 0


@pytest.mark.parametrize("args,status", [((None, P, None), cas.EINVAL), ((P, None, None), cas.EINVAL), ((P, P, P), cas.EINVAL)])
def test_pack_refuses(lib, args, status):
    assert lib.cascade_w4_pack(C.byref(weights()), *args, None) == status
    assert lib.cascade_w4_pack(C.byref(weights(zero_points=1)), P, P, None, None) == cas.EINVAL


@pytest.mark.parametrize("n,k,group,dtype,zeros", [(1, 32, 32, cas.BF16, 0), (16, 128, 128, cas.F32, 1), (17, 160, 32, cas.BF16, 1), (4096, 14336, 128, cas.BF16, 0)])
def test_bytes_of_packed_weights(lib, n, k, group, dtype, zeros):
    up = lambda v, to: -(-v // to) * to  # noqa: E731
    entries = up(n, 16) * (k // group)
    want = up(n, 16) * up(k, 128) // 2 + up(entries * (2 if dtype == cas.BF16 else 4), 256) + (up(entries, 256) if zeros else 0)
    assert lib.cascade_w4_bytes(C.byref(weights(n_out=n, k=k, group=group, dtype=dtype, zero_points=zeros))) == want


def gemm(lib, w=None, up=None, X=4 * P, x_scale=None, bias=None, residual=None, Y=8 * P, ws=P, ws_bytes=1 << 40, **change):
    d = cas.W4GemmDesc(4, 0, 0, 0, 0, 0, 0)
    for k, v in change.items():
        setattr(d, k, v)
    return lib.cascade_w4_gemm(C.byref(w or weights()), None if up is None else C.byref(up), C.byref(d), X, x_scale, bias, residual, Y, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(X=None), cas.EINVAL), (dict(Y=None), cas.EINVAL), (dict(Y=4 * P), cas.EINVAL), (dict(rows=-1), cas.EINVAL), (dict(x_format=3), cas.EINVAL),
    (dict(x_format=-1), cas.EINVAL), (dict(x_scale=P), cas.EINVAL), (dict(x_format=1), cas.EINVAL), (dict(x_group=-1), cas.EINVAL),
    (dict(epilogue=cas.EPI_BIAS), cas.EINVAL), (dict(bias=P), cas.EINVAL), (dict(epilogue=cas.EPI_RESIDUAL), cas.EINVAL), (dict(residual=P), cas.EINVAL),
    (dict(epilogue=cas.EPI_SWIGLU), cas.EINVAL), (dict(up=weights()), cas.EINVAL), (dict(up=weights(packed=None), epilogue=cas.EPI_SWIGLU), cas.EINVAL),
    (dict(x_stride=-1), cas.EINVAL), (dict(y_stride=-1), cas.EINVAL), (dict(residual_stride=-1), cas.EINVAL),
    (dict(epilogue=cas.EPI_ROPE), cas.EUNSUPPORTED), (dict(epilogue=64), cas.EUNSUPPORTED),
    (dict(epilogue=cas.EPI_GELU_ERF | cas.EPI_GELU_TANH), cas.EUNSUPPORTED), (dict(epilogue=cas.EPI_SWIGLU | cas.EPI_GELU_ERF), cas.EUNSUPPORTED),
    (dict(epilogue=cas.EPI_SWIGLU | cas.EPI_BIAS, up=weights(), bias=P), cas.EUNSUPPORTED),
    (dict(x_format=1, x_scale=P, x_group=48), cas.EUNSUPPORTED), (dict(x_format=2, x_scale=P, x_group=512), cas.EUNSUPPORTED),
    (dict(w=weights(k=320), x_format=2, x_scale=P, x_group=128), cas.ESHAPE),
    (dict(x_stride=248), cas.ESHAPE), (dict(y_stride=99), cas.ESHAPE), (dict(residual_stride=99, residual=P, epilogue=cas.EPI_RESIDUAL), cas.ESHAPE),
    (dict(residual=8 * P, residual_stride=104, epilogue=cas.EPI_RESIDUAL), cas.ESHAPE),
    (dict(up=weights(n_out=96), epilogue=cas.EPI_SWIGLU), cas.ESHAPE), (dict(up=weights(k=512), epilogue=cas.EPI_SWIGLU), cas.ESHAPE),
    (dict(up=weights(group=32), epilogue=cas.EPI_SWIGLU), cas.ESHAPE), (dict(up=weights(zero_points=1), epilogue=cas.EPI_SWIGLU), cas.ESHAPE),
    (dict(up=weights(dtype=cas.F32), epilogue=cas.EPI_SWIGLU), cas.ESHAPE), (dict(up=weights(packed=P + 16), epilogue=cas.EPI_SWIGLU), cas.EUNSUPPORTED),
    (dict(X=4 * P + 8), cas.EUNSUPPORTED), (dict(x_stride=260), cas.EUNSUPPORTED), (dict(x_stride=1 << 23), cas.EUNSUPPORTED),
    (dict(rows=(1 << 20) + 1), cas.EUNSUPPORTED), (dict(rows=0), cas.OK), (dict(rows=0, up=weights(), epilogue=cas.EPI_SWIGLU | cas.EPI_RESIDUAL, residual=8 * P), cas.OK)])
def test_w4_gemm_refuses(lib, change, status):
    assert gemm(lib, **change) == status


# ------------------------------------------------------------------ sampling
def sample(lib, logits=P, uniform=P, token=P, ws=P, ws_bytes=1 << 40, **change):
    d = cas.SampleDesc(cas.BF16, 4, 1000, 0, 0)
    for k, v in change.items():
        setattr(d, k, v)
    size = lib.cascade_sample_workspace_bytes(C.byref(d))
    return lib.cascade_sample(C.byref(d), logits, None, None, None, None, uniform, token, None, ws, ws_bytes if ws_bytes >= 0 else size + ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(logits=None), cas.EINVAL), (dict(uniform=None), cas.EINVAL), (dict(token=None), cas.EINVAL), (dict(rows=-1), cas.EINVAL), (dict(vocab=0), cas.EINVAL),
    (dict(stride=-1), cas.EINVAL), (dict(reserved=1), cas.EINVAL), (dict(dtype=2), cas.EUNSUPPORTED), (dict(vocab=(1 << 20) + 1), cas.EUNSUPPORTED),
    (dict(rows=(1 << 16) + 1), cas.EUNSUPPORTED), (dict(stride=999), cas.ESHAPE), (dict(ws=None), cas.EWORKSPACE), (dict(ws=P + 8), cas.EWORKSPACE),
    (dict(ws_bytes=-1), cas.EWORKSPACE), (dict(rows=0), cas.OK)])
def test_sample_refuses(lib, change, status):
    assert sample(lib, **change) == status


def test_binding_refuses_what_it_can_see_on_the_host():
    import torch
    x, gain = torch.zeros(4, 64), torch.zeros(64)
    for call in (lambda: cas.cascade_add_norm(x, gain, cas.NORM_RMSNORM, 1e-5, y=x),
                 lambda: cas.make_w4_weights(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2)),
                 lambda: cas.cascade_w4_gemm(weights(), x, x),
                 lambda: cas.cascade_sample(x, torch.zeros(4), torch.zeros(4, dtype=torch.int32))):
        with pytest.raises(cas.CascadeError) as e:
            call()
        assert e.value.status == cas.ESHAPE

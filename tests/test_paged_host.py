"""Rotary positions and the paged cache on the host: layouts of the descriptors, sizes, and what the entry points refuse before
they touch the GPU (pointers here are addresses that nothing reads)."""
import ctypes as C
import math
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
    fields = {"cascade_rope_desc": (cas.RopeDesc, "theta amplitude"), "cascade_paged_cache": (cas.PagedCache, "max_pages k_pages page_refs"),
              "cascade_paged_attn_desc": (cas.PagedAttnDesc, "o_dtype q_stride o_stride")}
    lines = [f'printf("%zu\\n", sizeof({c}));' + "".join(f'printf("%zu\\n", offsetof({c}, {f}));' for f in names.split())
             for c, (_, names) in fields.items()]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "cascade.h"\nint main(void){' + "".join(lines) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(t) for t in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [n for t, names in fields.values() for n in [C.sizeof(t)] + [getattr(t, f).offset for f in names.split()]]


def cache(**kw):
    c = cas.PagedCache(cas.BF16, 2, 100, 2, 64, 16, 4, 1, 8, P, P, P, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [(dict(k_pages=None), cas.EINVAL), (dict(page_refs=None), cas.EINVAL), (dict(n_layers=0), cas.EINVAL), (dict(n_pages=-1), cas.EINVAL),
              (dict(page_size=0), cas.EINVAL), (dict(max_pages=0), cas.EINVAL), (dict(dtype=2), cas.EUNSUPPORTED),
              (dict(head_dim=20), cas.EUNSUPPORTED), (dict(head_dim=264), cas.EUNSUPPORTED), (dict(page_size=8), cas.EUNSUPPORTED),
              (dict(page_size=48), cas.EUNSUPPORTED), (dict(page_size=1 << 17), cas.EUNSUPPORTED), (dict(n_shards=1025), cas.EUNSUPPORTED),
              (dict(n_pages=1 << 27), cas.EUNSUPPORTED), (dict(max_pages=1 << 27), cas.EUNSUPPORTED),
              (dict(n_seqs=1 << 20, max_pages=1 << 12), cas.EUNSUPPORTED),
              (dict(n_shards=64, max_pages=1 << 15, page_size=1 << 15, n_pages=1 << 10), cas.EUNSUPPORTED), (dict(v_pages=P + 8), cas.EUNSUPPORTED),
              (dict(dtype=cas.F32, head_dim=66), cas.EUNSUPPORTED)]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_every_entry_point_checks_the_cache(lib, change, status):
    c = C.byref(cache(**change))
    desc = cas.PagedAttnDesc(4, 4, 1.0, cas.BF16, 0, 0)
    assert lib.cascade_paged_extend(c, 1, P, P, P, P, P, None) == status
    assert lib.cascade_paged_append(c, 0, 1, P, P, P, 0, None, None, 0, None, 0, None, 0, None) == status
    assert lib.cascade_paged_attn(c, 0, C.byref(desc), P, P, P, P, P, P, 1 << 40, None) == status
    assert lib.cascade_pages_free(c, 1, P, None) == status
    assert lib.cascade_pages_fork(c, 1, P, P, P, P, 1 << 40, None) == status
    assert lib.cascade_pages_compact(c, P, P, 1 << 40, None) == status
    assert lib.cascade_pages_copy(c, 1, P, P, None) == status
    assert lib.cascade_pages_workspace_bytes(c) == 0 and lib.cascade_paged_attn_workspace_bytes(c, C.byref(desc)) == 0


def test_null_descriptors(lib):
    assert lib.cascade_paged_extend(None, 1, P, P, P, P, P, None) == cas.EINVAL
    assert lib.cascade_paged_attn(C.byref(cache()), 0, None, P, P, P, P, P, P, 1 << 40, None) == cas.EINVAL
    assert lib.cascade_rope(None, cas.F32, 1, 1, 64, P, P, 0, P, 0, None) == cas.EINVAL


ROPE = dict(layout=0, rot_dim=64, scaling=0, original_len=0, theta=1e4, factor=1.0, low=1.0, high=4.0, amplitude=1.0)


@pytest.mark.parametrize("change,status", [
    (dict(layout=2), cas.EINVAL), (dict(scaling=3), cas.EINVAL), (dict(rot_dim=0), cas.EINVAL), (dict(rot_dim=-2), cas.EINVAL),
    (dict(rot_dim=7), cas.EUNSUPPORTED), (dict(rot_dim=514), cas.EUNSUPPORTED), (dict(rot_dim=66), cas.ESHAPE), (dict(theta=0.0), cas.EINVAL),
    (dict(theta=math.nan), cas.EINVAL), (dict(theta=math.inf), cas.EINVAL), (dict(amplitude=math.nan), cas.EINVAL),
    (dict(scaling=1, factor=0.0), cas.EINVAL), (dict(scaling=1, factor=math.nan), cas.EINVAL), (dict(scaling=2, factor=2.0), cas.EINVAL),
    (dict(scaling=2, factor=2.0, original_len=8192, low=4.0), cas.EINVAL), (dict(scaling=2, factor=2.0, original_len=8192, high=math.nan), cas.EINVAL)])
def test_rope_descriptors(lib, change, status):
    desc = cas.RopeDesc(**{**ROPE, **change})
    assert lib.cascade_rope(C.byref(desc), cas.BF16, 1, 2, 64, P, P, 0, 2 * P, 0, None) == status
    assert lib.cascade_paged_append(C.byref(cache()), 0, 1, P, P, P, 0, C.byref(desc), P, 0, None, 0, None, 0, None) == status


@pytest.mark.parametrize("args,status", [
    ((0, 0, 1, 64, P, P, 0, P, 0), cas.EINVAL), ((0, 1, 0, 64, P, P, 0, P, 0), cas.EINVAL), ((0, 1, 1, 64, None, P, 0, P, 0), cas.EINVAL),
    ((0, 1, 1, 64, P, None, 0, P, 0), cas.EINVAL), ((0, 1, 1, 64, P, P, 0, None, 0), cas.EINVAL), ((3, 1, 1, 64, P, P, 0, P, 0), cas.EUNSUPPORTED),
    ((0, 1, 2, 64, P, P, 127, P, 0), cas.ESHAPE), ((0, 1, 2, 64, P, P, 0, 2 * P, 100), cas.ESHAPE), ((0, 1, 1, 64, P, P, 128, P, 64), cas.ESHAPE),
    ((0, 1, 1, 64, P, P, -64, P, 0), cas.EINVAL)])
def test_rope_arguments(lib, args, status):
    assert lib.cascade_rope(C.byref(cas.RopeDesc(**ROPE)), *args, None) == status


@pytest.mark.parametrize("change,status", [
    (dict(rows=0), cas.EINVAL), (dict(slots=None), cas.EINVAL), (dict(k=None), cas.EINVAL), (dict(v=None), cas.EINVAL), (dict(layer=2), cas.ESHAPE),
    (dict(layer=-1), cas.ESHAPE), (dict(kv_stride=127), cas.ESHAPE), (dict(kv_stride=-1), cas.EINVAL), (dict(positions=P), cas.EINVAL),
    (dict(q=P, q_out=P, heads=4), cas.EINVAL), (dict(rope=True), cas.EINVAL), (dict(rope=True, positions=P, q=P, heads=4), cas.EINVAL),
    (dict(rope=True, positions=P, q=P, q_out=P, heads=0), cas.EINVAL), (dict(rope=True, positions=P, q=P, q_out=P, heads=4, qs=255), cas.ESHAPE),
    (dict(rope=True, positions=P, q=P, q_out=P, heads=4, qs=512), cas.ESHAPE)])
def test_append_arguments(lib, change, status):
    a = {**dict(layer=0, rows=1, slots=P, k=P, v=P, kv_stride=0, rope=False, positions=None, heads=0, q=None, qs=0, q_out=None, qos=0), **change}
    desc = cas.RopeDesc(**ROPE)
    assert lib.cascade_paged_append(C.byref(cache()), a["layer"], a["rows"], a["slots"], a["k"], a["v"], a["kv_stride"],
                                    C.byref(desc) if a["rope"] else None, a["positions"], a["heads"], a["q"], a["qs"], a["q_out"], a["qos"],
                                    None) == status


@pytest.mark.parametrize("desc,args,status", [
    ((0, 4, 1.0, 1, 0, 0), {}, cas.EINVAL), ((4, 0, 1.0, 1, 0, 0), {}, cas.EINVAL), ((4, 4, 0.0, 1, 0, 0), {}, cas.EINVAL),
    ((4, 4, math.nan, 1, 0, 0), {}, cas.EINVAL), ((4, 3, 1.0, 1, 0, 0), {}, cas.ESHAPE), ((4, 4, 1.0, 2, 0, 0), {}, cas.EUNSUPPORTED),
    ((4, 4, 1.0, 1, 255, 0), {}, cas.ESHAPE), ((4, 4, 1.0, 1, 0, 248), {}, cas.ESHAPE), ((4, 4, 1.0, 1, 260, 0), {}, cas.EUNSUPPORTED),
    ((4, 4, 1.0, 1, 0, 260), {}, cas.EUNSUPPORTED), ((4, 4, 1.0, 1, 0, 0), dict(q_start=None), cas.EINVAL),
    ((4, 4, 1.0, 1, 0, 0), dict(q=None), cas.EINVAL), ((4, 4, 1.0, 1, 0, 0), dict(o=None), cas.EINVAL),
    ((4, 4, 1.0, 1, 0, 0), dict(q=P + 8), cas.EUNSUPPORTED), ((4, 4, 1.0, 1, 0, 0), dict(o=P + 2), cas.EUNSUPPORTED),
    ((4, 4, 1.0, 1, 0, 0), dict(layer=2), cas.ESHAPE), ((4, 4, 1.0, 1, 0, 0), dict(ws=None), cas.EWORKSPACE),
    ((4, 4, 1.0, 1, 0, 0), dict(ws=P + 4), cas.EWORKSPACE), ((4, 4, 1.0, 1, 0, 0), dict(bytes=1000), cas.EWORKSPACE)])
def test_attention_arguments(lib, desc, args, status):
    a = {**dict(layer=0, q_start=P, visible=None, q=P, o=P, ws=P, bytes=1 << 40), **args}
    assert lib.cascade_paged_attn(C.byref(cache()), a["layer"], C.byref(cas.PagedAttnDesc(*desc)), a["q_start"], a["visible"], a["q"], a["o"],
                                  None, a["ws"], a["bytes"], None) == status


@pytest.mark.parametrize("heads,dtype,d,rows", [(4, 0, 64, 1 << 27), (4, 1, 40, 1 << 27), (1024, 0, 4, 1 << 19)])
def test_attention_of_more_rows_than_a_launch_holds(lib, heads, dtype, d, rows):
    """16 rows of a kv head a workgroup of 256: 2^28 rows times heads are 2^32 threads."""
    c = cache(dtype=dtype, head_dim=d, n_kv_heads=heads, n_seqs=1, n_pages=4, max_pages=4, page_size=16)
    desc = cas.PagedAttnDesc(rows, heads, 1.0, dtype, 0, 0)
    assert rows * heads >= 1 << 28
    assert lib.cascade_paged_attn_workspace_bytes(C.byref(c), C.byref(desc)) == 0
    assert lib.cascade_paged_attn(C.byref(c), 0, C.byref(desc), P, None, P, P, None, P, 1 << 40, None) == cas.EUNSUPPORTED
    desc.rows = rows >> 4
    assert lib.cascade_paged_attn_workspace_bytes(C.byref(c), C.byref(desc)) > 0


def test_page_arguments(lib):
    c, many = C.byref(cache()), C.byref(cache(n_shards=3))
    assert lib.cascade_paged_extend(c, 0, P, None, P, P, P, None) == cas.EINVAL
    assert lib.cascade_paged_extend(c, 1, None, None, P, P, P, None) == cas.EINVAL
    assert lib.cascade_paged_extend(many, 1, P, None, P, P, P, None) == cas.EINVAL             # several shards: which row is whose?
    assert lib.cascade_pages_free(c, 0, P, None) == cas.EINVAL and lib.cascade_pages_free(c, 1, None, None) == cas.EINVAL
    assert lib.cascade_pages_fork(c, 1, P, None, P, P, 1 << 40, None) == cas.EINVAL
    assert lib.cascade_pages_fork(many, 8192, P, P, P, P, 1 << 40, None) == cas.EUNSUPPORTED
    assert lib.cascade_pages_fork(c, 1, P, P, P, None, 1 << 40, None) == cas.EWORKSPACE
    assert lib.cascade_pages_fork(c, 1, P, P, P, P, 16, None) == cas.EWORKSPACE
    assert lib.cascade_pages_compact(c, P, None, 1 << 40, None) == cas.EWORKSPACE
    assert lib.cascade_pages_compact(c, P, P + 4, 1 << 40, None) == cas.EWORKSPACE
    assert lib.cascade_pages_copy(c, 0, P, P, None) == cas.EINVAL and lib.cascade_pages_copy(c, 1, P, None, None) == cas.EINVAL


def test_the_binding_refuses_what_does_not_fit():
    import torch
    kp, t, n, r = torch.zeros(1, 4, 2, 16, 64), *(torch.zeros(s, dtype=torch.int32) for s in ((2, 1, 3), (2, 1), (4,)))
    for args in ((kp, kp, t, n, r), (kp, kp, t.long(), n, r)):       # not on the GPU; not int32
        with pytest.raises(cas.CascadeError) as e:
            cas.make_paged_cache(*args)
        assert e.value.status == cas.ESHAPE

"""Rotary positions and rows of a cache in numbers that one launch cannot hold."""
import numpy as np
import pytest

from test_gpu_paged_attn import cas  # noqa: F401

pytestmark = pytest.mark.gpu

ROWS = (1 << 27) + 9                                       # 8 rows a workgroup of 256 threads: 2^32 threads and more
LOOK = [0, 1, (1 << 26) - 1, 1 << 26, (1 << 26) + 1, (1 << 27) - 1, 1 << 27, ROWS - 1]


def test_rows_that_take_several_launches(cas):  # noqa: F811
    import torch
    from test_gpu_rope import check, desc_of, turned
    x = torch.zeros((ROWS, 1, 8), dtype=torch.bfloat16, device="cuda")
    look, pos = torch.tensor(LOOK, device="cuda"), torch.arange(ROWS, device="cuda", dtype=torch.int32)
    x[look] = torch.randn((len(LOOK), 1, 8), device="cuda").bfloat16()
    was = x[look].float().cpu().numpy().astype(np.float64)
    cas.cascade_rope(desc_of(cas, 8, 10000.0, "half"), x, pos)
    torch.cuda.synchronize()
    check(x[look], was, turned(was, LOOK, 8, 10000.0, "half"), "bf16", positions=LOOK)
    x[look] = 0
    assert not x.any()


def test_rows_of_a_cache_that_take_several_launches(cas):  # noqa: F811
    import torch
    from paged_reference import Cache
    cache = Cache(cas, "bf16", 1, 8, 16, [[33]], seed=1, filler=0.0)
    k, v = (torch.zeros((ROWS, 1, 8), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots, look = torch.full((ROWS,), -1, dtype=torch.int32, device="cuda"), torch.tensor(LOOK, device="cuda")
    k[look], v[look] = (torch.randn((len(LOOK), 1, 8), device="cuda").bfloat16() for _ in range(2))
    slots[look] = torch.arange(16, 16 + len(LOOK), device="cuda", dtype=torch.int32)
    kp, vp = cache.kp.clone(), cache.vp.clone()
    cas.cascade_paged_append(cache.handle, 0, slots, k, v)
    torch.cuda.synchronize()
    kp[0, 1, 0, :len(LOOK)], vp[0, 1, 0, :len(LOOK)] = k[look, 0], v[look, 0]
    assert torch.equal(cache.kp, kp) and torch.equal(cache.vp, vp)

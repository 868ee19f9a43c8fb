"""Limits of every size in both kernels of paged attention: none, the type's lowest and largest values, one key, all, in any order."""
import numpy as np
import pytest

from test_gpu_paged_attn import cas  # noqa: F401

pytestmark = pytest.mark.gpu

LOWEST, LARGEST = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("dtype,H,Hkv,d,new", [("bf16", 8, 2, 128, [1, 1, 1]), ("f32", 4, 2, 64, [1, 1, 1]), ("bf16", 8, 2, 64, [40, 1, 3]),
                                               ("f32", 4, 2, 16, [40, 1, 3]), ("bf16", 8, 2, 128, [100, 90, 1]),
                                               ("bf16", 8, 2, 64, [130, 80, 77])])
@pytest.mark.parametrize("shards", [1, 3])
def test_limits_of_every_size(cas, dtype, H, Hkv, d, new, shards):  # noqa: F811
    import torch
    from paged_reference import DT, Cache, attention, check_attention, dealt, i32, starts
    lens = dealt([300, 200, 77], shards)
    cache = Cache(cas, dtype, Hkv, d, 16, lens, seed=31)
    rng, rows = np.random.default_rng(32), sum(new)
    limits = rng.choice([LOWEST, LOWEST + 1, -1, 0, 1, 31, 33, 64, 65, 100, LARGEST - 1, LARGEST], (rows, shards))
    limits[:3] = LOWEST                                    # rows that see nothing; with one row each, all of a sequence
    visible, q_start = i32(limits), starts(new)
    q = torch.randn((rows, H, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(33)).to(DT[dtype])
    o, lse = torch.full_like(q, 7.0), torch.full((H, rows), 7.0, device="cuda")
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, rows, H))
    ws.fill_(0xff)
    cas.cascade_paged_attn(cache.handle, 0, q, o, i32(q_start), d ** -0.5, visible=visible, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    assert bool((o[:3] == 0).all())
    check_attention(cache, o, lse, attention(cache, 0, q, q_start, visible, d ** -0.5), 300)

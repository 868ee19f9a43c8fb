"""Weights of paged attention of few rows over a bf16 cache: 16 bits of them enter the product with the values."""
import math

import pytest

from test_gpu_paged_attn import cas  # noqa: F401

pytestmark = pytest.mark.gpu


def attend(cas, H, Hkv, d, context, new, seed, change=None, shards=1):  # noqa: F811
    import numpy as np
    import torch
    from paged_reference import Cache, attention, causal, dealt, i32, starts
    cache = Cache(cas, "bf16", Hkv, d, 16, dealt(np.add(context, new), shards), seed=seed)
    if change:
        change(cache)
    q_start, rows = starts(new), sum(new)
    q = torch.randn((rows, H, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed + 1)).bfloat16()
    visible, o = i32(causal(context, new, shards)), torch.full((rows, H, d), 7.0, device="cuda")
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, rows, H))
    cas.cascade_paged_attn(cache.handle, 0, q, o, i32(q_start), d ** -0.5, visible=visible, workspace=ws)
    torch.cuda.synchronize()
    return o, attention(cache, 0, q, q_start, visible, d ** -0.5)


@pytest.mark.parametrize("H,Hkv,d", [(8, 2, 128), (8, 2, 64), (4, 4, 96), (4, 2, 256)])
@pytest.mark.parametrize("context,new,shards", [([1, 2, 3, 7, 15, 40], [1] * 6, 1), ([300, 5], [1, 20], 2), ([3000], [1], 1), ([33, 2], [33, 5], 1)])
def test_weights_keep_16_bits(cas, H, Hkv, d, context, new, shards):  # noqa: F811
    """A weight is cut to its upper 8 bits, off by 2^-7 at most, and the rest rounded to 8 bits, off by 2^-8 of that; the 2^-18 that
    is added to every weight comes on top.  o is in fp32, so no rounding of it covers them.  The other terms as in
    paged_reference.check_attention."""
    o, (ro, _, av, mag) = attend(cas, H, Hkv, d, context, new, d)
    keys, eps = max(c + n for c, n in zip(context, new)), 2.0 ** -24
    weight = 2 * (d + 3) * eps * mag + (2 * keys + 64) * eps + 2.0 ** -15 + 2.0 ** -18
    err, bound = (o.double() - ro).abs(), av * weight[..., None] * 1.01 + ro.abs() * eps * 1.01 + 1e-30
    assert bool((err <= bound).all()), float((err / bound).max())


@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("new", [1, 16])
def test_infinite_values_that_every_row_sees(cas, bad, new):  # noqa: F811
    """Neither half of a weight is zero or of the other sign: infinity, never a NaN; also where the weight is exactly one."""
    def change(cache):
        for at in (0, 1, 9, 40):
            cache.vp[0, cache.table[0, 0, at // 16].item(), 0, at % 16, at] = bad
        cache.vp[0, cache.table[1, 0, 0].item(), 1, 0, 7] = bad        # of one key: weight 1
    import torch
    o, _ = attend(cas, 4, 2, 64, [96, 0], [new, 1], 5, change)
    for at in (0, 1, 9, 40):
        assert bool((o[:new, :2, at] == bad).all())
    assert bool((o[new, 2:, 7] == bad).all())
    assert int(torch.isfinite(o).logical_not().sum()) == new * 2 * 4 + 2

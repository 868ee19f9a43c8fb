"""A descriptor of some neighbouring sequences of a paged cache: the same pages, lists and references."""
import numpy as np
import pytest

from test_gpu_pages import Pool, cas  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shards", [1, 3])
def test_calls_on_some_sequences(cas, shards):  # noqa: F811
    """Extension, fork and freeing through part of the lists leave what the whole cache's calls leave."""
    import torch
    from paged_reference import i32
    rng = np.random.default_rng(shards)
    pool = Pool(cas, 9, shards, 16, 60 * shards, 9)
    pool.extend([40] * 9, rng.integers(0, shards, 360))
    a, b = 3, 6
    some = cas.make_paged_cache(pool.kp, pool.vp, pool.table[a:b], pool.lens[a:b], pool.refs)
    cas.cascade_pages_free(some, i32([1]))
    pool.sim.free([a + 1])
    pool.same()
    accepted = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    cas.cascade_pages_fork(some, i32([2]), i32([1]), accepted, pool.ws)
    want, _ = pool.sim.fork([a + 2], [a + 1])
    assert accepted.item() == want[0] == 1
    pool.same()
    new, shard = [5, 50, 1], rng.integers(0, shards, 56)
    slots, visible, accepted = (torch.full(n, 77, dtype=torch.int32, device="cuda") for n in ((56,), (56, shards), (3,)))
    cas.cascade_paged_extend(some, i32(np.concatenate([[0], np.cumsum(new)])), slots, visible, accepted, row_shard=i32(shard))
    all_new = [0] * a + new + [0] * (9 - b)
    want = pool.sim.extend(np.concatenate([[0], np.cumsum(all_new)]), shard, 56)
    for t, n in zip((slots, visible, accepted), (want[0], want[1], want[2][a:b])):
        assert np.array_equal(t.cpu().numpy(), n)
    pool.same()


def test_attention_over_one_of_many_sequences(cas):  # noqa: F811
    """A chunk of fewer rows than the cache has sequences, through the whole cache and through its own sequence alone, which takes
    the tiles."""
    import torch
    from launched import kernels_of
    from paged_reference import Cache, attention, causal, check_attention, i32
    lens = np.zeros((400, 1), int)
    lens[[7, 200, 399], 0] = 90, 350, 33
    cache = Cache(cas, "bf16", 2, 128, 16, lens, seed=61)
    rows, H = 150, 8
    q, visible = torch.randn((rows, H, 128), device="cuda").bfloat16(), i32(causal([200], [rows], 1))
    some = cas.make_paged_cache(cache.kp, cache.vp, cache.table[200:201], cache.lens[200:201], cache.refs)
    ref = attention(cache, 0, q, [0] * 201 + [rows] * 200, visible, 0.09)
    for handle, q_start, kernel in ((cache.handle, i32([0] * 201 + [rows] * 200), "paged_"), (some, i32([0, rows]), "paged_tile")):
        o, lse = torch.full_like(q, 7.0), torch.full((H, rows), 7.0, device="cuda")
        ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(handle, rows, H))
        names = kernels_of(lambda: cas.cascade_paged_attn(handle, 0, q, o, q_start, 0.09, visible=visible, lse=lse, workspace=ws))
        assert any(kernel in n for n in names)
        torch.cuda.synchronize()
        check_attention(cache, o, lse, ref, 350)

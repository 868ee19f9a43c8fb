"""Paged attention in tiles (more than 256 rows times heads of a sequence; bf16, heads of 64 and 128) where it could go wrong: every
call is checked to have run that kernel."""
import math

import numpy as np
import pytest

from test_gpu_paged_attn import cas  # noqa: F401

pytestmark = pytest.mark.gpu


def call(cas, cache, q, o, q_start, visible, lse, layer=0):  # noqa: F811
    import torch
    from launched import kernels_of
    from paged_reference import i32
    rows, H, d = q.shape
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, rows, H))
    ws.fill_(0xff)
    starts_dev = i32(q_start)
    names = kernels_of(lambda: cas.cascade_paged_attn(cache.handle, layer, q, o, starts_dev, d ** -0.5, visible=visible, lse=lse, workspace=ws))
    assert any("paged_tile" in n for n in names), names
    torch.cuda.synchronize()


def attend(cas, cache, q, o, q_start, visible, lse, layer=0):  # noqa: F811
    from paged_reference import attention
    call(cas, cache, q, o, q_start, visible, lse, layer)
    return attention(cache, layer, q, q_start, visible, q.shape[2] ** -0.5)


def queries(rows, H, d, seed):
    import torch
    return torch.randn((rows, H, d), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).bfloat16()


def part(ref, rows):
    return ref[0][rows], ref[1][:, rows], ref[2][rows], ref[3][rows]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv,rows", [(4, 2, 140), (8, 2, 100), (2, 2, 300), (16, 1, 20)])
@pytest.mark.parametrize("shards", [1, 2, 9])
def test_limits_of_every_size(cas, d, H, Hkv, rows, shards):  # noqa: F811
    """Rows that see nothing, limits in no order, below zero and behind the end; a sequence without keys."""
    import torch
    from paged_reference import Cache, check_attention, dealt, i32
    cache = Cache(cas, "bf16", Hkv, d, 16, dealt([123, 0, 400], shards), seed=41)
    rng = np.random.default_rng(42)
    limits = rng.integers(-3, 410 // shards, (3 * rows, shards))
    limits[::5] = 0
    limits[1::7] = rng.choice([-2 ** 31, -1, 0, 1, 63, 64, 65, 2 ** 31 - 1], (len(limits[1::7]), shards))
    limits[2 * rows:2 * rows + 64] = 0                     # whole wavefronts, and with 16 heads a whole tile and more
    q, o, lse = queries(3 * rows, H, d, 43), torch.full((3 * rows, H, d), 7.0, device="cuda").bfloat16(), torch.full((H, 3 * rows), 7.0, device="cuda")
    ref = attend(cas, cache, q, o, np.arange(4) * rows, i32(limits), lse)
    check_attention(cache, o, lse, ref, 400)


@pytest.mark.parametrize("mask", [True, False])
def test_rows_that_all_see_nothing(cas, mask):  # noqa: F811
    import torch
    from paged_reference import Cache, i32
    cache = Cache(cas, "bf16", 2, 128, 16, [[50 if mask else 0]], seed=44)
    q, o, lse = queries(200, 8, 128, 45), torch.full((200, 8, 128), 7.0, device="cuda").bfloat16(), torch.full((8, 200), 7.0, device="cuda")
    call(cas, cache, q, o, [0, 200], i32(np.zeros((200, 1))) if mask else None, lse)
    assert bool((o == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("masked", [True, False])
def test_entries_that_are_no_pages_hold_no_keys(cas, d, masked):  # noqa: F811
    """Pages of 16 and of 32 rows: a block of 16 keys of a tile, and half a tile; the first, one in the middle, the last."""
    import torch
    from paged_reference import Cache, check_attention, i32
    for page in (16, 32):
        lens = np.array([[20 * page], [7 * page]])
        cache = Cache(cas, "bf16", 2, d, page, lens, seed=46)
        whole, n_pages = cache.table.clone(), cache.kp.shape[1]
        gone = {0: {5: -1, 6: n_pages, 19: 2 ** 31 - 1}, 1: {0: -2 ** 31}}
        for b, entries in gone.items():
            for j, value in entries.items():
                cache.table[b, 0, j] = value
        rows = 100
        q, o, lse = queries(2 * rows, 8, d, 47), torch.full((2 * rows, 8, d), 7.0, device="cuda").bfloat16(), torch.full((8, 2 * rows), 7.0, device="cuda")
        # limits that grow through the lists: row i of a sequence sees the first (i + 1) / rows of its keys
        seen = np.concatenate([np.arange(1, rows + 1) * int(n) // rows for n in lens[:, 0]])
        call(cas, cache, q, o, [0, rows, 2 * rows], i32(seen[:, None]) if masked else None, lse)
        # the same without those pages: the ones behind them move up, and so do the limits
        rest = Cache(cas, "bf16", 2, d, page, [[17 * page], [6 * page]], seed=0)
        rest.kp, rest.vp, rest.table = cache.kp, cache.vp, torch.full_like(whole, -1)
        fewer = seen.copy()
        for b, entries in gone.items():
            kept = [j for j in range(int(lens[b, 0]) // page) if j not in entries]
            rest.table[b, 0, :len(kept)] = whole[b, 0, kept]
            for i in range(b * rows, (b + 1) * rows):
                fewer[i] -= sum(min(max(seen[i] - j * page, 0), page) for j in entries)
        from paged_reference import attention
        ref = attention(rest, 0, q, [0, rows, 2 * rows], i32(fewer[:, None]) if masked else None, d ** -0.5)
        check_attention(rest, o, lse, ref, int(lens.max()))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_keys_and_values_that_a_row_does_not_see(cas, d, bad):  # noqa: F811
    """One key in the middle and one value behind it are not finite: rows in front of them must not feel them."""
    import torch
    from paged_reference import Cache, causal, check_attention, i32, starts
    new, context, H, Hkv = 150, 90, 8, 2
    cache = Cache(cas, "bf16", Hkv, d, 16, [[context + new]], seed=48)
    at = lambda pool, token, head, col: (0, cache.table[0, 0, token // 16].item(), head, token % 16, col)  # noqa: E731
    key, value = context + 100, context + 40               # the key hits kv head 0 from row 100 on, the value kv head 1 from row 40 on
    cache.kp[at(cache.kp, key, 0, 3)] = math.nan
    cache.vp[at(cache.vp, value, 1, 5)] = bad
    q, o, lse = queries(new, H, d, 49), torch.full((new, H, d), 7.0, device="cuda").bfloat16(), torch.full((H, new), 7.0, device="cuda")
    visible = i32(causal([context], [new], 1))
    call(cas, cache, q, o, starts([new]), visible, lse)
    hit = o[40:, 4:, 5]
    assert bool((torch.isnan(hit) if math.isnan(bad) else hit == bad).all())
    assert bool(torch.isnan(o[100:, :4]).all()) and bool(torch.isnan(lse[:4, 100:]).all())
    # everywhere else as if both were zero
    from paged_reference import attention
    cache.kp[at(cache.kp, key, 0, 3)], cache.vp[at(cache.vp, value, 1, 5)] = 0.0, 0.0
    ref = attention(cache, 0, q, starts([new]), visible, d ** -0.5)
    check_attention(cache, o[:40], lse[:, :40], part(ref, slice(0, 40)), context + new)
    o[40:, 4:, 5] = ref[0][40:, 4:, 5].bfloat16()
    check_attention(cache, o[:100], lse[:, :100], part(ref, slice(0, 100)), context + new)
    upper = [t[:, 4:] if t.shape[1] == H else t[4:] for t in ref]
    check_attention(cache, o[:, 4:], lse[4:], upper, context + new)


@pytest.mark.parametrize("d", [64, 128])
def test_output_in_fp32_in_a_later_layer(cas, d):  # noqa: F811
    """Whole walks, written by the kernel itself, and cut ones, written by the merge."""
    import torch
    from paged_reference import Cache, causal, check_attention, i32, starts
    for new, context in (([70], [0]), ([70, 3, 200], [3000, 10, 77])):
        cache = Cache(cas, "bf16", 2, d, 32, np.add(new, context)[:, None], layers=3, seed=50)
        rows = sum(new)
        q, o, lse = queries(rows, 8, d, 51), torch.full((rows, 8, d), 7.0, device="cuda"), torch.full((8, rows), 7.0, device="cuda")
        ref = attend(cas, cache, q, o, starts(new), i32(causal(context, new, 1)), lse, layer=2)
        check_attention(cache, o, lse, ref, 3070)


@pytest.mark.parametrize("o_f32", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_strided_rows_and_rows_of_no_sequence(cas, d, o_f32):  # noqa: F811
    import torch
    from paged_reference import Cache, causal, check_attention, i32
    cache = Cache(cas, "bf16", 2, d, 32, [[190], [240]], seed=52)
    rows, H = 200, 4
    q_start = [2, 3, 195]                                  # rows 0, 1 and 195 .. 199 belong to nobody
    q = queries(rows, H + 4, d, 53)[:, 2:2 + H]
    wide = torch.full((rows, H + 2, d), 7.0, device="cuda", dtype=torch.float32 if o_f32 else torch.bfloat16)
    o, lse = wide[:, 1:1 + H], torch.full((H, rows), 7.0, device="cuda")
    visible = torch.zeros((rows, 1), dtype=torch.int32, device="cuda")
    visible[2:195] = i32(causal([189, 48], [1, 192], 1))
    ref = attend(cas, cache, q, o, q_start, visible, lse)
    inside = slice(2, 195)
    check_attention(cache, o[inside], lse[:, inside], part(ref, inside), 240)
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, H + 1] == 7).all()) and bool((wide[:2] == 7).all()) and bool((wide[195:] == 7).all())
    assert bool((lse[:, :2] == 7).all()) and bool((lse[:, 195:] == 7).all())


def test_many_heads_of_few_rows(cas):  # noqa: F811
    """One token whose heads fill more than a tile: its walk has one limit for all of them."""
    import torch
    from paged_reference import Cache, check_attention, i32
    cache = Cache(cas, "bf16", 1, 64, 16, [[700]], seed=54)
    q, o, lse = queries(1, 300, 64, 55), torch.full((1, 300, 64), 7.0, device="cuda").bfloat16(), torch.full((300, 1), 7.0, device="cuda")
    ref = attend(cas, cache, q, o, [0, 1], i32([[444]]), lse)
    check_attention(cache, o, lse, ref, 700)

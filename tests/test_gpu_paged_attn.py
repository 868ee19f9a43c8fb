"""Attention of new rows over a paged cache against 64-bit attention: numbers of rows, head layouts, lengths, shards and pages;
masks; values that are not finite; strides; graphs and streams."""
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


def run(cas, dtype, H, Hkv, d, page, context, new, shards=1, mask="causal", seed=0, amp=1.0, o_f32=False, layers=1, layer=0, **kw):
    import torch
    from paged_reference import DT, Cache, attention, causal, check_attention, dealt, i32, starts
    lens = dealt(np.add(context, new), shards)
    cache = Cache(cas, dtype, Hkv, d, page, lens, layers=layers, seed=seed, amp=amp, **kw)
    q_start, rows = starts(new), int(sum(new))
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    q = (amp * torch.randn((rows, H, d), device="cuda", generator=gen)).to(DT[dtype])
    visible = i32(causal(context, new, shards)) if mask == "causal" else None
    o = torch.full((rows, H, d), 7.0, device="cuda", dtype=torch.float32 if o_f32 else DT[dtype])
    lse = torch.full((H, rows), 7.0, device="cuda")
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, rows, H))
    ws.fill_(0xff)                                          # NaN wherever something is read before it is written
    cas.cascade_paged_attn(cache.handle, layer, q, o, i32(q_start), d ** -0.5, visible=visible, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    ref = attention(cache, layer, q, q_start, visible, d ** -0.5)
    check_attention(cache, o, lse, ref, int(lens.sum(1).max()))
    return cache, q, o, lse


HEADS = [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("bf16", 12, 4, 64), ("bf16", 16, 1, 128), ("bf16", 5, 1, 128), ("f32", 4, 2, 64),
         ("f32", 3, 3, 16)]


@pytest.mark.parametrize("dtype,H,Hkv,d", HEADS)
@pytest.mark.parametrize("page", [16, 64])
def test_one_token_each(cas, dtype, H, Hkv, d, page):
    run(cas, dtype, H, Hkv, d, page, [0, 1, 15, 16, 31, 32, 63, 200, 1000], [1] * 9, seed=d)


@pytest.mark.parametrize("dtype,H,Hkv,d", HEADS)
def test_chunks_and_tokens_in_one_batch(cas, dtype, H, Hkv, d):
    run(cas, dtype, H, Hkv, d, 32, [100, 0, 333, 64, 0, 7], [1, 130, 4, 64, 0, 33], seed=d + 1)


@pytest.mark.parametrize("dtype,d", [("bf16", 8), ("bf16", 32), ("bf16", 72), ("bf16", 96), ("bf16", 192), ("bf16", 256), ("f32", 4),
                                     ("f32", 36), ("f32", 100), ("f32", 128), ("f32", 132), ("f32", 256)])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 3]])
def test_head_dimensions(cas, dtype, d, new):
    run(cas, dtype, 4, 2, d, 16, [77, 300, 0], new, seed=d)


@pytest.mark.parametrize("dtype,shards", [("bf16", 2), ("bf16", 7), ("bf16", 100), ("f32", 3)])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [150, 1, 9, 0]])
def test_shards(cas, dtype, shards, new):
    run(cas, dtype, 8, 2, 64, 16, [500, 3, 129, 40], new, shards=shards, seed=shards)


def test_more_sequences_than_a_wavefront(cas):
    rng = np.random.default_rng(0)
    run(cas, "bf16", 4, 2, 64, 16, rng.integers(0, 150, 150), rng.integers(0, 3, 150), shards=2, seed=3)


def test_a_long_walk_is_cut(cas):
    run(cas, "bf16", 8, 2, 128, 64, [20000, 5], [1, 1], seed=4)
    run(cas, "bf16", 8, 2, 128, 128, [9000], [70], seed=5)
    run(cas, "f32", 2, 1, 64, 32, [7001], [5], seed=6)


def test_large_scores(cas):
    run(cas, "bf16", 8, 2, 128, 32, [700, 90], [1, 100], amp=5.0, seed=7)
    run(cas, "f32", 4, 2, 64, 32, [700, 90], [1, 100], amp=5.0, seed=8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_a_mask(cas, dtype):
    """A bidirectional chunk, and rows over cached states of another length (cross attention)."""
    run(cas, dtype, 8, 4, 64, 16, [37, 1, 0, 300], [50, 200, 77, 1], mask=None, seed=9)


def test_output_in_fp32_and_a_later_layer(cas):
    run(cas, "bf16", 8, 2, 128, 32, [100, 0], [3, 60], o_f32=True, layers=3, layer=2, seed=10)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 70])
def test_rows_that_see_nothing_or_little(cas, dtype, rows):
    import torch
    from paged_reference import DT, Cache, attention, check_attention, i32
    cache = Cache(cas, dtype, 2, 64, 16, [[50, 0], [0, 0], [33, 90]], seed=11)
    rng = np.random.default_rng(12)
    q_start = np.arange(4) * rows
    q = torch.randn((3 * rows, 4, 64), device="cuda").to(DT[dtype])
    # limits in any order; some are zero, some below it, some behind the end
    limits = rng.integers(-3, 60, (3 * rows, 2))
    limits[::5] = 0
    visible = i32(limits)
    o, lse = torch.full_like(q, 7.0), torch.full((4, 3 * rows), 7.0, device="cuda")
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, 3 * rows, 4))
    cas.cascade_paged_attn(cache.handle, 0, q, o, i32(q_start), 0.125, visible=visible, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    check_attention(cache, o, lse, attention(cache, 0, q, q_start, visible, 0.125), 200)


@pytest.mark.parametrize("dtype,H,Hkv,d", [("bf16", 4, 2, 128), ("bf16", 4, 2, 96), ("f32", 4, 2, 64)])
@pytest.mark.parametrize("new", [3, 100])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_unseen_values_that_are_not_finite(cas, dtype, H, Hkv, d, new, bad):
    """Later tokens of the chunk hold NaN or infinities: rows before them must not feel them, rows from there on must."""
    import torch
    from paged_reference import DT, Cache, attention, causal, check_attention, i32, starts
    context, at = 41, 41 + new // 2                        # token `at` is not finite, in one column of one head
    cache = Cache(cas, dtype, Hkv, d, 16, [[context + new]], seed=13)
    page = cache.table[0, 0, at // 16].item()
    cache.vp[0, page, 1, at % 16, 5] = bad
    cache.kp[0, cache.table[0, 0, (context + new - 1) // 16].item(), 0, (context + new - 1) % 16, 3] = math.nan
    q = torch.randn((new, H, d), device="cuda").to(DT[dtype])
    visible = i32(causal([context], [new], 1))
    o = torch.full_like(q, 7.0)
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, new, H))
    cas.cascade_paged_attn(cache.handle, 0, q, o, i32(starts([new])), d ** -0.5, visible=visible, workspace=ws)
    torch.cuda.synchronize()
    ro, _, av, mag = attention(cache, 0, q, starts([new]), visible, d ** -0.5)
    before = new // 2
    rep = H // Hkv
    # rows that do not see it: as if it were zero there
    clean = cache.vp.clone()
    clean[0, page, 1, at % 16, 5] = 0.0
    dirty, cache.vp = cache.vp, clean
    ref = attention(cache, 0, q, starts([new]), visible, d ** -0.5)
    cache.vp = dirty
    sub = lambda t: t[:before]  # noqa: E731
    check_attention(cache, sub(o), None, (sub(ref[0]), ref[1][:, :before], sub(ref[2]), sub(ref[3])), context + new)
    hit = o[before:, rep:, 5]
    assert bool((torch.isnan(hit) if math.isnan(bad) else hit == bad).all())
    other = torch.ones(d, dtype=torch.bool)
    other[5] = False
    assert bool(torch.isfinite(o[:new - 1][:, :, other.cuda()]).all())
    assert bool(torch.isnan(o[new - 1, :rep]).all())       # the last token's key is NaN, and only its own row sees it


def test_entries_that_are_no_pages_hold_no_keys(cas):
    import torch
    from paged_reference import Cache, attention, check_attention, i32
    for dtype, rows in (("bf16", 1), ("bf16", 80), ("f32", 2)):
        cache = Cache(cas, dtype, 2, 64, 16, [[100], [64]], seed=14)
        whole = cache.table.clone()
        cache.table[0, 0, 2], cache.table[1, 0, 0] = -1, cache.kp.shape[1]
        q = torch.randn((2 * rows, 4, 64), device="cuda").to(cache.kp.dtype)
        o, q_start = torch.full_like(q, 7.0), [0, rows, 2 * rows]
        ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, 2 * rows, 4))
        cas.cascade_paged_attn(cache.handle, 0, q, o, i32(q_start), 0.125, workspace=ws)
        torch.cuda.synchronize()
        # the same without those 16 keys: the pages behind them move up by one
        rest = Cache(cas, dtype, 2, 64, 16, [[84], [48]], seed=0)
        rest.kp, rest.vp = cache.kp, cache.vp
        rest.table = torch.full_like(whole, -1)
        rest.table[0, 0, :6] = whole[0, 0, [0, 1, 3, 4, 5, 6]]
        rest.table[1, 0, :3] = whole[1, 0, 1:4]
        check_attention(rest, o, None, attention(rest, 0, q, q_start, None, 0.125), 100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows_and_rows_of_no_sequence(cas, dtype):
    import torch
    from paged_reference import DT, Cache, attention, causal, check_attention, i32
    cache = Cache(cas, dtype, 2, 64, 32, [[90], [140]], seed=15)
    rows, H = 60, 4
    q_start = [2, 3, 55]                                   # rows 0, 1 and 55 .. 59 belong to nobody
    fused = torch.randn((rows, H + 4, 64), device="cuda").to(DT[dtype])
    q = fused[:, :H]
    wide = torch.full((rows, H + 1, 64), 7.0, device="cuda", dtype=DT[dtype])
    o, lse = wide[:, :H], torch.full((H, rows), 7.0, device="cuda")
    visible = torch.zeros((rows, 1), dtype=torch.int32, device="cuda")
    visible[2:55] = i32(causal([89, 88], [1, 52], 1))
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, rows, H))
    cas.cascade_paged_attn(cache.handle, 0, q, o, i32(q_start), 0.125, visible=visible, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    ref = attention(cache, 0, q, q_start, visible, 0.125)
    inside = slice(2, 55)
    check_attention(cache, o[inside], lse[:, inside], (ref[0][inside], ref[1][:, inside], ref[2][inside], ref[3][inside]), 140)
    assert bool((wide[:, H] == 7).all()) and bool((wide[:2] == 7).all()) and bool((wide[55:] == 7).all())
    assert bool((lse[:, :2] == 7).all()) and bool((lse[:, 55:] == 7).all())


def test_the_same_call_gives_the_same_bits(cas):
    import torch
    from paged_reference import Cache, causal, i32, starts
    context, new = [5000, 100, 0], [1, 200, 9]
    cache = Cache(cas, "bf16", 2, 128, 64, np.add(context, new)[:, None], seed=16)
    q = torch.randn((210, 8, 128), device="cuda").bfloat16()
    visible, q_start = i32(causal(context, new, 1)), i32(starts(new))
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, 210, 8))
    outs = []
    for _ in range(3):
        o, lse = torch.empty_like(q), torch.empty((8, 210), device="cuda")
        cas.cascade_paged_attn(cache.handle, 0, q, o, q_start, 0.1, visible=visible, lse=lse, workspace=ws)
        outs.append((o, lse))
    torch.cuda.synchronize()
    assert all(torch.equal(o, outs[0][0]) and torch.equal(lse, outs[0][1]) for o, lse in outs)


def test_a_captured_call_follows_lengths_and_limits(cas):
    """A graph is captured once and replayed while the sequences grow: lengths, limits and queries are read at replay."""
    import torch
    from paged_reference import Cache, attention, check_attention, i32
    cache = Cache(cas, "bf16", 2, 128, 16, [[1000], [500], [40]], seed=17)
    q, q_start = torch.randn((3, 8, 128), device="cuda").bfloat16(), i32([0, 1, 2, 3])
    visible, o, lse = i32([[100], [1], [5]]), torch.empty((3, 8, 128), device="cuda").bfloat16(), torch.empty((8, 3), device="cuda")
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, 3, 8))

    def call():
        cas.cascade_paged_attn(cache.handle, 0, q, o, q_start, 0.1, visible=visible, lse=lse, workspace=ws)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for limits, lens in (([999, 500, 7], [1000, 500, 40]), ([30, 2, 40], [31, 2, 40]), ([0, 400, 40], [1000, 450, 39])):
        visible.copy_(i32(limits)[:, None])
        cache.lens.copy_(i32(lens)[:, None])
        q.copy_(torch.randn((3, 8, 128), device="cuda"))
        o.fill_(7.0)
        ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(cache, o, lse, attention(cache, 0, q, [0, 1, 2, 3], visible, 0.1), 1000)


def test_two_streams_with_a_workspace_each(cas):
    import torch
    from paged_reference import Cache, attention, check_attention, i32
    jobs = []
    for i in range(2):
        cache = Cache(cas, "bf16", 2, 64, 16, [[3000 + 500 * i]], seed=18 + i)
        q = torch.randn((1, 8, 64), device="cuda").bfloat16()
        ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, 1, 8))
        jobs.append((cache, q, torch.empty_like(q), ws, torch.cuda.Stream(), i32([0, 1])))
    torch.cuda.synchronize()
    for _ in range(5):
        for cache, q, o, ws, stream, q_start in jobs:
            cas.cascade_paged_attn(cache.handle, 0, q, o, q_start, 0.125, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for cache, q, o, *_ in jobs:
        check_attention(cache, o, None, attention(cache, 0, q, [0, 1], None, 0.125), 3500)


def test_partials_of_several_parties_merge(cas):
    """Each party holds some shards and returns o in fp32 with lse; cascade_lse_merge combines them."""
    import torch
    from paged_reference import Cache, attention, check_attention, i32
    rows, H, d = 5, 4, 64
    lens = [[60, 0, 200]]
    whole = Cache(cas, "bf16", 2, d, 16, lens, seed=20)
    q = torch.randn((rows, H, d), device="cuda").bfloat16()
    limits = i32([[0, 0, 0], [0, 0, 9], [1, 0, 0], [60, 0, 199], [33, 0, 70]])
    m, u = torch.empty((1, H, 3, rows), device="cuda"), torch.empty((1, 3, H, rows, d), device="cuda")
    for s in range(3):
        table, own = whole.table[:, s:s + 1].contiguous(), whole.lens[:, s:s + 1].contiguous()
        party = cas.make_paged_cache(whole.kp, whole.vp, table, own, whole.refs)
        o, lse = torch.empty((rows, H, d), device="cuda"), torch.empty((H, rows), device="cuda")
        ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(party, rows, H))
        cas.cascade_paged_attn(party, 0, q, o, i32([0, rows]), 0.125, visible=limits[:, s:s + 1].contiguous(), lse=lse, workspace=ws)
        m[0, :, s], u[0, s] = lse, o.transpose(0, 1)
    plan = cas.cascade_plan_create(1, rows, 3, np.zeros(rows, np.int32))
    out, total = torch.empty((1, rows, H * d), device="cuda").bfloat16(), torch.empty((1, H, rows), device="cuda")
    cas.cascade_lse_merge(plan, m, torch.ones_like(m), u, out, H, 2, d, u_mode=cas.U_NORMALISED, lse_out=total)
    torch.cuda.synchronize()
    # (two more roundings of fp32 than a single call, far inside the allowance for the sums)
    ref = attention(whole, 0, q, [0, rows], limits, 0.125)
    live = slice(1, rows)
    check_attention(whole, out.view(rows, H, d)[live], None, (ref[0][live], ref[1][:, live], ref[2][live], ref[3][live]), 260)


def test_which_kernel_takes_which_rows(cas):
    """Sequences of more than 256 flattened rows go to the tiles, the others to the kernel for few rows; fp32 and other head
    dimensions always; no more rows than sequences: the kernel for few rows alone."""
    import torch
    from launched import kernels_of
    from paged_reference import DT, Cache, i32, starts

    def names(dtype, d, new, H=8, Hkv=2):
        cache = Cache(cas, dtype, Hkv, d, 16, np.add(new, 40)[:, None], seed=1)
        q = torch.randn((sum(new), H, d), device="cuda").to(DT[dtype])
        o, q_start = torch.empty_like(q), i32(starts(new))
        ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, sum(new), H))
        got = kernels_of(lambda: cas.cascade_paged_attn(cache.handle, 0, q, o, q_start, 0.1, workspace=ws))
        return ["tile" if "paged_tile" in n else "rows" if "paged_rows" in n else "merge" for n in got]
    assert names("bf16", 128, [100]) == ["tile", "merge"]
    assert names("bf16", 64, [100, 1]) == ["tile", "rows", "merge"]
    assert names("bf16", 128, [64]) == ["rows", "merge"]
    assert names("bf16", 96, [300]) == ["rows", "merge"] and names("f32", 64, [300]) == ["rows", "merge"]
    assert names("bf16", 128, [1] * 100) == ["rows", "merge"]


@pytest.mark.parametrize("new,rows", [([70], 200), ([64, 0, 0], 64), ([0] * 40 + [41], 41), ([0, 0, 0, 90], 90)])
def test_batches_that_guess_the_kernel_wrong(cas, new, rows):
    """Rows that make tiles possible where there are few, and as many sequences as rows where one has them all."""
    import torch
    from paged_reference import Cache, attention, causal, check_attention, i32, starts
    context = [30 + i for i in range(len(new))]
    if len(new) == 3:
        new, context = new + [0] * 61, context + [5] * 61   # as many sequences as rows
    cache = Cache(cas, "bf16", 2, 64, 16, np.add(new, context)[:, None], seed=21)
    q = torch.randn((rows, 8, 64), device="cuda").bfloat16()
    visible = torch.zeros((rows, 1), dtype=torch.int32, device="cuda")
    visible[:sum(new)] = i32(causal(context, new, 1))
    o, lse = torch.full_like(q, 7.0), torch.full((8, rows), 7.0, device="cuda")
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, rows, 8))
    ws.fill_(0xff)
    cas.cascade_paged_attn(cache.handle, 0, q, o, i32(starts(new)), 0.125, visible=visible, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    ref, n = attention(cache, 0, q, starts(new), visible, 0.125), sum(new)
    check_attention(cache, o[:n], lse[:, :n], (ref[0][:n], ref[1][:, :n], ref[2][:n], ref[3][:n]), 200)
    assert bool((o[n:] == 7).all()) and bool((lse[:, n:] == 7).all())


@pytest.mark.parametrize("shards,page", [(1, 16), (1, 256), (5, 32), (130, 16)])
@pytest.mark.parametrize("d", [64, 128])
def test_tiles(cas, shards, page, d):
    """Many rows: several tiles a sequence, ends inside pages and tiles, empty shards, pieces of a walk."""
    run(cas, "bf16", 8, 2, d, page, [0, 700, 63, 2000], [257, 64, 300, 90], shards=shards, seed=22)
    run(cas, "bf16", 6, 2, d, page, [1300], [129], shards=shards, mask=None, seed=23)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("at", [3, 200, 340])
def test_values_that_are_not_finite_in_tiles(cas, bad, at):
    """One value of a shard's row, early (every row of the tiles sees it), where the limit passes, and last of all."""
    import torch
    from paged_reference import Cache, attention, causal, check_attention, i32, starts
    new, context = [150], [200]
    cache = Cache(cas, "bf16", 2, 128, 16, [[175, 175]], seed=24)
    token = min(at, 349)
    s, r = token % 2, token // 2
    cache.vp[0, cache.table[0, s, r // 16].item(), 0, r % 16, 77] = bad
    q = torch.randn((150, 8, 128), device="cuda").bfloat16()
    visible = i32(causal(context, new, 2))
    o = torch.full_like(q, 7.0)
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(cache.handle, 150, 8))
    cas.cascade_paged_attn(cache.handle, 0, q, o, i32(starts(new)), 0.09, visible=visible, workspace=ws)
    torch.cuda.synchronize()
    sees = torch.arange(150, device="cuda") + 200 >= token
    hit = o[:, :4, 77]
    assert bool((torch.isnan(hit[sees]) if math.isnan(bad) else hit[sees] == bad).all())
    finite = torch.isfinite(o)
    finite[:, :4, 77] |= sees[:, None]
    assert bool(finite.all())
    cache.vp[0, cache.table[0, s, r // 16].item(), 0, r % 16, 77] = 0.0
    ref = attention(cache, 0, q, starts(new), visible, 0.09)
    o[:, :4, 77] = torch.where(sees[:, None], ref[0][:, :4, 77].bfloat16(), o[:, :4, 77])
    check_attention(cache, o, None, ref, 350)


def test_pools_beyond_32_bits_of_bytes(cas):
    """Pages whose bytes lie behind the first 4 GiB of a layer's pool, and whose elements lie behind 2^31."""
    import torch
    from paged_reference import Cache, attention, causal, check_attention, dealt, i32, starts
    page, Hkv, d, n_pages = 64, 8, 128, 34000              # 131072 bytes a page
    new, context = [1, 70], [500, 300]
    small = Cache(cas, "bf16", Hkv, d, page, dealt(np.add(context, new), 1), seed=25)
    used = small.kp.shape[1]
    kp, vp = (torch.empty((2, n_pages, Hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    far = n_pages - used - 1
    kp[1, far:far + used], vp[1, far:far + used] = small.kp[0], small.vp[0]
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[far:far + used] = small.refs
    big = cas.make_paged_cache(kp, vp, torch.where(small.table >= 0, small.table + far, -1).int(), small.lens, refs)
    q, visible = torch.randn((71, 32, d), device="cuda").bfloat16(), i32(causal(context, new, 1))
    o, lse = torch.empty_like(q), torch.empty((32, 71), device="cuda")
    ws = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(big, 71, 32))
    cas.cascade_paged_attn(big, 1, q, o, i32(starts(new)), d ** -0.5, visible=visible, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    check_attention(small, o, lse, attention(small, 0, q, starts(new), visible, d ** -0.5), 501)
    # rows written there, and a page copied from there
    slots = i32([(n_pages - 1) * page + 5, (n_pages - 1) * page + 6])
    k, v = torch.randn((2, Hkv, d), device="cuda").bfloat16(), torch.randn((2, Hkv, d), device="cuda").bfloat16()
    cas.cascade_paged_append(big, 1, slots, k, v)
    kp[0, 3] = 1.0
    cas.cascade_pages_copy(big, i32([n_pages - 1]), i32([3]))
    torch.cuda.synchronize()
    assert torch.equal(kp[1, n_pages - 1, :, 5:7].transpose(0, 1), k) and torch.equal(vp[1, 3, :, 5:7].transpose(0, 1), v)


def test_two_graphs_share_a_workspace_in_turn(cas):
    import torch
    from paged_reference import Cache, attention, causal, check_attention, i32, starts
    jobs = []
    ws = None
    for new, context in (([90, 1], [3000, 500]), ([1, 1, 1], [4000, 20, 900])):
        cache = Cache(cas, "bf16", 2, 128, 16, np.add(new, context)[:, None], seed=26)
        q, visible, q_start = torch.randn((sum(new), 8, 128), device="cuda").bfloat16(), i32(causal(context, new, 1)), i32(starts(new))
        jobs.append((cache, q, visible, q_start, torch.empty_like(q), torch.empty((8, sum(new)), device="cuda"), new))
    ws = cas.new_workspace(max(cas.cascade_paged_attn_workspace_bytes(c.handle, q.shape[0], 8) for c, q, *_ in jobs))
    graphs = []
    for cache, q, visible, q_start, o, lse, _ in jobs:
        def call():
            cas.cascade_paged_attn(cache.handle, 0, q, o, q_start, 0.09, visible=visible, lse=lse, workspace=ws)
        call()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    for _ in range(3):
        for graph, (cache, q, visible, q_start, o, lse, new) in zip(graphs, jobs):
            q.copy_(torch.randn(q.shape, device="cuda"))
            o.fill_(7.0)
            graph.replay()
        torch.cuda.synchronize()
        for cache, q, visible, q_start, o, lse, new in jobs:
            check_attention(cache, o, lse, attention(cache, 0, q, starts(new), visible, 0.09), 4001)

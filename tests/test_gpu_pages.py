"""Pages of a cache against a sequential simulation: taking, sharing, freeing, compacting and copying; refusals on the device;
graphs; and steps of a layer composed from all of it."""
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


class Simulation:
    """The rules, one page at a time."""

    def __init__(self, B, S, page, n_pages, max_pages):
        self.page, self.max_pages, self.S = page, max_pages, S
        self.table, self.lens, self.refs = np.full((B, S, max_pages), -1), np.zeros((B, S), int), np.zeros(n_pages, int)

    def _pages(self, n):
        return -(-n // self.page)

    def extend(self, q_start, shard, rows):
        S, B = self.S, len(self.lens)
        slots, visible, accepted = np.full(rows, -1), np.zeros((rows, S), int), np.ones(B, int)
        exhausted = False
        for b in range(B):
            mine = [int(s) for s in shard[q_start[b]:q_start[b + 1]]]
            after = self.lens[b] + np.array([mine.count(s) for s in range(S)])
            need = sum(self._pages(after[s]) - self._pages(self.lens[b, s]) for s in range(S))
            if (after > self.max_pages * self.page).any():
                accepted[b] = 0
                continue
            if need and (exhausted or need > (self.refs == 0).sum()):
                accepted[b], exhausted = 0, True
                continue
            for s in range(S):
                for j in range(self._pages(self.lens[b, s]), self._pages(after[s])):
                    self.table[b, s, j] = np.flatnonzero(self.refs == 0)[0]
                    self.refs[self.table[b, s, j]] = 1
            for i, s in enumerate(mine):
                t = q_start[b] + i
                if 0 <= s < S:
                    r = self.lens[b, s]
                    slots[t] = self.table[b, s, r // self.page] * self.page + r % self.page
                    self.lens[b, s] += 1
                visible[t] = self.lens[b]
        return slots, visible, accepted

    def free(self, seqs):
        for b in seqs:
            if 0 <= b < len(self.lens):
                for p in self.table[b][self.table[b] >= 0]:
                    self.refs[p] -= 1
                self.table[b], self.lens[b] = -1, 0

    def fork(self, src, dst):
        """accepted, and (old page, new page, rows) of the copies."""
        before, tables, accepted, copies, exhausted = self.lens.copy(), self.table.copy(), np.ones(len(src), int), [], False
        B = len(before)
        for i, (a, b) in enumerate(zip(src, dst)):
            if not (0 <= a < B and 0 <= b < B and a != b) or b in dst[:i] or before[b].any():
                accepted[i] = 0
                continue
            need = int((before[a] % self.page != 0).sum())
            if need and (exhausted or need > (self.refs == 0).sum()):
                accepted[i], exhausted = 0, True
                continue
            for s in range(self.S):
                full, part = divmod(before[a, s], self.page)
                self.table[b, s, :full] = tables[a, s, :full]
                for p in tables[a, s, :full]:
                    self.refs[p] += 1
                if part:
                    p = np.flatnonzero(self.refs == 0)[0]
                    self.refs[p] = 1
                    self.table[b, s, full] = p
                    copies.append((tables[a, s, full], p, part))
            self.lens[b] = before[a]
        return accepted, copies

    def compact(self):
        live = int((self.refs > 0).sum())
        moves = list(zip([p for p in range(live, len(self.refs)) if self.refs[p]], [p for p in range(live) if not self.refs[p]]))
        new = np.arange(len(self.refs))
        for a, b in moves:
            new[a], self.refs[b], self.refs[a] = b, self.refs[a], 0
        self.table = np.where(self.table >= 0, new[self.table], -1)
        return live, moves


class Pool:
    """A cache on the GPU next to its simulation; rows hold numbers that tell them apart."""

    def __init__(self, cas, B, S, page, n_pages, max_pages, Hkv=2, d=16, dtype="bf16", layers=2):
        import torch
        from paged_reference import DT, i32
        self.cas, self.sim = cas, Simulation(B, S, page, n_pages, max_pages)
        g = torch.Generator(device="cuda").manual_seed(1)
        self.kp, self.vp = (torch.randn((layers, n_pages, Hkv, page, d), device="cuda", generator=g).to(DT[dtype]) for _ in range(2))
        self.table, self.lens, self.refs = i32(self.sim.table), i32(self.sim.lens), i32(self.sim.refs)
        self.handle = cas.make_paged_cache(self.kp, self.vp, self.table, self.lens, self.refs)
        self.ws = cas.new_workspace(cas.cascade_pages_workspace_bytes(self.handle))
        self.ws.fill_(0xff)

    def same(self):
        for t, n in ((self.table, self.sim.table), (self.lens, self.sim.lens), (self.refs, self.sim.refs)):
            assert np.array_equal(t.cpu().numpy(), n)

    def extend(self, new, shard=None, pad=0):
        import torch
        from paged_reference import i32
        q_start, rows = np.concatenate([[0], np.cumsum(new)]), int(np.sum(new)) + pad
        if rows == 0:
            return None
        full = np.zeros(rows, int) if shard is None else np.concatenate([shard, np.zeros(pad, int)])
        slots, visible, accepted = (torch.full(n, 77, dtype=torch.int32, device="cuda") for n in ((rows,), (rows, self.sim.S), (len(new),)))
        self.cas.cascade_paged_extend(self.handle, i32(q_start), slots, visible, accepted, row_shard=None if shard is None else i32(full))
        want = self.sim.extend(q_start, full, rows)
        for t, n in zip((slots, visible, accepted), want):
            assert np.array_equal(t.cpu().numpy(), n)
        self.same()
        return slots, visible, accepted

    def free(self, seqs):
        from paged_reference import i32
        self.cas.cascade_pages_free(self.handle, i32(seqs))
        self.sim.free(seqs)
        self.same()

    def fork(self, src, dst):
        import torch
        from paged_reference import i32
        kp, vp, accepted = self.kp.clone(), self.vp.clone(), torch.full((len(src),), 77, dtype=torch.int32, device="cuda")
        self.cas.cascade_pages_fork(self.handle, i32(src), i32(dst), accepted, self.ws)
        want, copies = self.sim.fork(list(src), list(dst))
        assert np.array_equal(accepted.cpu().numpy(), want)
        self.same()
        for a, b, n in copies:
            kp[:, b, :, :n], vp[:, b, :, :n] = kp[:, a, :, :n], vp[:, a, :, :n]
        assert torch.equal(kp, self.kp) and torch.equal(vp, self.vp)

    def compact(self):
        import torch
        kp, vp, n_live = self.kp.clone(), self.vp.clone(), torch.full((1,), 77, dtype=torch.int32, device="cuda")
        self.cas.cascade_pages_compact(self.handle, n_live, self.ws)
        live, moves = self.sim.compact()
        assert n_live.item() == live
        self.same()
        for a, b in moves:
            kp[:, b], vp[:, b] = kp[:, a], vp[:, a]
        assert torch.equal(kp, self.kp) and torch.equal(vp, self.vp)


@pytest.mark.parametrize("S,page,dtype", [(1, 16, "bf16"), (3, 16, "f32"), (1, 128, "f32"), (20, 16, "bf16")])
def test_a_random_life(cas, S, page, dtype):
    rng = np.random.default_rng(S * page)
    B = 9
    pool = Pool(cas, B, S, page, 70 * S, 12, dtype=dtype)
    for step in range(40):
        what = rng.choice(["extend", "extend", "extend", "free", "fork", "compact"])
        if what == "extend":
            new = rng.integers(0, 60, B) * (rng.random(B) < 0.5)
            shard = None if S == 1 and step % 2 else rng.integers(0, S, new.sum())
            pool.extend(new, shard, pad=int(rng.integers(0, 3)))
        elif what == "free":
            pool.free(rng.integers(0, B, rng.integers(1, 3)).tolist())
        elif what == "fork":
            n = rng.integers(1, 5)
            pool.fork(rng.integers(0, B, n).tolist(), rng.integers(0, B, n).tolist())
        else:
            pool.compact()


def test_many_rows_and_sequences(cas):
    """Several passes of rows, several rounds of sequences, several passes over the references."""
    rng = np.random.default_rng(0)
    pool = Pool(cas, 5000, 1, 16, 20000, 5, Hkv=1, d=8, layers=1)
    pool.extend(rng.integers(0, 4, 5000))
    pool.extend(rng.integers(0, 9, 5000))
    pool.free(rng.permutation(5000)[:3000].tolist())
    pool.compact()
    pool.extend(rng.integers(0, 40, 5000))
    pool = Pool(cas, 300, 40, 16, 12000, 20, Hkv=1, d=8, layers=1)
    new = np.zeros(300, int)
    new[[3, 120, 299]] = 2500, 1, 3000
    pool.extend(new, rng.integers(0, 40, new.sum()))
    pool.extend(new, rng.integers(0, 40, new.sum()))
    pool.fork([3, 120, 3], [4, 5, 6])


def test_refusals_of_an_extension(cas):
    pool = Pool(cas, 4, 1, 16, 10, 6)
    pool.extend([97, 90, 0, 16])                           # 0: list full (6 pages of 16); 1: 6 pages; 3: 1
    pool.extend([0, 6, 64, 15])                            # 1 needs none, 2: 4 pages of the 3 left, 3 needs one, behind 2
    pool.extend([0, 0, 48, 0])                             # the last three
    pool.extend([1, 1, 1, 1])                              # none left; 1 is full
    pool = Pool(cas, 3, 2, 16, 100, 2)
    pool.extend([40, 20, 5], np.concatenate([np.zeros(33, int), np.ones(7, int), np.arange(20) % 2, [-1, 5, 0, 2, 1]]))


def test_refusals_of_a_fork(cas):
    pool = Pool(cas, 6, 2, 16, 12, 6)
    pool.extend([70, 3, 0, 0, 0, 0], np.arange(73) % 2)    # 35 and 35: 6 pages; 2 and 1: 2 pages
    pool.fork([0, 0, 0, 2, 7, 0, -1], [0, 1, 2, 2, 3, 9, 4])       # itself, occupied, good, named before, out of range three times
    pool.fork([1, 1, 0], [3, 4, 5])                        # good (the last two pages), none left, none left
    pool.fork([5, 4], [4, 5])                              # empty ones from empty ones
    pool.free([0, 0, 2, 99, -5])


def test_a_chain_takes_sources_as_they_were(cas):
    pool = Pool(cas, 4, 1, 16, 20, 6)
    pool.extend([40, 0, 0, 0])
    pool.fork([0, 1, 2], [1, 2, 3])                        # 1 and 2 were empty


def test_copies_of_pages(cas):
    import torch
    from paged_reference import i32
    for Hkv, d, page, dtype in ((2, 16, 16, "bf16"), (3, 8, 16, "bf16"), (5, 132, 64, "f32")):
        pool = Pool(cas, 1, 1, page, 12, 3, Hkv=Hkv, d=d, dtype=dtype, layers=3)
        kp, vp = pool.kp.clone(), pool.vp.clone()
        cas.cascade_pages_copy(pool.handle, i32([0, 5, 12, 7, 2, 3]), i32([1, 6, 2, -1, 11, 3]))
        for a, b in ((0, 1), (5, 6), (2, 11)):
            kp[:, b], vp[:, b] = kp[:, a], vp[:, a]
        assert torch.equal(kp, pool.kp) and torch.equal(vp, pool.vp)


def test_captured_calls(cas):
    """Extension, fork, freeing and compaction in one graph, replayed on changed states."""
    import torch
    from paged_reference import i32
    pool = Pool(cas, 4, 1, 16, 40, 8)
    pool.extend([50, 20, 0, 0])
    q_start, slots, visible = i32([0, 5, 5, 5, 9]), *(torch.empty(n, dtype=torch.int32, device="cuda") for n in ((9,), (9, 1)))
    accepted, forked, n_live = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (4, 1, 1))
    src, dst, gone = i32([0]), i32([2]), i32([2])

    def calls():
        cas.cascade_pages_free(pool.handle, gone)
        cas.cascade_pages_fork(pool.handle, src, dst, forked, pool.ws)
        cas.cascade_paged_extend(pool.handle, q_start, slots, visible, accepted)
        cas.cascade_pages_compact(pool.handle, n_live, pool.ws)

    def follow():
        pool.sim.free([int(gone)])
        fork, _ = pool.sim.fork([int(src)], [int(dst)])
        want = pool.sim.extend(q_start.cpu().numpy(), np.zeros(9, int), 9)
        live, _ = pool.sim.compact()
        for t, n in zip((forked, slots, visible, accepted), (fork, *want)):
            assert np.array_equal(t.cpu().numpy(), n)
        assert n_live.item() == live
        pool.same()
    calls()
    torch.cuda.synchronize()
    follow()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        gone.fill_([2, 1, 0, 2][i])
        dst.fill_([2, 1, 0, 2][i])
        src.fill_([1, 0, 3, 0][i])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        follow()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot,d", [(16, 16), (8, 24), (6, 32), (0, 16)])
def test_rows_written_to_their_slots(cas, dtype, layout, rot, d):
    """Keys rotated, values as they are, queries rotated beside them; a row without a slot is not stored; nothing else changes."""
    import torch
    from paged_reference import DT, i32
    from test_gpu_rope import check, desc_of, turned
    rng = np.random.default_rng(rot + d)
    for rows in (1, 6, 3000):
        pool = Pool(cas, 1, 1, 16, 256, 3, Hkv=3, d=d, dtype=dtype)
        kp, vp = pool.kp.clone(), pool.vp.clone()
        slots = rng.permutation(4096)[:rows]
        slots[1::7] = [-1, 4096, 2 ** 31 - 1, -2 ** 31][rows % 4]
        pos = rng.integers(0, 9999, rows)
        fused = torch.randn((rows, 4 + 6, d), device="cuda").to(DT[dtype])
        q, k, v = fused[:, :4], fused[:, 4:7], fused[:, 7:]
        qr, kr = (t.float().cpu().numpy().astype(np.float64) for t in (q, k))
        if rot:
            out = torch.full((rows, 4, d), 7.0, device="cuda").to(DT[dtype])
            cas.cascade_paged_append(pool.handle, 1, i32(slots), k, v, positions=i32(pos), rope=desc_of(cas, rot, 10000.0, layout), q=q, q_out=out)
            check(out, qr, turned(qr, pos, rot, 10000.0, layout), dtype, positions=pos)
            again = q.clone()
            cas.cascade_paged_append(pool.handle, 1, i32(slots), k, v, positions=i32(pos), rope=desc_of(cas, rot, 10000.0, layout), q=again)
            assert torch.equal(again, out)
        else:
            cas.cascade_paged_append(pool.handle, 1, i32(slots), k, v)
        want = turned(kr, pos, rot, 10000.0, layout) if rot else kr
        kept = np.flatnonzero((slots >= 0) & (slots < 4096))
        at = torch.from_numpy(slots[kept]).cuda()
        check(pool.kp[1, at // 16, :, at % 16], kr[kept], want[kept], dtype, positions=pos)
        assert torch.equal(pool.vp[1, at // 16, :, at % 16], v[torch.from_numpy(kept).cuda()])
        for now, was in ((pool.kp, kp), (pool.vp, vp)):
            now[1, at // 16, :, at % 16] = was[1, at // 16, :, at % 16]
            assert torch.equal(now, was)


@pytest.mark.parametrize("shards", [1, 3])
def test_a_prompt_in_chunks_is_a_prompt_at_once(cas, shards):
    """Two sequences pass through one layer chunk by chunk, composed from norm, projections, extension, append and attention over
    the pages, and a branch of one goes on with other tokens: as cascade_layer_forward gives for each whole sequence."""
    import torch
    from cascade_inputs import CONFIGS, make_layer_weights
    from paged_reference import i32, starts
    cfg = CONFIGS["C3"].with_(name="paged", d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ff=512, batch=1, n_shards=1)
    H, Hkv, d, D = 4, 2, 64, 256
    w = {k: cas.to_device(v, "bf16") for k, v in make_layer_weights(cfg).items()}
    wqkv = torch.cat([w["wq"], w["wk"], w["wv"]])
    rope = cas.make_rope_desc(d, cfg.rope_theta)
    lens = {0: 150, 1: 70, 2: 131}
    rng = np.random.default_rng(5)
    x = {b: torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32)).bfloat16().cuda() for b, n in lens.items()}
    x[2][:120] = x[0][:120]                                 # the branch leaves sequence 0 behind its 120th token
    owner = {b: rng.integers(0, shards, n) for b, n in lens.items()}
    owner[2][:120] = owner[0][:120]
    pool = Pool(cas, 3, shards, 16, 40 * shards, 12, Hkv=Hkv, d=d, layers=1)
    out = {b: torch.empty((n, D), device="cuda").bfloat16() for b, n in lens.items()}
    done = {0: 0, 1: 0, 2: 0}
    out[2][:120] = 0

    def chunk(new):
        rows = sum(new)
        part = [x[b][done[b]:done[b] + n] for b, n in enumerate(new)]
        h = torch.cat(part)
        pos = i32(np.concatenate([np.arange(done[b], done[b] + n) for b, n in enumerate(new)]))
        slots, visible, accepted = pool.extend(new, np.concatenate([owner[b][done[b]:done[b] + n] for b, n in enumerate(new)]))
        normed, qkv = torch.empty_like(h), torch.empty((rows, (H + 2 * Hkv) * d), device="cuda").bfloat16()
        cas.cascade_norm(h, w["norm1_g"], None, normed, cas.NORM_RMSNORM, cfg.eps)
        cas.cascade_shard_gemm(None, normed, wqkv, qkv)
        heads = qkv.view(rows, H + 2 * Hkv, d)
        q, k, v = heads[:, :H], heads[:, H:H + Hkv], heads[:, H + Hkv:]
        cas.cascade_paged_append(pool.handle, 0, slots, k, v, positions=pos, rope=rope, q=q)
        o, ws = torch.empty((rows, H, d), device="cuda").bfloat16(), cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(pool.handle, rows, H))
        cas.cascade_paged_attn(pool.handle, 0, q, o, i32(starts(new)), cfg.scale, visible=visible, workspace=ws)
        h1, act, y = torch.empty_like(h), torch.empty((rows, 512), device="cuda").bfloat16(), torch.empty_like(h)
        cas.cascade_shard_gemm(None, o.view(rows, H * d), w["wo"], h1, residual=h, epilogue=cas.EPI_RESIDUAL)
        cas.cascade_norm(h1, w["norm2_g"], None, normed, cas.NORM_RMSNORM, cfg.eps)
        cas.cascade_shard_gemm(None, normed, w["w_gate"], act, W_up=w["w_up"], epilogue=cas.EPI_SWIGLU)
        cas.cascade_shard_gemm(None, act, w["w_down"], y, residual=h1, epilogue=cas.EPI_RESIDUAL)
        for b, n in enumerate(new):
            out[b][done[b]:done[b] + n] = y[starts(new)[b]:starts(new)[b] + n]
            done[b] += n

    chunk([100, 1, 0])
    chunk([20, 33, 0])
    pool.fork([0], [2])
    done[2] = 120
    chunk([1, 1, 1])
    chunk([29, 35, 10])
    assert done == lens
    for b, n in lens.items():
        plan = cas.cascade_plan_create(1, n, 1, np.zeros(n, np.int32))
        desc = cas.make_layer_desc(cfg.with_(seq_len=n))
        ws = cas.new_workspace(cas.cascade_layer_workspace_bytes(plan, desc))
        want = torch.empty((1, n, D), device="cuda").bfloat16()
        weights = cas.make_layer_weights(w)
        cas.cascade_layer_forward(plan, desc, weights, x[b][None], want, ws)
        torch.cuda.synchronize()
        first = 120 if b == 2 else 0
        # both sides round q, k, v, o, h1 and the activation to bf16, after sums in another order
        err = (out[b][first:].double() - want[0, first:].double()).abs().max() / want.double().abs().max()
        assert err < 2e-2, (b, err)
    pool.free([0, 1, 2])
    assert not pool.refs.any()

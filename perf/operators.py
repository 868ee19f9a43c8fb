"""Cases that time the operators of a paged, token-sharded key/value cache: rotary positions, the pages themselves, and the
attention of new tokens over them.

A case is a dict of plain values (lengths of sequences as a text of numbers); its "kind" names the pass:

  rope     rotary positions of the heads of a batch of rows
  arrive   sequences leave the cache and others take their place: pages freed, pages and slots for the new rows, keys rotated
           and written with their values, queries rotated
  branch   the branches of a search are dropped and the surviving sequences forked again (full pages shared, the last one copied)
  compact  pages scattered over the pool move to its front
  attend   attention of the new rows of every sequence (one each, or a chunk) over the keys that the cache holds

`own` chooses between the plain form, elementary torch operations, and the library's calls.  Head counts and dimensions are
those of the workloads in cascade_inputs/configs.py.
"""
import math

import numpy as np
import torch

own = False

_THETA = 500000.0
# query heads, kv heads, head dim
_HEADS = {"tiny": (4, 4, 16), "gpt2": (12, 12, 64), "8b": (32, 8, 128), "70b": (64, 8, 128)}


def _heads(shape):
    return dict(zip(("H", "Hkv", "d"), _HEADS[shape]))


def _rope(rot, layout="half", theta=_THETA, scaling="none", factor=1.0, original=0, amplitude=1.0):
    return {"rot": rot, "layout": layout, "theta": theta, "scaling": scaling, "factor": factor, "original": original, "amplitude": amplitude}


def listed():
    return [
        # queries and keys of one new token of each of a few sequences: the smallest call
        {"name": "rope_tokens", "kind": "rope", "dtype": "bf16", **_heads("8b"), "rows": 4, "far": 2048, **_rope(128)},
        # a long prompt's chunk at positions past the length the model was trained for, frequencies scaled by a ramp
        {"name": "rope_long_prompt", "kind": "rope", "dtype": "bf16", **_heads("8b"), "rows": 8192, "far": 131072,
         **_rope(128, scaling="ramp", factor=8.0, original=8192)},
        # a quarter of each head rotated, neighbouring columns as pairs, fp32, an odd number of rows
        {"name": "rope_part_f32", "kind": "rope", "dtype": "f32", **_heads("gpt2"), "rows": 1021, "far": 4096,
         **_rope(16, layout="interleaved", theta=10000.0, scaling="linear", factor=4.0)},
        # short prompts of unequal lengths arrive together
        {"name": "arrive_short", "kind": "arrive", "dtype": "bf16", **_heads("8b"), "lens": "17 64 1 120 5 33 77 250", "shards": 1,
         "page": 16, **_rope(128)},
        # two documents arrive, their tokens dealt to the shards of the protocol
        {"name": "arrive_sharded", "kind": "arrive", "dtype": "bf16", **_heads("8b"), "lens": "2500 1596", "shards": 16, "page": 64,
         **_rope(128)},
        # a beam of four branches per sequence is dropped and forked again, the pages of eight layers at once
        {"name": "branch_beams", "kind": "branch", "dtype": "bf16", **_heads("8b"), "parents": 4, "branches": 4, "context": 1000,
         "shards": 1, "page": 64, "layers": 8},
        # a half-empty pool is compacted
        {"name": "compact_pool", "kind": "compact", "dtype": "bf16", **_heads("8b"), "seqs": 12, "context": 700, "shards": 1, "page": 64,
         "layers": 8, "share": 0.5},
        # one new token for a few sequences: latency
        {"name": "attend_tokens", "kind": "attend", "dtype": "bf16", **_heads("8b"), "new": "1 1 1 1", "context": "2048 1500 700 333",
         "shards": 1, "page": 16},
        # generation over long contexts of unequal lengths: the cache is what has to be read
        {"name": "attend_long_caches", "kind": "attend", "dtype": "bf16", **_heads("8b"), "new": _text([1] * 32),
         "context": _text(8192 - 211 * i for i in range(32)), "shards": 1, "page": 64},
        # a prompt's chunk among sequences that generate, caches in shards
        {"name": "attend_mixed_sharded", "kind": "attend", "dtype": "bf16", **_heads("70b"), "new": _text([509] + [1] * 11 + [4] * 4),
         "context": _text(1500 + 111 * i for i in range(16)), "shards": 8, "page": 32},
        # a long prompt's chunk over what was cached before it
        {"name": "attend_chunk", "kind": "attend", "dtype": "bf16", **_heads("8b"), "new": "4096", "context": "12288", "shards": 1, "page": 64},
        # fp32, small heads: a few prompts' chunks
        {"name": "attend_f32", "kind": "attend", "dtype": "f32", **_heads("gpt2"), "new": "100 37 1", "context": "900 411 0", "shards": 1,
         "page": 32},
    ]


def _ints(text):
    return [int(t) for t in text.split()]


def _text(ints):
    return " ".join(str(i) for i in ints)


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "arrive", "branch", "compact", "attend", "attend", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads = _heads(rng.choice(["tiny", "gpt2"] if dtype == "f32" else ["gpt2", "8b", "8b", "70b"]))
    case = {"kind": kind, "dtype": dtype, **heads}
    if kind in ("rope", "arrive"):
        d = heads["d"]
        scaling = rng.choice(["none", "linear", "ramp"])
        case.update(_rope(rng.choice([d, d, d // 2]), rng.choice(["half", "interleaved"]), rng.choice([10000.0, _THETA]), scaling,
                          1.0 if scaling == "none" else rng.uniform(1.5, 32.0), 8192 if scaling == "ramp" else 0,
                          rng.choice([1.0, 1.0, 1.2])))
    if kind == "rope":
        return {**case, "rows": _log_int(rng, 1, 4000), "far": _log_int(rng, 100, 1 << 20)}
    shards, page = rng.choice([1, 1, 1, 4, 16]), rng.choice([16, 32, 64, 128])
    if kind == "arrive":
        return {**case, "lens": _text(_log_int(rng, 1, 600) for _ in range(_log_int(rng, 1, 6))), "shards": shards, "page": page}
    if kind == "branch":
        return {**case, "parents": rng.randint(1, 6), "branches": rng.randint(1, 4), "context": _log_int(rng, 20, 1000), "shards": shards,
                "page": page, "layers": rng.randint(1, 4)}
    if kind == "compact":
        return {**case, "seqs": rng.randint(2, 12), "context": _log_int(rng, 50, 700), "shards": shards, "page": page,
                "layers": rng.randint(1, 4), "share": rng.uniform(0.3, 0.9)}
    if rng.random() < 0.5:                                  # generation: one row each, now and then a few
        n = _log_int(rng, 1, 24)
        new = [rng.choice([1, 1, 1, 1, 3]) for _ in range(n)]
        return {**case, "new": _text(new), "context": _text(_log_int(rng, 1, 6000) for _ in new), "shards": shards, "page": page}
    new = [_log_int(rng, 2, 1024)] + [_log_int(rng, 1, 64) for _ in range(rng.randint(0, 5))]
    return {**case, "new": _text(new), "context": _text(_log_int(rng, 1, 3000) for _ in new), "shards": shards, "page": page}


# ---------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _draws(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *shape: torch.randn(shape, device="cuda", generator=g).to(_dtype(case))


def _int32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _tables(lens, page, n_pages, max_pages, rng):
    """Page lists [B, S, max_pages] of the given lengths [B, S], pages in an order that a used pool has, and the references."""
    B, S = lens.shape
    table, refs = np.full((B, S, max_pages), -1, np.int64), np.zeros(n_pages, np.int64)
    used = -(-lens // page)
    ids = rng.permutation(n_pages)[:used.sum()]
    table[np.arange(max_pages) < used[:, :, None]] = ids
    refs[ids] = 1
    return table, refs


def _dealt(lens, shards):
    """Rows of each shard where the tokens of a sequence are dealt to the shards in turn."""
    lens = np.asarray(lens, np.int64)[:, None]
    return lens // shards + (np.arange(shards) < lens % shards)


def _parent_lens(case):
    return [max(1, case["context"] - 13 * i) for i in range(case["parents"])]


def _pool_lens(case):
    return [max(1, case["context"] - 29 * (i % 5)) for i in range(case["seqs"])]


def prepare(case, seed):
    """What a program has in hand: rows, positions, the cache and its tables; with the library, the handle of the cache
    and the workspace that it keeps."""
    rng, normal, kind = np.random.default_rng(seed), _draws(case, seed), case["kind"]
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    st = {"case": case}
    if kind == "rope":
        st["x0"] = normal(case["rows"], H + Hkv, d)
        st["x"] = torch.empty_like(st["x0"])
        st["positions"] = _int32(rng.integers(0, case["far"], case["rows"]))
        if own:
            st["rope"] = _rope_desc(case)
        return st
    S, page, layers = case["shards"], case["page"], case.get("layers", 1)
    if kind == "arrive":
        new = _ints(case["lens"])
        rows, final, lens = sum(new), _dealt(new, S), np.zeros((len(new), S), np.int64)
        st["q_start"] = _int32(np.concatenate([[0], np.cumsum(new)]))
        st["shard"] = _int32(np.concatenate([np.arange(n) % S for n in new]))
        st["positions"] = _int32(np.concatenate([np.arange(n) for n in new]))
        qkv = normal(rows, H + 2 * Hkv, d)                 # rows as a fused projection leaves them
        st["q0"], st["k"], st["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        st["q"] = torch.empty_like(st["q0"])
        st["slots"], st["visible"] = _int32(np.zeros(rows)), _int32(np.zeros((rows, S)))
        st["accepted"], st["all"] = _int32(np.zeros(len(lens))), _int32(np.arange(len(lens)))
        spare = 7
    elif kind == "branch":
        n = case["parents"] * case["branches"]
        final = lens = _dealt(_parent_lens(case) + [0] * n, S)
        st["src"], st["dst"] = _int32(np.arange(n) // case["branches"]), _int32(case["parents"] + np.arange(n))
        st["accepted"] = _int32(np.zeros(n))
        spare = n * S + 5
    elif kind == "compact":
        final = lens = _dealt(_pool_lens(case), S)
        st["n_live"] = _int32([0])
        spare = int((-(-lens // page)).sum() * (1 / case["share"] - 1)) + 1
    else:
        context, new = _ints(case["context"]), _ints(case["new"])
        final = lens = _dealt(np.add(context, new), S)
        rows = sum(new)
        st["q_start"] = _int32(np.concatenate([[0], np.cumsum(new)]))
        st["visible"] = _int32(np.concatenate([_dealt(c + 1 + np.arange(n), S) for c, n in zip(context, new)]))
        st["q"], st["o"] = normal(rows, H, d), torch.empty((rows, H, d), device="cuda", dtype=_dtype(case))
        st["lse"] = torch.empty((H, rows), device="cuda")
        spare = 11
    used = -(-final // page)
    n_pages, max_pages = int(used.sum()) + spare, int(used.max()) + 1
    table, refs = _tables(lens, page, n_pages, max_pages, rng)
    st["table"], st["lens"], st["refs"] = _int32(table), _int32(lens), _int32(refs)
    st["kp"], st["vp"] = normal(layers, n_pages, Hkv, page, d), normal(layers, n_pages, Hkv, page, d)
    if kind == "compact":
        st["table0"], st["refs0"] = st["table"].clone(), st["refs"].clone()
    if own:
        import paper_2507_05228_amd as cas
        st["cache"] = cas.make_paged_cache(st["kp"], st["vp"], st["table"], st["lens"], st["refs"])
        if kind == "arrive":
            st["rope"] = _rope_desc(case)
        elif kind == "attend":
            st["ws"] = cas.new_workspace(cas.cascade_paged_attn_workspace_bytes(st["cache"], rows, H))
        else:
            st["ws"] = cas.new_workspace(cas.cascade_pages_workspace_bytes(st["cache"]))
    return st


# ---------------------------------------------------------------------------- one pass, by the library's calls
def _rope_desc(case):
    import paper_2507_05228_amd as cas
    return cas.make_rope_desc(case["rot"], case["theta"], layout=cas.ROPE_HALF if case["layout"] == "half" else cas.ROPE_INTERLEAVED,
                              scaling={"none": cas.ROPE_UNSCALED, "linear": cas.ROPE_LINEAR, "ramp": cas.ROPE_RAMP}[case["scaling"]],
                              factor=case["factor"], low=1.0, high=4.0, original_len=case["original"], amplitude=case["amplitude"])


def _run_own(st, case):
    import paper_2507_05228_amd as cas
    kind = case["kind"]
    if kind == "rope":
        cas.cascade_rope(st["rope"], st["x0"], st["positions"], st["x"])
        return {"x": st["x"]}
    cache = st["cache"]
    if kind == "arrive":
        cas.cascade_pages_free(cache, st["all"])
        cas.cascade_paged_extend(cache, st["q_start"], st["slots"], st["visible"], st["accepted"],
                                 row_shard=st["shard"] if case["shards"] > 1 else None)
        cas.cascade_paged_append(cache, 0, st["slots"], st["k"], st["v"], positions=st["positions"], rope=st["rope"], q=st["q0"], q_out=st["q"])
    elif kind == "branch":
        cas.cascade_pages_free(cache, st["dst"])
        cas.cascade_pages_fork(cache, st["src"], st["dst"], st["accepted"], st["ws"])
    elif kind == "compact":
        st["table"].copy_(st["table0"])
        st["refs"].copy_(st["refs0"])
        cas.cascade_pages_compact(cache, st["n_live"], st["ws"])
    else:
        cas.cascade_paged_attn(cache, 0, st["q"], st["o"], st["q_start"], case["d"] ** -0.5, visible=st["visible"], lse=st["lse"], workspace=st["ws"])
    return _outputs(st, kind)


def _outputs(st, kind):
    names = {"arrive": ("q", "slots", "visible", "accepted"), "branch": ("accepted",), "compact": ("n_live",), "attend": ("o", "lse")}[kind]
    return {k: st[k] for k in names + (() if kind == "attend" else ("table", "lens", "refs", "kp", "vp"))}


# ---------------------------------------------------------------------------- one pass, in elementary operations
def _frequencies(case, device):
    f = case["theta"] ** (-torch.arange(0, case["rot"], 2, device=device, dtype=torch.float64) / case["rot"])
    if case["scaling"] == "linear":
        f = f / case["factor"]
    elif case["scaling"] == "ramp":
        g = ((case["original"] * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        f = f * ((1 - g) / case["factor"] + g)
    return f


def _rotate(case, x, positions):
    """x [rows, heads, d] with its first `rot` columns rotated, in fp32."""
    rot, x = case["rot"], x.float()
    angle = (positions.double()[:, None] * _frequencies(case, x.device))[:, None]
    c, s = (angle.cos() * case["amplitude"]).float(), (angle.sin() * case["amplitude"]).float()
    if case["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat([a * c - b * s, a * s + b * c, x[..., rot:]], -1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat([torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2), x[..., rot:]], -1)


def _freed(table, lens, refs, seqs):
    gone = table[seqs].flatten().long()
    taken = torch.zeros_like(refs).scatter_add_(0, gone.clamp_min(0), (gone >= 0).int())
    refs.sub_(taken)
    table[seqs], lens[seqs] = -1, 0


def _lowest_free(refs):
    """Page ids, free ones first, in ascending order."""
    return torch.argsort((refs > 0).int(), stable=True).int()


def _run_plain(st, case):
    kind = case["kind"]
    if kind == "rope":
        st["x"].copy_(_rotate(case, st["x0"], st["positions"]))
        return {"x": st["x"]}
    if kind == "attend":
        _attend_plain(st, case)
        return _outputs(st, kind)
    table, lens, refs, kp, vp, page = (*(st[k] for k in ("table", "lens", "refs", "kp", "vp")), case["page"])
    ids = torch.arange(table.shape[2], device="cuda")
    if kind == "arrive":
        _freed(table, lens, refs, st["all"].long())
        rows, S = st["visible"].shape
        seq = torch.searchsorted(st["q_start"][1:].contiguous(), torch.arange(rows, device="cuda", dtype=torch.int32), right=True)
        mine = (st["shard"].long()[:, None] == torch.arange(S, device="cuda")).int()
        running = torch.cat([mine.new_zeros(1, S), mine.cumsum(0, dtype=torch.int32)])
        before = running[st["q_start"][:-1].long()]
        st["visible"].copy_(lens[seq] + running[1:] - before[seq])
        after = lens + running[st["q_start"][1:].long()] - before
        first, last = (lens + page - 1) // page, (after + page - 1) // page
        need = (last - first).flatten()
        base = (need.cumsum(0) - need).view_as(first)
        free = _lowest_free(refs)
        new = (ids >= first[..., None]) & (ids < last[..., None])
        table.copy_(torch.where(new, free[(base[..., None] + ids - first[..., None]).clamp(0, len(free) - 1)], table))
        is_free = refs == 0
        refs.copy_(torch.where(is_free & (is_free.cumsum(0) <= need.sum()), 1, refs))
        lens.copy_(after)
        st["accepted"].fill_(1)
        at = st["visible"].gather(1, st["shard"].long()[:, None])[:, 0] - 1
        pages = table[seq, st["shard"].long(), (at // page).long()]
        st["slots"].copy_(pages * page + at % page)
        kp[0, pages.long(), :, (at % page).long()] = _rotate(case, st["k"], st["positions"]).to(kp.dtype)
        vp[0, pages.long(), :, (at % page).long()] = st["v"]
        st["q"].copy_(_rotate(case, st["q0"], st["positions"]))
    elif kind == "branch":
        src, dst = st["src"].long(), st["dst"].long()
        _freed(table, lens, refs, dst)
        part = lens[src] % page                             # rows of the last page where that is partly filled
        need = (part > 0).flatten()
        new = _lowest_free(refs)[(need.cumsum(0) - 1).clamp_min(0)].view_as(part)
        at = (ids == (lens[src] // page)[..., None]) & (part > 0)[..., None]
        parent = table[src]
        child = torch.where(at, new[..., None], parent)
        is_free = refs == 0
        refs.copy_(torch.where(is_free & (is_free.cumsum(0) <= need.sum()), 1, refs))
        shared = torch.where(at, -1, parent).flatten().long()
        refs.add_(torch.zeros_like(refs).scatter_add_(0, shared.clamp_min(0), (shared >= 0).int()))
        table[dst], lens[dst] = child, lens[src]
        old, new = (torch.where(at, t, 0).sum(-1).flatten()[need].long() for t in (parent, child))
        held = (torch.arange(page, device="cuda") < part.flatten()[need][:, None])[None, :, None, :, None]
        kp[:, new] = torch.where(held, kp[:, old], kp[:, new])
        vp[:, new] = torch.where(held, vp[:, old], vp[:, new])
        st["accepted"].fill_(1)
    else:
        table.copy_(st["table0"])
        refs.copy_(st["refs0"])
        live, page_ids = refs > 0, torch.arange(len(refs), device="cuda")
        st["n_live"].copy_(live.sum())
        old, new = (live & (page_ids >= st["n_live"])).nonzero()[:, 0], (~live & (page_ids < st["n_live"])).nonzero()[:, 0]
        kp[:, new], vp[:, new] = kp[:, old], vp[:, old]
        refs[new], refs[old] = refs[old], 0
        page_ids[old] = new
        table.copy_(torch.where(table >= 0, page_ids[table.clamp_min(0).long()], -1))
    return _outputs(st, kind)


def _attend_plain(st, case):
    """All sequences at once, padded to the longest chunk and to the length of the page lists."""
    H, Hkv, d, page, S, n = case["H"], case["Hkv"], case["d"], case["page"], case["shards"], max(_ints(case["new"]))
    q_start, table = st["q_start"].long(), st["table"]
    B, cols = len(_ints(case["new"])), table.shape[2] * page
    row = q_start[:-1, None] + torch.arange(n, device="cuda")
    real = row < q_start[1:, None]
    row = row.clamp_max(len(st["q"]) - 1)
    k, v = (p[0, table.clamp_min(0).long()].float().permute(0, 3, 1, 2, 4, 5).reshape(B, Hkv, S * cols, d) for p in (st["kp"], st["vp"]))
    q = st["q"][row].float().view(B, n, Hkv, H // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    seen = torch.minimum(st["visible"][row], st["lens"][:, None]) * real[..., None]              # [B, n, S]
    seen = (torch.arange(cols, device="cuda") < seen[..., None]).view(B, 1, 1, n, S * cols)
    a = (q @ k.transpose(2, 3).contiguous()).view(B, Hkv, H // Hkv, n, S * cols) * d ** -0.5
    a = a.masked_fill_(~seen, -math.inf)
    m = a.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = a.sub_(m).exp_()
    total = p.sum(-1)
    o = (p.view(B, Hkv, -1, S * cols) @ v).view(B, Hkv, H // Hkv, n, d) / torch.where(total > 0, total, 1.0)[..., None]
    lse = m[..., 0] + total.log()
    rows = torch.arange(len(st["q"]), device="cuda")
    seq = torch.searchsorted(q_start[1:].contiguous(), rows, right=True)
    at = (seq, slice(None), slice(None), rows - q_start[seq])
    st["o"].copy_(o[at].reshape(len(rows), H, d))
    st["lse"].copy_(lse[at].reshape(len(rows), H).t())


def run(st):
    return _run_own(st, st["case"]) if own else _run_plain(st, st["case"])


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    es, kind = (2 if case["dtype"] == "bf16" else 4), case["kind"]
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    if kind == "rope":
        return {"bytes": 2 * es * case["rows"] * (H + Hkv) * d + 4 * case["rows"], "flops": 3.0 * case["rows"] * (H + Hkv) * case["rot"]}
    if kind == "arrive":
        rows = sum(_ints(case["lens"]))
        return {"bytes": es * rows * d * 2 * (H + 2 * Hkv) + 4 * rows * (case["shards"] + 3), "flops": 3.0 * rows * (H + Hkv) * case["rot"]}
    row, page = case.get("layers", 1) * 2 * es * Hkv * d, case["page"]
    if kind == "branch":
        lens = _dealt(_parent_lens(case), case["shards"])
        return {"bytes": 2.0 * row * case["branches"] * int((lens % page).sum()), "flops": 0.0}
    if kind == "compact":
        lens = _dealt(_pool_lens(case), case["shards"])
        live = int((-(-lens // page)).sum())
        return {"bytes": 2.0 * row * page * live * (1 - live / (live + int(live * (1 / case["share"] - 1)) + 1)), "flops": 0.0}
    context, new = _ints(case["context"]), _ints(case["new"])
    pairs = sum(n * c + n * (n + 1) / 2 for c, n in zip(context, new))
    return {"bytes": es * (2 * (sum(context) + sum(new)) * Hkv * d + 2 * sum(new) * H * d), "flops": 4.0 * d * H * pairs}


# ---------------------------------------------------------------------------- the same results in 64 bits
def _turned(case, x, positions):
    """Pairs as complex numbers times e^(i angle)."""
    rot, x = case["rot"], x.double()
    i = torch.arange(case["rot"] // 2, device=x.device, dtype=torch.float64)
    f = torch.exp(-2 * i / rot * math.log(case["theta"]))
    if case["scaling"] == "linear":
        f = f / case["factor"]
    if case["scaling"] == "ramp":
        turns = case["original"] * f / (2 * math.pi)       # of the original length; fewer than 1: scaled, more than 4: not
        kept = torch.where(turns < 1, 0.0, torch.where(turns > 4, 1.0, (turns - 1) / 3))
        f = (1 - kept) * f / case["factor"] + kept * f
    turn = torch.polar(torch.full_like(f, case["amplitude"])[None], positions.double()[:, None] * f)[:, None]
    y = x.clone()
    if case["layout"] == "half":
        z = torch.complex(x[..., :rot // 2].contiguous(), x[..., rot // 2:rot].contiguous()) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.view_as_complex(x[..., :rot].contiguous().view(*x.shape[:2], rot // 2, 2)) * turn
        y[..., :rot] = torch.view_as_real(z).flatten(-2)
    return y


def exact(case, seed):
    st = _exact_state(case, seed)
    kind, page = case["kind"], case.get("page")
    if kind == "rope":
        return {"x": _turned(case, st["x0"], st["positions"])}
    if kind == "attend":
        return _attend_exact(case, st)
    # pages are whole numbers and copies; of an arrival, what is computed
    if kind != "arrive":
        return None
    q, k, kp, vp = _turned(case, st["q0"], st["positions"]), _turned(case, st["k"], st["positions"]), st["kp"].double(), st["vp"].double()
    free, held, table = 0, 0, {}
    lens, S = _ints(case["lens"]), case["shards"]
    for b, n in enumerate(lens):                            # an empty pool: pages in order, list by list
        for s in range(S):
            for j in range(-(-len(range(s, n, S)) // page)):
                table[b, s, j], free = free, free + 1
    for b, n in enumerate(lens):
        for t in range(n):
            p, r = table[b, t % S, t // S // page], t // S % page
            kp[0, p, :, r], vp[0, p, :, r] = k[held], st["v"][held].double()
            held += 1
    return {"q": q, "slots": None, "visible": None, "accepted": None, "table": None, "lens": None, "refs": None, "kp": kp, "vp": vp}


def _exact_state(case, seed):
    global own
    was, own = own, False                                   # the inputs, without a handle of the library
    try:
        return prepare(case, seed)
    finally:
        own = was


def _attend_exact(case, st):
    H, Hkv, d, page = case["H"], case["Hkv"], case["d"], case["page"]
    o, lse = torch.zeros(st["q"].shape, device="cuda", dtype=torch.float64), torch.zeros(st["lse"].shape, device="cuda", dtype=torch.float64)
    lo = 0
    for b, (c, n) in enumerate(zip(_ints(case["context"]), _ints(case["new"]))):
        shard_keys = _dealt([c + n], case["shards"])[0]
        pages = [st["table"][b, s, :-(-int(m) // page)].long() for s, m in enumerate(shard_keys)]
        for g in range(Hkv):
            k, v = (torch.cat([p[0, ids, g].reshape(-1, d)[:m] for ids, m in zip(pages, shard_keys)]).double() for p in (st["kp"], st["vp"]))
            # token j of the sequence lies in shard j mod S, at row j // S of it: seen by the rows at or after it
            token = torch.cat([torch.arange(int(m), device="cuda") * case["shards"] + s for s, m in enumerate(shard_keys)])
            hidden = token[None] > c + torch.arange(n, device="cuda")[:, None]
            for h in range(g * (H // Hkv), (g + 1) * (H // Hkv)):
                a = (st["q"][lo:lo + n, h].double() @ k.t() * d ** -0.5).masked_fill(hidden, -math.inf)
                lse[h, lo:lo + n] = torch.logsumexp(a, -1)
                o[lo:lo + n, h] = torch.softmax(a, -1) @ v
        lo += n
    return {"o": o, "lse": lse}

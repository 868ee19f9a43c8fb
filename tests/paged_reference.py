"""Plain 64-bit references of the paged cache's operators, and caches to try them on."""
import math

import numpy as np
import torch

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}         # a rounding's largest error, relative


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class Cache:
    """Pools, lists and references, with the library's handle.  lens [B][S]; pages in shuffled order; every row that no list
    holds is `filler`."""

    def __init__(self, cas, dtype, Hkv, d, page, lens, layers=1, spare=3, max_pages=None, seed=0, filler=math.nan, amp=1.0):
        rng = np.random.default_rng(seed)
        lens = np.asarray(lens, np.int64)
        B, S = lens.shape
        used = -(-lens // page)
        n_pages = int(used.sum()) + spare
        self.max_pages = int(used.max()) + 1 if max_pages is None else max_pages
        table, refs = np.full((B, S, self.max_pages), -1), np.zeros(n_pages)
        ids = iter(rng.permutation(n_pages))
        gen = torch.Generator(device="cuda").manual_seed(seed)
        shape = (layers, n_pages, Hkv, page, d)
        self.kp, self.vp = (torch.full(shape, filler, device="cuda", dtype=DT[dtype]) for _ in range(2))
        for b in range(B):
            for s in range(S):
                for j in range(used[b, s]):
                    table[b, s, j] = next(ids)
                    refs[table[b, s, j]] = 1
                    n = min(page, lens[b, s] - j * page)
                    for pool, a in ((self.kp, amp), (self.vp, 1.0)):
                        pool[:, table[b, s, j], :, :n] = (a * torch.randn((layers, Hkv, n, d), device="cuda", generator=gen)).to(DT[dtype])
        self.table, self.lens, self.refs = i32(table), i32(lens), i32(refs)
        self.handle = cas.make_paged_cache(self.kp, self.vp, self.table, self.lens, self.refs)
        self.page, self.d, self.Hkv, self.dtype = page, d, Hkv, dtype

    def rows(self, pool, layer, b, s, n):
        """The first n rows of a list: [Hkv, n, d] in 64 bits."""
        pages = self.table[b, s, :-(-n // self.page)].long()
        return pool[layer, pages].transpose(0, 1).reshape(self.Hkv, -1, self.d)[:, :n].double()


def attention(cache, layer, q, q_start, visible, scale):
    """o [rows, H, d], lse [H, rows], and for the bounds: weights times |v| [rows, H, d], and the largest of the sums of
    |q||k| scale that a row's scores are made of [rows, H]."""
    rows, H, d = q.shape
    lens = cache.lens.cpu().numpy()
    o, av = (torch.zeros((rows, H, d), dtype=torch.float64, device="cuda") for _ in range(2))
    lse, mag = torch.full((H, rows), -math.inf, dtype=torch.float64, device="cuda"), torch.zeros((rows, H), dtype=torch.float64, device="cuda")
    for b in range(lens.shape[0]):
        lo, hi = q_start[b], q_start[b + 1]
        if hi <= lo:
            continue
        ks, vs, seen = [], [], []
        for s in range(lens.shape[1]):
            n = int(lens[b, s])
            ks.append(cache.rows(cache.kp, layer, b, s, n))
            vs.append(cache.rows(cache.vp, layer, b, s, n))
            limit = torch.full((hi - lo,), n, device="cuda") if visible is None else visible[lo:hi, s].clamp_max(n)
            seen.append(torch.arange(n, device="cuda") < limit[:, None])
        k, v, seen = torch.cat(ks, 1), torch.cat(vs, 1), torch.cat(seen, 1)
        for h in range(H):
            g = h // (H // cache.Hkv)
            x = q[lo:hi, h].double()
            a = (x @ k[g].t() * scale).masked_fill(~seen, -math.inf)
            some = seen.any(1)
            w = torch.where(some[:, None], torch.softmax(a, 1), 0.0)
            for r in range(hi - lo) if not torch.isfinite(v[g]).all() else ():
                o[lo + r, h] = w[r, seen[r]] @ v[g][seen[r]]
            if torch.isfinite(v[g]).all():
                o[lo:hi, h], av[lo:hi, h] = w @ v[g], w @ v[g].abs()
            lse[h, lo:hi] = torch.where(some, torch.logsumexp(a, 1), -math.inf)
            if k.shape[1]:
                mag[lo:hi, h] = ((x.abs() @ k[g].abs().t()) * scale).masked_fill(~seen, 0.0).amax(1)
    return o, lse, av, mag


def check_attention(cache, o, lse, ref, keys):
    """Bounds.  A score is a sum of d products in fp32: it is off by (d + 3) 2^-24 of the sum of their magnitudes, and a weight by
    that much, relatively, twice (its own and the sum's), besides the exponential and the sum over the keys, 2^-24 each.  The
    weights are rounded to the cache's type in front of the second product and so is the result."""
    ro, rl, av, mag = ref
    eps, half = 2.0 ** -24, HALF_STEP[cache.dtype]
    score = (cache.d + 3) * eps * mag
    weight = 2 * score + (2 * keys + 64) * eps + (half if cache.dtype == "bf16" else 0.0)
    out = HALF_STEP["bf16" if o.dtype == torch.bfloat16 else "f32"]
    err, bound = (o.double() - ro).abs(), av * weight[..., None] * 1.01 + ro.abs() * out * 1.01 + 1e-30
    assert torch.isfinite(o[torch.isfinite(ro)]).all()
    assert bool((err <= bound).all()), float((err / bound).max())
    if lse is not None:
        dead = rl == -math.inf
        assert bool((lse[dead] == -math.inf).all()) and bool((o.permute(1, 0, 2)[dead] == 0).all())
        live = ~dead
        err = (lse.double() - rl).abs()[live]
        bound = (score.t() + (2 * keys + 64) * eps + 4 * eps * rl.abs().clamp_max(1e30))[live]
        assert bool((err <= bound).all()), float((err / bound).max())


def dealt(lens, shards):
    lens = np.asarray(lens, np.int64)[..., None]
    return lens // shards + (np.arange(shards) < lens % shards)


def causal(context, new, shards):
    """visible [rows, S] of new tokens dealt to the shards in turn behind `context` ones."""
    return np.concatenate([dealt(c + 1 + np.arange(n), shards) for c, n in zip(context, new)]) if sum(new) else np.zeros((0, shards))


def starts(new):
    return np.concatenate([[0], np.cumsum(new)])

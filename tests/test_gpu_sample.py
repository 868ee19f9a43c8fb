"""Tokens from logits against the definition in 64 bits (numpy, a whole sort): equal tokens; prob within 2^-22 (a rounding to fp32,
2^-24, and weights exact to 2^-30)."""
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


def reference(logits, u, t, k, p, least):
    l = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64)) + 0.0
    most = l.max()
    if most == -np.inf:
        return 0, 0.0
    order = np.argsort(-l, kind="stable")
    if not t > 0:
        return int(order[0]), 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        # an infinite distance has no weight, at a temperature of infinity either (where the quotient says nothing)
        w = np.where(l == most, 1.0, np.where(np.isinf(l - most), 0.0, np.exp((l - most) / np.float64(t))))
    w = w[order]
    if k > 0:
        w = w[:k]
    if p < 1:
        w = w[:np.searchsorted(np.cumsum(w), p * w.sum()) + 1]
    if least > 0:
        w = w[:max(1, int((w >= np.float64(least)).sum()))]
    running = np.cumsum(w)
    target = (u if u >= 0 else 0.0) * running[-1]
    at = np.searchsorted(running, target, side="right") if target < running[-1] else int((w > 0).sum()) - 1
    return int(order[at]), w[at] / running[-1]


def run(cas, logits, u, t=None, k=None, p=None, least=None, stream=None):
    import torch
    rows = len(logits)

    def dev(v, dt):
        return None if v is None else torch.as_tensor(np.broadcast_to(np.asarray(v), (rows,)).copy()).to(dt).cuda()

    args = dict(temperature=dev(t, torch.float32), top_k=dev(k, torch.int32), top_p=dev(p, torch.float32), min_p=dev(least, torch.float32))
    uu = dev(u, torch.float32)
    token, prob = torch.full((rows,), -7, device="cuda", dtype=torch.int32), torch.full((rows,), -7.0, device="cuda")
    ws = cas.new_workspace(cas.cascade_sample_workspace_bytes(rows, logits.shape[1], logits.dtype))
    ws.fill_(0xa5)
    torch.cuda.synchronize()
    cas.cascade_sample(logits, uu, token, prob=prob, workspace=ws, stream=stream, **args)
    torch.cuda.synchronize()
    host = [np.full(rows, d, np.float32) if v is None else v.cpu().numpy() for v, d in zip(args.values(), (1.0, 0, 1.0, 0.0))]
    l, uh = logits.float().cpu().numpy(), uu.cpu().numpy()
    for r in range(rows):
        want = reference(l[r], uh[r], host[0][r], int(host[1][r]), host[2][r], host[3][r])
        got = (int(token[r]), float(prob[r]))
        assert got[0] == want[0], (r, got, want, [h[r] for h in host], uh[r])
        assert abs(got[1] - want[1]) <= 2.0 ** -22 * want[1], (r, got, want)
    return token, prob


def make(rows, V, dtype, seed=0, spread=2.5):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    return (spread * torch.randn((rows, V), device="cuda", generator=g)).to(dt), np.random.default_rng(seed)


VOCABS = [1, 2, 3, 7, 8, 9, 100, 1023, 1025, 8191, 8193, 50257, 128256, 131077]


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sizes_and_settings(cas, V, dtype):
    rows = 24
    logits, rng = make(rows, V, dtype, seed=V)
    u = rng.random(rows)
    run(cas, logits, u)
    run(cas, logits, u, t=rng.choice([0.0, 0.5, 1.0, 1.7], rows), k=rng.choice([0, 1, 2, 50, 900, 5000, V, V + 3, -4], rows),
        p=rng.choice([1.0, 0.99, 0.9, 0.5, 0.01], rows), least=rng.choice([0.0, 0.001, 0.05, 0.5, 1.0], rows))
    run(cas, logits, u, t=0.8, k=50, p=0.95)
    run(cas, logits, u, k=min(V, 3000))
    run(cas, logits, u, p=0.999)
    run(cas, logits, u, least=0.0005)


@pytest.mark.parametrize("V", [5, 3000, 70001])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_flat_rows_have_borders_inside_full_bins(cas, V, dtype):
    rows = 12
    logits, rng = make(rows, V, dtype, seed=V + 1)
    u = rng.random(rows)
    for t in (20.0, 1000.0, float("inf")):
        run(cas, logits, u, t=t)
        run(cas, logits, u, t=t, k=V // 2 + 1, p=0.7)
        run(cas, logits, u, t=t, k=V // 3 + 1, least=0.9)
        run(cas, logits, u, t=t, p=0.4, least=0.97)
        run(cas, logits, u, t=t, k=2, p=0.1)


@pytest.mark.parametrize("V", [4, 1500, 40000, 128256])
@pytest.mark.parametrize("values", [1, 2, 5])
def test_rows_of_few_values(cas, V, values):
    """Ties by the thousand: the lowest index first."""
    import torch
    rng = np.random.default_rng(V + values)
    for dtype in (torch.bfloat16, torch.float32):
        logits = torch.from_numpy(rng.choice(np.array([-2.0, 0.0, 0.5, 1.0, 3.0])[:values], (9, V))).to(dtype).cuda()
        u = np.array([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 0.1, 0.3, 0.9, 0.99])
        run(cas, logits, u)
        run(cas, logits, u, k=V // 2 + 1)
        run(cas, logits, u, p=0.5)
        run(cas, logits, u, t=0.3, k=V // 2 + 1, p=0.77, least=0.2)


def test_minus_zero_ties_with_zero(cas):
    import torch
    logits = torch.full((4, 3000), -1e4, device="cuda")
    logits[:, 10], logits[:, 20], logits[:, 30] = 0.0, -0.0, 0.0
    for u, want in ((0.0, 10), (0.4, 20), (0.9, 30)):
        token, _ = run(cas, logits, u)
        assert (token == want).all()
    run(cas, logits, 0.7, k=2)


def test_values_next_to_zero_on_either_side(cas):
    """Windows of finer bins that end right below zero."""
    import torch
    for least in (-1e-40, -1e-45, 1e-45):
        logits = torch.full((6, 2600), -5.0, device="cuda")
        logits[:, 100:1300:2] = 0.0
        logits[:, 101:1301:2] = least
        logits[3:, 1300:2500] = least
        logits[:, 120] = -0.0
        for u in (0.05, 0.2, 0.3, 0.45, 0.6, 0.9):
            run(cas, logits, u, t=float("inf"))
            run(cas, logits, u, t=float("inf"), k=700)
            run(cas, logits, u, t=1e30, p=0.3)


@pytest.mark.parametrize("t", [1e-30, 1e-6, 1e-3, 1e30, 1.4e-45, float("nan"), -1.0, 0.0, float("inf")])
def test_temperatures(cas, t):
    import torch
    for dtype in ("bf16", "f32"):
        logits, rng = make(8, 5000, dtype, seed=2)
        logits[:4, 77] = logits[:4].amax(1)                # a tie at the top
        run(cas, logits, rng.random(8), t=t)
        run(cas, logits, rng.random(8), t=t, k=3, p=0.9, least=0.1)
    big = torch.tensor([[3e38, 2.9e38, -3e38, 3e38]] * 3, device="cuda")
    run(cas, big, [0.1, 0.6, 0.9], t=t)


@pytest.mark.parametrize("u", [0.0, 2.0 ** -30, 1 - 2.0 ** -24, 1.0, 5.0, -1.0, float("nan"), float("inf")])
def test_uniforms_at_and_behind_the_ends(cas, u):
    logits, _ = make(6, 2000, "bf16", seed=3)
    run(cas, logits, u)
    run(cas, logits, u, k=5)
    run(cas, logits, u, t=200.0, p=0.9)
    logits, _ = make(2, 40000, "f32", seed=3, spread=0.1)
    run(cas, logits, u)


@pytest.mark.parametrize("setting", [dict(p=0.0), dict(p=-1.0), dict(p=float("nan")), dict(p=2.0), dict(p=1e-9), dict(least=float("nan")), dict(least=-1.0),
                                     dict(least=1.0), dict(least=2.0), dict(least=float("inf")), dict(least=1e-38), dict(k=-(1 << 31)), dict(k=(1 << 31) - 1),
                                     dict(k=1), dict(k=1, p=0.0, least=2.0)])
def test_settings_at_and_behind_their_ends(cas, setting):
    for V, spread in ((3000, 2.5), (40000, 0.05)):
        logits, rng = make(6, V, "f32", seed=4, spread=spread)
        run(cas, logits, rng.random(6), **setting)


def test_masked_rows(cas):
    import torch
    inf, nan = float("inf"), float("nan")
    for V in (50, 9000):
        for dtype in (torch.bfloat16, torch.float32):
            lowest = torch.finfo(dtype).min
            logits = torch.full((9, V), -inf, device="cuda", dtype=dtype)
            logits[1] = nan
            logits[2, 3::7] = nan                          # nothing to choose in rows 0 .. 2
            logits[3, V - 1] = 1.0
            logits[4, 5:9] = torch.tensor([1.0, 2.0, 2.0, nan], dtype=dtype)
            logits[5] = lowest
            logits[6] = lowest
            logits[6, 40] = -3.0
            logits[7, 11] = inf
            logits[7, 30] = inf
            logits[7, 12] = 100.0
            logits[8, 30:] = -torch.finfo(dtype).tiny
            for u in (0.0, 0.3, 0.8):
                run(cas, logits, u)
                run(cas, logits, u, k=3, p=0.9, least=0.05)
                run(cas, logits, u, t=0.0)
                run(cas, logits, u, t=inf)
                run(cas, logits, u, t=1e-40)


def test_infinities_by_the_thousand(cas):
    import torch
    logits = torch.randn((3, 20000), device="cuda")
    logits[:, 100:9000] = float("inf")
    run(cas, logits, [0.1, 0.5, 0.99])
    run(cas, logits, [0.1, 0.5, 0.99], k=5000, p=0.7, least=0.5)


def test_strides_and_addresses_off_any_boundary(cas):
    import torch
    for dtype in (torch.bfloat16, torch.float32):
        for V in (5, 4001, 33000):
            big = (2.5 * torch.randn(7 * (V + 5) + 3, device="cuda")).to(dtype)
            logits = big[3:].view(7, V + 5)[:, :V]
            u = np.random.default_rng(V).random(7)
            run(cas, logits, u, p=0.9)
            run(cas, logits, u, t=30.0)


def test_offsets_beyond_32_bits(cas):
    import torch
    V, stride = 50257, (1 << 31) + 64
    for dtype in (torch.bfloat16, torch.float32):
        room = torch.empty(2 * stride + V, device="cuda", dtype=dtype)
        logits = room.as_strided((3, V), (stride, 1))
        logits.copy_(2.5 * torch.randn((3, V), device="cuda"))
        run(cas, logits, [0.2, 0.6, 0.9], p=0.9)
        run(cas, logits, [0.2, 0.6, 0.9], t=[0.0, 1.0, 30.0])


def test_many_rows(cas):
    logits, rng = make(3000, 700, "f32", seed=6)
    run(cas, logits, rng.random(3000), t=rng.choice([0.0, 0.7, 1.0], 3000), k=rng.choice([0, 40], 3000), p=rng.choice([0.9, 1.0], 3000))
    logits, rng = make(300, 40000, "bf16", seed=7)         # large chunks
    run(cas, logits, rng.random(300), t=rng.choice([0.0, 0.7, 1.0], 300), k=rng.choice([0, 40], 300), p=rng.choice([0.9, 1.0], 300))


def test_largest_vocabulary(cas):
    logits, rng = make(2, 1 << 20, "f32", seed=8)
    run(cas, logits, rng.random(2), p=0.9)
    run(cas, logits, rng.random(2), t=50.0)


def test_a_row_has_the_same_token_whatever_the_others(cas):
    import torch
    logits, rng = make(400, 20000, "bf16", seed=9)
    u = rng.random(400)
    token, prob = run(cas, logits, u, p=0.95, t=1.3)
    few, fprob = run(cas, logits[17:20].clone(), u[17:20], p=0.95, t=1.3)
    assert torch.equal(token[17:20], few) and torch.equal(prob[17:20], fprob)


def test_greedy_rows_are_cascade_greedy_token(cas):
    import torch
    for dtype in ("bf16", "f32"):
        logits, _ = make(40, 30011, dtype, seed=10)
        a, b = torch.empty(40, device="cuda", dtype=torch.int32), torch.empty(40, device="cuda", dtype=torch.int32)
        cas.cascade_greedy_token(logits, a)
        ws = cas.new_workspace(cas.cascade_sample_workspace_bytes(40, 30011, logits.dtype))
        cas.cascade_sample(logits, torch.rand(40, device="cuda"), b, temperature=torch.zeros(40, device="cuda"), workspace=ws)
        assert torch.equal(a, b)


def test_shares_of_tokens(cas):
    """Evenly spaced random numbers give every token its share to one part in their number."""
    import torch
    V, n = 50, 4096
    logits, _ = make(1, V, "f32", seed=11, spread=1.0)
    token, _ = run(cas, logits.expand(n, V).contiguous(), (np.arange(n) + 0.5) / n)
    got = torch.bincount(token.long(), minlength=V).double() / n
    assert (got - logits[0].double().softmax(0)).abs().max().item() <= 1.0 / n


def test_no_rows_and_other_stream(cas):
    import torch
    logits, rng = make(5, 9000, "bf16", seed=12)
    cas.cascade_sample(logits[:0], torch.empty(0, device="cuda"), torch.empty(0, device="cuda", dtype=torch.int32))
    run(cas, logits, rng.random(5), p=0.9, stream=torch.cuda.Stream())


def test_binding_refuses(cas):
    import torch
    logits, _ = make(4, 100, "bf16")
    u, token = torch.rand(4, device="cuda"), torch.empty(4, device="cuda", dtype=torch.int32)
    ws = cas.new_workspace(cas.cascade_sample_workspace_bytes(4, 100, logits.dtype))

    def refused(logits=logits, u=u, token=token, ws=ws, **kw):
        with pytest.raises(cas.CascadeError):
            cas.cascade_sample(logits, u, token, workspace=ws, **kw)

    refused(logits=logits.half())
    refused(logits=logits.t())
    refused(logits=logits[:1].expand(4, 100))
    refused(logits=logits.cpu())
    refused(u=u[:3])
    refused(u=u.double())
    refused(token=token.long())
    refused(ws=None)
    refused(ws=ws[:-1])
    refused(temperature=u[:2])
    refused(top_k=u)
    refused(prob=u.double())

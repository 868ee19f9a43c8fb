"""Tokens from logits at the ends of the settings: a top_p that is no number behind a top_k that cuts, random numbers of 1 and more,
weights too small for the bins.  Tolerances as in test_gpu_sample."""
import numpy as np
import pytest

from test_gpu_sample import make, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cas():
    import torch
    assert torch.cuda.is_available()
    import paper_2507_05228_amd as cas
    cas.load_library()
    return cas


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,spread,k", [(40000, 0.05, 5000), (40000, 0.05, 39999), (128256, 0.01, 1025), (9000, 2.5, 8000), (3000, 0.05, 50), (40000, 0.05, 0)])
@pytest.mark.parametrize("least", [None, 0.0, 0.97, float("nan")])
def test_top_p_that_is_no_number_is_off(cas, dtype, V, spread, k, least):
    import torch
    logits, rng = make(6, V, dtype, seed=V + k, spread=spread)
    u = rng.random(6)
    token, prob = run(cas, logits, u, k=k, p=float("nan"), least=least)
    off, off_prob = run(cas, logits, u, k=k, p=1.0, least=least)
    assert torch.equal(token, off) and torch.equal(prob, off_prob)


@pytest.mark.parametrize("u", [1.0, 1.0 + 2.0 ** -23, 7.0, float("inf")])
def test_a_random_number_of_one_takes_the_last_place(cas, u):
    """A few large weights and many below the last bit of their sum: running sums in fixed trees are not monotone there, and the
    last one is not the largest."""
    import torch
    rows, V, tiny = 300, 700, 90
    g = np.random.default_rng(0)
    logits = np.full((rows, V), -np.inf, np.float32)
    for r in range(rows):
        n = int(g.integers(3, 40))
        at = g.permutation(V)[:n + tiny]
        logits[r, at] = np.concatenate([g.normal(size=n), g.uniform(-38.0, -36.2, tiny)])
    logits = torch.from_numpy(logits).cuda()
    run(cas, logits, u)
    run(cas, logits, u, k=60)
    run(cas, logits, u, least=1e-18)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [500, 40000])
@pytest.mark.parametrize("setting", [dict(), dict(k=300), dict(p=0.999), dict(least=1e-25), dict(t=0.25, k=450, least=1e-30)])
def test_weights_below_the_bins_count_as_none(cas, dtype, V, setting):
    """Finite logits 50 to 100 temperatures below the largest are as if they were -inf, for random numbers of 1 and more too."""
    import torch
    logits, rng = make(8, V, dtype, seed=V, spread=1.0)
    t = setting.get("t", 1.0)
    logits = torch.where(logits < 0.5, t * (logits.amax(1, keepdim=True).float() - 75 - 3 * logits.float()), t * logits.float()).to(logits.dtype)
    most = logits.amax(1, keepdim=True).float()
    below = (most - logits.float()) / t
    assert ((below < 20) | (below > 50)).all()             # none near the bins' end
    cut = torch.where(below > 50, float("-inf"), logits.float()).to(logits.dtype)
    for u in (0.3, 0.999, 1.0, 3.0, float("inf")):
        want = run(cas, cut, u, **setting)
        rows = len(logits)
        token, prob = torch.empty(rows, device="cuda", dtype=torch.int32), torch.empty(rows, device="cuda")
        dev = {name: None if key not in setting else torch.full((rows,), setting[key], device="cuda", dtype=torch.int32 if key == "k" else torch.float32)
               for name, key in (("temperature", "t"), ("top_k", "k"), ("top_p", "p"), ("min_p", "least"))}
        cas.cascade_sample(logits, torch.full((rows,), u, device="cuda"), token, prob=prob,
                           workspace=cas.new_workspace(cas.cascade_sample_workspace_bytes(rows, V, logits.dtype)), **dev)
        assert torch.equal(token, want[0]) and torch.equal(prob, want[1])


@pytest.mark.parametrize("most,few,V", [(65, 64, 128256), (200, 146, 50257), (300, 1, 32000)])
def test_a_workspace_for_many_rows_serves_fewer(cas, most, few, V):
    import torch
    logits, rng = make(few, V, "bf16", seed=V)
    u, t = torch.from_numpy(rng.random(few)).float().cuda(), torch.full((few,), 0.7, device="cuda")
    results = []
    for rows in (most, few):
        token, prob = torch.empty(few, device="cuda", dtype=torch.int32), torch.empty(few, device="cuda")
        cas.cascade_sample(logits, u, token, temperature=t, prob=prob, workspace=cas.new_workspace(cas.cascade_sample_workspace_bytes(rows, V, logits.dtype)))
        results.append((token, prob))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])

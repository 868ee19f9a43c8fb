"""Tokens from logits at the ends of the settings: a top_p that is no number behind a top_k that cuts, random numbers of 1 and more.
Tolerances as in test_gpu_sample."""
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

"""Tokens from logits at the ends of the settings: a top_p that is no number behind a top_k that cuts.
Tolerances as in test_gpu_sample."""
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

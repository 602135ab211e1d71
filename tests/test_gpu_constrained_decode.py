"""The example that runs the operators together with the framework's step."""
import pytest
import torch

from paper_2605_15609_b200.examples import constrained_decode as ex

pytestmark = pytest.mark.gpu


def test_every_slot_gets_a_legal_token_and_the_cache_stays_in_its_budget():
    B, blocks, budget = 3, 6, 64
    out, cache, legal, passes = ex.decode(B=B, D=3, blocks=blocks, budget=budget, V=1000, seed=3)
    assert out.shape == (B, blocks * ex.M) and bool((out >= 0).all()) and bool((out < 1000).all())
    assert bool(legal[out.long()].all())
    assert cache.n <= budget + 2 * ex.M and cache.length.tolist() == [cache.n] * B
    w = cache.weight[:, :, :cache.n]
    assert bool(torch.isfinite(w).all()) and bool((w >= 0).all()) and float(w.sum()) > 0
    assert passes < blocks * 2 * ex.M                 # several tokens per pass


def test_the_same_decode_again():
    a = ex.decode(B=2, D=4, blocks=3, budget=48, V=700, seed=5)
    b = ex.decode(B=2, D=4, blocks=3, budget=48, V=700, seed=5)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1].k[:, :a[1].n], b[1].k[:, :b[1].n])

"""Rows without a token (token < 0, as psd_confidence_logits writes them) in the policy, the drafts and the acceptance: parity
with the oracle on random states in which many predictions are missing, and the chain from masked logits to the commit."""
import numpy as np
import pytest
import torch

import oracle
import paper_2605_15609_b200 as psd
from paper_2605_15609_b200.examples import constrained_decode as ex
from psd_testlib import GpuChain, dev, f32, np_

pytestmark = pytest.mark.gpu
MASK_ID = 70000


def _case(seed, B, M, missing):
    rng = np.random.default_rng(seed)
    tok = rng.integers(0, 60000, size=(B, M)).astype(np.int32)
    conf = rng.random((B, M)).astype(np.float32)
    none = rng.random((B, M)) < missing
    tok[none] = -1 - rng.integers(0, 3, size=int(none.sum()))       # any negative token
    conf[none & (rng.random((B, M)) < 0.7)] = 0.0                   # (with a confidence of 0, mostly)
    mask = (rng.random((B, M)) < 0.7).astype(np.int32)
    tok[0], mask[0] = -1, 1                                          # a block of dead ends
    tokens = np.where(mask == 1, MASK_ID, rng.integers(0, 60000, size=(B, M))).astype(np.int32)
    return conf, tok, tokens, mask, rng


def _pols(tau, k_min, k_max, D, mode):
    kw = dict(tau=f32(tau), k_min=k_min, k_max=k_max, depth=D, accept_mode=mode, mask_id=MASK_ID)
    return oracle.Policy(**kw), psd.policy(**kw)


@pytest.mark.parametrize("B,M", [(3, 1), (6, 33), (4, 64), (2, 200)])
@pytest.mark.parametrize("missing", [0.2, 0.9])
@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("tau,k_min,k_max,D", [(0.6, 1, 0, 4), (-1.0, 2, 3, 6), (0.99, 8, 0, 3)])
def test_stages_against_the_oracle(B, M, missing, mode, tau, k_min, k_max, D):
    po, pg = _pols(tau, k_min, k_max, D, mode)
    conf, tok, tokens, mask, rng = _case(B * 1000 + M + D, B, M, missing)
    g = GpuChain(B, M, D)
    t, m = dev(tokens), dev(mask)
    psd.psd_select_unmask(dev(conf), dev(tok), t, m, pg, g.sel, g.n_sel, g.sel_pos)
    want = oracle.select_unmask(conf, tok, tokens, mask, po)
    for w, x in zip(want, (t, m, g.sel, g.n_sel, g.sel_pos)):
        assert np.array_equal(w, np_(x))
    assert int(want[3][0]) == 0 and want[1][0].all()                # nothing to commit: the block is as it was
    tokens, mask = want[:2]
    psd.psd_build_drafts(dev(conf), dev(tok), t, m, pg, g.sigma, g.n_fill, g.draft_tokens, g.draft_mask)
    drafts = oracle.build_drafts(conf, tok, tokens, mask, po)
    for w, x in zip(drafts, (g.sigma, g.n_fill, g.draft_tokens, g.draft_mask)):
        assert np.array_equal(w, np_(x))
    assert (drafts[2] >= 0).all()
    # a verifier that mostly agrees, and has no token here and there
    tokV = np.repeat(tok[:, None], D, 1)
    tokV[rng.random(tokV.shape) < 0.1] += 1
    tokV[rng.random(tokV.shape) < 0.2 * missing] = -1
    tokV = tokV.astype(np.int32)
    confV = (rng.random((B, D, M)) ** 0.25).astype(np.float32)
    tV, cV = dev(tokV), dev(confV)
    psd.psd_verify_accept(tV, cV, g.sigma, g.n_fill, g.draft_tokens, g.draft_mask, pg, g.tokens_out, g.mask_out, g.k_star, g.n_spec,
                          g.n_comm, g.accepted)
    want = oracle.verify_accept(tokV, confV, *drafts, po)
    for w, x in zip(want, (g.tokens_out, g.mask_out, g.k_star, g.n_spec, g.n_comm, g.accepted)):
        assert np.array_equal(w, np_(x))
    assert (want[0] >= 0).all()
    # drafts made elsewhere, in which some filled slots hold no token: a verifier without one there does not agree
    bad = (rng.random((B, 1, M)) < 0.2) & (mask[:, None] == 1) & (drafts[3] == 0)
    dt2, tokV2 = np.where(bad, -1, drafts[2]).astype(np.int32), np.where(bad.any(1, keepdims=True), -1, tokV).astype(np.int32)
    psd.psd_verify_accept(dev(tokV2), cV, g.sigma, g.n_fill, dev(dt2), g.draft_mask, pg, g.tokens_out, g.mask_out, g.k_star,
                          g.n_spec, g.n_comm, g.accepted)
    for w, x in zip(oracle.verify_accept(tokV2, confV, *drafts[:2], dt2, drafts[3], po),
                    (g.tokens_out, g.mask_out, g.k_star, g.n_spec, g.n_comm, g.accepted)):
        assert np.array_equal(w, np_(x))
    # the same drafts as a graph
    ranks = oracle.chain_as_dag(D, po.step)
    dag = psd.psd_dag_init(ranks)
    g2 = GpuChain(B, M, D)
    psd.psd_build_drafts_dag(dev(conf), dev(tok), t, m, pg, dag, g2.sigma, g2.n_fill, g2.draft_tokens, g2.draft_mask)
    psd.psd_verify_accept_dag(tV, cV, g2.sigma, g2.draft_tokens, g2.draft_mask, pg, dag, g2.tokens_out, g2.mask_out, g2.k_star,
                              g2.n_spec, g2.n_comm, g2.accepted)
    drafts = oracle.build_drafts_dag(conf, tok, tokens, mask, po, ranks)
    want = oracle.verify_accept_dag(tokV, confV, drafts[0], *drafts[2:], po, ranks)
    for w, x in zip((*drafts, *want), (g2.sigma, g2.n_fill, g2.draft_tokens, g2.draft_mask, g2.tokens_out, g2.mask_out, g2.k_star,
                                       g2.n_spec, g2.n_comm, g2.accepted)):
        assert np.array_equal(w, np_(x))


@pytest.mark.parametrize("k_min", [1, 3, 8])
def test_from_masked_logits_to_the_state(k_min):
    """Slots whose grammar allows nothing stay masked whatever k_min asks for."""
    M, V = 8, 500
    lg = torch.randn(M, V, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    allow = torch.full((M, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
    dead = [0, 2, 3, 6, 7]
    allow[dead] = 0
    tok, conf = torch.zeros(1, M, dtype=torch.int32, device="cuda"), torch.zeros(1, M, device="cuda")
    ws = torch.empty(psd.psd_logits_workspace_bytes(M, V), dtype=torch.uint8, device="cuda")
    psd.psd_confidence_logits(lg, tok, conf, M=M, allow=allow, workspace=ws)
    tokens, mask = torch.full((1, M), V, dtype=torch.int32, device="cuda"), torch.ones(1, M, dtype=torch.int32, device="cuda")
    g = GpuChain(1, M, 4)
    for _ in range(4):
        psd.psd_select_unmask(conf, tok, tokens, mask, psd.policy(tau=0.9, k_min=k_min), g.sel, g.n_sel, g.sel_pos)
    assert mask[0].tolist() == [int(i in dead) for i in range(M)] and int(g.n_sel[0]) == 0
    assert tokens[0, dead].tolist() == [V] * len(dead) and bool((tokens >= 0).all())


def test_the_example_stops_at_a_dead_end():
    with pytest.raises(RuntimeError, match="grammar"):
        ex.decode(B=2, D=3, blocks=1, budget=64, V=300, allowed=0.0)

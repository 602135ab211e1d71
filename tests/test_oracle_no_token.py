"""A prediction without a token (token < 0: psd_confidence_logits' answer for a row in which nothing may be chosen) is no
candidate: it is not committed, not speculated, agrees with nothing and is not counted.  The oracle, on the CPU."""
import numpy as np
import pytest

import oracle

M = 6
MASK = 900


def _state():
    """Slots 0, 2 committed; of the masked slots 1, 3, 4, 5 slots 1 and 4 have no token."""
    tokens = np.array([[10, MASK, 12, MASK, MASK, MASK]], np.int32)
    mask = np.array([[0, 1, 0, 1, 1, 1]], np.int32)
    tok = np.array([[1, -1, 3, 40, -1, 60]], np.int32)
    conf = np.array([[0.9, 0.0, 0.9, 0.2, 0.0, 0.3]])
    return tokens, mask, tok, conf


@pytest.mark.parametrize("k_min,tau", [(1, 0.9), (3, 0.9), (6, 0.9), (1, -1.0)])
def test_select_commits_only_slots_with_a_token(k_min, tau):
    tokens, mask, tok, conf = _state()
    t, m, sel, n_sel, pos = oracle.select_unmask(conf, tok, tokens, mask, oracle.Policy(tau=tau, k_min=k_min, mask_id=MASK))
    n = 1 if (k_min, tau) == (1, 0.9) else 2
    assert n_sel[0] == n and pos[0].tolist() == [5, 3][:n] + [-1] * (M - n)
    assert m[0].tolist() == [0, 1, 0, int(n < 2), 1, 0] and t[0].tolist() == [10, MASK, 12, MASK if n < 2 else 40, MASK, 60]
    assert sel[0].sum() == n


def test_select_with_dead_ends_only_leaves_the_block_alone():
    tokens, mask, tok, conf = _state()
    t, m, sel, n_sel, pos = oracle.select_unmask(conf, np.full_like(tok, -1), tokens, mask, oracle.Policy(k_min=4, tau=-1.0))
    assert n_sel[0] == 0 and np.array_equal(t, tokens) and np.array_equal(m, mask) and (pos == -1).all() and (sel == 0).all()


def _drafts(p, dag):
    tokens, mask, tok, conf = _state()
    if dag:
        return oracle.build_drafts_dag(conf, tok, tokens, mask, p, oracle.chain_as_dag(p.depth, p.step))
    return oracle.build_drafts(conf, tok, tokens, mask, p)


@pytest.mark.parametrize("dag", [False, True])
def test_drafts_speculate_only_slots_with_a_token(dag):
    sigma, n_fill, dt, dm = _drafts(oracle.Policy(depth=5, k_min=1), dag)
    assert sigma[0].tolist() == [5, 3, -1, -1, -1, -1] and n_fill[0].tolist() == [0, 1, 2, 2, 2]
    assert (dt >= 0).all() and dm[0, :, 1].all() and dm[0, :, 4].all() and dm[0, 4].tolist() == [0, 1, 0, 0, 1, 0]


@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("dag", [False, True])
def test_acceptance_takes_no_missing_token(mode, dag):
    """The verifier has no token for slot 3 on the node before it is filled, nor for slots 1 and 4 anywhere; a threshold below
    every confidence commits none of them."""
    p = oracle.Policy(tau=-1.0, depth=3, k_min=1, accept_mode=mode, mask_id=MASK)
    sigma, n_fill, dt, dm = _drafts(p, dag)
    tokV = np.array([[[1, -1, 3, 40, -1, 60], [1, -1, 3, -1, -1, 60], [1, 5, 3, 40, -1, 60]]], np.int32)
    confV = np.full((1, 3, M), 0.5)
    if dag:
        t, m, ks, ns, nc, acc = oracle.verify_accept_dag(tokV, confV, sigma, dt, dm, p, oracle.chain_as_dag(3, 1))
        # (the graph has the edge root -> node 2 as well, and the root does predict slot 3)
        want = (2, 2, 3, [1, 1, 1], [10, 5, 12, 40, MASK, 60], [0, 0, 0, 0, 1, 0])
    else:
        t, m, ks, ns, nc, acc = oracle.verify_accept(tokV, confV, sigma, n_fill, dt, dm, p)
        want = (1, 1, 1, [1, 1, 0], [10, MASK, 12, MASK, MASK, 60], [0, 1, 0, 1, 1, 0])
    assert (int(ks[0]), int(ns[0]), int(nc[0]), acc[0].tolist(), t[0].tolist(), m[0].tolist()) == want


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_a_draft_that_holds_no_token_agrees_with_nothing(mode):
    """Drafts made elsewhere: -1 in a filled slot is not accepted by a verifier that says -1."""
    p = oracle.Policy(tau=-1.0, depth=2, k_min=1, accept_mode=mode, mask_id=MASK)
    sigma, n_fill = np.array([[0, -1]], np.int32), np.array([[0, 1]], np.int32)
    dt, dm = np.array([[[MASK, MASK], [-1, MASK]]], np.int32), np.array([[[1, 1], [0, 1]]], np.int32)
    tokV, confV = np.array([[[-1, 7], [-1, 7]]], np.int32), np.full((1, 2, 2), 0.5)
    t, m, ks, ns, nc, acc = oracle.verify_accept(tokV, confV, sigma, n_fill, dt, dm, p)
    assert int(ks[0]) == 0 and acc[0].tolist() == [1, 0] and t[0].tolist() == [MASK, 7] and m[0].tolist() == [1, 0] and int(nc[0]) == 1
    t, m, ks, ns, nc, acc = oracle.verify_accept_dag(tokV, confV, sigma, dt, dm, p, [set(), {0}])
    assert int(ks[0]) == 0 and acc[0].tolist() == [1, 0] and t[0].tolist() == [MASK, 7] and m[0].tolist() == [1, 0] and int(nc[0]) == 1

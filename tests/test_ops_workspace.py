"""Workspace sizes of the operators around the step grow with what changes while a service runs, so that a workspace made for its
largest batch serves the smaller ones.  (No GPU: sizes only.)"""
import random

import pytest

import paper_2605_15609_b200 as psd

HEADS = [(32, 8, 128), (28, 4, 128), (4, 4, 64), (8, 2, 64), (128, 1, 96), (16, 16, 64), (2, 1, 8)]


def test_a_batch_that_shrinks():
    """Sizes that a service meets while its sequences finish: 4 drafts of 32 tokens, 32 heads over 8 key heads of 128."""
    a = [psd.psd_attention_workspace_bytes(B, 4, 32, 32, 8, 128, 2000, 32) for B in (16, 8, 4, 2, 1)]
    assert a == sorted(a, reverse=True)
    a = [psd.psd_attention_workspace_bytes(1, 4, 32, 32, 8, 128, P, 32) for P in (2000, 513, 512, 257, 1, 0)]
    assert a == sorted(a, reverse=True)
    a = [psd.psd_weights_workspace_bytes(B, 4, 32, 32, 8, 128, 1000) for B in (8, 4, 2, 1)]
    assert a == sorted(a, reverse=True)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("M", [1, 2, 7, 16, 32, 64, 150])
def test_attention_grows_with_batch_drafts_and_lengths(heads, M):
    r = random.Random(hash((heads, M)) & 0xffff)
    for _ in range(400):
        big = [int(2 ** r.uniform(0, 7)), int(2 ** r.uniform(0, 5)), int(2 ** r.uniform(0, 15)) - 1, int(2 ** r.uniform(0, 11)) - 1]
        small = [r.choice((x, r.randint(lo, x))) for x, lo in zip(big, (1, 1, 0, 0))]
        w = [psd.psd_attention_workspace_bytes(B, D, M, *heads, P, S) for B, D, P, S in (big, small)]
        assert w[0] >= w[1] >= 256, (big, small, w)


@pytest.mark.parametrize("heads", HEADS)
def test_prefix_weights_grow_with_all_sizes(heads):
    r = random.Random(heads[0])
    for _ in range(2000):
        big = [int(2 ** r.uniform(0, 7)), int(2 ** r.uniform(0, 5)), int(2 ** r.uniform(0, 9)), int(2 ** r.uniform(0, 15))]
        small = [r.choice((x, r.randint(1, x))) for x in big]
        w = [psd.psd_weights_workspace_bytes(B, D, M, *heads, P) for B, D, M, P in (big, small)]
        assert w[0] >= w[1] >= 256, (big, small, w)


def test_logits_grow_with_rows_and_vocabulary():
    r = random.Random(1)
    for _ in range(2000):
        big = [int(2 ** r.uniform(0, 14)), int(2 ** r.uniform(0, 18))]
        small = [r.choice((x, r.randint(1, x))) for x in big]
        w = [psd.psd_logits_workspace_bytes(*x) for x in (big, small)]
        assert w[0] >= w[1] > 0, (big, small, w)


def test_sizes_stay_near_what_is_used():
    """A split form's partial results: two tiles of 128 rows per SM at most, 129 words a row."""
    assert psd.psd_attention_workspace_bytes(16, 8, 64, 32, 8, 128, 8192, 64) <= 148 * 256 * 129 * 4 + 256
    assert psd.psd_weights_workspace_bytes(16, 8, 64, 32, 8, 128, 8192) <= 148 * 256 * 4 + 256
    assert psd.psd_attention_workspace_bytes(1, 4, 32, 4, 4, 64, 257, 32) == 256


def test_logits_workspace_stays_near_what_is_used():
    """One record of 16 bytes per row and warp: 31 warps of 4096 columns for a row of 126464 in a large batch (it was 558 records)."""
    assert psd.psd_logits_workspace_bytes(8192, 126464) <= 8192 * 3 * 31 * 16
    assert psd.psd_logits_workspace_bytes(1, 126464) <= 558 * 16 + 256

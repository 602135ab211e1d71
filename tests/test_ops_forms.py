"""Which form the drafts' attention takes at shapes where both sides were measured (no GPU: names only).  us: the form named here
against the other."""
import pytest

import paper_2605_15609_b200 as psd

ONE, FUSED, JOINED = "draft_attention_kernel", "prefix_attention_kernel", "prefix_attention_kernel+draft_attention_kernel"

MEASURED = [  # B, D, M, Hq, Hkv, Dh, P, S
    # short prefixes, few rows: one launch
    ((1, 4, 32, 4, 4, 64, 257, 32), ONE), ((1, 4, 32, 4, 4, 64, 1024, 32), ONE), ((1, 4, 32, 32, 8, 128, 512, 32), ONE),        # 7:15 14:17 18:20
    ((16, 1, 1, 32, 8, 128, 512, 32), ONE), ((8, 8, 4, 16, 2, 128, 257, 8), ONE), ((1, 4, 2, 32, 8, 128, 257, 2), ONE),         # 14:17 14:24 11:14
    ((5, 4, 33, 16, 16, 64, 64, 33), ONE), ((40, 8, 4, 32, 4, 128, 64, 4), ONE), ((5, 4, 33, 16, 16, 128, 64, 33), ONE),        # 11:17 35:40 17:18
    # long prefixes, few rows: split
    ((1, 4, 32, 4, 4, 64, 2048, 32), JOINED), ((1, 4, 32, 32, 8, 128, 1024, 32), JOINED), ((1, 1, 1, 32, 8, 128, 1024, 32), JOINED),   # 17:23 22:30 14:23
    # many rows: the own keys behind the prefix, short prefixes among them
    ((4, 4, 32, 32, 8, 128, 128, 32), FUSED), ((16, 4, 32, 32, 8, 128, 64, 32), FUSED), ((16, 4, 32, 32, 8, 128, 128, 32), FUSED),     # 13:26 28:53 28:63
    ((8, 4, 32, 32, 4, 64, 512, 32), FUSED), ((20, 4, 8, 32, 4, 128, 257, 8), FUSED), ((5, 4, 33, 16, 16, 128, 257, 33), FUSED),       # 17:50 20:35 23:30
    ((16, 16, 8, 32, 8, 128, 1024, 32), FUSED), ((16, 16, 4, 32, 8, 128, 1024, 32), FUSED), ((8, 64, 3, 64, 8, 128, 1024, 32), FUSED),  # 71:111 47:61 117:174
    ((8, 64, 2, 64, 8, 128, 1024, 32), FUSED), ((16, 32, 16, 16, 16, 64, 1024, 32), FUSED),                                            # 90:114 154:174
    # more drafts to a tile than pays
    ((16, 32, 12, 16, 16, 64, 1024, 32), JOINED), ((5, 40, 4, 16, 16, 64, 1100, 4), JOINED),                                           # 158:177
]


@pytest.mark.parametrize("shape,form", MEASURED)
def test_the_faster_form_is_taken(shape, form):
    assert psd.psd_attention_kernel_names(*shape)[0] == form


def test_without_a_prefix_there_is_one_form():
    for M, S in ((1, 0), (32, 32), (700, 700)):
        assert psd.psd_attention_kernel_names(16, 8, M, 32, 8, 128, 0, S) == (ONE, 0)


def test_bad_sizes_have_no_form():
    assert psd.psd_attention_kernel_names(0, 1, 1, 1, 1, 8, 1, 1) is None and psd.psd_attention_kernel_names(1, 1, 1, 3, 2, 8, 1, 1) is None

"""Sizes that the library takes in 32 bits: the binding refuses larger ones, which would arrive as other sizes (no GPU; tensors without memory)."""
import pytest
import torch

import paper_2605_15609_b200 as psd
from test_ops_devices import _Elsewhere, launches  # noqa: F401  (a fixture)

FAR = 1 << 32


class _Empty(_Elsewhere):
    def data_ptr(self):
        return 0x10000


def _t(*shape, dtype=torch.bfloat16):
    return _Empty(torch.empty(*shape, dtype=dtype, device="meta"), 0)


def test_rows_of_more_than_32_bits(launches):  # noqa: F811
    args = lambda H: (_t(1, H), _t(1, H, dtype=torch.int8), _t(1, dtype=torch.float32))  # noqa: E731
    psd.psd_quantize_rows(*args(64))
    assert launches == ["psd_quantize_rows"]
    with pytest.raises(ValueError, match="32 bits"):
        psd.psd_quantize_rows(*args(FAR + 64))
    assert launches == ["psd_quantize_rows"]


def test_head_rows_of_more_than_32_bits(launches):  # noqa: F811
    def call(H):
        psd.psd_confidence_q8(_t(2, H), _t(3, H, dtype=torch.int8), _t(3, dtype=torch.float32), _t(2, dtype=torch.int32), _t(2, dtype=torch.float32),
                              workspace=_t(1024, dtype=torch.uint8))
    call(64)
    assert launches == ["psd_confidence_q8"]
    with pytest.raises(ValueError, match="32 bits"):
        call(FAR + 64)
    assert launches == ["psd_confidence_q8"]


def test_blocks_of_more_than_32_bits(launches):  # noqa: F811
    """One scale per key head would be handed to a call that reads one for each 32 tokens."""
    def call(block):
        blocks = -(-100 // block)
        psd.psd_draft_attention_q8(_t(2, 1, 4, 64), *[_t(1, 100, 2, 64, dtype=torch.int8) for _ in "kv"], *[_t(1, 2, blocks, dtype=torch.float32) for _ in "kv"],
                                   _t(2, 1, 4, 64), block=block, workspace=_t(1024, dtype=torch.uint8))
    call(32)
    assert launches == ["psd_draft_attention_q8"]
    with pytest.raises(ValueError, match="32 bits"):
        call(FAR + 32)
    assert launches == ["psd_draft_attention_q8"]


@pytest.mark.parametrize("bad", [dict(rotary=FAR + 64), dict(rotary=64, kind=FAR + 1)])
def test_frequencies_of_more_than_32_bits(bad):
    with pytest.raises(ValueError, match="32 bits"):
        psd.psd_rope_frequencies(**bad)


def test_workspaces_of_more_than_32_bits():
    for i in range(8):
        sizes = [2, 2, 4, 8, 2, 64, 100, 4]
        sizes[i] += FAR
        for f in (psd.psd_attention_q8_workspace_bytes, psd.psd_attention_q8_kernel_names):
            with pytest.raises(ValueError, match="32 bits"):
                f(*sizes)
    for sizes in ((FAR + 4, 128, 100), (4, FAR + 128, 100), (4, 128, FAR + 100)):
        with pytest.raises(ValueError, match="32 bits"):
            psd.psd_confidence_q8_workspace_bytes(*sizes)

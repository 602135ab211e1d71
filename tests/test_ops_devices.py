"""The operators around the step refuse tensors that are not on the current CUDA device, before anything is launched.  (No GPU:
every tensor is on the host, or says that it is elsewhere.)"""
import pytest
import torch

import paper_2605_15609_b200 as psd
from paper_2605_15609_b200 import binding


class _Elsewhere:
    """A tensor's shape, type and strides with another device."""

    def __init__(self, t, device):
        self.t, self.index = t, device

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.index

    @property
    def device(self):
        return f"cuda:{self.index}"


@pytest.fixture
def launches(monkeypatch):
    """What would have been launched; device 0 is current."""
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: seen.append(name) or 0
    monkeypatch.setattr(binding, "LIB", Library())
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    return seen


def _calls():
    h = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    ws = torch.zeros(1024, dtype=torch.uint8)
    return {
        "psd_draft_attention": dict(q=h(4, 2, 4, 64), k_prefix=h(2, 9, 2, 64), v_prefix=h(2, 9, 2, 64), out=h(4, 2, 4, 64),
                                    lse=f(4, 2, 4), k_own=h(4, 3, 2, 64), v_own=h(4, 3, 2, 64), prefix_len=i(2), own_len=i(4),
                                    workspace=ws, status=i(1)),
        "psd_prefix_weights": dict(q=h(4, 2, 4, 64), k_prefix=h(2, 9, 2, 64), lse=f(4, 2, 4), acc_out=f(2, 2, 9), acc_in=f(2, 2, 9),
                                   prefix_len=i(2), workspace=ws, status=i(1)),
        "psd_prefix_evict": dict(scores=f(2, 2, 9), k=h(2, 9, 2, 64), v=h(2, 9, 2, 64), k_out=h(2, 5, 2, 64), v_out=h(2, 5, 2, 64),
                                 index=i(2, 2, 5), scores_out=f(2, 2, 5), len_out=i(2), prefix_len=i(2)),
        "psd_confidence_logits": dict(logits=f(8, 70), out_token=i(8), out_conf=f(8), out_lse=f(8), history=i(2, 6), history_len=i(2),
                                      draft_tokens=i(4, 2), draft_mask=i(4, 2), bias=f(70), allow=i(8, 3), workspace=ws,
                                      status=i(1)),
    }


EXTRA = {"psd_confidence_logits": dict(D=2, M=2, repetition=1.2)}


@pytest.mark.parametrize("name", list(_calls()))
def test_host_tensors_are_refused(name, launches):
    args = _calls()[name]
    with pytest.raises(ValueError, match="device"):
        getattr(psd, name)(**args, **EXTRA.get(name, {}))                  # everything on the host
    for left in args:                                                      # one tensor left on the host
        mixed = {k: t if k == left else _Elsewhere(t, 0) for k, t in args.items()}
        with pytest.raises(ValueError, match="device"):
            getattr(psd, name)(**mixed, **EXTRA.get(name, {}))
    assert launches == []


@pytest.mark.parametrize("name", list(_calls()))
def test_tensors_of_another_device_are_refused(name, launches):
    args = _calls()[name]
    with pytest.raises(ValueError, match="device"):
        getattr(psd, name)(**{k: _Elsewhere(t, 1) for k, t in args.items()}, **EXTRA.get(name, {}))
    for other in args:
        mixed = {k: _Elsewhere(t, int(k == other)) for k, t in args.items()}
        with pytest.raises(ValueError, match="device"):
            getattr(psd, name)(**mixed, **EXTRA.get(name, {}))
    assert launches == []
    getattr(psd, name)(**{k: _Elsewhere(t, 0) for k, t in args.items()}, **EXTRA.get(name, {}))
    assert launches == [name]

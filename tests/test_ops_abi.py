"""Refusals of the operators around the step, on the host, before anything is launched (no GPU)."""
import ctypes

import pytest

import paper_2605_15609_b200 as psd
from paper_2605_15609_b200 import binding

L = binding.LIB
FAKE = 0x10000      # non-NULL and well aligned; never dereferenced


def _att(**kw):
    f = dict(B=2, D=3, M=4, Hq=8, Hkv=2, Dh=64, P=100, S=4, dtype=psd.PSD_BF16, causal=0, scale=0.125, reserved=0, q_token=512,
             q_head=64, out_token=512, out_head=64)
    st = {n: psd.PsdKvStrides(12800, 128, 64) for n in ("kp", "vp", "ko", "vo")}
    for k, v in kw.items():
        if k in st:
            st[k] = psd.PsdKvStrides(*v)
        else:
            f[k] = v
    return psd.PsdAttention(**f, **st)


def _attention(q=FAKE, plen=None, out=FAKE, ws=FAKE, n=1 << 40, **kw):
    return L.psd_draft_attention(q, FAKE, FAKE, plen, FAKE, FAKE, None, ctypes.byref(_att(**kw)), out, None, ws, n, None, None)


BAD_SHAPES = [dict(B=0), dict(D=0), dict(M=0), dict(M=-1), dict(Hq=7), dict(Hkv=0), dict(Hq=258, Hkv=2), dict(Dh=0), dict(Dh=136),
              dict(Dh=60), dict(P=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
              dict(q_token=0), dict(q_head=-64), dict(kp=(-8, 128, 64)), dict(kp=(0, 0, 64)), dict(B=1 << 20, D=1 << 20),
              dict(q_token=1 << 39), dict(kp=(1 << 40, 128, 64))]


@pytest.mark.parametrize("kw", BAD_SHAPES)
def test_shapes(kw):
    assert _attention(**kw) == psd.PSD_ERR_SHAPE
    assert L.psd_prefix_weights(FAKE, FAKE, None, FAKE, ctypes.byref(_att(**kw)), 1.0, None, FAKE, FAKE, 1 << 40, None,
                                None) == psd.PSD_ERR_SHAPE


def test_attention_refusals():
    assert _attention(q=None) == psd.PSD_ERR_NULL and _attention(out=None) == psd.PSD_ERR_NULL
    assert _attention(ws=None) == psd.PSD_ERR_NULL
    call = lambda **kw: L.psd_draft_attention(*[kw.get(n, FAKE) for n in ("q", "k", "v")], None, kw.get("ko", FAKE),  # noqa: E731
                                              kw.get("vo", FAKE), None, ctypes.byref(kw.get("a", _att())), FAKE, None, FAKE,
                                              kw.get("n", 1 << 40), None, None)
    assert call(k=None) == psd.PSD_ERR_NULL and call(v=None) == psd.PSD_ERR_NULL
    assert call(ko=None) == psd.PSD_ERR_NULL and call(vo=None) == psd.PSD_ERR_NULL
    assert L.psd_draft_attention(FAKE, FAKE, FAKE, None, FAKE, FAKE, None, None, FAKE, None, FAKE, 1 << 40, None, None) == psd.PSD_ERR_NULL
    for a in (_att(S=-1), _att(causal=2), _att(vp=(0, -8, 0)), _att(ko=(0, 0, 0)), _att(out_token=0)):
        assert call(a=a) == psd.PSD_ERR_SHAPE
    for a in (_att(dtype=psd.PSD_FP32), _att(dtype=-1), _att(reserved=1)):
        assert call(a=a) == psd.PSD_ERR_UNSUPPORTED
    for a in (_att(q_token=516), _att(out_head=68), _att(kp=(12800, 124, 64)), _att(vo=(12801, 128, 64))):
        assert call(a=a) == psd.PSD_ERR_ALIGN
    assert call(q=FAKE + 8) == psd.PSD_ERR_ALIGN and call(v=FAKE + 2) == psd.PSD_ERR_ALIGN
    assert _attention(plen=FAKE + 2) == psd.PSD_ERR_ALIGN and _attention(ws=FAKE + 16) == psd.PSD_ERR_ALIGN
    assert call(n=0) == psd.PSD_ERR_WORKSPACE
    need = psd.psd_attention_workspace_bytes(2, 3, 4, 8, 2, 64, 100, 4)
    assert need >= 256 and call(n=need - 1) == psd.PSD_ERR_WORKSPACE


def test_workspaces():
    assert psd.psd_attention_workspace_bytes(1, 4, 32, 32, 8, 128, 2000, 32) >= 256
    for bad in ((0, 4, 32, 32, 8, 128, 2000, 32), (1, 4, 32, 32, 5, 128, 2000, 32), (1, 4, 32, 32, 8, 129, 2000, 32),
                (1, 4, 32, 32, 8, 128, -1, 32)):
        assert psd.psd_attention_workspace_bytes(*bad) == 0
    assert psd.psd_weights_workspace_bytes(1, 4, 32, 32, 8, 128, 0) == 0 < psd.psd_weights_workspace_bytes(1, 4, 32, 32, 8, 128, 1)
    assert psd.psd_logits_workspace_bytes(0, 5) == psd.psd_logits_workspace_bytes(5, 0) == 0 < psd.psd_logits_workspace_bytes(1, 1)


def test_weights_refusals():
    def call(q=FAKE, k=FAKE, lse=FAKE, out=FAKE, ws=FAKE, n=1 << 40, beta=1.0, acc=None, **kw):
        return L.psd_prefix_weights(q, k, None, lse, ctypes.byref(_att(**kw)), beta, acc, out, ws, n, None, None)
    for name in ("q", "k", "lse", "out", "ws"):
        assert call(**{name: None}) == psd.PSD_ERR_NULL
    assert call(P=0) == psd.PSD_ERR_SHAPE and call(beta=float("nan")) == psd.PSD_ERR_SHAPE
    assert call(dtype=5) == psd.PSD_ERR_UNSUPPORTED
    assert call(lse=FAKE + 1) == psd.PSD_ERR_ALIGN and call(acc=FAKE + 2) == psd.PSD_ERR_ALIGN and call(q=FAKE + 4) == psd.PSD_ERR_ALIGN
    assert call(n=0) == psd.PSD_ERR_WORKSPACE


def test_evict_refusals():
    def call(ptr=None, **kw):
        f = dict(B=2, Hkv=2, Dh=64, P=100, keep=10, n_sink=2, n_recent=3, dtype=psd.PSD_BF16)
        st = {n: (12800, 128, 64) for n in ("k", "v", "k_out", "v_out")}
        for k, v in kw.items():
            (st if k in st else f)[k] = v
        e = psd.PsdEvict(**f, **{k: psd.PsdKvStrides(*v) for k, v in st.items()})
        p = [FAKE, FAKE, FAKE, None, ctypes.byref(e), FAKE, FAKE, FAKE, None, None]
        for i, v in (ptr or {}).items():
            p[i] = v
        return L.psd_prefix_evict(*p, None)
    for i in (0, 1, 2, 4, 5, 6, 7):
        assert call({i: None}) == psd.PSD_ERR_NULL
    for kw in (dict(B=0), dict(Hkv=0), dict(Dh=4), dict(P=0), dict(keep=0), dict(n_sink=-1), dict(n_recent=9), dict(k=(0, 0, 0)),
               dict(k_out=(0, 128, 64)), dict(v_out=(12800, 128, 0))):
        assert call(**kw) == psd.PSD_ERR_SHAPE, kw
    assert call(dtype=psd.PSD_FP32) == psd.PSD_ERR_UNSUPPORTED
    assert call(v=(12800, 132, 64)) == psd.PSD_ERR_ALIGN and call({1: FAKE + 8}) == psd.PSD_ERR_ALIGN
    assert call({0: FAKE + 2}) == psd.PSD_ERR_ALIGN and call({7: FAKE + 1}) == psd.PSD_ERR_ALIGN


def test_logits_refusals():
    def call(ptr=None, dtype=psd.PSD_BF16, stride=1000, B=2, D=2, M=3, V=1000, n=1 << 40, **kw):
        f = dict(history=FAKE, history_len=FAKE, draft_tokens=FAKE, draft_mask=FAKE, bias=FAKE, allow=FAKE, history_cap=5, bias_rows=1,
                 allow_rows=12, repetition=1.1, presence=0.0, frequency=0.0, reserved=0)
        f.update(kw)
        e = psd.PsdLogitsEdit(**f)
        p = dict(lg=FAKE, tok=FAKE, conf=FAKE, lse=None, ws=FAKE)
        p.update(ptr or {})
        return L.psd_confidence_logits(p["lg"], dtype, stride, B, D, M, V, ctypes.byref(e), p["tok"], p["conf"], p["lse"], p["ws"],
                                       n, None, None)
    for name in ("lg", "tok", "conf", "ws"):
        assert call({name: None}) == psd.PSD_ERR_NULL
    for kw in (dict(B=0), dict(D=0), dict(M=0), dict(V=0), dict(stride=999), dict(repetition=0.0), dict(repetition=float("nan")),
               dict(presence=float("inf")), dict(frequency=float("nan")), dict(history_cap=-1), dict(bias_rows=5), dict(bias_rows=0),
               dict(allow_rows=7), dict(B=1 << 20, D=1 << 20)):
        assert call(**kw) == psd.PSD_ERR_SHAPE, kw
    assert call(draft_mask=None) == psd.PSD_ERR_NULL and call(history=None) == psd.PSD_ERR_NULL
    assert call(dtype=3) == psd.PSD_ERR_UNSUPPORTED and call(reserved=1) == psd.PSD_ERR_UNSUPPORTED
    assert call({"lg": FAKE + 1}) == psd.PSD_ERR_ALIGN and call({"ws": FAKE + 4}) == psd.PSD_ERR_ALIGN
    assert call({"lg": FAKE + 2}, dtype=psd.PSD_FP32) == psd.PSD_ERR_ALIGN and call(allow=FAKE + 2) == psd.PSD_ERR_ALIGN
    assert call(n=16) == psd.PSD_ERR_WORKSPACE


def test_lengths_whose_last_step_would_overflow_are_refused():
    """Kernels walk these lengths in steps of thousands with 32-bit positions."""
    far = (1 << 30) + 1
    st = psd.PsdKvStrides(12800, 128, 64)
    for kw in (dict(P=far), dict(keep=far)):
        f = dict(B=1, Hkv=2, Dh=64, P=100, keep=10, n_sink=2, n_recent=3, dtype=psd.PSD_BF16)
        f.update(kw)
        e = psd.PsdEvict(**f, k=st, v=st, k_out=st, v_out=st)
        assert L.psd_prefix_evict(FAKE, FAKE, FAKE, None, ctypes.byref(e), FAKE, FAKE, FAKE, None, None, None) == psd.PSD_ERR_SHAPE, kw
    for B, M, V, cap in ((1, 1, far, 0), (1, far, 8, 0), (far, 1, 8, 0), (1, 1, 8, far)):
        e = psd.PsdLogitsEdit(history=FAKE, history_cap=cap, bias_rows=1, allow_rows=1, repetition=1.0)
        assert L.psd_confidence_logits(FAKE, psd.PSD_BF16, V, B, 1, M, V, ctypes.byref(e), FAKE, FAKE, None, FAKE, 1 << 50, None,
                                       None) == psd.PSD_ERR_SHAPE
    assert psd.psd_logits_workspace_bytes(far, 8) == psd.psd_logits_workspace_bytes(8, far) == 0


def test_struct_layouts():
    assert ctypes.sizeof(psd.PsdKvStrides) == 24 and ctypes.sizeof(psd.PsdAttention) == 48 + 32 + 96
    assert ctypes.sizeof(psd.PsdEvict) == 32 + 96 and ctypes.sizeof(psd.PsdLogitsEdit) == 48 + 28 + 4


def test_packed_descriptors_are_the_structs():
    """The bytes the binding packs are those of the C structs."""
    st = [psd.PsdKvStrides(i, i + 1, i + 2) for i in (100, 200, 300, 400)]
    flat = [v for s in st for v in (s.outer, s.token, s.head)]
    head = (1, 2, 3, 4, 5, 6, 7, 8, 1, 1, 0.5, 0, 11, 12, 13, 14)
    assert bytes(psd.PsdAttention(*head, *st)) == binding._pack_attention(*head, *flat)
    head = (1, 2, 3, 4, 5, 6, 7, 1)
    assert bytes(psd.PsdEvict(*head, *st)) == binding._pack_evict(*head, *flat)
    edit = (1 << 40, 2, 3, 4, 5, 6, 7, 8, 9, 1.5, 0.25, -1.0, 0)
    assert bytes(psd.PsdLogitsEdit(*edit)) == binding._pack_edit(*edit)

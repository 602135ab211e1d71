"""Refusals of the 8-bit operators and of the rotation, on the host, before anything is launched; workspaces; frequencies; tensors on
other devices (no GPU)."""
import ctypes
import random

import numpy as np
import pytest
import torch

import paper_2605_15609_b200 as psd
from paper_2605_15609_b200 import binding
from test_ops_devices import _Elsewhere, launches  # noqa: F401  (a fixture)

L = binding.LIB
FAKE = 0x10000      # non-NULL and well aligned; never dereferenced
NULL, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = (getattr(psd, "PSD_ERR_" + n) for n in ("NULL", "SHAPE", "ALIGN", "WORKSPACE", "UNSUPPORTED"))


# ---- frequencies -------------------------------------------------------------------------------------------------

def test_frequencies():
    R, base, factor, original, low, high = 64, 500000.0, 8.0, 8192.0, 1.0, 4.0
    j = np.arange(R // 2)
    f = base ** (-2 * j / R)
    w = np.clip((original * f / (2 * np.pi) - low) / (high - low), 0, 1)
    want = [f, f / factor, (base * factor ** (R / (R - 2))) ** (-2 * j / R), w * f + (1 - w) * f / factor]
    for kind, x in enumerate(want):
        got, gain = psd.psd_rope_frequencies(R, base, kind, factor, original, low, high)
        assert got.dtype is torch.float64 and got.shape == (R // 2,)
        assert np.allclose(got.numpy(), x, rtol=1e-13, atol=0)
        assert gain == pytest.approx(0.1 * np.log(factor) + 1 if kind == psd.PSD_ROPE_BY_PARTS else 1.0, rel=1e-6)
    assert w[0] == 1 and w[-1] == 0 and ((w > 0) & (w < 1)).any()      # all three parts occur


@pytest.mark.parametrize("bad, code", [(dict(rotary=0), SHAPE), (dict(rotary=7), SHAPE), (dict(rotary=130), SHAPE), (dict(base=1.0), SHAPE),
                                       (dict(base=float("nan")), SHAPE), (dict(factor=0.5), SHAPE), (dict(factor=float("inf")), SHAPE),
                                       (dict(kind=4), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED), (dict(kind=2, rotary=2), SHAPE),
                                       (dict(kind=3, original=0.0), SHAPE), (dict(kind=3, original=100, low=4.0, high=4.0), SHAPE),
                                       (dict(kind=3, original=100, low=-1.0), SHAPE)])
def test_frequencies_refused(bad, code):
    with pytest.raises(psd.PsdError) as e:
        psd.psd_rope_frequencies(**{"rotary": 64, **bad})
    assert e.value.code == code
    assert L.psd_rope_frequencies(64, 10000.0, 0, 1.0, 0.0, 0.0, 0.0, None, None) == NULL


# ---- rotation -----------------------------------------------------------------------------------------------------

ROT = dict(n_tokens=5, Hq=8, Hkv=2, Dh=64, dtype=psd.PSD_BF16, rotary=64, interleaved=0, n_slots=9, eps=1e-6, gain=1.0)
ROT.update({f"{n}_token": 512 for n in ("q", "k", "v", "q_out", "k_out", "v_out")})
ROT.update({f"{n}_head": 64 for n in ("q", "k", "v", "q_out", "k_out", "v_out")})


def _rotate(r=None, **ptr):
    a = [ptr.get(n, FAKE) for n in ("q", "k", "v", "position", "frequency", "q_norm", "k_norm", "slot")]
    b = [ptr.get(n, FAKE) for n in ("q_out", "k_out", "v_out")]
    return L.psd_rotate_qk(*a, ctypes.byref(psd.PsdRotate(**{**ROT, **(r or {})})), *b, None)


@pytest.mark.parametrize("r", [dict(n_tokens=0), dict(n_tokens=-1), dict(n_tokens=2 ** 31 - 1), dict(Hq=-1), dict(Hkv=-1), dict(Hq=0, Hkv=0), dict(Hq=16385),
                               dict(Dh=0), dict(Dh=12), dict(Dh=136), dict(rotary=-2), dict(rotary=66), dict(rotary=3), dict(interleaved=2), dict(eps=0.0),
                               dict(eps=float("nan")), dict(gain=0.0), dict(gain=float("inf")), dict(n_slots=-1), dict(q_token=0), dict(k_head=-64),
                               dict(v_out_token=0)])
def test_rotate_shapes(r):
    assert _rotate(r) == SHAPE


def test_rotate_refusals():
    assert L.psd_rotate_qk(*[FAKE] * 8, None, *[FAKE] * 3, None) == NULL
    for n in ("q", "k", "q_out", "k_out", "v_out", "position", "frequency"):
        assert _rotate(**{n: None}) == NULL
    assert _rotate(dict(Hkv=0), k=None, k_out=None) == NULL                     # values without keys
    for n in (psd.PSD_FP32, -1):
        assert _rotate(dict(dtype=n)) == UNSUPPORTED
    for n in ("q", "k", "v", "q_out", "k_out", "v_out", "q_norm", "k_norm"):
        assert _rotate(**{n: FAKE + 8}) == ALIGN
    assert _rotate(position=FAKE + 2) == ALIGN and _rotate(slot=FAKE + 1) == ALIGN and _rotate(frequency=FAKE + 4) == ALIGN
    for n in ("q_token", "k_head", "v_token", "q_out_head", "k_out_token", "v_out_head"):
        assert _rotate({n: 516}) == ALIGN


def test_rotate_binding():
    h = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    p, f = torch.zeros(5, dtype=torch.int32), torch.zeros(32, dtype=torch.float64)
    ok = dict(q=h(5, 4, 64), k=h(5, 2, 64), q_out=h(5, 4, 64), k_out=h(5, 2, 64), position=p, frequency=f)
    for bad in (dict(q_out=None), dict(v=h(5, 2, 64)), dict(q_out=h(4, 4, 64)), dict(k=h(4, 2, 64)), dict(k_out=h(6, 2, 64)), dict(q=None, k=None, q_out=None, k_out=None),
                dict(k=None, k_out=None, v=h(5, 2, 64), v_out=h(5, 2, 64)), dict(v=h(5, 3, 64), v_out=h(5, 3, 64)), dict(k=h(5, 2, 128), k_out=h(5, 2, 128)),
                dict(q=torch.zeros(5, 4, 64)), dict(q=h(64, 4, 5).permute(2, 1, 0)), dict(slot=p, v=h(5, 2, 64), v_out=h(7, 2, 64))):
        with pytest.raises(ValueError):
            psd.psd_rotate_qk(**{**ok, **bad})


# ---- rows and prefix -------------------------------------------------------------------------------------------------

def _rows(x=FAKE, dtype=psd.PSD_BF16, stride=64, n=4, H=64, codes=FAKE, cs=64, scale=FAKE):
    return L.psd_quantize_rows(x, dtype, stride, n, H, codes, cs, scale, None)


def test_rows_refusals():
    assert _rows(x=None) == _rows(codes=None) == _rows(scale=None) == NULL
    for bad in (dict(n=0), dict(n=-3), dict(n=2 ** 31), dict(H=0), dict(H=4), dict(H=60), dict(stride=56), dict(cs=63)):
        assert _rows(**bad) == SHAPE
    assert _rows(dtype=psd.PSD_FP32) == UNSUPPORTED
    for bad in (dict(stride=68), dict(cs=68), dict(x=FAKE + 8), dict(codes=FAKE + 4), dict(scale=FAKE + 2)):
        assert _rows(**bad) == ALIGN


QUANT = dict(B=2, Hkv=2, Dh=64, P=100, block=32, dtype=psd.PSD_BF16, span=0, reserved=0)


def _prefix(q=None, k=FAKE, v=FAKE, begin=None, end=None, kc=FAKE, vc=FAKE, ks=FAKE, vs=FAKE, **st):
    s = {n: psd.PsdKvStrides(*st.get("s_" + n, (12800, 128, 64))) for n in ("k", "v", "k_codes", "v_codes")}
    return L.psd_prefix_quantize(k, v, begin, end, ctypes.byref(psd.PsdQuantize(**{**QUANT, **(q or {})}, **s)), kc, vc, ks, vs, None)


def test_prefix_refusals():
    for n in ("k", "v", "kc", "vc", "ks", "vs"):
        assert _prefix(**{n: None}) == NULL
    assert L.psd_prefix_quantize(FAKE, FAKE, None, None, None, FAKE, FAKE, FAKE, FAKE, None) == NULL
    for q in (dict(B=0), dict(Hkv=0), dict(Dh=12), dict(Dh=136), dict(P=0), dict(P=2 ** 30 + 1), dict(block=0), dict(block=48), dict(block=256), dict(span=-1),
              dict(B=2 ** 20, Hkv=2 ** 11)):
        assert _prefix(q) == SHAPE
    for q in (dict(dtype=2), dict(reserved=1)):
        assert _prefix(q) == UNSUPPORTED
    for st in (dict(s_k=(-8, 128, 64)), dict(s_v=(0, 0, 64)), dict(s_k_codes=(0, 128, 64)), dict(s_v_codes=(12800, 128, 0))):
        assert _prefix(**st) == SHAPE
    for st in (dict(s_k=(12804, 128, 64)), dict(s_v_codes=(12800, 132, 64)), dict(kc=FAKE + 4), dict(k=FAKE + 8), dict(ks=FAKE + 2), dict(begin=FAKE + 2)):
        assert _prefix(**st) == ALIGN


# ---- attention ----------------------------------------------------------------------------------------------------------

def _att(**kw):
    f = dict(B=2, D=3, M=4, Hq=8, Hkv=2, Dh=64, P=100, S=4, dtype=psd.PSD_BF16, causal=0, scale=0.125, reserved=0, q_token=512, q_head=64, out_token=512,
             out_head=64)
    st = {n: psd.PsdKvStrides(12800, 128, 64) for n in ("kp", "vp", "ko", "vo")}
    for k, v in kw.items():
        if k in st:
            st[k] = psd.PsdKvStrides(*v)
        else:
            f[k] = v
    return psd.PsdAttention(**f, **st)


def _attend(block=32, n=1 << 40, a=None, **ptr):
    g = lambda x: ptr.get(x, FAKE)  # noqa: E731
    return L.psd_draft_attention_q8(g("q"), g("kc"), g("vc"), g("ks"), g("vs"), block, ptr.get("plen"), g("ko"), g("vo"), ptr.get("olen"),
                                    ctypes.byref(a or _att()), g("out"), ptr.get("lse"), g("ws"), n, None, None)


@pytest.mark.parametrize("kw", [dict(B=0), dict(D=0), dict(M=0), dict(Hq=7), dict(Hkv=0), dict(Hq=258, Hkv=2), dict(Dh=0), dict(Dh=136), dict(Dh=72), dict(Dh=60), dict(P=-1),
                                dict(S=-1), dict(scale=0.0), dict(scale=float("nan")), dict(causal=2), dict(q_token=0), dict(kp=(-16, 128, 64)), dict(vp=(0, 0, 64)),
                                dict(kp=(1 << 40, 128, 64)), dict(B=1 << 20, D=1 << 20)])
def test_attention_shapes(kw):
    assert _attend(a=_att(**kw)) == SHAPE


def test_attention_refusals():
    for n in ("q", "kc", "vc", "ks", "vs", "ko", "vo", "out", "ws"):
        assert _attend(**{n: None}) == NULL
    for block in (0, -32, 8, 24, 256):
        assert _attend(block=block) == SHAPE
    for a in (_att(dtype=psd.PSD_FP32), _att(reserved=1)):
        assert _attend(a=a) == UNSUPPORTED
    for a in (_att(kp=(12800, 128, 72)), _att(vp=(12808, 128, 64)), _att(q_token=516), _att(ko=(12800, 124, 64))):
        assert _attend(a=a) == ALIGN
    for n in ("q", "kc", "vc", "ko", "out"):
        assert _attend(**{n: FAKE + 8}) == ALIGN
    assert _attend(ks=FAKE + 2) == ALIGN and _attend(plen=FAKE + 2) == ALIGN and _attend(ws=FAKE + 16) == ALIGN and _attend(lse=FAKE + 1) == ALIGN
    assert _attend(n=0) == WORKSPACE and _attend(n=255) == WORKSPACE


def test_attention_workspace_grows():
    """What a large batch gets serves every smaller one."""
    r = random.Random(1)
    for bad in ((0, 1, 1, 1, 1, 16, 1, 1), (1, 1, 1, 3, 2, 16, 1, 1), (1, 1, 1, 1, 1, 24, 1, 1), (1, 1, 1, 1, 1, 16, -1, 1)):
        assert psd.psd_attention_q8_workspace_bytes(*bad) == 0
    for _ in range(3000):
        B, D, M = int(2 ** r.uniform(0, 8)), int(2 ** r.uniform(0, 6)), r.choice([1, 1, 2, 5, 32, 64])
        Hq, Hkv = r.choice([(1, 1), (8, 1), (32, 8), (28, 4), (128, 1), (40, 8)])
        Dh, P, S = r.choice([16, 64, 128]), int(2 ** r.uniform(0, 17)), r.choice([0, M, 200])
        n = psd.psd_attention_q8_workspace_bytes(B, D, M, Hq, Hkv, Dh, P, S)
        assert n >= 256 and n % 256 == 0
        assert psd.psd_attention_q8_workspace_bytes(r.randint(1, B), r.randint(1, D), M, Hq, Hkv, Dh, r.randint(0, P), r.randint(0, S)) <= n


def test_attention_kernel_names():
    """Few rows per key head, query tiles with and without partial results, no prefix; the splits of the partial results."""
    names = lambda *a: psd.psd_attention_q8_kernel_names(*a)  # noqa: E731
    assert names(64, 1, 1, 32, 8, 128, 16384, 64)[0] == "prefix_rows_q8_kernel+draft_attention_kernel"
    assert names(1, 16, 1, 32, 8, 128, 4000, 8) == ("prefix_tiles_q8_kernel+draft_attention_kernel", 16)
    which, splits = names(1, 4, 32, 32, 8, 128, 2000, 32)
    assert which == "prefix_tiles_q8_kernel" and 2 <= splits <= 8                        # joined by a cluster
    assert names(16, 8, 64, 32, 8, 128, 8192, 64) == ("prefix_tiles_q8_kernel", 1)
    assert names(16, 8, 64, 32, 8, 128, 0, 64)[0] == "draft_attention_kernel"
    assert names(1, 1, 1, 32, 8, 128, 100, 8) == ("draft_attention_kernel", 0) and names(1, 4, 32, 4, 4, 64, 500, 32) == ("draft_attention_kernel", 0)
    assert names(1, 1, 1, 3, 2, 128, 100, 1) is None and names(1, 1, 1, 2, 2, 72, 100, 1) is None


# ---- head ---------------------------------------------------------------------------------------------------------------

def _head(hidden=FAKE, dtype=psd.PSD_BF16, w=FAKE, ws=FAKE, R=4, H=128, V=100, tok=FAKE, conf=FAKE, lse=None, space=FAKE, n=1 << 40):
    return L.psd_confidence_q8(hidden, dtype, w, ws, R, H, V, tok, conf, lse, space, n, None, None)


def test_head_refusals():
    for n in ("hidden", "w", "ws", "tok", "conf", "space"):
        assert _head(**{n: None}) == NULL
    for bad in (dict(R=0), dict(R=2 ** 30 + 1), dict(H=32), dict(H=96), dict(H=131136), dict(V=0), dict(V=2 ** 31 - 100)):
        assert _head(**bad) == SHAPE
    assert _head(dtype=psd.PSD_FP32) == UNSUPPORTED
    for bad in (dict(hidden=FAKE + 8), dict(w=FAKE + 8), dict(ws=FAKE + 2), dict(space=FAKE + 128), dict(lse=FAKE + 2)):
        assert _head(**bad) == ALIGN
    need = psd.psd_confidence_q8_workspace_bytes(4, 128, 100)
    assert need >= 4 * 128 + 4 * 4 + 12 * 4 and _head(n=need - 1) == WORKSPACE
    assert psd.psd_confidence_q8_workspace_bytes(0, 128, 100) == 0 and psd.psd_confidence_q8_workspace_bytes(4, 100, 100) == 0


# ---- devices ------------------------------------------------------------------------------------------------------------

def _calls():
    h = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    f = lambda *s: torch.zeros(*s)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    c = lambda *s: torch.zeros(*s, dtype=torch.int8)  # noqa: E731
    ws = torch.zeros(1024, dtype=torch.uint8)
    return {
        "psd_rotate_qk": dict(q=h(5, 4, 64), k=h(5, 2, 64), q_out=h(5, 4, 64), k_out=h(7, 2, 64), v=h(5, 2, 64), v_out=h(7, 2, 64), position=i(5),
                              frequency=torch.zeros(32, dtype=torch.float64), slot=i(5), q_norm=h(64), k_norm=h(64)),
        "psd_quantize_rows": dict(x=h(3, 64), codes=c(3, 64), scale=f(3)),
        "psd_prefix_quantize": dict(k=h(2, 70, 2, 64), v=h(2, 70, 2, 64), k_codes=c(2, 70, 2, 64), v_codes=c(2, 70, 2, 64), k_scale=f(2, 2, 3), v_scale=f(2, 2, 3),
                                    begin=i(2), end=i(2)),
        "psd_draft_attention_q8": dict(q=h(4, 2, 4, 64), k_codes=c(2, 70, 2, 64), v_codes=c(2, 70, 2, 64), k_scale=f(2, 2, 3), v_scale=f(2, 2, 3), out=h(4, 2, 4, 64),
                                       lse=f(4, 2, 4), k_own=h(4, 3, 2, 64), v_own=h(4, 3, 2, 64), prefix_len=i(2), own_len=i(4), workspace=ws, status=i(1)),
        "psd_confidence_q8": dict(hidden=h(5, 64), w_codes=c(9, 64), w_scale=f(9), out_token=i(5), out_conf=f(5), out_lse=f(5), workspace=ws, status=i(1)),
    }


@pytest.mark.parametrize("name", list(_calls()))
def test_tensors_elsewhere_are_refused(name, launches):  # noqa: F811
    args = _calls()[name]
    with pytest.raises(ValueError, match="device"):
        getattr(psd, name)(**args)                                             # everything on the host
    for other in args:                                                         # one tensor on the host, or on another GPU
        for mixed in ({k: t if k == other else _Elsewhere(t, 0) for k, t in args.items()}, {k: _Elsewhere(t, int(k == other)) for k, t in args.items()}):
            with pytest.raises(ValueError, match="device"):
                getattr(psd, name)(**mixed)
    assert launches == []
    getattr(psd, name)(**{k: _Elsewhere(t, 0) for k, t in args.items()})
    assert launches == [name]


@pytest.mark.parametrize("name, bad", [("psd_quantize_rows", dict(codes=torch.zeros(3, 32, dtype=torch.int8))), ("psd_quantize_rows", dict(codes=torch.zeros(3, 64))),
                                       ("psd_quantize_rows", dict(scale=torch.zeros(4))), ("psd_prefix_quantize", dict(k_scale=torch.zeros(2, 2, 2))),
                                       ("psd_prefix_quantize", dict(v_codes=torch.zeros(2, 70, 2, 64, dtype=torch.uint8))), ("psd_prefix_quantize", dict(block=64)),
                                       ("psd_draft_attention_q8", dict(k_scale=torch.zeros(2, 2, 4))), ("psd_draft_attention_q8", dict(block=16)),
                                       ("psd_draft_attention_q8", dict(k_codes=torch.zeros(2, 70, 2, 64))), ("psd_draft_attention_q8", dict(v_own=None)),
                                       ("psd_confidence_q8", dict(w_codes=torch.zeros(9, 128, dtype=torch.int8))), ("psd_confidence_q8", dict(w_scale=torch.zeros(8)))])
def test_shapes_and_types_are_refused(name, bad, launches):  # noqa: F811
    args = {k: _Elsewhere(t, 0) for k, t in _calls()[name].items()}
    with pytest.raises((ValueError, TypeError)):
        getattr(psd, name)(**{**args, **{k: _Elsewhere(t, 0) if isinstance(t, torch.Tensor) else t for k, t in bad.items()}})
    assert launches == []

"""The 8-bit operators and the rotation against plain implementations.

Codes and scales are exact: fp32 operations in a stated order.  Tolerances of the others, from the arithmetic (u = half a step
of the type: 2^-9 bf16 and 2^-12 fp16 relative to the power of two above, 2^-8 and 2^-11 relative to the value):
  rotation: sines of an angle rounded to fp32 after its whole turns are dropped (2^-23 of a radian-sized angle), norm, weight and two
  products in fp32: 2^-20 of the size of the terms, then the output's rounding;
  scores: fp32 sums of Dh products, error e <= (Dh + 6) * 2^-24 * max_j sum_d |q_d k_d| * scale and 2^-22 of the largest exponent
  argument; weights carry a relative 2 e + 2^-17; weights over the prefix are rounded to fp16 (2^-11), those of own keys
  to the type, and the output once;
  confidences: the exponential's 2^-22 of its argument and 2^-24 per addend of a lane's sum: a relative 6e-5."""
import numpy as np
import pytest
import torch

import ops_plain as plain
import paper_2605_15609_b200 as psd
import q8_plain as q8

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _f64(t):
    return t.detach().double().cpu().numpy()


def _rnd(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


def _lens(n, most, seed):
    r = np.random.default_rng(seed)
    x = [int(v) for v in r.integers(0, most + 1, n)]
    x[0] = most
    if n > 1:
        x[1] = min(1, most)
    if n > 2:
        x[2] = 0
    return x


# ---- rows ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R, H", [(1, 8), (3, 64), (130, 264), (128, 4096), (5, 4104), (9, 8192), (2, 16384), (3, 16392), (1, 50000), (700, 512),
                                  (3000, 1024)])
def test_rows(R, H, dtype):
    x = (_rnd(R + H)(R, H) * 0.3).to(DT[dtype])
    codes, scale = torch.full((R, H), 99, dtype=torch.int8, device="cuda"), torch.full((R,), 7.0, device="cuda")
    psd.psd_quantize_rows(x, codes, scale)
    want, s = q8.code_rows(x.float().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), s)
    assert np.array_equal(_f64(codes), want)
    assert int(codes.abs().max()) <= 127 and int(codes.abs().max()) == 127


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_rows_special(dtype):
    """Zeros, the type's extremes, subnormals, NaN and infinities; rows that are views of wider ones."""
    H, top = 1000, torch.finfo(DT[dtype]).max
    x = _rnd(1)(12, H)
    x[0] = 0
    x[1, 5], x[2, 999], x[3, 0] = float("nan"), float("inf"), -float("inf")
    x[4] = top
    x[5] = -top
    x[6] = 0
    x[6, 7] = torch.finfo(DT[dtype]).smallest_normal / 4
    x[7] *= 1e-6
    x[8, 17] = 1000
    wide = torch.full((12, H + 24), float("nan"), dtype=DT[dtype], device="cuda")
    wide[:, 16:16 + H] = x.to(DT[dtype])
    out = torch.full((12, H + 16), 55, dtype=torch.int8, device="cuda")
    scale = torch.empty(12, device="cuda")
    psd.psd_quantize_rows(wide[:, 16:16 + H], out[:, 8:8 + H], scale)
    want, s = q8.code_rows(wide[:, 16:16 + H].float().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True)
    assert np.array_equal(_f64(out[:, 8:8 + H]), want)
    assert bool((out[:, :8] == 55).all()) and bool((out[:, 8 + H:] == 55).all())


# ---- the prefix's cache ----------------------------------------------------------------------------------------------

PREFIX = [  # B, P, Hkv, Dh, block, begin, end
    (1, 1, 1, 8, 16, None, None), (2, 100, 2, 64, 32, None, None), (3, 300, 3, 128, 64, "some", "some"), (4, 129, 1, 80, 128, None, "some"),
    (2, 515, 8, 128, 16, "some", "some"), (5, 70, 4, 72, 32, "some", None), (1, 2000, 2, 128, 128, [1990], [2000]), (3, 96, 2, 96, 32, [31, 32, 33], [32, 64, 96]),
    (2, 64, 2, 64, 16, [-5, 60], [500, 30]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout", ["dense", "heads_first"])
@pytest.mark.parametrize("case", PREFIX)
def test_prefix(case, layout, dtype):
    B, P, Hkv, Dh, block, begin, end = case
    rnd = _rnd(P + Dh)
    nb = -(-P // block)
    some = lambda how, other, seed: None if how is None else _lens(B, P, seed) if how == "some" else how  # noqa: E731
    begin, end = some(begin, 0, 5), some(end, P, 3)
    lo, hi = begin or [0] * B, end or [P] * B
    k, v = (rnd(B, P, Hkv, Dh).to(DT[dtype]) for _ in "kv")
    for b in range(B):
        k[b, max(hi[b], 0):] = float("nan")
        v[b, max(hi[b], 0):] = float("inf")
    if layout == "heads_first":
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    old = [torch.randint(-127, 128, (B, P, Hkv, Dh), device="cuda").to(torch.int8) for _ in "kv"]
    if layout == "heads_first":
        old = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in old]
    olds = [torch.rand(B, Hkv, nb, device="cuda") for _ in "kv"]
    want = [q8.prefix_quantize(x.float().cpu().numpy(), lo, hi, block, c.cpu().numpy(), s.cpu().numpy()) for x, c, s in zip((k, v), old, olds)]
    span = max([1] + [min(max(h, 0), P) - min(max(l, 0), P) for l, h in zip(lo, hi)])
    for sp in (0, span):
        c, s = [x.clone(memory_format=torch.preserve_format) for x in old], [x.clone() for x in olds]
        psd.psd_prefix_quantize(k, v, *c, *s, block=block, begin=None if begin is None else _i32(begin), end=None if end is None else _i32(end),
                                span=sp)
        for x, y, (wc, ws) in zip(c, s, want):
            assert np.array_equal(y.cpu().numpy(), ws)
            assert np.array_equal(_f64(x), wc)


def test_prefix_non_finite_block():
    """A NaN marks its block of its head, keys or values, and no other."""
    k, v = torch.ones(1, 64, 2, 64, device="cuda", dtype=torch.bfloat16), torch.ones(1, 64, 2, 64, device="cuda", dtype=torch.bfloat16)
    k[0, 40, 1, 3], v[0, 2, 0, 9] = float("nan"), float("-inf")
    c = [torch.full((1, 64, 2, 64), 5, dtype=torch.int8, device="cuda") for _ in "kv"]
    s = [torch.zeros(1, 2, 2, device="cuda") for _ in "kv"]
    psd.psd_prefix_quantize(k, v, *c, *s, block=32)
    assert torch.isnan(s[0]).tolist() == [[[False, False], [False, True]]] and torch.isnan(s[1]).tolist() == [[[True, False], [False, False]]]
    assert bool((c[0][0, 32:, 1] == 0).all()) and bool((c[0][0, :32] == 127).all()) and bool((c[1][0, :32, 0] == 0).all())


# ---- rotation ----------------------------------------------------------------------------------------------------------

ROTATE = [  # T, Hq, Hkv, Dh, rotary, interleaved, norm, values
    (1, 1, 1, 8, 8, False, True, True), (3, 4, 2, 64, 64, False, True, True), (5, 4, 2, 64, 64, True, False, True), (7, 28, 4, 128, 128, False, True, True),
    (33, 3, 3, 128, 64, True, True, False), (33, 5, 1, 96, 32, False, False, True), (9, 6, 2, 80, 20, False, True, True), (9, 6, 2, 80, 20, True, True, True),
    (4, 2, 2, 72, 72, False, True, True), (4, 2, 2, 72, 10, True, True, False), (2, 3, 1, 24, 2, False, False, True), (6, 4, 4, 128, 0, False, True, True),
    (900, 40, 8, 128, 128, False, True, True), (2500, 32, 8, 64, 32, True, True, True), (1200, 40, 8, 120, 60, False, False, True), (1, 128, 1, 128, 128, True, True, True),
    (1300, 4, 4, 80, 40, False, True, True), (2000, 3, 1, 64, 64, True, True, True), (1500, 2, 5, 128, 96, False, False, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", ROTATE)
def test_rotate(case, dtype):
    T, Hq, Hkv, Dh, R, inter, norm, values = case
    rnd = _rnd(T + Dh + R)
    qkv = rnd(T, Hq + 2 * Hkv, Dh).to(DT[dtype])
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    wq, wk = ((1 + 0.2 * rnd(Dh)).to(DT[dtype]) for _ in "qk") if norm else (None, None)
    pos = torch.randint(0, 3_000_000, (T,), device="cuda", dtype=torch.int32)
    pos[0] = 2 ** 31 - 1
    if T > 2:
        pos[1], pos[2] = 0, -77
    freq = psd.psd_rope_frequencies(R, 10000.0, psd.PSD_ROPE_BY_PARTS, 4.0, 4096)[0].cuda() if R else None
    gain, slots = 1.25, T + 5
    slot = torch.randperm(slots, device="cuda")[:T].to(torch.int32)
    if T > 3:
        slot[3] = -1
    if T > 4:
        slot[4] = slots
    qo = torch.full((T, Hq, Dh), 7.0, dtype=DT[dtype], device="cuda")
    ko, vo = (torch.full((slots, Hkv, Dh), 7.0, dtype=DT[dtype], device="cuda") for _ in "kv")
    psd.psd_rotate_qk(q, k, qo, ko, pos if R else None, freq, v=v if values else None, v_out=vo if values else None, slot=slot, q_norm=wq,
                      k_norm=wk, eps=1e-6, interleaved=inter, gain=gain)
    f = _f64(freq) if R else np.zeros(0)
    at = slot.cpu().numpy()
    filed = (at >= 0) & (at < slots)
    for x, w, got in ((q, wq, _f64(qo)), (k, wk, _f64(ko))):
        want, size = q8.rotate(_f64(x), pos.cpu().numpy(), f, None if w is None else _f64(w), 1e-6, inter, gain)
        if x is k:
            rest = np.delete(got, at[filed], 0)
            assert np.all(rest == 7.0)
            got, want, size = got[at[filed]], want[filed], size[filed]
        tol = 2.0 ** -20 * size + U[dtype] * np.abs(want) * (1 + 2.0 ** -18) + U[dtype] * 2.0 ** -14 * (dtype == "fp16")
        assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) - tol).max())
        if not norm and R < Dh:
            assert np.array_equal(got[..., R:], want[..., R:])
    if values:
        assert np.array_equal(_f64(vo)[at[filed]], _f64(v)[filed])
        assert np.all(np.delete(_f64(vo), at[filed], 0) == 7.0)
    else:
        assert bool((vo == 7.0).all())


def test_rotate_in_place_alone_and_batched():
    """Outputs that are the inputs, queries without keys, keys without queries, nodes of M tokens: the same numbers."""
    rnd, N, M, Hq, Hkv, Dh = _rnd(3), 3, 5, 4, 2, 64
    qkv = rnd(N, M, Hq + 2 * Hkv, Dh).bfloat16()
    pos = torch.randint(0, 5000, (N * M,), device="cuda", dtype=torch.int32)
    freq = psd.psd_rope_frequencies(Dh)[0].cuda()
    q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
    qo, ko = torch.empty(N, M, Hq, Dh, device="cuda", dtype=q.dtype), torch.empty(N, M, Hkv, Dh, device="cuda", dtype=q.dtype)
    psd.psd_rotate_qk(q, k, qo, ko, pos, freq)
    a, b = torch.empty_like(qo), torch.empty_like(ko)
    psd.psd_rotate_qk(q, None, a, None, pos, freq)
    psd.psd_rotate_qk(None, k, None, b, pos, freq)
    assert torch.equal(a, qo) and torch.equal(b, ko)
    keep = qkv[:, :, Hq + Hkv:].clone()
    psd.psd_rotate_qk(q, k, q, k, pos, freq)
    assert torch.equal(q, qo) and torch.equal(k, ko) and torch.equal(qkv[:, :, Hq + Hkv:], keep)


def test_rotate_keeps_non_finite_numbers_apart():
    """An infinity reaches its partner in a rotated pair and no other number where there is no norm."""
    for inter in (False, True):
        x = torch.ones(1, 1, 64, device="cuda", dtype=torch.bfloat16)
        x[0, 0, 40] = float("inf")                  # behind the rotated part
        x[0, 0, 3] = float("nan")
        y = torch.empty_like(x)
        psd.psd_rotate_qk(x, None, y, None, _i32([5]), psd.psd_rope_frequencies(32)[0].cuda(), interleaved=inter)
        bad = (~torch.isfinite(y[0, 0])).nonzero().flatten().tolist()
        assert bad == ([2, 3, 40] if inter else [3, 19, 40])


# ---- attention over an 8-bit prefix --------------------------------------------------------------------------------------

def _cache(rnd, B, P, Hkv, Dh, block, plen, layout):
    """Codes and scales of a random cache; what lies past a length is not to be used."""
    codes = (rnd(B, P, Hkv, Dh) * 40).clamp(-127, 127).round().to(torch.int8)
    nb = -(-P // block)
    scale = (rnd(B, Hkv, nb).abs() + 0.3) / 40
    for b in range(B):
        codes[b, plen[b]:] = 127
        scale[b, :, -(-plen[b] // block):] = float("nan")
    values = _f64(codes) * np.repeat(_f64(scale).transpose(0, 2, 1), block, 1)[:, :P, :, None]
    if layout == "heads_first":
        codes = codes.transpose(1, 2).contiguous().transpose(1, 2)
    elif layout == "padded":
        pad = torch.full((B, P, Hkv + 1, Dh + 16), 126, dtype=torch.int8, device="cuda")
        pad[:, :, 1:, 16:] = codes
        codes = pad[:, :, 1:, 16:]
    return codes, scale, values


def _check(out, lse, q, kp, vp, ko, vo, plen, olen, scale, causal, dtype):
    want, wlse, absv, big = plain.draft_attention(_f64(q), kp, vp, plen, ko, vo, olen, scale, causal)
    e = (q.shape[3] + 6) * 2.0 ** -24 * big + 2.0 ** -22 * max(1.0, big)
    got, glse = _f64(out), _f64(lse)
    empty = np.isinf(wlse)
    assert np.array_equal(np.isinf(glse), empty) and np.all(got[empty] == 0)
    assert np.all(np.abs(glse[~empty] - wlse[~empty]) <= 2 * e + 2.0 ** -18 + 2.0 ** -22 * np.abs(wlse[~empty]))
    rel = 2 * e + 2.0 ** -17
    weights = 2.0 ** -11 if max(olen) == 0 else U[dtype]
    tol = (weights * absv + U[dtype] * np.abs(want)) * (1 + rel) + rel * absv + 1e-7
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) - tol).max())


def _attention(shape, block, dtype, layout="dense", causal=False, seed=0, full=False, scale=None):
    B, D, M, Hq, Hkv, Dh, P, S = shape
    rnd, N = _rnd(seed + P + Dh), B * D
    plen, olen = ([P] * B, [S] * N) if full else (_lens(B, P, seed), _lens(N, S, seed + 1))
    kc, ks, kp = _cache(rnd, B, P, Hkv, Dh, block, plen, layout)
    vc, vs, vp = _cache(rnd, B, P, Hkv, Dh, block, plen, layout)
    q = (rnd(N, M, Hq, Dh) * 0.7).to(DT[dtype])
    ko, vo = (rnd(N, S, Hkv, Dh).to(DT[dtype]) for _ in "kv")
    for n in range(N):
        ko[n, olen[n]:] = float("nan")
        vo[n, olen[n]:] = float("inf")
    scale = Dh ** -0.5 if scale is None else scale
    out, lse, status = torch.full_like(q, 7.0), torch.full((N, M, Hq), 7.0, device="cuda"), _i32([0])
    ws = torch.full((psd.psd_attention_q8_workspace_bytes(B, D, M, Hq, Hkv, Dh, P, S),), 255, dtype=torch.uint8, device="cuda")
    psd.psd_draft_attention_q8(q, kc, vc, ks, vs, out, lse, ko, vo, block=block, prefix_len=_i32(plen), own_len=_i32(olen), scale=scale,
                               causal=causal, workspace=ws, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    _check(out, lse, q, kp, vp, _f64(ko), _f64(vo), plen, olen, scale, causal, dtype)


ATT = [  # B, D, M, Hq, Hkv, Dh, P, S
    (1, 1, 1, 1, 1, 16, 1, 1), (1, 1, 1, 8, 8, 64, 300, 5), (2, 3, 1, 8, 2, 128, 129, 70), (3, 2, 5, 6, 2, 64, 127, 5), (1, 4, 32, 4, 4, 64, 257, 32),
    (2, 2, 32, 14, 2, 128, 200, 32), (3, 1, 7, 7, 1, 80, 385, 9), (1, 2, 64, 4, 2, 128, 700, 64), (1, 8, 3, 128, 1, 96, 140, 3), (4, 1, 40, 2, 2, 128, 0, 40),
    (4, 2, 16, 3, 3, 48, 130, 0), (3, 1, 2, 2, 1, 32, 0, 0), (2, 9, 33, 5, 5, 128, 1030, 33), (1, 64, 1, 8, 2, 128, 1500, 40), (40, 1, 1, 8, 2, 112, 600, 20),
    (5, 1, 17, 1, 1, 128, 33, 4),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", ATT)
def test_attention(shape, dtype):
    _attention(shape, 32, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", [(*s[:6], s[6] + 577, s[7]) for s in ATT if s[6]])
def test_attention_past_the_short_prefixes(shape, dtype):
    """The same rows over prefixes that one launch does not take."""
    _attention(shape, 32, dtype)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("layout", ["dense", "heads_first", "padded"])
@pytest.mark.parametrize("shape", [(3, 1, 1, 8, 2, 128, 500, 3), (2, 4, 32, 8, 2, 64, 400, 32), (2, 3, 30, 16, 4, 128, 333, 30), (3, 1, 1, 8, 2, 128, 950, 3),
                                   (2, 4, 32, 8, 2, 64, 1100, 32), (3, 2, 9, 6, 2, 112, 201, 9), (2, 1, 1, 5, 5, 32, 140, 2),
                                   (40, 3, 9, 16, 8, 64, 20, 9), (30, 2, 10, 32, 32, 96, 70, 10)])
def test_attention_blocks_and_layouts(shape, layout, block):
    _attention(shape, block, "bf16", layout)
    _attention(shape, block, "fp16", layout, causal=True, seed=9)


@pytest.mark.parametrize("shape", [(2, 2, 1, 8, 2, 128, 3000, 0), (1, 1, 1, 4, 4, 64, 5000, 0), (1, 4, 32, 8, 1, 128, 2049, 0), (1, 2, 64, 8, 4, 80, 4096, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_long_prefixes(shape, dtype):
    """Prefix only: the weights' rounding is fp16's whatever the type."""
    _attention(shape, 64, dtype, full=True)


# ---- confidences over a head in codes ---------------------------------------------------------------------------------------

HEAD = [(1, 64, 1), (1, 64, 17), (5, 128, 300), (128, 256, 1024), (130, 192, 1000), (257, 320, 515), (300, 4096, 2049), (1000, 512, 700), (3, 8192, 5000)]


def _head_inputs(R, H, V, dtype, seed=0):
    rnd = _rnd(seed + R + H + V)
    w, ws = torch.empty(V, H, dtype=torch.int8, device="cuda"), torch.empty(V, device="cuda")
    head = (rnd(V, H) * 0.05).bfloat16()
    psd.psd_quantize_rows(head, w, ws)
    hidden = rnd(R, H)
    hidden += head[torch.randint(0, V, (R,), device="cuda")].float() * 3 / (H * 0.05 ** 2) * (torch.arange(R, device="cuda") % 2)[:, None]
    return hidden.to(DT[dtype]), w, ws


def _run_head(hidden, w, ws):
    R, H, V = *hidden.shape, w.shape[0]
    tok, conf, lse, status = _i32([-5] * R), torch.full((R,), 7.0, device="cuda"), torch.full((R,), 7.0, device="cuda"), _i32([0])
    space = torch.full((psd.psd_confidence_q8_workspace_bytes(R, H, V),), 255, dtype=torch.uint8, device="cuda")
    psd.psd_confidence_q8(hidden, w, ws, tok, conf, lse, workspace=space, status=status)
    torch.cuda.synchronize()
    return tok, conf, lse, int(status.item())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R, H, V", HEAD)
def test_head(R, H, V, dtype):
    hidden, w, ws = _head_inputs(R, H, V, dtype)
    tok, conf, lse, status = _run_head(hidden, w, ws)
    want, wconf, wlse, _ = q8.head(hidden.float().cpu().numpy(), w.cpu().numpy(), ws.cpu().numpy())
    assert status == 0 and np.array_equal(tok.cpu().numpy(), want)
    assert np.all(np.abs(_f64(conf) - wconf) <= 6e-5 * wconf)
    assert np.all(np.abs(_f64(lse) - wlse) <= 6e-5 + 2.0 ** -22 * np.abs(wlse))

"""The 8-bit operators and the rotation as a service calls them: graphs, streams, workspaces, strides past 32 bits, lengths that are cut,
special scales, isolation of drafts, the give-up path, and a run of all of them together.  Tolerances as in test_gpu_q8.py."""
import math

import numpy as np
import pytest
import torch

import paper_2605_15609_b200 as psd
import q8_plain as q8
from test_gpu_q8 import _cache, _check, _f64, _head_inputs, _i32, _rnd, _run_head

pytestmark = pytest.mark.gpu

ROWS = (3, 1, 1, 8, 2, 128, 700, 6)           # few rows per key head
PARTIAL = (1, 16, 2, 8, 2, 128, 700, 2)       # a query tile, keys split, a second kernel joins
JOINED = (1, 4, 32, 8, 2, 128, 700, 32)       # query tiles, keys split over a cluster that joins
JOINED_ONE = (1, 1, 32, 8, 2, 64, 900, 32)    # the same with one query tile
FUSED = (16, 4, 64, 32, 8, 128, 300, 64)      # query tiles, own keys in the same kernel
SMALL = (40, 4, 33, 16, 4, 64, 200, 33)       # the same with heads of 64, two drafts to a tile
SHORT = (2, 2, 21, 8, 2, 96, 150, 40)         # a short prefix and the own keys, no query tiles
SHORT_ONE = (3, 1, 1, 4, 4, 64, 300, 6)       # the same of single tokens
SHORT_MANY = (40, 3, 9, 16, 8, 64, 80, 9)     # the same with several waves of CTAs
FORMS = {ROWS: "prefix_rows_q8_kernel+draft_attention_kernel", PARTIAL: "prefix_tiles_q8_kernel+draft_attention_kernel",
         JOINED: "prefix_tiles_q8_kernel", JOINED_ONE: "prefix_tiles_q8_kernel", FUSED: "prefix_tiles_q8_kernel", SMALL: "prefix_tiles_q8_kernel",
         SHORT: "draft_attention_kernel", SHORT_ONE: "draft_attention_kernel", SHORT_MANY: "draft_attention_kernel"}


def _space(n):
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")


def _inputs(shape, seed=0, dtype=torch.bfloat16, block=32, plen=None, olen=None):
    B, D, M, Hq, Hkv, Dh, P, S = shape
    rnd, N = _rnd(seed), B * D
    plen = plen or [P - 3 * (b % 5) for b in range(B)]
    kc, ks, kp = _cache(rnd, B, P, Hkv, Dh, block, plen, "dense")
    vc, vs, vp = _cache(rnd, B, P, Hkv, Dh, block, plen, "dense")
    t = dict(q=(0.7 * rnd(N, M, Hq, Dh)).to(dtype), k_codes=kc, v_codes=vc, k_scale=ks, v_scale=vs, k_own=rnd(N, S, Hkv, Dh).to(dtype), v_own=rnd(N, S, Hkv, Dh).to(dtype),
             prefix_len=_i32(plen), own_len=_i32(olen or [S] * N))
    return t, kp, vp


def _attend(t, ws=None, block=32, status=None, **kw):
    N, M, Hq, Dh = t["q"].shape
    B, P, Hkv, _ = t["k_codes"].shape
    if ws is None:
        ws = _space(psd.psd_attention_q8_workspace_bytes(B, N // B, M, Hq, Hkv, Dh, P, t["k_own"].shape[1]))
    out, lse = torch.full_like(t["q"], 7.0), torch.full((N, M, Hq), 7.0, device="cuda")
    psd.psd_draft_attention_q8(**t, out=out, lse=lse, block=block, workspace=ws, status=status, **kw)
    return out, lse


@pytest.mark.parametrize("shape", list(FORMS))
def test_shapes_reach_their_form(shape):
    names, splits = psd.psd_attention_q8_kernel_names(*shape)
    assert names == FORMS[shape] and (splits > 1) == (shape in (PARTIAL, JOINED, JOINED_ONE, ROWS))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(1, 4, 32, 8, 2, 128, 700, 32), (1, 1, 32, 8, 2, 64, 900, 32), (1, 2, 16, 8, 2, 64, 900, 40), (2, 4, 33, 14, 2, 96, 1500, 33), (1, 1, 300, 2, 2, 128, 1025, 300),
                                   (3, 2, 40, 4, 2, 80, 600, 129), (1, 4, 32, 16, 4, 128, 2000, 32)])
def test_keys_split_over_a_cluster(shape, causal, dtype):
    """Sequences shorter than the splits, without a prefix, own keys of several tiles dealt out to the cluster."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    names, splits = psd.psd_attention_q8_kernel_names(*shape)
    assert names == "prefix_tiles_q8_kernel" and splits > 1
    for plen in ([P] * B, [P // 3 + 1] * B, [[100, 0, P][b % 3] for b in range(B)], [0] * B):
        for olen in ([S] * (B * D), [[0, S, 1][n % 3] for n in range(B * D)]):
            t, kp, vp = _inputs(shape, 4, {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype], 32, plen, olen)
            past = torch.arange(S, device="cuda")[None] >= t["own_len"][:, None]
            t["k_own"][past], t["v_own"][past] = math.nan, math.inf
            out, lse = _attend(t, causal=causal)
            _check(out, lse, t["q"], kp, vp, np.nan_to_num(_f64(t["k_own"])), np.nan_to_num(_f64(t["v_own"]), posinf=0), plen, olen, Dh ** -0.5, causal, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 700, 2, 1, 64, 33, 700), (2, 1, 3, 4, 2, 128, 64, 1500), (1, 2, 70, 4, 4, 32, 129, 90), (45, 3, 9, 16, 8, 64, 5, 9), (3, 1, 1, 128, 1, 112, 1, 1)])
def test_short_prefixes_in_one_launch(shape, causal, dtype):
    """Many query rows or own keys beside a few prefix keys, ragged and empty lengths, strided queries, outputs and own keys."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    assert psd.psd_attention_q8_kernel_names(*shape) == ("draft_attention_kernel", 0)
    plen, olen = [(P * (b % 4) + 2) // 3 for b in range(B)], [[S, 0, S // 2, 1][n % 4] for n in range(B * D)]
    t, kp, vp = _inputs(shape, 13, {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype], 32, plen, olen)
    for n in ("q", "k_own", "v_own"):
        x = t[n]
        wide = torch.full((x.shape[0], x.shape[1], x.shape[2] + 2, x.shape[3] + 16), math.nan, dtype=x.dtype, device="cuda")
        wide[:, :, 1:-1, 8:-8] = x
        t[n] = wide[:, :, 1:-1, 8:-8]
    past = torch.arange(S, device="cuda")[None] >= t["own_len"][:, None]
    t["k_own"][past], t["v_own"][past] = math.nan, math.inf
    out, lse = _attend(t, causal=causal)
    plen = [min(p, P) for p in plen]
    _check(out, lse, t["q"], kp, vp, np.nan_to_num(_f64(t["k_own"])), np.nan_to_num(_f64(t["v_own"]), posinf=0), plen, olen, Dh ** -0.5, causal, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(16, 4, 32, 16, 8, 128, 130, 32), (20, 3, 33, 16, 8, 64, 300, 33), (17, 3, 70, 8, 4, 80, 129, 70), (40, 8, 32, 8, 2, 128, 1, 32),
                                   (19, 4, 40, 16, 8, 128, 257, 40), (12, 6, 32, 28, 4, 128, 200, 32), (10, 2, 150, 8, 4, 96, 200, 170)])
def test_own_keys_behind_an_unsplit_prefix(shape, causal, dtype):
    """Ragged lengths of the prefix (none at all among them) and of the drafts, several drafts to a query tile."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    assert psd.psd_attention_q8_kernel_names(*shape) == ("prefix_tiles_q8_kernel", 1)
    plen = [(P * (b % 4)) // 3 for b in range(B)]
    olen = [[S, 0, S // 2, 1][n % 4] for n in range(B * D)]
    t, kp, vp = _inputs(shape, 3, {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype], 32, plen, olen)
    past = torch.arange(S, device="cuda")[None] >= t["own_len"][:, None]
    t["k_own"][past], t["v_own"][past] = math.nan, math.inf
    out, lse = _attend(t, causal=causal)
    some = list(range(0, B, 5)) + [B - 1]                       # (a plain loop over all of them would take minutes)
    pick = [b * D + d for b in some for d in range(D)]
    g = lambda x: _f64(x)[pick]  # noqa: E731
    _check(out[pick], lse[pick], t["q"][pick], kp[some], vp[some], np.nan_to_num(g(t["k_own"])), np.nan_to_num(g(t["v_own"]), posinf=0), [plen[b] for b in some],
           [olen[n] for n in pick], Dh ** -0.5, causal, dtype)


@pytest.mark.parametrize("shape", list(FORMS))
def test_same_bits_and_no_lse(shape):
    """Equal inputs give equal bits; lse, lengths and own keys may be left out; lengths outside the cache are cut."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    t, _, _ = _inputs(shape, 5, plen=[P] * B)
    out, lse = _attend(t)
    again = torch.empty_like(out)
    ws = _space(psd.psd_attention_q8_workspace_bytes(*shape))
    rest = {k: v for k, v in t.items() if k not in ("prefix_len", "own_len")}
    psd.psd_draft_attention_q8(**rest, out=again, workspace=ws)
    assert torch.equal(again, out)
    t["prefix_len"], t["own_len"] = _i32([P + 1000] * B), _i32([S + 5] * (B * D))
    o, l = _attend(t)
    assert torch.equal(o, out) and torch.equal(l, lse)
    t["prefix_len"] = _i32([-4] * B)
    o, l = _attend(t)
    zero, z = _attend({**t, "prefix_len": _i32([0] * B)})
    assert torch.equal(o, zero) and torch.equal(l, z)
    none = {k: v for k, v in t.items() if k not in ("k_own", "v_own", "own_len")}
    o, l = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    psd.psd_draft_attention_q8(**none, out=o, lse=l, workspace=ws)
    assert bool((o == 0).all()) and bool((l == -math.inf).all())      # neither prefix nor own keys


@pytest.mark.parametrize("shape", list(FORMS))
def test_scales(shape):
    """A scale NaN makes NaN of what draws on its block and of nothing else; scales of 0, very small and very large ones."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    G = Hq // Hkv
    t, kp, vp = _inputs(shape, 6, plen=[P] * B)
    out, lse = _attend(t)
    for name in ("k_scale", "v_scale"):
        bad = {**t, name: t[name].clone()}
        bad[name][B - 1, 1, 2] = math.nan
        o, l = _attend(bad)
        hit = torch.zeros_like(out, dtype=torch.bool)
        hit[(B - 1) * D:, :, G:2 * G] = True
        assert bool(torch.isnan(o[hit]).all()) and torch.equal(o[~hit], out[~hit])
        if name == "k_scale":
            assert bool(torch.isnan(l[(B - 1) * D:, :, G:2 * G]).all())
        else:
            assert torch.equal(l, lse)
    # values of one block that stand for nothing, tiny ones and (bf16) huge ones
    vs = t["v_scale"].clone()
    vs[:, :, 0], vs[:, :, 1], vs[:, :, 2] = 0.0, 1e-30, 1e25
    o, _ = _attend({**t, "v_scale": vs})
    v = _f64(t["v_codes"]) * np.repeat(_f64(vs).transpose(0, 2, 1), 32, 1)[:, :P, :, None]
    b, n = 0, 0
    s = np.einsum("ihd,khd->hik", _f64(t["q"])[n].reshape(M, Hq, Dh), np.concatenate([kp[b], _f64(t["k_own"])[n]])[:, np.arange(Hq) // G]) * Dh ** -0.5
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    allv = np.concatenate([v[b], _f64(t["v_own"])[n]])[:, np.arange(Hq) // G]
    want, size = np.einsum("hik,khd->ihd", p, allv), np.einsum("hik,khd->ihd", p, np.abs(allv))
    assert np.all(np.abs(_f64(o)[n] - want) <= 2.0 ** -7 * size + 2.0 ** -8 * np.abs(want))
    # keys whose scale is 0 are scored 0
    ks = torch.zeros_like(t["k_scale"])
    _, l = _attend({**t, "k_scale": ks, "own_len": _i32([0] * (B * D))})
    assert bool((l - math.log(P)).abs().max() <= 1e-5)


@pytest.mark.parametrize("shape", [PARTIAL, JOINED, FUSED, SMALL, SHORT])
def test_a_draft_does_not_reach_another(shape):
    """NaN and infinities in one draft's own keys and values leave all other drafts' bits as they were."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    t, _, _ = _inputs(shape, 7)
    out, lse = _attend(t)
    n = D // 2
    t["k_own"][n], t["v_own"][n] = math.nan, math.inf
    o, l = _attend(t)
    keep = [x for x in range(B * D) if x != n]
    assert torch.equal(o[keep], out[keep]) and torch.equal(l[keep], lse[keep])
    assert bool((~torch.isfinite(o[n].float())).all())


@pytest.mark.parametrize("shape", [ROWS, PARTIAL, JOINED])
def test_a_cache_shared_by_all_heads_and_sequences(shape):
    """Stride 0 of the outer dimension and of the heads."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    B, shape = 2, (2, *shape[1:])
    t, kp, vp = _inputs(shape, 8, plen=[P] * B)
    for n in ("k", "v"):
        t[n + "_codes"] = t[n + "_codes"][:1, :, :1].expand(B, P, Hkv, Dh)
    out, lse = _attend(t)
    full = {**t, **{n + "_codes": t[n + "_codes"].contiguous() for n in "kv"}}
    o, l = _attend(full)
    assert torch.equal(o, out) and torch.equal(l, lse)


def test_strides_past_32_bits():
    """Caches, rows and tokens more than 2^32 bytes apart."""
    far = (1 << 32) + 64
    mem = torch.empty(far + (1 << 20), dtype=torch.int8, device="cuda")
    for P, M, D in ((1000, 1, 1), (1000, 32, 4), (100, 1, 1), (100, 32, 4)):
        B, Hkv, Dh = 2, 2, 64
        shape, spread = (B, D, M, 4, Hkv, Dh, P, 3), mem.as_strided((B, P, Hkv, Dh), (far, Hkv * Dh, Dh, 1))
        t, _, _ = _inputs(shape, 9)
        out, lse = _attend(t)
        spread.copy_(t["k_codes"])
        o, l = _attend({**t, "k_codes": spread})
        assert torch.equal(o, out) and torch.equal(l, lse)
    # codes written there, from numbers that lie as far apart
    wide = torch.empty((far // 2) + (1 << 20), dtype=torch.bfloat16, device="cuda")
    k = wide.as_strided((B, P, Hkv, Dh), (far // 2, Hkv * Dh, Dh, 1))
    k.copy_(_rnd(1)(B, P, Hkv, Dh))
    dense, v = k.contiguous(), torch.zeros(B, P, Hkv, Dh, dtype=torch.bfloat16, device="cuda")
    s = [torch.empty(B, Hkv, 4, device="cuda") for _ in range(4)]
    a, vc = torch.empty(B, P, Hkv, Dh, dtype=torch.int8, device="cuda"), torch.empty(B, P, Hkv, Dh, dtype=torch.int8, device="cuda")
    psd.psd_prefix_quantize(dense, v, a, vc, s[0], s[1])
    psd.psd_prefix_quantize(k, v, spread, vc, s[2], s[3])
    assert torch.equal(spread, a) and torch.equal(s[0], s[2])
    x = wide.as_strided((2, 512), (far // 2, 1))
    r, out_codes, ref = torch.empty(2, device="cuda"), mem.as_strided((2, 512), (far, 1)), torch.empty(2, 512, dtype=torch.int8, device="cuda")
    psd.psd_quantize_rows(x, out_codes, r)
    r2 = torch.empty(2, device="cuda")
    psd.psd_quantize_rows(x.contiguous(), ref, r2)
    assert torch.equal(out_codes, ref) and torch.equal(r, r2)
    q, pos, f = wide.as_strided((2, 4, 64), (far // 2, 64, 1)), _i32([5, 9]), psd.psd_rope_frequencies(64)[0].cuda()
    want = torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    psd.psd_rotate_qk(q.contiguous(), None, want, None, pos, f)
    psd.psd_rotate_qk(q, None, q, None, pos, f)
    assert torch.equal(q, want)


# ---- head ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("R, H, V", [(1500, 512, 20000), (4097, 128, 3001), (129, 1088, 40000)])
def test_head_at_larger_sizes(R, H, V):
    """Several row tiles and bands, against exact sums in 64 bits on the GPU."""
    hidden, w, ws = _head_inputs(R, H, V, "bf16", 2)
    tok, conf, lse, status = _run_head(hidden, w, ws)
    c, s = q8.code_rows(hidden.float().cpu().numpy())
    n = torch.from_numpy(c).cuda() @ w.double().t()
    l = (n.float() * ws) * torch.from_numpy(s).cuda()[:, None]
    m = l.amax(1)
    first = torch.where(l == m[:, None], torch.arange(V, device="cuda"), V).amin(1)
    z = torch.logsumexp(l.double(), 1)
    assert status == 0 and torch.equal(tok.long(), first)
    want = torch.exp(m.double() - z)
    assert bool(((conf.double() - want).abs() <= 6e-5 * want).all()) and bool(((lse.double() - z).abs() <= 6e-5 + 2.0 ** -22 * z.abs()).all())


@pytest.mark.parametrize("R, H, V", [(128 * 37 + 5, 128, 2500), (128 * 74, 64, 1999), (128 * 111 - 1, 64, 777), (200001, 64, 33), (60000, 64, 300), (20000, 64, 1), (641, 64, 16),
                                     (2, 64, 100003), (700, 576, 4000), (50000, 768, 1000), (9000, 4608, 1200)])
def test_head_row_tiles_and_bands(R, H, V):
    """Counts of row tiles that share different factors with the number of SMs (bands are cut shorter), fewer tiles than SMs, rows larger than a band;
    equal logits in all parts of a tile and in several tiles: the lowest token."""
    rnd = _rnd(R + V)
    hidden, w, ws = rnd(R, H).bfloat16(), (rnd(V, H) * 40).clamp(-127, 127).round().to(torch.int8), (rnd(V).abs() + 0.1) * 2e-2 / H
    for v in range(V // 3, V, max(1, V // 7)):
        w[v], ws[v] = w[0], ws[0]
    hidden[::2] = w[0].to(torch.bfloat16)
    tok, conf, lse, status = _run_head(hidden, w, ws)
    c, s = torch.empty(R, H, dtype=torch.int8, device="cuda"), torch.empty(R, device="cuda")
    psd.psd_quantize_rows(hidden, c, s)
    assert status == 0
    for r in range(0, R, 1 << 13):
        n = c[r:r + (1 << 13)].double() @ w.double().t()                    # exact
        l = (n.float() * ws) * s[r:r + (1 << 13), None]
        m = l.amax(1)
        first = torch.where(l == m[:, None], torch.arange(V, device="cuda"), V).amin(1)
        z = torch.logsumexp(l.double(), 1)
        want = torch.exp(m.double() - z)
        got = slice(r, r + (1 << 13))
        assert torch.equal(tok[got].long(), first)
        assert bool(((conf[got].double() - want).abs() <= 6e-5 * want).all()) and bool(((lse[got].double() - z).abs() <= 6e-5 + 2.0 ** -22 * z.abs()).all())


def test_head_special_rows():
    """Rows with a NaN or an infinity have confidence NaN and are counted; a row of zeros is uniform; equal logits: the lowest token; a scale NaN of
    one vocabulary row reaches every confidence."""
    R, H, V = 140, 128, 900
    hidden, w, ws = _head_inputs(R, H, V, "bf16", 3)
    hidden[3, 7], hidden[130, 0], hidden[50] = math.nan, math.inf, 0
    w[400], ws[400] = w[77], ws[77]                                  # equal rows of the head
    hidden[9] = w[77].to(torch.bfloat16)
    tok, conf, lse, status = _run_head(hidden, w, ws)
    assert status == 2 and torch.isnan(conf).nonzero().flatten().tolist() == [3, 130]
    assert int(tok[50]) == 0 and float(conf[50]) == pytest.approx(1 / V, rel=1e-5) and int(tok[9]) == 77
    ws2 = ws.clone()
    ws2[V - 1] = math.nan
    _, conf, _, status = _run_head(hidden, w, ws2)
    assert status == R and bool(torch.isnan(conf).all())


@pytest.mark.parametrize("order", [1, 2])
def test_head_tile_orders(order):
    hidden, w, ws = _head_inputs(700, 128, 3000, "fp16", 4)
    want = _run_head(hidden, w, ws)
    assert psd.psd_set_tuning(psd.PSD_TUNE_TILE_ORDER, order) == 0
    assert psd.psd_set_tuning(psd.PSD_TUNE_BAND_BYTES, 40000) == 0
    try:
        got = _run_head(hidden, w, ws)
    finally:
        psd.psd_set_tuning(psd.PSD_TUNE_TILE_ORDER, 0)
        psd.psd_set_tuning(psd.PSD_TUNE_BAND_BYTES, 36 << 20)
    assert torch.equal(got[0], want[0]) and bool(((got[1] - want[1]).abs() <= 1e-5 * want[1]).all()) and got[3] == 0


# ---- graphs, streams, time limits ---------------------------------------------------------------------------------------------

class _Step:
    """Rotate, file, code, attend, score: one step of a service on fixed buffers."""
    B, D, M, HQ, HKV, DH, P, V, H = 2, 4, 32, 8, 2, 128, 512, 3000, 8 * 128

    def __init__(self, seed, ws=None, space=None):
        rnd, B, N, T = _rnd(seed), self.B, self.B * self.D, self.B * self.D * self.M
        HQ, HKV, DH, P, M = self.HQ, self.HKV, self.DH, self.P, self.M
        self.qkv = rnd(T, HQ + 2 * HKV, DH).bfloat16()
        self.norms = [(1 + 0.1 * rnd(DH)).bfloat16() for _ in range(2)]
        self.freq, self.gain = psd.psd_rope_frequencies(DH, kind=psd.PSD_ROPE_BY_PARTS, factor=4.0, original=256)
        self.freq = self.freq.cuda()
        self.length = _i32([300, 411])
        self.position = (self.length[:, None, None] + torch.arange(M, device="cuda")[None, None]).expand(B, self.D, M).reshape(-1).to(torch.int32).contiguous()
        self.q = torch.empty(N, M, HQ, DH, device="cuda", dtype=torch.bfloat16)
        self.ko, self.vo = (torch.empty(N, M, HKV, DH, device="cuda", dtype=torch.bfloat16) for _ in "kv")
        self.k, self.v = (rnd(B, P, HKV, DH).bfloat16() for _ in "kv")
        self.begin = _i32([0, 0])
        self.codes = [torch.zeros(B, P, HKV, DH, dtype=torch.int8, device="cuda") for _ in "kv"]
        self.scale = [torch.zeros(B, HKV, P // 32, device="cuda") for _ in "kv"]
        self.out, self.lse = torch.empty_like(self.q), torch.empty(N, M, HQ, device="cuda")
        head = (0.05 * rnd(self.V, self.H)).bfloat16()
        self.w, self.ws = torch.empty(self.V, self.H, dtype=torch.int8, device="cuda"), torch.empty(self.V, device="cuda")
        psd.psd_quantize_rows(head, self.w, self.ws)
        self.tok, self.conf = torch.empty(T, dtype=torch.int32, device="cuda"), torch.empty(T, device="cuda")
        self.space = _space(psd.psd_attention_q8_workspace_bytes(B, self.D, M, HQ, HKV, DH, P, M)) if ws is None else ws
        self.space2 = _space(psd.psd_confidence_q8_workspace_bytes(T, self.H, self.V)) if space is None else space
        self.status = _i32([0])

    def run(self):
        HQ, HKV = self.HQ, self.HKV
        psd.psd_rotate_qk(self.qkv[:, :HQ], self.qkv[:, HQ:HQ + HKV], self.q, self.ko, self.position, self.freq, v=self.qkv[:, HQ + HKV:], v_out=self.vo,
                          q_norm=self.norms[0], k_norm=self.norms[1], gain=self.gain)
        psd.psd_prefix_quantize(self.k, self.v, *self.codes, *self.scale, begin=self.begin, end=self.length)
        psd.psd_draft_attention_q8(self.q, *self.codes, *self.scale, self.out, self.lse, self.ko, self.vo, prefix_len=self.length, workspace=self.space, status=self.status)
        psd.psd_confidence_q8(self.out.view(-1, self.H), self.w, self.ws, self.tok, self.conf, workspace=self.space2, status=self.status)

    def results(self):
        return [x.clone() for x in (self.q, self.ko, self.vo, *self.codes, *self.scale, self.out, self.lse, self.tok, self.conf)]


def test_a_step_of_all_of_them():
    """The rotated queries attend over the coded prefix and their own rotated keys, and the result is scored: each stage against the
    plain implementation of the same stage, then the policy takes the confidences."""
    s = _Step(1)
    s.run()
    torch.cuda.synchronize()
    B, D, M, HQ, HKV, DH, N = s.B, s.D, s.M, s.HQ, s.HKV, s.DH, s.B * s.D
    pos = s.position.cpu().numpy()
    for x, w, got in ((s.qkv[:, :HQ], s.norms[0], s.q), (s.qkv[:, HQ:HQ + HKV], s.norms[1], s.ko)):
        want, size = q8.rotate(_f64(x), pos, _f64(s.freq), _f64(w), 1e-6, False, s.gain)
        assert np.all(np.abs(_f64(got).reshape(want.shape) - want) <= 2.0 ** -20 * size + 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -18))
    lens, kv = s.length.tolist(), []
    for x, c, sc in zip((s.k, s.v), s.codes, s.scale):
        wc, wsc = q8.prefix_quantize(x.float().cpu().numpy(), [0, 0], lens, 32, np.zeros(c.shape, dtype=np.int8), np.zeros(sc.shape, dtype=np.float32))
        assert np.array_equal(_f64(c), wc) and np.array_equal(sc.cpu().numpy(), wsc)
        kv.append(wc * np.repeat(wsc.astype(np.float64).transpose(0, 2, 1), 32, 1)[..., None])
    _check(s.out, s.lse, s.q, *kv, _f64(s.ko), _f64(s.vo), lens, [M] * N, DH ** -0.5, False, "bf16")
    want, wconf, _, _ = q8.head(s.out.view(-1, s.H).float().cpu().numpy(), s.w.cpu().numpy(), s.ws.cpu().numpy())
    assert np.array_equal(s.tok.cpu().numpy(), want) and np.all(np.abs(_f64(s.conf) - wconf) <= 6e-5 * wconf)
    assert int(s.status.item()) == 0
    p = psd.policy(tau=0.9, k_min=2, depth=D, mask_id=s.V)
    tokens, mask = torch.full((B, M), s.V, dtype=torch.int32, device="cuda"), torch.ones(B, M, dtype=torch.int32, device="cuda")
    sel, n_sel, where = _i32([[0] * M] * B), _i32([0] * B), _i32([[0] * M] * B)
    psd.psd_select_unmask(s.conf.view(B, D, M), s.tok.view(B, D, M), tokens, mask, p, sel, n_sel, where, node=_i32([1] * B), n_nodes=D)
    top = s.conf.view(B, D, M)[:, 1].sort(dim=1, descending=True, stable=True).indices[:, :2]
    assert n_sel.tolist() == [2, 2] and bool((mask.gather(1, top) == 0).all())
    assert torch.equal(tokens.gather(1, top), s.tok.view(B, D, M)[:, 1].gather(1, top))


def test_captured_steps_share_workspaces():
    """Two graphs over different buffers and the same workspaces, replayed in turn on new inputs, on a stream of their own."""
    a = _Step(2)
    b = _Step(3, a.space, a.space2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for s in (a, b):
            s.run()                                            # (the kernels are loaded before the capture)
        for s in (a, b):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                s.run()
            graphs.append(g)
        for turn in range(3):
            for s in (a, b):
                s.qkv.copy_(_rnd(10 + turn)(*s.qkv.shape))
                s.k.copy_(_rnd(20 + turn)(*s.k.shape))
                s.length.copy_(_i32([200 + 50 * turn, 512 - turn]))
            for g in graphs:
                g.replay()
            for g in reversed(graphs):
                g.replay()
    side.synchronize()
    replayed = [s.results() for s in (a, b)]
    for s, want in zip((a, b), replayed):
        for x in (s.q, s.ko, s.vo, s.out, s.lse, s.tok, s.conf):
            x.fill_(3)
        s.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(s.results(), want)) and int(s.status.item()) == 0
    del graphs


def test_two_streams_at_once():
    """Two steps with workspaces of their own, on two streams, give what each gives alone."""
    steps = [_Step(4), _Step(5)]
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append(s.results())
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(10):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert all(torch.equal(x, y) for x, y in zip(s.results(), w))


def test_a_workspace_for_the_largest_batch_serves_smaller_ones():
    big = _space(psd.psd_attention_q8_workspace_bytes(32, 4, 32, 8, 2, 128, 2000, 32))
    for B, D, M in ((32, 4, 32), (5, 4, 32), (1, 1, 32), (32, 4, 1), (3, 1, 1), (1, 4, 32)):
        shape = (B, D, M, 8, 2, 128, 2000, M)
        if M == 1:
            big_one = _space(psd.psd_attention_q8_workspace_bytes(32, 4, 1, 8, 2, 128, 2000, 32))
        t, _, _ = _inputs(shape, 11)
        out, lse = _attend(t, big if M > 1 else big_one)
        o, l = _attend(t)
        assert torch.equal(o, out) and torch.equal(l, lse)


@pytest.mark.parametrize("what", [ROWS, PARTIAL, JOINED, JOINED_ONE, FUSED, "head"])
def test_a_wait_that_runs_out(what):
    """With the loaders told to wait on a barrier that nothing arrives on, the call and its kernels return and the status word says so; the next call is
    as ever."""
    if what == "head":
        hidden, w, ws = _head_inputs(130, 256, 2000, "bf16", 6)
        call = lambda: _run_head(hidden, w, ws)  # noqa: E731
    else:
        t, _, _ = _inputs(what, 12)

        def call():
            status = _i32([0])
            r = _attend(t, status=status)
            torch.cuda.synchronize()
            return (*r, int(status.item()))
    want = call()
    assert want[-1] == 0
    assert psd.psd_set_tuning(psd.PSD_TUNE_WAIT_LIMIT, 400) == 0          # 400 000 cycles: about 0.2 ms
    assert psd.psd_set_tuning(psd.PSD_TUNE_SELFTEST_STALL, 1) == 0
    try:
        assert call()[-1] == psd.PSD_ERR_TIMEOUT
    finally:
        psd.psd_set_tuning(psd.PSD_TUNE_SELFTEST_STALL, 0)
        psd.psd_set_tuning(psd.PSD_TUNE_WAIT_LIMIT, 4_000_000)
    got = call()
    assert got[-1] == 0 and all(torch.equal(x, y) for x, y in zip(got[:-1], want[:-1]))

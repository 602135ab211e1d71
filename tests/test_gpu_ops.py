"""The operators around the step against plain 64-bit implementations.

Tolerances, from the arithmetic (u = unit roundoff of the inputs' type, 2^-8 for bf16, 2^-11 for fp16):
  scores: fp32 sums of Dh products, error e <= (Dh + 4) * 2^-24 * max_j sum_d |q_d k_d| * scale, plus 2^-22 times the
  largest exponent argument for its rounding; weights carry a relative 2 * that plus 2^-18 for the exponential;
  attention: each weight is rounded to the type (u * sum_j p_j |v_j|) and the output once (u * |out|);
  prefix weights: the relative error of the weights, plus 2^-24 per addend for the sum;
  confidences: 2^-24 per addend of a lane's sum (at most 600) and the exponential: a relative 6e-5."""
import numpy as np
import pytest
import torch

import ops_plain as plain
import paper_2605_15609_b200 as psd

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _f64(t):
    return t.detach().double().cpu().numpy()


def _lens(n, most, seed):
    r = np.random.default_rng(seed)
    x = [int(v) for v in r.integers(0, most + 1, n)]
    x[0] = most
    if n > 1:
        x[1] = min(1, most)
    if n > 2:
        x[2] = 0
    return x


def _layout(t, how):
    """The same values in another memory layout."""
    if how == "dense":
        return t
    if how == "heads_first":                 # [outer, head, token, Dh]
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    pad = torch.full((*t.shape[:2], t.shape[2] + 2, t.shape[3] + 8), float("nan"), dtype=t.dtype, device=t.device)
    v = pad[:, :, 1:-1, 8:] if t.shape[3] % 8 == 0 else pad
    v.copy_(t)
    return v


def _attention_case(B, D, M, Hq, Hkv, Dh, P, S, dtype, seed, layout="dense", full=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(DT[dtype])  # noqa: E731
    N = B * D
    plen = [P] * B if full else _lens(B, P, seed)
    olen = [S] * N if full else _lens(N, S, seed + 1)
    q, kp, vp, ko, vo = rnd(N, M, Hq, Dh), rnd(B, P, Hkv, Dh), rnd(B, P, Hkv, Dh), rnd(N, S, Hkv, Dh), rnd(N, S, Hkv, Dh)
    for b in range(B):
        kp[b, plen[b]:] = float("nan")
        vp[b, plen[b]:] = float("inf")
    for n in range(N):
        ko[n, olen[n]:] = float("inf")
        vo[n, olen[n]:] = float("nan")
    kp, vp, ko, vo = (_layout(t, layout) for t in (kp, vp, ko, vo))
    if layout == "heads_first":              # a run of tokens per head (nodes stay M tokens apart)
        q = q.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    else:
        q = _layout(q, layout)
    return q, kp, vp, ko, vo, plen, olen


def _run_attention(q, kp, vp, ko, vo, plen, olen, scale, causal, out=None):
    N, M, Hq, Dh = q.shape
    B, P, Hkv, _ = kp.shape
    S = ko.shape[1] if ko is not None else 0
    out = torch.full((N, M, Hq, Dh), 7.0, dtype=q.dtype, device="cuda") if out is None else out
    lse = torch.full((N, M, Hq), 7.0, device="cuda")
    status = _i32([0])
    ws = torch.full((psd.psd_attention_workspace_bytes(B, N // B, M, Hq, Hkv, Dh, P, S),), 255, dtype=torch.uint8, device="cuda")
    psd.psd_draft_attention(q, kp, vp, out, lse, ko, vo, prefix_len=None if plen is None else _i32(plen),
                            own_len=None if olen is None else _i32(olen), scale=scale, causal=causal, workspace=ws,
                            status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return out, lse


def _check_attention(out, lse, q, kp, vp, ko, vo, plen, olen, scale, causal, dtype):
    want, wlse, absv, big = plain.draft_attention(_f64(q), _f64(kp), _f64(vp), plen, _f64(ko), _f64(vo), olen, scale, causal)
    e = (q.shape[3] + 4) * 2.0 ** -24 * big + 2.0 ** -22 * max(1.0, big)
    got, glse = _f64(out), _f64(lse)
    empty = np.isinf(wlse)
    assert np.array_equal(np.isinf(glse), empty) and np.all(got[empty] == 0)
    assert np.all(np.abs(glse[~empty] - wlse[~empty]) <= 2 * e + 2.0 ** -18 + 2.0 ** -22 * np.abs(wlse[~empty]))
    rel = 2 * e + 2.0 ** -17
    tol = U[dtype] * (absv + np.abs(want)) * (1 + rel) + rel * absv + 1e-7
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) - tol).max())


ATT = [  # B, D, M, Hq, Hkv, Dh, P, S
    (1, 1, 1, 1, 1, 8, 1, 1), (1, 1, 1, 8, 8, 64, 300, 5), (2, 3, 1, 8, 2, 128, 129, 70), (3, 2, 5, 6, 2, 64, 127, 5),
    (1, 4, 32, 4, 4, 64, 257, 32), (2, 2, 32, 14, 2, 128, 200, 32), (3, 1, 7, 7, 1, 80, 385, 9), (1, 2, 64, 4, 2, 128, 700, 64),
    (1, 8, 3, 128, 1, 96, 140, 3), (4, 1, 40, 2, 2, 128, 0, 40), (4, 2, 16, 3, 3, 72, 130, 0), (3, 1, 2, 2, 1, 32, 0, 0),
    (2, 9, 33, 5, 5, 128, 1030, 33), (1, 1, 300, 2, 2, 64, 64, 300), (1, 64, 1, 8, 2, 128, 1500, 40),
]


@pytest.mark.parametrize("shape", ATT)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention(shape, dtype):
    B, D, M, Hq, Hkv, Dh, P, S = shape
    for causal in (False, True):
        c = _attention_case(*shape, dtype, seed=sum(shape))
        out, lse = _run_attention(*c, Dh ** -0.5, causal)
        _check_attention(out, lse, *c, Dh ** -0.5, causal, dtype)


# several query tiles over an unsplit prefix: the own keys are further tiles of the same kernel, up to five drafts per tile
ATT_FUSED = [(2, 6, 32, 2, 2, 64, 100, 32), (3, 6, 32, 3, 1, 128, 255, 32), (4, 5, 33, 2, 2, 72, 140, 150), (3, 3, 150, 4, 2, 128, 1, 150),
             (4, 9, 31, 7, 1, 96, 200, 40)]


# prefixes long enough for the tensor-core kernel: split along the keys, one and several query tiles
ATT_LONG = [(1, 1, 1, 2, 1, 64, 2100, 3), (2, 3, 1, 8, 2, 128, 1153, 70), (1, 4, 32, 4, 4, 64, 3001, 32), (3, 2, 5, 6, 2, 128, 1279, 5),
            (2, 2, 40, 14, 2, 80, 1400, 40), (1, 8, 3, 128, 1, 96, 900, 3), (1, 2, 150, 3, 3, 128, 1025, 150)]
# the same with enough sequences and heads that nothing is split
ATT_UNSPLIT = [(5, 6, 32, 16, 16, 64, 1200, 32), (4, 5, 33, 20, 20, 72, 700, 150), (10, 3, 20, 56, 8, 128, 650, 20)]


@pytest.mark.parametrize("shape", ATT_LONG)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout", ["dense", "heads_first"])
def test_attention_long_prefix(shape, dtype, layout):
    for causal in (False, True):
        c = _attention_case(*shape, dtype, seed=sum(shape) + causal, layout=layout)
        out, lse = _run_attention(*c, shape[5] ** -0.5, causal)
        _check_attention(out, lse, *c, shape[5] ** -0.5, causal, dtype)


@pytest.mark.parametrize("shape", ATT_UNSPLIT)
@pytest.mark.parametrize("causal", [False, True])
def test_attention_unsplit_prefix(shape, causal):
    dtype = "fp16" if causal else "bf16"
    c = _attention_case(*shape, dtype, seed=sum(shape), layout="padded" if causal else "dense")
    out, lse = _run_attention(*c, shape[5] ** -0.5, causal)
    _check_attention(out, lse, *c, shape[5] ** -0.5, causal, dtype)


def test_attention_unsplit_isolation_and_far_scores():
    """Five drafts to a query tile: NaN in one draft's keys reaches no other draft; scores of one draft far above or below
    another's of the same tile, with and without a prefix."""
    q, kp, vp, ko, vo, plen, olen = _attention_case(5, 6, 32, 16, 16, 64, 1200, 32, "bf16", 31, full=True)
    q[..., 0], ko[..., 0] = 8.0, 0.0
    for n in range(30):
        ko[n, :, :, 0] = (-120.0, 60.0, 0.0, -30.0, 90.0, -200.0)[n % 6]
    plen = [0, 1200, 37, 1, 640]
    a = _run_attention(q, kp, vp, ko, vo, plen, olen, 1.0, False)
    _check_attention(*a, q, kp, vp, ko, vo, plen, olen, 1.0, False, "bf16")
    for bad in (1, 2, 27):
        ko2, vo2 = ko.clone(), vo.clone()
        ko2[bad], vo2[bad] = float("nan"), float("inf")
        b = _run_attention(q, kp, vp, ko2, vo2, plen, olen, 1.0, False)
        others = [n for n in range(30) if n != bad]
        assert torch.equal(a[0][others], b[0][others]) and torch.equal(a[1][others], b[1][others])
        assert bool(torch.isnan(b[0][bad]).all())


def test_attention_long_prefix_extreme_scores():
    """Raises of the running maximum by far more than its threshold, in both directions, in several tiles."""
    c = list(_attention_case(1, 2, 64, 4, 2, 128, 2500, 64, "bf16", 37, full=True))
    for at, f in ((5, 20.0), (500, -60.0), (1300, 60.0), (2499, 90.0)):
        c[1][0, at] *= f
    out, lse = _run_attention(*c, 0.5, False)
    _check_attention(out, lse, *c, 0.5, False, "bf16")


@pytest.mark.parametrize("shape", ATT_FUSED)
@pytest.mark.parametrize("layout", ["dense", "padded"])
def test_attention_own_keys_after_an_unsplit_prefix(shape, layout):
    for causal in (False, True):
        for dtype in ("bf16", "fp16"):
            c = _attention_case(*shape, dtype, seed=sum(shape) + causal, layout=layout)
            out, lse = _run_attention(*c, 0.3, causal)
            _check_attention(out, lse, *c, 0.3, causal, dtype)


def test_attention_own_scores_far_from_the_prefix():
    """Rows whose first keys are their own, far below or above anything another draft of the same tile has; no prefix for
    one sequence, a long way up from the prefix for another."""
    q, kp, vp, ko, vo, plen, olen = _attention_case(3, 6, 32, 2, 2, 64, 100, 32, "bf16", 29, full=True)
    q[:, :, :, 0], ko[..., 0] = 8.0, 0.0
    for n in range(18):
        ko[n, :, :, 0] = (-120.0, 60.0, 0.0, -30.0, 90.0, -200.0)[n % 6]
    plen = [0, 100, 37]
    c = (q, kp, vp, ko, vo, plen, olen)
    for causal in (False, True):
        out, lse = _run_attention(*c, 1.0, causal)
        _check_attention(out, lse, *c, 1.0, causal, "bf16")


@pytest.mark.parametrize("layout", ["heads_first", "padded"])
@pytest.mark.parametrize("shape", [ATT[2], ATT[5], ATT[7], ATT[12]])
def test_attention_strides(shape, layout):
    Dh = shape[5]
    c = _attention_case(*shape, "bf16", seed=3, layout=layout)
    q = c[0]
    wide = torch.full((q.shape[0], q.shape[1], q.shape[2] + 1, Dh + 16), 5.0, dtype=q.dtype, device="cuda")
    out, lse = _run_attention(*c, 0.2, False, out=wide[:, :, 1:, 16:])
    _check_attention(out, lse, *c, 0.2, False, "bf16")
    assert bool((wide[:, :, :1] == 5).all()) and bool((wide[..., :16] == 5).all())     # nothing beside the output is written


def test_attention_shared_prefix_of_all_sequences():
    """One prefix for the whole batch, given as an expanded tensor (stride 0), is read in place."""
    q, kp, vp, ko, vo, plen, olen = _attention_case(3, 2, 4, 8, 2, 64, 300, 4, "bf16", 5, full=True)
    kp, vp = kp[:1].expand(3, -1, -1, -1), vp[:1].expand(3, -1, -1, -1)
    plen = [300, 17, 128]
    out, lse = _run_attention(q, kp, vp, ko, vo, plen, olen, 0.125, False)
    _check_attention(out, lse, q, kp, vp, ko, vo, plen, olen, 0.125, False, "bf16")


def test_attention_lengths_are_clamped_and_default_to_the_capacity():
    c = _attention_case(2, 2, 4, 4, 2, 64, 150, 6, "bf16", 9, full=True)
    a = _run_attention(*c[:5], None, None, 0.125, False)
    b = _run_attention(*c[:5], [1 << 30, 151], [7, 1 << 30, 6, 6], 0.125, False)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    z = _run_attention(*c[:5], [-5, -1], [-1, -7, 0, -2], 0.125, False)
    assert bool((z[0] == 0).all()) and bool((z[1] == -float("inf")).all())


@pytest.mark.parametrize("shape", [ATT[4], ATT[5], ATT[14], ATT_FUSED[0], ATT_FUSED[1], ATT_FUSED[4]])
def test_a_draft_never_sees_another_drafts_keys(shape):
    """NaN and infinities in one draft's own keys and values change no other draft's outputs, bit for bit."""
    q, kp, vp, ko, vo, plen, olen = _attention_case(*shape, "bf16", 11, full=True)
    a = _run_attention(q, kp, vp, ko, vo, plen, olen, 0.1, False)
    ko2, vo2 = ko.clone(), vo.clone()
    ko2[1], vo2[1] = float("nan"), float("inf")
    b = _run_attention(q, kp, vp, ko2, vo2, plen, olen, 0.1, False)
    others = [n for n in range(q.shape[0]) if n != 1]
    assert torch.equal(a[0][others], b[0][others]) and torch.equal(a[1][others], b[1][others])
    assert bool(torch.isnan(b[0][1]).all())


def test_attention_extreme_scores():
    """Large scores of either sign in one row: the running maximum carries them."""
    c = list(_attention_case(1, 2, 8, 4, 2, 64, 900, 8, "bf16", 13, full=True))
    c[1][0, 5] *= 60.0
    c[1][0, 500] *= -60.0
    c[1][0, 899] *= 90.0
    out, lse = _run_attention(*c, 1.0, False)
    _check_attention(out, lse, *c, 1.0, False, "bf16")


def test_attention_equal_bits_again_and_on_another_stream():
    c = _attention_case(2, 4, 32, 8, 2, 128, 2100, 32, "bf16", 17)
    a = _run_attention(*c, 0.09, False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = _run_attention(*c, 0.09, False)
    s.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_attention_far_offsets():
    """A cache whose sequences start beyond 2^32 elements."""
    P, Hkv, Dh = 8, 1, 64
    far = (1 << 32) + 4096                      # elements: 8.6 GB of bf16
    big = torch.empty(far + P * Hkv * Dh, dtype=torch.bfloat16, device="cuda")
    kp = big.as_strided((2, P, Hkv, Dh), (far, Hkv * Dh, Dh, 1))
    q, k0, v0, ko, vo, plen, olen = _attention_case(2, 1, 4, 2, Hkv, Dh, P, 4, "bf16", 19, full=True)
    kp.copy_(k0)
    out, lse = _run_attention(q, kp, kp, ko, vo, plen, olen, 0.125, False)
    _check_attention(out, lse, q, k0, k0, ko, vo, plen, olen, 0.125, False, "bf16")
    del big, kp


def test_binding_refuses_queries_that_are_no_run_of_tokens():
    q, kp, vp, ko, vo, plen, olen = _attention_case(2, 2, 4, 4, 2, 64, 50, 4, "bf16", 1)
    with pytest.raises(ValueError):
        _run_attention(_layout(q, "heads_first"), kp, vp, ko, vo, plen, olen, 0.125, False)
    with pytest.raises(ValueError):
        _run_attention(q, kp, vp.half(), ko, vo, plen, olen, 0.125, False)
    with pytest.raises(psd.PsdError):
        _run_attention(*(t.float() for t in (q, kp, vp, ko, vo)), plen, olen, 0.125, False)


# ---- prefix weights -----------------------------------------------------------------------------------------------------

WEIGHTS = [  # B, D, M, Hq, Hkv, Dh, P
    (1, 1, 1, 1, 1, 8, 1), (2, 3, 1, 8, 2, 128, 129), (3, 2, 5, 6, 2, 64, 127), (1, 4, 32, 14, 2, 80, 257), (2, 2, 33, 4, 4, 128, 300),
    (1, 2, 3, 128, 1, 96, 140), (1, 1, 300, 2, 2, 64, 515), (1, 8, 64, 2, 1, 128, 1000),
]


@pytest.mark.parametrize("shape", WEIGHTS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout", ["dense", "padded"])
def test_prefix_weights(shape, dtype, layout):
    B, D, M, Hq, Hkv, Dh, P = shape
    q, kp, _, _, _, plen, _ = _attention_case(B, D, M, Hq, Hkv, Dh, P, 1, dtype, sum(shape), layout)
    scale = Dh ** -0.5
    g = torch.Generator(device="cuda").manual_seed(4)
    lse = 4 + torch.rand(B * D, M, Hq, generator=g, device="cuda")
    lse.view(-1)[::5] = -float("inf")            # rows that saw no keys
    if M * Hq * B * D > 1:
        lse.view(-1)[1] = 2.0
    acc = torch.rand(B, Hkv, P, generator=g, device="cuda")
    ws = torch.full((psd.psd_weights_workspace_bytes(B, D, M, Hq, Hkv, Dh, P),), 255, dtype=torch.uint8, device="cuda")
    big = plain.draft_attention(_f64(q), _f64(kp), _f64(kp), plen, np.zeros((B * D, 0, Hkv, Dh)), np.zeros((B * D, 0, Hkv, Dh)),
                                [0] * (B * D), scale, False)[3]
    e = (Dh + 4) * 2.0 ** -24 * big + 2.0 ** -22 * (big + 5)
    rel = 2 * e + 2.0 ** -18 + D * M * (Hq // Hkv) * 2.0 ** -24
    for acc_in, beta in ((None, 1.0), (acc, 0.75)):
        out = torch.full_like(acc, 9.0)
        status = _i32([0])
        psd.psd_prefix_weights(q, kp, lse, out, acc_in=acc_in, beta=beta, prefix_len=_i32(plen), scale=scale, workspace=ws,
                               status=status)
        again = acc.clone()                      # in place
        psd.psd_prefix_weights(q, kp, lse, again, acc_in=again if acc_in is not None else None, beta=beta,
                               prefix_len=_i32(plen), scale=scale, workspace=ws, status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and torch.equal(out, again)
        want = plain.prefix_weights(_f64(q), _f64(kp), plen, _f64(lse), scale, beta, None if acc_in is None else _f64(acc_in))
        assert np.all(np.abs(_f64(out) - want) <= rel * np.abs(want) + 1e-30)


def test_weights_of_an_attention_pass_sum_to_its_rows():
    """With lse from psd_draft_attention and no own keys, every row spreads a weight of one."""
    B, D, M, Hq, Hkv, Dh, P = 2, 3, 16, 8, 2, 64, 333
    q, kp, vp, _, _, plen, _ = _attention_case(B, D, M, Hq, Hkv, Dh, P, 1, "bf16", 23, full=True)
    _, lse = _run_attention(q, kp, vp, None, None, plen, None, 0.125, False)
    out = torch.empty(B, Hkv, P, device="cuda")
    ws = torch.empty(psd.psd_weights_workspace_bytes(B, D, M, Hq, Hkv, Dh, P), dtype=torch.uint8, device="cuda")
    psd.psd_prefix_weights(q, kp, lse, out, scale=0.125, workspace=ws)
    assert np.allclose(_f64(out).sum(-1), D * M * (Hq // Hkv), rtol=1e-4)


# ---- eviction -------------------------------------------------------------------------------------------------------------

EVICT = [  # B, Hkv, Dh, P, keep, sink, recent
    (1, 1, 8, 1, 1, 0, 0), (1, 2, 64, 50, 50, 1, 1), (1, 2, 64, 50, 80, 1, 1), (2, 3, 128, 1000, 250, 4, 32), (3, 2, 96, 1025, 1, 0, 0),
    (3, 4, 80, 3000, 1000, 0, 1000), (2, 1, 64, 5000, 700, 700, 0), (1, 2, 128, 2048, 2047, 3, 5), (1, 1, 64, 60000, 5000, 4, 100),
    # several CTAs per head, some with nothing to do; keys that stay in shared memory and (the last) that do not
    (3, 2, 64, 9001, 3000, 4, 64), (5, 3, 8, 16385, 1, 0, 0), (4, 8, 64, 20000, 19990, 100, 9000), (3, 16, 16, 33000, 2500, 30, 40),
    (1, 2, 8, 300000, 9000, 4, 100),
]


@pytest.mark.parametrize("shape", EVICT)
@pytest.mark.parametrize("kind", ["tails", "ties", "odd"])
def test_evict(shape, kind):
    B, Hkv, Dh, P, keep, sink, recent = shape
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    sc = torch.randn(B, Hkv, P, generator=g, device="cuda")
    if kind == "tails":
        sc = torch.exp(3 * sc)
    elif kind == "ties":
        sc = torch.round(sc)
        sc[sc == 1] = -0.0
    else:
        sc[..., ::7] = float("nan")
        sc[..., 1::11] = float("inf")
        sc[..., 2::13] = -float("inf")
        sc[..., 3::5] = torch.finfo(torch.float32).min
        sc[..., 4::9] = 1e-42
    plen = _lens(B, P, 3)
    dt = torch.float16 if kind == "odd" else torch.bfloat16
    k, v = (_layout(torch.randn(B, P, Hkv, Dh, generator=g, device="cuda").to(dt), lay) for lay in ("padded", "heads_first"))
    k_out = torch.full((B, Hkv, keep, Dh), 3.0, dtype=dt, device="cuda").transpose(1, 2)
    v_out = torch.full((B, keep, Hkv, Dh), 3.0, dtype=dt, device="cuda")
    index = torch.full((B, Hkv, keep), -9, dtype=torch.int32, device="cuda")
    so = torch.full((B, Hkv, keep), 9.0, device="cuda")
    ln = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    psd.psd_prefix_evict(sc, k, v, k_out, v_out, index, so, ln, prefix_len=_i32(plen), n_sink=sink, n_recent=recent)
    torch.cuda.synchronize()
    want = plain.prefix_evict(sc.cpu().numpy(), plen, keep, sink, recent)
    assert ln.tolist() == [min(x, keep) for x in plen]
    for b in range(B):
        for h in range(Hkv):
            w = want[b][h]
            n = len(w)
            assert index[b, h].tolist() == w + [-1] * (keep - n)
            at = torch.tensor(w, dtype=torch.int64, device="cuda")
            assert torch.equal(k_out[b, :n, h], k[b, at, h]) and torch.equal(v_out[b, :n, h], v[b, at, h])
            assert bool((k_out[b, n:, h] == 3).all()) and bool((v_out[b, n:, h] == 3).all())
            assert torch.equal(torch.nan_to_num(so[b, h, :n], nan=77.0), torch.nan_to_num(sc[b, h, at], nan=77.0))
            assert bool((so[b, h, n:] == 0).all())


# ---- confidences from logits ------------------------------------------------------------------------------------------------

LOGITS = [  # B, D, M, V, T
    (1, 1, 1, 1, 0), (1, 1, 1, 33, 5), (1, 1, 1, 5000, 40), (2, 3, 1, 2049, 7), (1, 2, 5, 4096, 64), (3, 1, 2, 777, 1), (2, 2, 4, 1000, 30),
    (1, 4, 32, 8193, 100), (2, 1, 70, 640, 20), (1, 1, 3, 40000, 3000),
]


def _logits_case(B, D, M, V, T, dtype, seed, padded=False):
    rng = np.random.default_rng(seed)
    R, N = B * D * M, B * D
    x = torch.from_numpy(rng.normal(scale=2.0, size=(R, V)).astype(np.float32)).to(DT[dtype])
    if padded:
        wide = torch.full((R, V + 3), float("nan"), dtype=DT[dtype], device="cuda")
        wide[:, :V] = x.cuda()
        lg = wide[:, :V]
    else:
        lg = x.cuda()
    hist = rng.integers(-2, V + 2, size=(B, T)).astype(np.int32) if T else None
    if T > 3:
        hist[:, 1::2] = hist[:, :1]                         # one token many times
    hl = _lens(B, T, seed) if T else None
    dmask = rng.integers(0, 2, size=(N, M)).astype(np.int32)
    dtok = rng.integers(0, V + 1, size=(N, M)).astype(np.int32)
    return lg, x.float().numpy(), hist, hl, dtok, dmask, rng


def _run_logits(lg, B, D, M, **kw):
    R, V = lg.shape
    tok = torch.full((R,), -7, dtype=torch.int32, device="cuda")
    conf, lse = torch.full((R,), -7.0, device="cuda"), torch.full((R,), -7.0, device="cuda")
    status = _i32([0])
    ws = torch.full((psd.psd_logits_workspace_bytes(R, V),), 255, dtype=torch.uint8, device="cuda")
    psd.psd_confidence_logits(lg, tok, conf, lse, B=B, D=D, M=M, workspace=ws, status=status, **kw)
    torch.cuda.synchronize()
    return tok.cpu().numpy(), _f64(conf), _f64(lse), int(status.item())


def _check_logits(got, x, n_bad=0):
    tok, conf, lse, status = got
    wt, wc, wl = plain.confidence(x)
    bad = np.isnan(wc)
    assert status == int(bad.sum()) == n_bad
    assert np.array_equal(tok[~bad], wt[~bad])
    assert np.all(np.isnan(conf[bad])) and np.all(np.isnan(lse[bad]))
    assert np.all(np.abs(conf[~bad] - wc[~bad]) <= 6e-5 * wc[~bad])
    fin = ~bad & np.isfinite(wl)
    assert np.array_equal(lse[~bad & ~fin], wl[~bad & ~fin])
    assert np.all(np.abs(lse[fin] - wl[fin]) <= 6e-5 + 2.0 ** -22 * np.abs(wl[fin]))


@pytest.mark.parametrize("shape", LOGITS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("padded", [False, True])
def test_logits_all_edits(shape, dtype, padded):
    B, D, M, V, T = shape
    lg, x, hist, hl, dtok, dmask, rng = _logits_case(*shape, dtype, sum(shape), padded)
    R, words = B * D * M, (V + 31) // 32
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    allow = rng.integers(-2 ** 31, 2 ** 31, size=(R, words)).astype(np.int32)
    if R > 2:
        allow[1] = 0                                        # a row with nothing left
        allow[2] = -1
    for bias_rows in sorted({1, B, R}):
        bias = np.zeros((bias_rows, V), np.float32)
        bias[:, ::17] = rng.normal(size=bias[:, ::17].shape)
        bias[:, 5::101] = np.finfo(np.float32).min
        want = plain.edited_logits(x, D, M, hist, hl, dtok, dmask, 1.3, 0.4, 0.15, bias, allow)
        got = _run_logits(lg, B, D, M, history=dev(hist), history_len=_i32(hl) if T else None, draft_tokens=dev(dtok),
                          draft_mask=dev(dmask), repetition=1.3, presence=0.4, frequency=0.15,
                          bias=dev(bias) if bias_rows > 1 else dev(bias[0]), allow=dev(allow))
        _check_logits(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_logits_one_edit_at_a_time(dtype):
    B, D, M, V, T = 2, 2, 3, 3001, 50
    lg, x, hist, hl, dtok, dmask, rng = _logits_case(B, D, M, V, T, dtype, 5)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    none = dict(history=None, hist_len=None, draft_tokens=None, draft_mask=None, rep=1.0, pres=0.0, freq=0.0, bias=None, allow=None)
    _check_logits(_run_logits(lg, B, D, M), plain.edited_logits(x, D, M, **none))
    for rep, pres, freq in ((0.5, 0.0, 0.0), (1.0, 2.0, 0.0), (1.0, 0.0, -1.0)):
        w = plain.edited_logits(x, D, M, **dict(none, history=hist, hist_len=hl, rep=rep, pres=pres, freq=freq))
        _check_logits(_run_logits(lg, B, D, M, history=dev(hist), history_len=_i32(hl), repetition=rep, presence=pres,
                                  frequency=freq), w)
    w = plain.edited_logits(x, D, M, **dict(none, draft_tokens=dtok, draft_mask=dmask, pres=30.0))
    _check_logits(_run_logits(lg, B, D, M, draft_tokens=dev(dtok), draft_mask=dev(dmask), presence=30.0), w)
    allow = rng.integers(-2 ** 31, 2 ** 31, size=(B, (V + 31) // 32)).astype(np.int32)
    w = plain.edited_logits(x, D, M, **dict(none, allow=allow))
    _check_logits(_run_logits(lg, B, D, M, allow=dev(allow)), w)
    bias = rng.normal(size=(1, V)).astype(np.float32)       # a dense bias
    _check_logits(_run_logits(lg, B, D, M, bias=dev(bias[0])), plain.edited_logits(x, D, M, **dict(none, bias=bias)))


def test_logits_ties_take_the_lowest_token():
    lg = torch.full((3, 20000), -1.0, dtype=torch.bfloat16, device="cuda")
    lg[1, [19999, 700, 13000]] = 4.0
    lg[2, [3, 9000]] = 4.0
    bias = torch.zeros(20000, device="cuda")
    bias[2] = 5.0                                           # an edited token ties with unedited ones
    got = _run_logits(lg, 1, 1, 3, bias=bias)
    assert got[0].tolist() == [2, 2, 2]
    assert _run_logits(lg, 1, 1, 3)[0].tolist() == [0, 700, 3]
    allow = torch.full((1, 625), -1, dtype=torch.int32, device="cuda")
    allow[0, 0] = 0
    assert _run_logits(lg, 1, 1, 3, allow=allow)[0].tolist() == [32, 700, 9000]


def test_logits_non_finite_values_and_lowest_values():
    V = 5000
    x = np.zeros((9, V), np.float32)
    low = float(torch.finfo(torch.bfloat16).min)
    x[0, 17] = np.nan
    x[1, 4999] = np.inf
    x[2] = -np.inf                                          # nothing left
    x[3] = low                                              # a row of the type's lowest value: uniform
    x[4] = -np.inf
    x[4, 44] = low
    x[5] = np.nan
    x[6, 100] = np.nan                                      # forbidden below: not seen
    x[7] = low
    x[7, 8] = 3.0
    x[8, 3] = -np.inf
    allow = np.full((9, (V + 31) // 32), -1, np.int32)
    allow[6, 3] &= ~(1 << 4)
    lg = torch.from_numpy(x).to(torch.bfloat16).cuda()
    want = lg.float().cpu().numpy()
    want[6, 100] = -np.inf
    for pad in (False, True):
        t = lg
        if pad:
            t = torch.zeros(9, V + 1, dtype=torch.bfloat16, device="cuda")
            t[:, :V] = lg
            t = t[:, :V]
        got = _run_logits(t, 1, 1, 9, allow=torch.from_numpy(allow).cuda())
        _check_logits(got, want, n_bad=3)
        assert got[0][2] == -1 and got[1][2] == 0 and got[2][2] == -np.inf
        assert abs(got[1][3] * V - 1) < 1e-4


def test_logits_feed_the_policy():
    """The confidences go straight into psd_select_unmask: a row without a token (confidence 0) is ranked last."""
    B, M, V = 1, 8, 1000
    lg = torch.randn(B * M, V, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    lg[torch.arange(M), torch.arange(M) * 7] = 20.0
    allow = torch.full((M, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
    allow[2] = 0
    tok, conf, lse, _ = _run_logits(lg, B, 1, M, allow=allow)
    t, c = torch.from_numpy(tok).cuda().view(1, 1, M), torch.from_numpy(conf.astype(np.float32)).cuda().view(1, 1, M)
    tokens, mask = torch.full((1, M), V, dtype=torch.int32, device="cuda"), torch.ones(1, M, dtype=torch.int32, device="cuda")
    sel, n_sel, pos = torch.zeros_like(mask), _i32([0]), torch.zeros_like(mask)
    psd.psd_select_unmask(c, t, tokens, mask, psd.policy(tau=0.9, k_min=1), sel, n_sel, pos)
    assert sel[0].tolist() == [1, 1, 0, 1, 1, 1, 1, 1] and mask[0, 2].item() == 1
    assert tokens[0].tolist() == [V if i == 2 else i * 7 for i in range(M)]


# ---- waits that run out -------------------------------------------------------------------------------------------------------

def test_waits_that_run_out_are_reported_and_the_next_call_is_fine():
    """With PSD_TUNE_SELFTEST_STALL the loader of every CTA waits, after its first tile, on a barrier that nothing arrives on: the
    wait runs out (400 000 cycles here), the kernels report PSD_ERR_TIMEOUT, let their own copies and products finish and return;
    with the knobs back the next call is right."""
    c = _attention_case(1, 2, 64, 8, 2, 128, 2500, 64, "bf16", 41, full=True)
    q, kp, vp, ko, vo, plen, olen = c
    N, M, Hq, Dh = q.shape
    out, lse = torch.empty_like(q), torch.zeros(N, M, Hq, device="cuda")
    ws = torch.zeros(psd.psd_attention_workspace_bytes(1, 2, 64, 8, 2, 128, 2500, 64), dtype=torch.uint8, device="cuda")
    acc = torch.zeros(1, 2, 2500, device="cuda")
    ws2 = torch.zeros(psd.psd_weights_workspace_bytes(1, 2, 64, 8, 2, 128, 2500), dtype=torch.uint8, device="cuda")
    s1, s2 = _i32([0]), _i32([0])
    assert psd.psd_set_tuning(psd.PSD_TUNE_WAIT_LIMIT, 400) == 0 and psd.psd_set_tuning(psd.PSD_TUNE_SELFTEST_STALL, 1) == 0
    try:
        psd.psd_draft_attention(q, kp, vp, out, lse, ko, vo, workspace=ws, status=s1)
        torch.cuda.synchronize()
        psd.psd_prefix_weights(q, kp, lse, acc, workspace=ws2, status=s2)
        torch.cuda.synchronize()
    finally:
        psd.psd_set_tuning(psd.PSD_TUNE_SELFTEST_STALL, 0)
        psd.psd_set_tuning(psd.PSD_TUNE_WAIT_LIMIT, 4_000_000)
    assert int(s1.item()) == int(s2.item()) == psd.PSD_ERR_TIMEOUT
    out, lse = _run_attention(*c, Dh ** -0.5, False)
    _check_attention(out, lse, *c, Dh ** -0.5, False, "bf16")

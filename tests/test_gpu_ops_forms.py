"""Every form that the drafts' attention and the prefix weights take, at shapes that are asserted to reach it: own keys behind an
unsplit prefix in one kernel, prefixes split up to 64 ways, caches shared by stride 0 and with offsets past 2^32 under a tensor map,
many sequences, and prefix weights with several units per CTA and several query tiles per unit.

Tolerances are those of test_gpu_ops.py: attention's from the rounding of weights and outputs (u sum_j p_j |v_j| + u |out|) and of
fp32 scores; prefix weights' relative error from the scores', the exponential's and 2^-24 per addend."""
import pytest
import torch

import ops_gpu64 as ref
import paper_2605_15609_b200 as psd
from test_gpu_ops import _attention_case, _i32, _lens, _run_attention, U

pytestmark = pytest.mark.gpu

ONE, FUSED, JOINED = "draft_attention_kernel", "prefix_attention_kernel", "prefix_attention_kernel+draft_attention_kernel"


def _form(shape):
    return psd.psd_attention_kernel_names(*shape)


def _check(got, c, scale, causal, dtype):
    q, kp, vp, ko, vo, plen, olen = c
    out, lse = got
    want, wlse, absv, big = ref.draft_attention(q, kp, vp, plen, ko, vo, olen, scale, causal)
    e = (q.shape[3] + 4) * 2.0 ** -24 * big + 2.0 ** -22 * max(1.0, big)
    empty = torch.isinf(wlse)
    assert torch.equal(torch.isinf(lse), empty) and bool((out[empty] == 0).all())
    lse, wlse = lse.double()[~empty], wlse[~empty]
    assert bool(((lse - wlse).abs() <= 2 * e + 2.0 ** -18 + 2.0 ** -22 * wlse.abs()).all())
    rel = 2 * e + 2.0 ** -17
    tol = U[dtype] * (absv + want.abs()) * (1 + rel) + rel * absv + 1e-7
    assert bool(((out.double() - want).abs() <= tol).all()), float(((out.double() - want).abs() - tol).max())


# B, D, M, Hq, Hkv, Dh, P, S: one and several drafts per query tile, odd numbers of query tiles, own keys of none to two tiles,
# head sizes between 64 and 128, groups of 1 to 128 heads
FUSED_SHAPES = [(6, 3, 43, 16, 16, 64, 1100, 32), (5, 5, 60, 16, 16, 64, 1100, 0), (4, 6, 31, 28, 4, 128, 700, 40), (3, 9, 33, 20, 10, 96, 900, 33),
                (2, 4, 150, 16, 8, 80, 1030, 150), (7, 7, 16, 24, 12, 72, 640, 16), (25, 3, 2, 128, 1, 64, 1300, 5), (5, 6, 32, 16, 16, 128, 1200, 23)]


@pytest.mark.parametrize("shape", FUSED_SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("full", [False, True])
def test_own_keys_behind_an_unsplit_prefix(shape, dtype, causal, full):
    assert _form(shape) == (FUSED, 1)
    c = list(_attention_case(*shape, dtype, seed=sum(shape) + causal, layout="padded" if full else "dense", full=full))
    if not full:
        c[6] = [min(x, shape[7]) if i % 5 else 0 for i, x in enumerate(c[6])]          # drafts without own keys among the others
    got = _run_attention(*c, 0.2, causal)
    _check(got, c, 0.2, causal, dtype)


@pytest.mark.parametrize("shape", [FUSED_SHAPES[2], FUSED_SHAPES[3], FUSED_SHAPES[7]])
def test_a_draft_behind_an_unsplit_prefix_never_sees_anothers_keys(shape):
    assert _form(shape) == (FUSED, 1)
    q, kp, vp, ko, vo, plen, olen = _attention_case(*shape, "bf16", 43, full=True)
    N = q.shape[0]
    plen = _lens(shape[0], shape[6], 3)
    a = _run_attention(q, kp, vp, ko, vo, plen, olen, 0.1, False)
    _check(a, (q, kp, vp, ko, vo, plen, olen), 0.1, False, "bf16")
    for bad in (0, 1, N // 2, N - 1):
        ko2, vo2 = ko.clone(), vo.clone()
        ko2[bad], vo2[bad] = float("nan"), float("inf")
        b = _run_attention(q, kp, vp, ko2, vo2, plen, olen, 0.1, False)
        others = [n for n in range(N) if n != bad]
        assert torch.equal(a[0][others], b[0][others]) and torch.equal(a[1][others], b[1][others])
        assert bool(torch.isnan(b[0][bad]).all())


def test_far_scores_behind_an_unsplit_prefix():
    shape = (5, 6, 32, 32, 16, 128, 700, 32)
    assert _form(shape) == (FUSED, 1)
    q, kp, vp, ko, vo, plen, olen = _attention_case(*shape, "bf16", 47, full=True)
    q[..., 0], ko[..., 0] = 8.0, 0.0
    for n in range(30):
        ko[n, :, :, 0] = (-120.0, 60.0, 0.0, -30.0, 90.0, -200.0)[n % 6]
    c = (q, kp, vp, ko, vo, [0, 700, 37, 1, 640], olen)
    for causal in (False, True):
        _check(_run_attention(*c, 1.0, causal), c, 1.0, causal, "bf16")


JOINED_SHAPES = [((1, 1, 8, 4, 1, 64, 16500, 5), 64), ((1, 4, 64, 2, 1, 128, 16400, 9), 64), ((2, 2, 40, 8, 1, 64, 9000, 9), 24),
                 # not split, many drafts per query tile; one query tile over two halves, as many sequences as are put in order, and more
                 ((5, 40, 4, 16, 16, 64, 1100, 4), 1), ((128, 2, 3, 4, 2, 64, 1100, 3), 2), ((150, 2, 3, 2, 1, 128, 1100, 3), 2)]


@pytest.mark.parametrize("shape,splits", JOINED_SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_partial_results_and_join(shape, splits, dtype):
    assert _form(shape) == (JOINED, splits)
    for full in (False, True):
        c = list(_attention_case(*shape, dtype, seed=sum(shape), full=full))
        if not full and shape[0] == 1:
            c[5] = [shape[6] // 3]                        # (the splits share what there is: some of one tile)
        causal = not full
        _check(_run_attention(*c, 0.15, causal), c, 0.15, causal, dtype)
    if shape[0] == 1:
        for L in (1, 127, 129, 700):                      # fewer tiles than splits
            c[5] = [L]
            _check(_run_attention(*c, 0.15, False), c, 0.15, False, dtype)


def test_unsplit_sequences_beyond_those_put_in_order():
    for B in (128, 129):
        shape = (B, 3, 50, 2, 2, 64, 1100, 20)
        assert _form(shape) == (FUSED, 1)
        c = _attention_case(*shape, "bf16", seed=B)
        _check(_run_attention(*c, 0.15, False), c, 0.15, False, "bf16")


def test_a_prompt():
    """Long own keys, causal, no prefix: a block of queries that are their own keys, and one behind earlier own keys."""
    for shape in ((1, 1, 1000, 4, 2, 128, 0, 1000), (2, 1, 70, 4, 4, 64, 0, 1500)):
        assert _form(shape) == (ONE, 0)
        c = _attention_case(*shape, "bf16", seed=3, full=True)
        _check(_run_attention(*c, 0.1, True), c, 0.1, True, "bf16")


def _weights(q, kp, plen, lse, scale, beta=1.0, acc_in=None):
    N, M, Hq, Dh = q.shape
    B, P, Hkv, _ = kp.shape
    status, out = _i32([0]), torch.full((B, Hkv, P), 9.0, device="cuda")
    ws = torch.full((psd.psd_weights_workspace_bytes(B, N // B, M, Hq, Hkv, Dh, P),), 255, dtype=torch.uint8, device="cuda")
    before = psd.psd_launch_count()
    psd.psd_prefix_weights(q, kp, lse, out, acc_in=acc_in, beta=beta, prefix_len=None if plen is None else _i32(plen), scale=scale,
                           workspace=ws, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return out, psd.psd_launch_count() - before


def _check_weights(out, q, kp, plen, lse, scale, beta=1.0, acc_in=None):
    N, M, Hq, Dh = q.shape
    B, P, Hkv, _ = kp.shape
    plen = [P] * B if plen is None else plen
    want, big = ref.prefix_weights(q, kp, plen, lse, scale, beta, acc_in)
    rows = N // B * M * (Hq // Hkv)
    far = float(lse[lse > -float("inf")].abs().max())
    rel = 2 * ((Dh + 4) * 2.0 ** -24 * big + 2.0 ** -22 * (big + far)) + 2.0 ** -18 + rows * 2.0 ** -24
    assert bool(((out.double() - want).abs() <= rel * want.abs() + 1e-30).all())
    for b in range(B):
        assert bool((out[b, :, plen[b]:] == 0).all())


def _weights_case(B, D, M, Hq, Hkv, Dh, P, dtype, seed, lens=True):
    q, kp, _, _, _, plen, _ = _attention_case(B, D, M, Hq, Hkv, Dh, P, 1, dtype, seed, full=not lens)
    g = torch.Generator(device="cuda").manual_seed(seed)
    lse = 4 + 2 * torch.rand(B * D, M, Hq, generator=g, device="cuda")
    lse.view(-1)[::7] = -float("inf")
    lse[-1] = -float("inf")                              # a draft that saw no keys
    return q, kp, plen if lens else None, lse, torch.rand(B, Hkv, P, generator=g, device="cuda")


# several units of 256 keys per CTA, one to eleven query tiles in a unit (the query ring holds four)
WEIGHTS = [(6, 8, 40, 16, 8, 128, 3000), (6, 3, 43, 16, 16, 64, 2600), (40, 4, 32, 14, 2, 80, 1300), (9, 11, 64, 16, 16, 128, 900)]


@pytest.mark.parametrize("shape", WEIGHTS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lens", [True, False])
def test_weights_with_several_units_per_cta(shape, dtype, lens):
    B, D, M, Hq, Hkv, Dh, P = shape
    q, kp, plen, lse, acc = _weights_case(*shape, dtype, sum(shape), lens)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    units = sum(-(-n // 256) for n in (plen or [P] * B)) * Hkv
    assert units > 1.5 * sms
    for acc_in, beta in ((None, 1.0), (acc, 0.75)):
        out, launches = _weights(q, kp, plen, lse, 0.2, beta, acc_in)
        assert launches == 1                              # the query rows are not split
        _check_weights(out, q, kp, plen, lse, 0.2, beta, acc_in)


def test_weights_of_units_with_one_and_two_key_tiles():
    """Lengths around the tiles' and units' ends, in turn, so that a CTA's units differ from one to the next."""
    B, P = 24, 1024
    q, kp, _, lse, acc = _weights_case(B, 4, 40, 16, 16, 64, P, "bf16", 5, lens=False)
    plen = ([1024, 1, 0, 127, 128, 129, 255, 256, 257, 383, 384, 385, 511, 640, 897, 1023] * 2)[:B]
    out, launches = _weights(q, kp, plen, lse, 0.2, 0.5, acc)
    assert launches == 1
    _check_weights(out, q, kp, plen, lse, 0.2, 0.5, acc)


@pytest.mark.parametrize("B", [256, 257, 300])
def test_weights_of_more_sequences_than_are_counted(B):
    c = _weights_case(B, 2, 100, 3, 3, 64, 600, "bf16", B)
    out, launches = _weights(*c[:4], 0.2, 0.5, c[4])
    assert launches == 1
    _check_weights(out, *c[:4], 0.2, 0.5, c[4])


@pytest.mark.parametrize("shape", [(4, 1, 1, 32, 8, 128, 9000), (1, 1, 1, 8, 1, 64, 20000), (64, 1, 1, 16, 16, 128, 1500)])
def test_weights_of_single_tokens(shape):
    q, kp, plen, lse, acc = _weights_case(*shape, "bf16", 11)
    lse[-1] = 5.0
    out, _ = _weights(q, kp, plen, lse, 0.2, 0.9, acc)
    _check_weights(out, q, kp, plen, lse, 0.2, 0.9, acc)


def test_weights_of_split_query_rows():
    """Few keys and many rows: the rows' sums come from several CTAs and are joined."""
    shape = (1, 8, 300, 8, 2, 128, 700)
    q, kp, plen, lse, acc = _weights_case(*shape, "fp16", 13)
    out, launches = _weights(q, kp, plen, lse, 0.2, 0.5, acc)
    assert launches == 2
    _check_weights(out, q, kp, plen, lse, 0.2, 0.5, acc)


SHARED = [(3, 4, 32, 8, 4, 64, 1500, 16), (5, 6, 32, 16, 16, 64, 1200, 32), (4, 1, 1, 8, 2, 128, 3000, 4)]


@pytest.mark.parametrize("shape", SHARED)
@pytest.mark.parametrize("what", ["sequences", "heads", "both", "own"])
def test_caches_shared_by_stride_zero(shape, what):
    """One cache for all sequences, for all key heads, or both; one set of own keys for all drafts and heads."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    assert _form(shape)[0] != ONE
    q, kp, vp, ko, vo, plen, olen = _attention_case(*shape, "bf16", 17, full=True)
    if what in ("sequences", "both"):
        kp, vp = kp[:1].expand(B, -1, -1, -1), vp[:1].expand(B, -1, -1, -1)
    if what in ("heads", "both"):
        kp, vp = (t[:, :, :1].expand(-1, -1, Hkv, -1) for t in (kp, vp))
    if what == "own":
        ko, vo = (t[:1, :, :1].expand(B * D, -1, Hkv, -1) for t in (ko, vo))
    c = (q, kp, vp, ko, vo, _lens(B, P, 5), olen)
    got = _run_attention(*c, 0.15, False)
    _check(got, c, 0.15, False, "bf16")
    lse = torch.where(torch.isinf(got[1]), got[1], got[1] + 1)
    out, _ = _weights(q, kp, c[5], lse, 0.15)
    _check_weights(out, q, kp, c[5], lse, 0.15)


@pytest.mark.parametrize("far", ["sequence", "token"])
def test_offsets_past_32_bits_under_a_tensor_map(far):
    """Sequences, or tokens, whose addresses pass 2^32 elements (9 to 10 GB of bf16)."""
    B, D, M, Hq, Hkv, Dh, P, S = 2, 3, 40, 4, 2, 64, 1100, 8
    assert _form((B, D, M, Hq, Hkv, Dh, P, S))[0] != ONE
    row = Hkv * Dh
    if far == "sequence":
        strides = ((1 << 32) + 4096, row, Dh, 1)
        n = strides[0] + P * row
    else:
        strides = (row, 1 << 22, Dh, 1)                   # the sequences next to each other within a token
        n = (P - 1) * strides[1] + B * row
    assert n > 1 << 32
    big = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    kp = big.as_strided((B, P, Hkv, Dh), strides)
    q, k0, v0, ko, vo, plen, olen = _attention_case(B, D, M, Hq, Hkv, Dh, P, S, "bf16", 19, full=True)
    kp.copy_(k0)
    got = _run_attention(q, kp, kp, ko, vo, plen, olen, 0.125, False)
    _check(got, (q, k0, k0, ko, vo, plen, olen), 0.125, False, "bf16")
    out, _ = _weights(q, kp, plen, got[1], 0.125)
    _check_weights(out, q, k0, plen, got[1], 0.125)
    del big, kp


def test_kernel_names():
    assert psd.psd_attention_kernel_names(0, 1, 1, 1, 1, 8, 1, 1) is None
    assert psd.psd_attention_kernel_names(1, 1, 1, 1, 1, 8, 0, 1) == (ONE, 0)


@pytest.mark.parametrize("P", [1, 30, 100, 128, 130])
@pytest.mark.parametrize("shape", [(16, 4, 32, 32, 8, 128, 32), (8, 4, 32, 32, 4, 64, 20), (16, 16, 4, 32, 8, 128, 4), (12, 9, 16, 8, 8, 64, 3)])
def test_own_keys_behind_a_short_unsplit_prefix(shape, P):
    """Prefixes shorter than a tile of keys, up to nine drafts to a tile."""
    drafts = (128 // (shape[3] // shape[4]) + shape[2] - 2) // shape[2] + 1
    shape = (*shape[:6], P + 321 if drafts > 3 else P, shape[6])           # (several drafts to a tile: from longer prefixes on)
    assert _form(shape) == (FUSED, 1)
    for causal in (False, True):
        c = _attention_case(*shape, "bf16", seed=P + causal)
        _check(_run_attention(*c, 0.2, causal), c, 0.2, causal, "bf16")


@pytest.mark.parametrize("shape", [(16, 16, 4, 32, 8, 128, 1024, 32), (8, 64, 2, 64, 8, 128, 1024, 2), (16, 32, 16, 16, 16, 64, 700, 16)])
def test_nine_drafts_to_a_tile(shape):
    assert _form(shape) == (FUSED, 1)
    q, kp, vp, ko, vo, plen, olen = c = _attention_case(*shape, "fp16", seed=5)
    a = _run_attention(*c, 0.2, True)
    _check(a, c, 0.2, True, "fp16")
    ko2, vo2 = ko.clone(), vo.clone()
    ko2[9], vo2[9] = float("nan"), float("nan")
    b = _run_attention(q, kp, vp, ko2, vo2, plen, olen, 0.2, True)
    others = [n for n in range(q.shape[0]) if n != 9]
    assert torch.equal(a[0][others], b[0][others]) and torch.equal(a[1][others], b[1][others])

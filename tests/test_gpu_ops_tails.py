"""Attention whose weight is spread over many keys far below the highest score, in a type of narrow range.

fp16 holds nothing below 2^-25, so a weight kept relative to the row's maximum would be lost below that, although thousands of such
keys together count.  Weights are therefore kept relative to a reference 2^7 or more below the maximum: a weight is off by at most
2^-32 of the largest, and the output by N * 2^-32 * max |v| over N keys, beside what rounding the weights and the output costs."""
import numpy as np
import pytest
import torch

import ops_plain as plain
import paper_2605_15609_b200 as psd

pytestmark = pytest.mark.gpu
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _one_high_key(N, H, Dh, n, dtype, at, score):
    """Keys [N, n, H, Dh] that all score 0 but the one at `at`, whose value is 0 where the others' are 1."""
    k, v = torch.zeros(N, n, H, Dh, dtype=DT[dtype], device="cuda"), torch.ones(N, n, H, Dh, dtype=DT[dtype], device="cuda")
    k[:, at, :, 0], v[:, at] = score / 4.0, 0.0
    return k, v


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("score", [10.0, 16.0, 18.5])
@pytest.mark.parametrize("form", ["split", "one tile of queries", "two halves", "unsplit", "own keys", "short prefix"])
def test_many_keys_far_below_the_highest(form, score, dtype):
    B, D, M, Hq, Hkv, Dh, P, S = {"split": (1, 4, 32, 4, 2, 64, 20000, 3), "one tile of queries": (1, 1, 4, 2, 1, 128, 20000, 0),
                                  "two halves": (5, 4, 16, 32, 32, 64, 4000, 2), "unsplit": (5, 4, 40, 16, 16, 64, 4000, 2), "own keys": (1, 1, 3, 2, 1, 128, 0, 6000),
                                  "short prefix": (2, 2, 8, 2, 2, 64, 900, 0)}[form]
    N = B * D
    q = torch.zeros(N, M, Hq, Dh, dtype=DT[dtype], device="cuda")
    q[..., 0] = 4.0
    at = {"own keys": 0, "split": 700}.get(form, 130)
    kp, vp = _one_high_key(B, Hkv, Dh, P, dtype, at, score) if P else (torch.empty(B, 0, Hkv, Dh, dtype=q.dtype, device="cuda"),) * 2
    ko, vo = _one_high_key(N, Hkv, Dh, S, dtype, 0, score if not P else 0.0) if S else (None, None)
    out, lse = torch.full_like(q, 7.0), torch.full((N, M, Hq), 7.0, device="cuda")
    ws = torch.full((psd.psd_attention_workspace_bytes(B, D, M, Hq, Hkv, Dh, P, S),), 255, dtype=torch.uint8, device="cuda")
    psd.psd_draft_attention(q, kp, vp, out, lse, ko, vo, scale=1.0, workspace=ws)
    torch.cuda.synchronize()
    # every row is the same: one high key, the others at 0 (of the own keys beside a prefix the first has value 0)
    n_zero = P + S - 1
    w = float(np.exp(-score))
    total = 1.0 + n_zero * w
    want = (n_zero - (1 if P and S else 0)) * w / total
    tol = U[dtype] * 2 * want * (1 + 2.0 ** -16) + 2.0 ** -16 * want + (P + S) * 2.0 ** -32 + 1e-7
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol), (float((out.double() - want).abs().max()), want, tol)
    assert np.all(np.abs(lse.double().cpu().numpy() - (score + np.log(total))) <= 2.0 ** -17 + 2.0 ** -22 * score)


def test_the_widest_weights_stay_finite():
    """fp16 with the largest values there are, a maximum that rises just short of the threshold from tile to tile, and from far below."""
    B, D, M, Hq, Hkv, Dh, P = 1, 4, 32, 4, 2, 64, 4000
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.zeros(D, M, Hq, Dh, dtype=torch.float16, device="cuda")
    q[..., 0] = 1.0
    k = torch.zeros(B, P, Hkv, Dh, dtype=torch.float16, device="cuda")
    k[0, :, :, 0] = (torch.arange(P, device="cuda") // 128 * 5.5 + 0.25 * torch.rand(P, generator=g, device="cuda"))[:, None].half()
    v = torch.where(torch.rand(B, P, Hkv, Dh, generator=g, device="cuda") < 0.5, 65504.0, -65504.0).half()
    out, lse = torch.zeros_like(q), torch.zeros(D, M, Hq, device="cuda")
    ws = torch.empty(psd.psd_attention_workspace_bytes(B, D, M, Hq, Hkv, Dh, P, 0), dtype=torch.uint8, device="cuda")
    psd.psd_draft_attention(q, k, v, out, lse, scale=1.0, workspace=ws)
    torch.cuda.synchronize()
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    none = np.zeros((D, 0, Hkv, Dh))
    want, wlse, absv, _ = plain.draft_attention(f(q)[:1, :1], f(k), f(v), [P], none[:1], none[:1], [0], 1.0, False)
    tol = U["fp16"] * (absv + np.abs(want)) * 1.001 + P * 2.0 ** -32 * 65504 + 2.0 ** -16 * absv
    assert np.all(np.abs(f(out) - want) <= tol)
    assert np.all(np.abs(f(lse) - wlse) <= 2.0 ** -16 + 2.0 ** -22 * np.abs(wlse))

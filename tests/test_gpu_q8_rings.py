"""Own keys behind prefixes in codes that are long enough for both rings of the query tiles' kernel (codes, and 16-bit tiles) to have wrapped several
times when the first own tile arrives.  Against 64 bits on the GPU; tolerances as in test_gpu_q8.py."""
import math

import pytest
import torch

import ops_gpu64
import paper_2605_15609_b200 as psd
from test_gpu_q8 import U
from test_gpu_q8_service import _attend, _inputs

pytestmark = pytest.mark.gpu

FUSED = [(20, 3, 33, 16, 8, 64, 3000, 33), (16, 4, 32, 16, 8, 128, 2500, 32), (17, 3, 70, 8, 4, 80, 2100, 70), (12, 6, 32, 28, 4, 128, 3900, 40), (10, 2, 150, 8, 4, 96, 2300, 170)]
JOINED = [(1, 1, 32, 32, 8, 128, 8192, 32), (1, 2, 16, 8, 2, 64, 9000, 40), (2, 1, 20, 8, 2, 96, 12000, 150), (2, 4, 33, 14, 2, 64, 8192, 33), (1, 4, 32, 32, 8, 128, 6000, 100)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", FUSED + JOINED)
def test_own_keys_behind_a_long_prefix(shape, causal, dtype):
    B, D, M, Hq, Hkv, Dh, P, S = shape
    names, splits = psd.psd_attention_q8_kernel_names(*shape)
    assert names == "prefix_tiles_q8_kernel" and (splits == 1) == (shape in FUSED)
    plen = [P - (b % 4) * 129 - (b % 3) for b in range(B)]
    olen = [[S, S // 2, 1, 0][n % 4] for n in range(B * D)]
    t, kp, vp = _inputs(shape, 31, {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype], 32, plen, olen)
    past = torch.arange(S, device="cuda")[None] >= t["own_len"][:, None]
    t["k_own"][past], t["v_own"][past] = math.nan, math.inf
    out, lse = _attend(t, causal=causal)
    some = [0, B - 1] if B > 1 else [0]
    pick = [b * D + d for b in some for d in range(D)]
    kp, vp = (torch.from_numpy(x[some]).cuda() for x in (kp, vp))
    want, wlse, absv, big = ops_gpu64.draft_attention(t["q"][pick], kp, vp, [plen[b] for b in some], t["k_own"][pick], t["v_own"][pick], [olen[n] for n in pick],
                                                      Dh ** -0.5, causal)
    e = (Dh + 6) * 2.0 ** -24 * big + 2.0 ** -22 * max(1.0, big)
    rel = 2 * e + 2.0 ** -17
    tol = (U[dtype] * absv + U[dtype] * want.abs()) * (1 + rel) + rel * absv + 1e-7
    assert bool(((out[pick].double() - want).abs() <= tol).all()), float(((out[pick].double() - want).abs() - tol).max())
    assert bool(((lse[pick].double() - wlse).abs() <= 2 * e + 2.0 ** -18 + 2.0 ** -22 * wlse.abs()).all())

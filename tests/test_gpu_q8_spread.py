"""Attention over codes whose value scales lie far apart, or near the ends of fp32, in every form of the operator.  Tolerances as in
test_gpu_q8.py: they go by what a row draws on (sum_j p_j |v_j|), so a block that a row does not attend to may not cost it anything."""
import math

import numpy as np
import pytest
import torch

import paper_2605_15609_b200 as psd
from test_gpu_q8 import _check, _f64, _i32
from test_gpu_q8_service import FORMS, _attend, _inputs

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
LOUD = slice(64, 96)                 # tokens of block 2


def _spread(shape, dtype, octaves, gap, both, seed=21):
    """Inputs of `shape` whose block 2 has value scales 2^octaves times the others', with scores `gap` nats below theirs; with `both`,
    above them for every other row."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    t, kp, vp = _inputs(shape, seed, DT[dtype])
    side = torch.sign(torch.randn(Dh, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
    q = t["q"].float() + side
    if both:
        q[:, :, 1::2] *= -1          # heads in turn; of a single row per key head, key heads in turn
    t["q"] = q.to(DT[dtype])
    # q . side is about Dh: the block's keys along -side score -gap
    t["k_codes"][:, LOUD] = (-100 * side).to(torch.int8)
    t["k_scale"][:, :, 2] = gap / (100 * math.sqrt(Dh))
    t["v_scale"][:, :, 2] *= 2.0 ** octaves
    for b in range(B):
        n = int(t["prefix_len"][b])
        t["k_codes"][b, n:] = 127
        k = _f64(t["k_codes"][b]) * np.repeat(_f64(t["k_scale"][b]).T, 32, 0)[:P, :, None]
        v = _f64(t["v_codes"][b]) * np.repeat(_f64(t["v_scale"][b]).T, 32, 0)[:P, :, None]
        kp[b, :n], vp[b, :n] = k[:n], v[:n]
    return t, kp, vp


def _expect(shape, dtype, t, kp, vp, power=0, **kw):
    """Against 64 bits, outputs and values in units of 2^power; a few sequences (a plain loop over all would take minutes)."""
    B, D, M, Hq, Hkv, Dh, P, S = shape
    out, lse = _attend(t, **kw)
    some = sorted({0, B - 1, B // 2})[:2]
    pick = [b * D + d for b in some for d in range(D)]
    unit = 2.0 ** -power
    own = [_f64(t[n])[pick] for n in ("k_own", "v_own")]
    _check(out[pick].double() * unit, lse[pick], t["q"][pick], kp[some], vp[some] * unit, own[0], own[1] * unit, [int(t["prefix_len"][b]) for b in some],
           [int(t["own_len"][n]) for n in pick], Dh ** -0.5, kw.get("causal", False), dtype)


@pytest.mark.parametrize("octaves, gap", [(10, 40), (20, 40), (30, 40), (60, 70)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", list(FORMS))
def test_a_loud_block_that_few_attend_to(shape, dtype, octaves, gap):
    """Rows that attend elsewhere keep their precision beside rows that attend to the loud block (fp16 outputs would not hold those)."""
    t, kp, vp = _spread(shape, dtype, octaves, gap, dtype == "bf16")
    _expect(shape, dtype, t, kp, vp)
    _expect(shape, dtype, {**t, "own_len": _i32([0] * len(t["own_len"]))}, kp, vp)


@pytest.mark.parametrize("octaves", [-10, -20, -30, -60])
@pytest.mark.parametrize("shape", list(FORMS))
def test_a_quiet_block_that_some_attend_to(shape, octaves):
    """Rows whose weight lies on one block of small values, and whose result is that block's."""
    t, kp, vp = _spread(shape, "bf16", octaves, 40 - octaves, True)
    _expect(shape, "bf16", {**t, "own_len": _i32([0] * len(t["own_len"]))}, kp, vp, octaves)


@pytest.mark.parametrize("power", [-110, -60, 60, 112])
@pytest.mark.parametrize("shape", list(FORMS))
def test_scales_near_the_ends(shape, power):
    """All values in units of 2^power: results that bf16 holds are not lost on the way."""
    t, kp, vp = _inputs(shape, 22)
    t["v_scale"], t["v_own"] = t["v_scale"] * 2.0 ** power, t["v_own"] * 2.0 ** power
    _expect(shape, "bf16", t, kp, vp * 2.0 ** power, power)
    _expect(shape, "bf16", {**t, "own_len": _i32([0] * len(t["own_len"]))}, kp, vp * 2.0 ** power, power)


@pytest.mark.parametrize("shape", list(FORMS))
def test_blocks_of_scale_zero_beside_loud_ones(shape):
    """Keys whose values stand for nothing still count in the sum of weights, whatever the other scales are."""
    t, kp, vp = _spread(shape, "bf16", 100, 40, False)
    t["k_scale"][:, :, 2], t["v_scale"][:, :, 2] = t["k_scale"][:, :, 2] * 2.5, 2.0 ** 100       # 100 nats: 2^100 * e^-100 is nothing
    t["v_scale"][:, :, 0] = 0.0
    kp[:, LOUD] *= 2.5
    vp[:, :32] = 0.0
    vp[:, LOUD] = _f64(t["v_codes"][:, LOUD]) * 2.0 ** 100
    for b in range(shape[0]):
        n = int(t["prefix_len"][b])
        kp[b, n:], vp[b, n:] = 0.0, 0.0
    _expect(shape, "bf16", t, kp, vp)

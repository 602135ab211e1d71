"""psd_confidence_logits at the sizes of a serving batch: several rows per warp, several groups of columns per row, every edit.

Tolerances as in test_gpu_ops.py: a relative 6e-5 for sums of a few hundred terms per lane; tokens are exact."""
import pytest
import torch

import ops_gpu64 as ref
import paper_2605_15609_b200 as psd

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
V, T = 20001, 60


def _plant(x):
    """Maxima, ties, NaN, infinities and lowest values in the second to fourth group (of 512 or 1024 columns) of warps' columns."""
    V = x.shape[1]
    r = torch.arange(len(x), device=x.device)
    col = torch.arange(V, device=x.device)
    x[r % 16 == 0, 4096 + 2 * 1024 + 17] = 40.0
    for c in (4096 + 3 * 1024 + 5, 2 * 4096 + 1024 + 9):
        x[r % 16 == 1, c] = 30.0
    for c in (4096 + 1024 + 300, 4096 + 1024 + 3, 4096 + 1024 + 301):
        x[r % 16 == 2, c] = 30.0
    x[r % 16 == 3, 3 * 4096 + 2050] = float("nan")
    x[r % 16 == 4, 2 * 4096 + 3000] = float("inf")
    x[r % 16 == 5, 4096 + 1500] = 60.0                                      # closed below
    x[(r % 16 == 7)[:, None] & (col % 4096 < 3072)[None]] = -float("inf")
    x[(r % 16 == 8)[:, None] & (col < V - 700)[None]] = torch.finfo(x.dtype).min
    x += torch.where(r % 16 == 9, 1.0, 0.0)[:, None].to(x.dtype) * (col // 512 * 0.75).to(x.dtype)       # rises group by group
    x[r % 16 == 10] = torch.finfo(x.dtype).min
    return r


def _allow(R, V, g, r):
    words = (V + 31) // 32
    a = torch.randint(-2 ** 31, 2 ** 31, (R, words), generator=g, device="cuda").to(torch.int32)
    a[(r % 16 < 5) | (r % 16 > 6)] |= torch.randint(-2 ** 31, 2 ** 31, (1, words), generator=g, device="cuda").to(torch.int32)
    a[:, [(4096 + 3 * 1024 + 5) // 32, (4096 + 1024 + 3) // 32, 4096 // 32 + 64]] = -1
    a[r % 16 == 5, (4096 + 1024) // 32:(4096 + 3072) // 32] = 0             # whole groups closed, a maximum among them
    only = r % 16 == 6
    a[only] = 0
    a[only, (V - 1) // 32] = 1 << (V - 1) % 32                              # the last column alone
    a[r % 32 == 12] = 0                                                     # nothing at all
    return a


# B, D, M, warps that share a row, columns of a warp
SHAPES = [(40, 4, 32, 1, 4096), (100, 4, 5, 2, 4096), (200, 2, 3, 4, 4096), (600, 1, 1, 8, 2048)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_all_edits(shape, dtype, padded):
    B, D, M, wpr, cols = shape
    R, N = B * D * M, B * D
    g = torch.Generator(device="cuda").manual_seed(R + len(dtype))
    x = (2 * torch.randn(R, V, generator=g, device="cuda")).to(DT[dtype])
    r = _plant(x)
    lg = x
    if padded:
        wide = torch.full((R, V + 3), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, :V] = x
        lg = wide[:, :V]
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda").to(torch.int32)  # noqa: E731
    history, hlen = ints(-2, V + 2, B, T), ints(0, T + 1, B)
    history[:, ::3] = history[:, :1]
    dtok, dmask = ints(0, V + 1, N, M), ints(0, 2, N, M)
    dtok[:, 0], dmask[:, 0] = 4096 + 3 * 1024 + 5, 0                        # an edited column among the planted ones
    allow = _allow(R, V, g, r)
    for bias_rows in (1, B):
        bias = torch.zeros(bias_rows, V, device="cuda")
        bias[:, ::37] = torch.randn(bias_rows, len(range(0, V, 37)), generator=g, device="cuda")
        bias[:, 11::1001] = torch.finfo(torch.float32).min
        want = ref.confidences(x, D, M, history, hlen, dtok, dmask, 1.3, 0.4, 0.15, bias, allow)
        tok, conf, lse = ints(-9, -8, R), torch.full((R,), -7.0, device="cuda"), torch.full((R,), -7.0, device="cuda")
        status = ints(0, 1, 1)
        ws = torch.full((psd.psd_logits_workspace_bytes(R, V),), 255, dtype=torch.uint8, device="cuda")
        psd.psd_confidence_logits(lg, tok, conf, lse, B=B, D=D, M=M, history=history, history_len=hlen, draft_tokens=dtok,
                                  draft_mask=dmask, repetition=1.3, presence=0.4, frequency=0.15, bias=bias if bias_rows > 1 else bias[0],
                                  allow=allow, workspace=ws, status=status)
        torch.cuda.synchronize()
        # the form this test is about: records of 16 bytes per row and warp, as many as warps of `cols` columns make
        written = int((ws.view(torch.int64) != -1).nonzero().max()) // 2 + 1
        assert written == R * (-(-V // (cols * wpr)) * wpr), "another form than the one under test"
        wt, wc, wl, bad = want
        assert int(status.item()) == int(bad.sum()) > 0
        assert torch.equal(tok[~bad], wt[~bad])
        assert bool(torch.isnan(conf[bad]).all()) and bool(torch.isnan(lse[bad]).all())
        ok = ~bad
        assert bool(((conf[ok].double() - wc[ok]).abs() <= 6e-5 * wc[ok]).all())
        fin = ok & torch.isfinite(wl)
        assert torch.equal(lse[ok & ~fin].double(), wl[ok & ~fin])
        assert bool(((lse[fin].double() - wl[fin]).abs() <= 6e-5 + 2.0 ** -22 * wl[fin].abs()).all())
        assert int((wt == -1).sum()) >= R // 32 and int((wt == V - 1).sum()) > 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_edits(dtype):
    B, D, M = 40, 4, 32
    R = B * D * M
    x = (2 * torch.randn(R, V, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")).to(DT[dtype])
    _plant(x)
    wt, wc, wl, bad = ref.confidences(x, D, M, None, None, None, None, 1.0, 0.0, 0.0, None, None)
    tok, conf, lse = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, device="cuda"), torch.zeros(R, device="cuda")
    ws = torch.full((psd.psd_logits_workspace_bytes(R, V),), 255, dtype=torch.uint8, device="cuda")
    psd.psd_confidence_logits(x, tok, conf, lse, B=B, D=D, M=M, workspace=ws)
    torch.cuda.synchronize()
    ok = ~bad
    assert torch.equal(tok[ok], wt[ok]) and bool(torch.isnan(conf[bad]).all())
    assert bool(((conf[ok].double() - wc[ok]).abs() <= 6e-5 * wc[ok]).all())
    assert bool(((lse[ok].double() - wl[ok]).abs() <= 6e-5 + 2.0 ** -22 * wl[ok].abs()).all())

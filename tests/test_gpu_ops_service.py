"""The operators around the step as a service calls them: one workspace for batches that shrink, calls that follow one another
without a synchronisation, calls captured in a CUDA graph."""
import pytest
import torch

import paper_2605_15609_b200 as psd

pytestmark = pytest.mark.gpu

D, M, HQ, HKV, DH, P, S = 4, 32, 32, 8, 128, 2000, 32


def _tensors(B, seed, P=P):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    N = B * D
    return dict(q=h(N, M, HQ, DH), k_prefix=h(B, P, HKV, DH), v_prefix=h(B, P, HKV, DH), k_own=h(N, S, HKV, DH), v_own=h(N, S, HKV, DH),
                prefix_len=torch.randint(0, P + 1, (B,), generator=g, device="cuda").to(torch.int32))


def _attend(t, ws):
    out, lse = torch.full_like(t["q"], 7.0), torch.full(t["q"].shape[:3], 7.0, device="cuda")
    psd.psd_draft_attention(**t, out=out, lse=lse, workspace=ws)
    return out, lse


def _weigh(t, lse, ws):
    B, P = t["k_prefix"].shape[:2]
    acc = torch.full((B, HKV, P), 7.0, device="cuda")
    psd.psd_prefix_weights(t["q"], t["k_prefix"], lse, acc, prefix_len=t["prefix_len"], workspace=ws)
    return acc


def _space(n):
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")


def test_one_workspace_serves_batches_that_shrink():
    """Sized for 16 sequences, used for fewer; every call follows the one before without a synchronisation."""
    a = _space(psd.psd_attention_workspace_bytes(16, D, M, HQ, HKV, DH, P, S))
    w = _space(psd.psd_weights_workspace_bytes(16, D, M, HQ, HKV, DH, P))
    batches = [_tensors(B, B) for B in (16, 8, 4, 3, 2, 1)]
    got = []
    for t in batches:
        out, lse = _attend(t, a)
        got.append((out, lse, _weigh(t, lse, w)))
    torch.cuda.synchronize()
    for t, (out, lse, acc) in zip(batches, got):
        B = t["k_prefix"].shape[0]
        o, s = _attend(t, _space(psd.psd_attention_workspace_bytes(B, D, M, HQ, HKV, DH, P, S)))
        torch.cuda.synchronize()
        c = _weigh(t, s, _space(psd.psd_weights_workspace_bytes(B, D, M, HQ, HKV, DH, P)))
        torch.cuda.synchronize()
        assert torch.equal(out, o) and torch.equal(lse, s) and torch.equal(acc, c)
        assert bool(torch.isfinite(o.float()).all()) and bool((c >= 0).all())


def test_calls_in_a_row_share_a_workspace():
    """The partial results of one call are read by its second launch before the next call writes its own over them."""
    n = psd.psd_attention_workspace_bytes(2, D, M, HQ, HKV, DH, P, S)
    ws = _space(n)
    a, b = _tensors(1, 1), _tensors(2, 2)
    want = []
    for t in (a, b):
        want.append(_attend(t, ws))
        torch.cuda.synchronize()
    got = [_attend(t, ws) for _ in range(40) for t in (a, b)]
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(got):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])


def test_calls_captured_in_a_graph():
    """Attention, weights, eviction and confidences in one graph, replayed on other inputs."""
    B, keep, V = 2, 300, 5000
    first, second = _tensors(B, 5), _tensors(B, 6)
    a, w = _space(psd.psd_attention_workspace_bytes(B, D, M, HQ, HKV, DH, P, S)), _space(psd.psd_weights_workspace_bytes(B, D, M, HQ, HKV, DH, P))
    c = _space(psd.psd_logits_workspace_bytes(B * D * M, V))
    g = torch.Generator(device="cuda").manual_seed(7)
    logits = torch.randn(B * D * M, V, generator=g, device="cuda").bfloat16()
    history = torch.randint(0, V, (B, 50), generator=g, device="cuda").to(torch.int32)
    out, lse = torch.empty_like(first["q"]), torch.empty(B * D, M, HQ, device="cuda")
    acc = torch.empty(B, HKV, P, device="cuda")
    small = [torch.zeros(B, keep, HKV, DH, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    index = torch.empty(B, HKV, keep, dtype=torch.int32, device="cuda")
    tok, conf = torch.empty(B * D * M, dtype=torch.int32, device="cuda"), torch.empty(B * D * M, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    results = (out, lse, acc, *small, index, tok, conf)

    def call():
        psd.psd_draft_attention(**first, out=out, lse=lse, workspace=a, status=status)
        psd.psd_prefix_weights(first["q"], first["k_prefix"], lse, acc, prefix_len=first["prefix_len"], workspace=w, status=status)
        psd.psd_prefix_evict(acc, first["k_prefix"], first["v_prefix"], *small, index, prefix_len=first["prefix_len"], n_sink=4,
                             n_recent=M)
        psd.psd_confidence_logits(logits, tok, conf, D=D, M=M, history=history, repetition=1.2, workspace=c, status=status)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()                                             # (the kernels are loaded before the capture)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for t in (second, _tensors(B, 8)):
        for k, v in t.items():
            first[k].copy_(v)
        logits.copy_(torch.randn(B * D * M, V, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [x.clone() for x in results]
        for x in results:
            x.fill_(3)
        small[0].zero_(), small[1].zero_()
        replayed[3][(index_past := replayed[5].transpose(1, 2) < 0)] = 0
        replayed[4][index_past] = 0
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(replayed, results))
    assert int(status.item()) == 0
    del graph

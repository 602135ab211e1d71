#!/usr/bin/env python
"""Decode blocks with one attention layer end to end on one GPU: the drafts of a sequence attend over its shared prefix
(psd_draft_attention), logits are penalised, biased and masked before their confidences (psd_confidence_logits), the policy
and acceptance run on them (psd_select_unmask, psd_build_drafts, psd_verify_accept), finished blocks join the prefix's cache,
and the cache is cut by the attention weight its keys have drawn (psd_prefix_weights, psd_prefix_evict).

    python -m paper_2605_15609_b200.examples.constrained_decode [--blocks 4] [--sequences 4] [--depth 4] [--budget 96]

The layer has random weights and stands in for a transformer; a real caller runs its own layers around the same calls.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2605_15609_b200 as psd  # noqa: E402

HQ, HKV, DH, H, M = 8, 2, 64, 256, 16        # heads, key heads, head size, hidden size, slots of a block


class Layer:
    """Embedding, one attention layer, output head."""

    def __init__(self, V, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device="cuda") / s[-1] ** 0.5).bfloat16()  # noqa: E731
        self.embed, self.slot = w(V + 1, H), w(M, H)        # row V of the table is the mask token
        self.qkv, self.back, self.head = w((HQ + 2 * HKV) * DH, H), w(H, HQ * DH), 64.0 * w(V, H)

    def qkv_of(self, tokens):
        """tokens [N, M] -> q [N, M, HQ, DH], k and v [N, M, HKV, DH]: views of one projection, not copies."""
        x = self.embed[tokens.long()] + self.slot
        y = (x @ self.qkv.t()).view(*tokens.shape, HQ + 2 * HKV, DH)
        return x, y[:, :, :HQ], y[:, :, HQ:HQ + HKV], y[:, :, HQ + HKV:]


class Cache:
    """Keys and values of the sequences' prefixes, the weight each key has drawn, and a second buffer to evict into."""

    def __init__(self, B, capacity, budget):
        kv = lambda n: torch.empty(B, n, HKV, DH, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.k, self.v, self.budget, self.capacity = kv(capacity), kv(capacity), budget, capacity
        self.small = kv(budget), kv(budget)
        self.weight = torch.zeros(B, HKV, capacity, device="cuda")
        self.length = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.n = 0                                          # the same in every sequence of this example

    def append(self, k, v):
        m = k.shape[1]
        self.k[:, self.n:self.n + m], self.v[:, self.n:self.n + m] = k, v
        self.weight[:, :, self.n:self.n + m] = 0
        self.n += m
        self.length.fill_(self.n)

    def evict(self):
        """Down to the budget: the first 4 keys, the last two blocks, and the best of the others."""
        B, keep = self.k.shape[0], self.budget
        index = torch.empty(B, HKV, keep, dtype=torch.int32, device="cuda")
        scores = torch.empty(B, HKV, keep, device="cuda")
        psd.psd_prefix_evict(self.weight, self.k, self.v, *self.small, index, scores, prefix_len=self.length, n_sink=4,
                             n_recent=2 * M)
        self.k[:, :keep], self.v[:, :keep] = self.small
        self.weight[:, :, :keep], self.n = scores, keep
        self.length.fill_(keep)
        return index


def decode(B=4, D=4, blocks=4, budget=96, V=4000, seed=0, allowed=0.5):
    """Returns the decoded tokens [B, blocks * M], the cache, the allowed tokens [V] bool and how many passes were made."""
    layer, p = Layer(V, seed), psd.policy(tau=0.6, k_min=1, k_max=8, depth=D, mask_id=V)
    cache = Cache(B, budget + 2 * M, budget)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    # a grammar: which tokens may appear at all (one row of bits for every row of logits)
    legal = torch.rand(V, generator=g, device="cuda") < allowed
    legal[:2] = allowed > 0        # (0: a grammar that allows nothing, a dead end)
    bits = torch.zeros((V + 31) // 32 * 32, dtype=torch.int64, device="cuda")
    bits[:V] = legal
    allow = (bits.view(-1, 32) << torch.arange(32, device="cuda")).sum(1).to(torch.int32)[None]
    text = torch.randint(0, V, (B, 2 * M), generator=g, device="cuda").to(torch.int32)     # the prompt
    status, passes = i32(1), 0
    attn_ws = psd_ws = None

    def forward(tokens, mask, drafts):
        """One pass over B * drafts token states: tokens, mask [B * drafts, M] -> token and confidence [B, drafts, M]; keeps the
        pass's queries, lse, keys and values."""
        nonlocal attn_ws, psd_ws, passes
        passes += 1
        N = B * drafts
        x, q, k, v = layer.qkv_of(tokens)
        out, lse = torch.empty(N, M, HQ, DH, dtype=q.dtype, device="cuda"), torch.empty(N, M, HQ, device="cuda")
        n = psd.psd_attention_workspace_bytes(B, drafts, M, HQ, HKV, DH, cache.capacity, M)
        if attn_ws is None or attn_ws.numel() < n:
            attn_ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        psd.psd_draft_attention(q, cache.k, cache.v, out, lse, k, v, prefix_len=cache.length, workspace=attn_ws, status=status)
        y = x + out.view(N, M, HQ * DH) @ layer.back.t()
        logits = (y.view(N * M, H) @ layer.head.t())
        tok, conf = i32(B, drafts, M), torch.empty(B, drafts, M, device="cuda")
        n = psd.psd_logits_workspace_bytes(N * M, V)
        if psd_ws is None or psd_ws.numel() < n:
            psd_ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        psd.psd_confidence_logits(logits, tok, conf, B=B, D=drafts, M=M, history=text, draft_tokens=tokens, draft_mask=mask,
                                  repetition=1.3, presence=0.2, allow=allow, workspace=psd_ws, status=status)
        return tok, conf, (q, lse, k, v)

    def store(tokens):
        """A block (or prompt piece) of known tokens: its keys join the cache, the keys there get the weight it gave them."""
        _, _, (q, lse, k, v) = forward(tokens, i32(B, M), 1)
        if cache.n:
            ws = torch.empty(psd.psd_weights_workspace_bytes(B, 1, M, HQ, HKV, DH, cache.capacity), dtype=torch.uint8,
                             device="cuda")
            psd.psd_prefix_weights(q, cache.k, lse, cache.weight, acc_in=cache.weight, beta=0.9, prefix_len=cache.length,
                                   workspace=ws, status=status)
        if cache.n + M > cache.capacity:
            cache.evict()
        cache.append(k, v)

    for i in range(0, text.shape[1], M):
        store(text[:, i:i + M].contiguous())
    for _ in range(blocks):
        tokens, mask = torch.full((B, M), V, dtype=torch.int32, device="cuda"), torch.ones(B, M, dtype=torch.int32, device="cuda")
        while int(mask.sum()):
            tok, conf, _ = forward(tokens, mask, 1)
            n_sel = i32(B)
            psd.psd_select_unmask(conf, tok, tokens, mask, p, i32(B, M), n_sel, i32(B, M))
            if bool(((n_sel == 0) & (mask.sum(1) > 0)).any()):
                raise RuntimeError("dead end: the grammar leaves no token for any masked slot of a sequence")
            sigma, n_fill, draft_tokens, draft_mask = i32(B, M), i32(B, D), i32(B, D, M), i32(B, D, M)
            psd.psd_build_drafts(conf, tok, tokens, mask, p, sigma, n_fill, draft_tokens, draft_mask)
            tok, conf, _ = forward(draft_tokens.view(B * D, M), draft_mask.view(B * D, M), D)
            psd.psd_verify_accept(tok, conf, sigma, n_fill, draft_tokens, draft_mask, p, tokens, mask, i32(B), i32(B), i32(B))
        store(tokens)
        text = torch.cat([text, tokens], 1)
    if int(status.item()) < 0:
        raise RuntimeError(psd.status_string(int(status.item())))
    return text[:, 2 * M:], cache, legal, passes


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--blocks", type=int, default=8)
    ap.add_argument("--sequences", type=int, default=4)
    ap.add_argument("--depth", type=int, default=4, help="drafts per sequence, the root included")
    ap.add_argument("--budget", type=int, default=96, help="keys per sequence and key head kept by an eviction")
    a = ap.parse_args()
    out, cache, legal, passes = decode(a.sequences, a.depth, a.blocks, a.budget)
    print(f"{a.sequences} sequences x {a.blocks} blocks of {M} tokens in {passes} passes; cache holds {cache.n} keys; "
          f"tokens outside the grammar: {int((~legal[out.long()]).sum())}")
    print("first sequence:", out[0].tolist())


if __name__ == "__main__":
    main()

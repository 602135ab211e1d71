"""Timed cases of the operators around a decoding step: attention of the drafts over the prefix that a sequence's
drafts share, the attention weight each cached key has drawn, eviction from the cache by that weight, and the
confidence pass over logits under penalties, biases and grammar masks.

A case is a dict of plain values; ``prepare`` makes what a user's program holds before the call, ``run`` is one
pass (with ``own`` the library's call, otherwise the same mathematics in elementary torch operations in fp32).
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # one sequence of the smallest benchmark shape (hidden 256): latency of a call
        dict(name="attn_tiny", op="attention", B=1, D=4, M=32, Hq=4, Hkv=4, Dh=64, P=257, S=32, causal=False,
             ragged=False, dtype="bf16"),
        # single request, hidden 4096 as 32 heads, four drafts of a block of 32 behind a prompt of 2000
        dict(name="attn_single_request", op="attention", B=1, D=4, M=32, Hq=32, Hkv=8, Dh=128, P=2000, S=32,
             causal=False, ragged=False, dtype="bf16"),
        # hidden 3584 as 28 heads over 4 key heads (7 query heads share a key head), 8 sequences of unequal length
        dict(name="attn_class_7b", op="attention", B=8, D=6, M=32, Hq=28, Hkv=4, Dh=128, P=1531, S=32, causal=False,
             ragged=True, dtype="bf16"),
        # the deep speculation sweep: 16 sequences, 8 drafts of 64 slots, long prefixes
        dict(name="attn_deep_sweep", op="attention", B=16, D=8, M=64, Hq=32, Hkv=8, Dh=128, P=8192, S=64,
             causal=False, ragged=True, dtype="bf16"),
        # serving token by token: 64 continuations of one long prefix, each with its own tokens so far
        dict(name="attn_single_tokens", op="attention", B=1, D=64, M=1, Hq=32, Hkv=8, Dh=128, P=16384, S=200,
             causal=True, ragged=True, dtype="fp16"),
        # accumulated weight of one request's prefix
        dict(name="weights_single_request", op="weights", B=1, D=4, M=32, Hq=32, Hkv=8, Dh=128, P=4095, ragged=False,
             dtype="bf16"),
        # the same for the deep sweep
        dict(name="weights_deep_sweep", op="weights", B=16, D=8, M=64, Hq=32, Hkv=8, Dh=128, P=8192, ragged=True,
             dtype="bf16"),
        # a small cache cut to a quarter
        dict(name="evict_small", op="evict", B=1, Hkv=4, Dh=64, P=1000, keep=250, sink=4, recent=32, ragged=False,
             dtype="bf16"),
        # a batch of long caches cut to a quarter
        dict(name="evict_large", op="evict", B=8, Hkv=8, Dh=128, P=32768, keep=8192, sink=4, recent=256, ragged=True,
             dtype="bf16"),
        # one token of one request over a vocabulary of 126464
        dict(name="logits_single_token", op="logits", B=1, D=1, M=1, V=126464, T=900, dtype="bf16"),
        # the verification batch of one request in fp32 logits, an odd vocabulary
        dict(name="logits_single_request", op="logits", B=1, D=4, M=32, V=126465, T=512, dtype="fp32"),
        # the batched serving step: 8192 rows
        dict(name="logits_batched_serving", op="logits", B=64, D=4, M=32, V=126464, T=512, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "weights", "evict", "logits"])
    top = {}
    for c in listed():
        w = _cost(c)
        top[c["op"]] = max(top.get(c["op"], 0), w)
    while True:
        if op in ("attention", "weights"):
            hq, hkv = rng.choice([(4, 4), (8, 1), (12, 4), (16, 2), (28, 4), (32, 8), (32, 32), (40, 8)])
            one = op == "attention" and rng.random() < 0.3
            M = 1 if one else _log(rng, 2, 64)
            c = dict(op=op, B=_log(rng, 1, 16), D=_log(rng, 1, 64) if one else _log(rng, 1, 8), M=M, Hq=hq, Hkv=hkv,
                     Dh=rng.choice([64, 80, 96, 128, 128]), P=_log(rng, 1, 16384), ragged=rng.random() < 0.5,
                     dtype=rng.choice(["bf16", "bf16", "fp16"]))
            if op == "attention":
                c["causal"] = one or rng.random() < 0.3
                c["S"] = _log(rng, 1, 300) if one else M + (_log(rng, 1, 64) if c["causal"] else 0)
        elif op == "evict":
            P = _log(rng, 64, 32768)
            keep = max(8, int(P * rng.uniform(0.05, 0.9)))
            c = dict(op=op, B=_log(rng, 1, 16), Hkv=rng.choice([1, 2, 4, 8, 32]), Dh=rng.choice([64, 80, 96, 128]),
                     P=P, keep=keep, sink=rng.choice([0, 1, 4]), recent=_log(rng, 1, max(1, keep // 4)),
                     ragged=rng.random() < 0.5, dtype=rng.choice(["bf16", "fp16"]))
        else:
            one = rng.random() < 0.3
            c = dict(op=op, B=_log(rng, 1, 64), D=1 if one else _log(rng, 1, 8), M=1 if one else _log(rng, 2, 64),
                     V=rng.choice([1024, 32000, 50257, 126464, 126465, 152064]), T=_log(rng, 1, 4096),
                     dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
        if _cost(c) <= top[op]:
            return c


def _cost(c):
    w = work(c)
    return w["bytes"] / 6.5e12 + w["flops"] / 1.6e15


# ---- sizes that differ from sequence to sequence (host numbers, a program knows them) ------------------------------------------

def _gen(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed))
    return g


def _lens(n, most, ragged, seed):
    """n lengths: all `most`, or spread between a fifth of it and all of it."""
    if not ragged:
        return [most] * n
    f = torch.rand(n, generator=_gen(seed, "cpu")).tolist()
    r = [max(0, min(most, int(round(most * (0.2 + 0.8 * x))))) for x in f]
    r[0] = most
    return r


# ---- inputs -------------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    return {"attention": _prepare_attention, "weights": _prepare_weights, "evict": _prepare_evict,
            "logits": _prepare_logits}[case["op"]](case, seed)


def _cache(case, g, lens):
    """K and V of the prefixes [B, P, Hkv, Dh]: unit normal keys, the first few (which draw much of the weight in
    trained models) along a direction that queries share; what lies past a sequence's end is memory nobody wrote."""
    B, P, Hkv, Dh, dt = case["B"], case["P"], case["Hkv"], case["Dh"], _DT[case["dtype"]]
    k = torch.randn(B, P, Hkv, Dh, generator=g, device="cuda", dtype=torch.float32).to(dt)
    v = torch.randn(B, P, Hkv, Dh, generator=g, device="cuda", dtype=torch.float32).to(dt)
    k[:, :4] += 0.6
    for b, n in enumerate(lens):
        k[b, n:] = math.nan
        v[b, n:] = math.nan
    return k, v


def _prepare_attention(case, seed):
    B, D, M, Hq, Hkv, Dh, P, S = (case[n] for n in ("B", "D", "M", "Hq", "Hkv", "Dh", "P", "S"))
    g, dt, N = _gen(seed), _DT[case["dtype"]], case["B"] * case["D"]
    plen = _lens(B, P, case["ragged"], seed + 1)
    olen = _lens(N, S, case["ragged"] and M == 1, seed + 2)
    kp, vp = _cache(case, g, plen)
    q = (torch.randn(N, M, Hq, Dh, generator=g, device="cuda") + 0.3).to(dt)
    ko = torch.randn(N, S, Hkv, Dh, generator=g, device="cuda").to(dt)
    vo = torch.randn(N, S, Hkv, Dh, generator=g, device="cuda").to(dt)
    past = torch.arange(S, device="cuda")[None, :] >= torch.tensor(olen, device="cuda")[:, None]
    ko[past] = math.nan
    vo[past] = math.nan
    st = dict(case, q=q, kp=kp, vp=vp, ko=ko, vo=vo, plen=plen, olen=olen,
              plen_dev=torch.tensor(plen, dtype=torch.int32, device="cuda"),
              olen_dev=torch.tensor(olen, dtype=torch.int32, device="cuda"), scale=1.0 / math.sqrt(Dh))
    if own:
        import paper_2605_15609_b200 as psd
        st.update(psd=psd, out=torch.empty_like(q), lse=torch.empty(N, M, Hq, device="cuda"),
                  ws=torch.empty(psd.psd_attention_workspace_bytes(B, D, M, Hq, Hkv, Dh, P, S), dtype=torch.uint8,
                                 device="cuda"))
    return st


def _prepare_weights(case, seed):
    B, D, M, Hq, Hkv, Dh, P = (case[n] for n in ("B", "D", "M", "Hq", "Hkv", "Dh", "P"))
    g, dt, N, G = _gen(seed), _DT[case["dtype"]], case["B"] * case["D"], Hq // Hkv
    plen = _lens(B, P, case["ragged"], seed + 1)
    kp, _ = _cache(case, g, plen)
    q = (torch.randn(N, M, Hq, Dh, generator=g, device="cuda") + 0.3).to(dt)
    scale = 1.0 / math.sqrt(Dh)
    # the log-sum-exp that the attention pass returned for each row: over the prefix, and some of the row's weight
    # on the draft's own keys
    lse = torch.empty(N, M, Hq, device="cuda")
    for b, n in enumerate(plen):
        qb = q[b * D:(b + 1) * D].reshape(D * M, Hkv, G, Dh)
        for h in range(Hkv):
            s = (qb[:, h].reshape(-1, Dh) @ kp[b, :n, h].t()).float() * scale
            lse[b * D:(b + 1) * D, :, h * G:(h + 1) * G] = torch.logsumexp(s, -1).reshape(D, M, G)
    lse += 0.3 * torch.rand(N, M, Hq, generator=g, device="cuda")
    st = dict(case, q=q, kp=kp, lse=lse, plen=plen, plen_dev=torch.tensor(plen, dtype=torch.int32, device="cuda"),
              scale=scale, beta=0.875, acc=torch.rand(B, Hkv, P, generator=g, device="cuda").pow(4))
    if own:
        import paper_2605_15609_b200 as psd
        st.update(psd=psd, acc_out=torch.empty_like(st["acc"]),
                  ws=torch.empty(psd.psd_weights_workspace_bytes(B, D, M, Hq, Hkv, Dh, P), dtype=torch.uint8,
                                 device="cuda"))
    return st


def _prepare_evict(case, seed):
    B, Hkv, Dh, P, keep = (case[n] for n in ("B", "Hkv", "Dh", "P", "keep"))
    g, dt = _gen(seed), _DT[case["dtype"]]
    plen = _lens(B, P, case["ragged"], seed + 1)
    kp, vp = _cache(case, g, plen)
    # accumulated weights: heavy-tailed, some keys never looked at (equal scores)
    sc = torch.exp(2.0 * torch.randn(B, Hkv, P, generator=g, device="cuda"))
    sc[torch.rand(B, Hkv, P, generator=g, device="cuda") < 0.1] = 0.0
    st = dict(case, kp=kp, vp=vp, scores=sc, plen=plen,
              plen_dev=torch.tensor(plen, dtype=torch.int32, device="cuda"),
              k_out=torch.zeros(B, keep, Hkv, Dh, device="cuda", dtype=dt),
              v_out=torch.zeros(B, keep, Hkv, Dh, device="cuda", dtype=dt))
    if own:
        import paper_2605_15609_b200 as psd
        st.update(psd=psd, index=torch.empty(B, Hkv, keep, dtype=torch.int32, device="cuda"),
                  scores_out=torch.empty(B, Hkv, keep, device="cuda"),
                  len_out=torch.empty(B, dtype=torch.int32, device="cuda"))
    return st


def _prepare_logits(case, seed):
    B, D, M, V, T = (case[n] for n in ("B", "D", "M", "V", "T"))
    g, N, R = _gen(seed), case["B"] * case["D"], case["B"] * case["D"] * case["M"]
    lg = torch.empty(R, V, device="cuda", dtype=_DT[case["dtype"]])
    for r in range(0, R, 512):      # piecewise: the fp32 draw of all rows at once would be large
        n = min(512, R - r)
        lg[r:r + n] = (2.0 * torch.randn(n, V, generator=g, device="cuda")).to(lg.dtype)
    peak = torch.randint(0, V, (R,), generator=g, device="cuda")
    lg[torch.arange(R, device="cuda"), peak] = (8.0 + 10.0 * torch.rand(R, generator=g, device="cuda")).to(lg.dtype)
    # tokens of the text so far: skewed, some of them the peaks of the sequence's rows
    hist = (V * torch.rand(B, T, generator=g, device="cuda").pow(3)).to(torch.int32)
    few = min(T, D * M)
    hist[:, :few] = peak.view(B, D * M)[:, :few].to(torch.int32)
    hist[:, T // 2:T // 2 + few // 2] = hist[:, :few // 2][:, :hist[:, T // 2:T // 2 + few // 2].shape[1]]
    hlen = _lens(B, T, True, seed + 1)
    # the drafts: a third of their slots hold tokens, the others are masked (token id V)
    dmask = (torch.rand(N, M, generator=g, device="cuda") < 0.67).to(torch.int32)
    dtok = torch.where(dmask > 0, V, torch.randint(0, V, (N, M), generator=g, device="cuda")).to(torch.int32)
    # a bias on a few hundred tokens, a few of them forbidden outright
    bias = torch.zeros(V, device="cuda")
    at = torch.randperm(V, generator=g, device="cuda")[:300]
    bias[at] = torch.randn(at.numel(), generator=g, device="cuda")
    bias[at[:10]] = torch.finfo(torch.float32).min
    # grammar: per row, one word of 32 tokens in ten is cut down; a row with four tokens left now and then; row 3 has none
    words = (V + 31) // 32
    allow = torch.full((R, words), -1, dtype=torch.int32, device="cuda")
    cut = torch.rand(R, words, generator=g, device="cuda") < 0.1
    allow[cut] = torch.randint(-2 ** 31, 2 ** 31 - 1, (int(cut.sum()),), generator=g, device="cuda").to(torch.int32)
    few_rows = torch.arange(R, device="cuda")[5::16]
    if few_rows.numel():
        allow[few_rows] = 0
        for j in range(4):
            tok = torch.randint(0, V, (few_rows.numel(),), generator=g, device="cuda")
            allow[few_rows, tok // 32] |= (1 << (tok % 32)).to(torch.int64).to(torch.int32)
    if R > 3:
        allow[3] = 0
    st = dict(case, lg=lg, hist=hist, hlen=hlen, hlen_dev=torch.tensor(hlen, dtype=torch.int32, device="cuda"),
              dtok=dtok, dmask=dmask, bias=bias, allow=allow, repetition=1.25, presence=0.25, frequency=0.125)
    if own:
        import paper_2605_15609_b200 as psd
        st.update(psd=psd, tok=torch.empty(R, dtype=torch.int32, device="cuda"), conf=torch.empty(R, device="cuda"),
                  lse=torch.empty(R, device="cuda"),
                  ws=torch.empty(psd.psd_logits_workspace_bytes(R, V), dtype=torch.uint8, device="cuda"))
    return st


# ---- one pass -----------------------------------------------------------------------------------------------------------------

def run(st):
    if own:
        return {"attention": _own_attention, "weights": _own_weights, "evict": _own_evict,
                "logits": _own_logits}[st["op"]](st)
    return {"attention": _plain_attention, "weights": _plain_weights, "evict": _plain_evict,
            "logits": _plain_logits}[st["op"]](st)


def _own_attention(st):
    st["psd"].psd_draft_attention(st["q"], st["kp"], st["vp"], st["out"], st["lse"], st["ko"], st["vo"],
                                  prefix_len=st["plen_dev"], own_len=st["olen_dev"], scale=st["scale"],
                                  causal=st["causal"], workspace=st["ws"])
    return {"out": st["out"], "lse": st["lse"]}


def _own_weights(st):
    st["psd"].psd_prefix_weights(st["q"], st["kp"], st["lse"], st["acc_out"], acc_in=st["acc"], beta=st["beta"],
                                 prefix_len=st["plen_dev"], scale=st["scale"], workspace=st["ws"])
    return {"acc": st["acc_out"]}


def _own_evict(st):
    st["psd"].psd_prefix_evict(st["scores"], st["kp"], st["vp"], st["k_out"], st["v_out"], st["index"],
                               scores_out=st["scores_out"], len_out=st["len_out"], prefix_len=st["plen_dev"],
                               n_sink=st["sink"], n_recent=st["recent"])
    return {"k": st["k_out"], "v": st["v_out"], "index": st["index"], "scores": st["scores_out"],
            "len": st["len_out"]}


def _own_logits(st):
    st["psd"].psd_confidence_logits(st["lg"], st["tok"], st["conf"], st["lse"], B=st["B"], D=st["D"], M=st["M"],
                                    history=st["hist"], history_len=st["hlen_dev"], draft_tokens=st["dtok"],
                                    draft_mask=st["dmask"], repetition=st["repetition"], presence=st["presence"],
                                    frequency=st["frequency"], bias=st["bias"], allow=st["allow"],
                                    workspace=st["ws"])
    return {"tok": st["tok"], "conf": st["conf"], "lse": st["lse"]}


def _plain_attention(st):
    B, D, M, Hq, Hkv, Dh, S = (st[n] for n in ("B", "D", "M", "Hq", "Hkv", "Dh", "S"))
    G = Hq // Hkv
    out, lse = torch.empty_like(st["q"]), torch.empty(B * D, M, Hq, device="cuda")
    slot = torch.arange(S, device="cuda")
    for b in range(B):
        n = slice(b * D, (b + 1) * D)
        L = st["plen"][b]
        q = st["q"][n].float().reshape(D, M, Hkv, G, Dh).permute(2, 0, 1, 3, 4).reshape(Hkv, D, M * G, Dh)
        kp, vp = (st[x][b, :L].float().permute(1, 0, 2) for x in ("kp", "vp"))
        sp = ((q.reshape(Hkv, -1, Dh) @ kp.transpose(1, 2)) * st["scale"]).reshape(Hkv, D, M * G, L)
        # own keys: slot s of node d counts where s < its length, and, causally, s <= length - M + i for query i
        limit = st["olen_dev"][n][:, None].expand(D, M)
        there = slot[None, :] < limit[:, :1]
        ko, vo = (torch.where(there[:, :, None, None], st[x][n].float(), 0.0).permute(2, 0, 1, 3) for x in ("ko", "vo"))
        if st["causal"]:
            limit = limit - M + 1 + torch.arange(M, device="cuda")[None, :]
        seen = (slot[None, None, :] < limit[:, :, None]).repeat_interleave(G, 1)
        so = torch.where(seen[None], (q @ ko.transpose(2, 3)) * st["scale"], -math.inf)
        m = so.amax(-1, keepdim=True)
        if L:
            m = torch.maximum(m, sp.amax(-1, keepdim=True))
        m = torch.where(m == -math.inf, 0.0, m)
        pp, po = torch.exp(sp - m), torch.exp(so - m)
        del sp, so
        l = pp.sum(-1, keepdim=True) + po.sum(-1, keepdim=True)
        o = (pp.reshape(Hkv, -1, L) @ vp).reshape(Hkv, D, M * G, Dh) + po @ vo
        o = torch.where(l > 0, o / l, 0.0)
        back = lambda x, w: x.reshape(Hkv, D, M, G, w).permute(1, 2, 0, 3, 4).reshape(D, M, Hq, w)  # noqa: E731
        out[n] = back(o, Dh).to(out.dtype)
        lse[n] = back(m + torch.log(l), 1)[..., 0]
    return {"out": out, "lse": lse}


def _plain_weights(st):
    B, D, M, Hq, Hkv, Dh, P = (st[n] for n in ("B", "D", "M", "Hq", "Hkv", "Dh", "P"))
    acc = torch.zeros(B, Hkv, P, device="cuda")
    for b in range(B):
        L, n = st["plen"][b], slice(b * D, (b + 1) * D)
        q = st["q"][n].float().reshape(D * M, Hkv, Hq // Hkv, Dh).permute(1, 0, 2, 3).reshape(Hkv, -1, Dh)
        lse = st["lse"][n].reshape(D * M, Hkv, Hq // Hkv).permute(1, 0, 2).reshape(Hkv, -1, 1)
        s = (q @ st["kp"][b, :L].float().permute(1, 2, 0)) * st["scale"]
        acc[b, :, :L] = st["beta"] * st["acc"][b, :, :L] + torch.exp(s - lse).sum(1)
    return {"acc": acc}


def _plain_evict(st):
    B, Hkv, Dh, keep = (st[n] for n in ("B", "Hkv", "Dh", "keep"))
    index = torch.full((B, Hkv, keep), -1, dtype=torch.int32, device="cuda")
    scores = torch.zeros(B, Hkv, keep, device="cuda")
    k_out, v_out = st["k_out"], st["v_out"]
    heads = torch.arange(Hkv, device="cuda")[None, :]
    for b in range(B):
        L = st["plen"][b]
        n = min(L, keep)
        at = torch.arange(L, device="cuda")
        forced = (at < st["sink"]) | (at >= L - st["recent"])
        key = torch.where(forced[None], math.inf, st["scores"][b, :, :L])
        best = torch.sort(key, dim=-1, descending=True, stable=True).indices[:, :n]
        best = torch.sort(best, dim=-1).values
        index[b, :, :n] = best.to(torch.int32)
        scores[b, :, :n] = torch.gather(st["scores"][b], 1, best)
        k_out[b, :n] = st["kp"][b][best.t(), heads]
        v_out[b, :n] = st["vp"][b][best.t(), heads]
    length = torch.tensor([min(x, keep) for x in st["plen"]], dtype=torch.int32).to("cuda", non_blocking=True)
    return {"k": k_out, "v": v_out, "index": index, "scores": scores, "len": length}


def _plain_logits(st):
    B, D, M, V, T = (st[n] for n in ("B", "D", "M", "V", "T"))
    R = B * D * M
    tok = torch.empty(R, dtype=torch.int32, device="cuda")
    conf, lse = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    ones = torch.ones(T + M, device="cuda")
    bit = torch.arange(32, device="cuda", dtype=torch.int32)
    for b in range(B):
        r = slice(b * D * M, (b + 1) * D * M)
        count = torch.zeros(D, V + 1, device="cuda")        # the last column takes what is no token
        count[:, :V] += torch.zeros(V, device="cuda").index_add_(0, st["hist"][b, :st["hlen"][b]], ones[:st["hlen"][b]])
        n = slice(b * D, (b + 1) * D)
        filled = torch.where(st["dmask"][n] == 0, st["dtok"][n], V).to(torch.int64)
        count.scatter_add_(1, filled, ones[:M].expand(D, M))
        count = count[:, None, :V].expand(D, M, V).reshape(D * M, V)
        x = st["lg"][r].float()
        pen = torch.where(x > 0, x / st["repetition"], x * st["repetition"]) - (st["frequency"] * count + st["presence"])
        x = torch.where(count > 0, pen, x) + st["bias"]
        ok = ((st["allow"][r][:, :, None] >> bit) & 1).reshape(D * M, -1)[:, :V] > 0
        x = torch.where(ok, x, -math.inf)
        m, a = x.max(-1)
        first = torch.where(x == m[:, None], torch.arange(V, device="cuda", dtype=torch.int32), V).amin(-1)
        none = m == -math.inf
        s = torch.exp(x - torch.where(none, 0.0, m)[:, None]).sum(-1)
        tok[r] = torch.where(none, -1, first).to(torch.int32)
        conf[r] = torch.where(none, 0.0, 1.0 / s)
        lse[r] = torch.where(none, -math.inf, m + torch.log(s))
    return {"tok": tok, "conf": conf, "lse": lse}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------

def exact(case, seed):
    """What run() returns for these inputs, in fp64: row block by row block, keys laid end to end."""
    st = prepare(case, seed)
    return {"attention": _exact_attention, "weights": _exact_weights, "evict": _exact_evict,
            "logits": _exact_logits}[case["op"]](st)


def _exact_attention(st):
    N, M, Hq, Dh = st["q"].shape
    G, D = Hq // st["Hkv"], st["D"]
    out = torch.zeros(N, M, Hq, Dh, dtype=torch.float64, device="cuda")
    lse = torch.full((N, M, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for h in range(st["Hkv"]):
        hq = slice(h * G, (h + 1) * G)
        for n in range(N):
            L, o = st["plen"][n // D], st["olen"][n]
            k = torch.cat([st["kp"][n // D, :L, h], st["ko"][n, :o, h]]).double()
            v = torch.cat([st["vp"][n // D, :L, h], st["vo"][n, :o, h]]).double()
            if k.shape[0] == 0:
                continue
            s = torch.einsum("igd,kd->igk", st["q"][n, :, hq].double(), k) * st["scale"]
            if st["causal"] and M > 1:
                for i in range(M):
                    s[i, :, max(L, L + o - M + 1 + i):] = -math.inf
            z = torch.logsumexp(s, -1)
            lse[n, :, hq] = z
            dead = torch.isinf(z)
            p = torch.exp(s - torch.where(dead, 0.0, z)[..., None])
            out[n, :, hq] = torch.einsum("igk,kd->igd", p, v)
    return {"out": out, "lse": lse}


def _exact_weights(st):
    B, D, Hkv, P = st["B"], st["D"], st["Hkv"], st["P"]
    G = st["Hq"] // Hkv
    acc = torch.zeros(B, Hkv, P, dtype=torch.float64, device="cuda")
    for b in range(B):
        for h in range(Hkv):
            L = st["plen"][b]
            acc[b, h, :L] = st["beta"] * st["acc"][b, h, :L].double()
            k = st["kp"][b, :L, h].double()
            for n in range(b * D, (b + 1) * D):
                for g in range(h * G, (h + 1) * G):
                    s = k @ st["q"][n, :, g].double().t() * st["scale"]
                    acc[b, h, :L] += torch.exp(s - st["lse"][n, :, g].double()).sum(1)
    return {"acc": acc}


def _exact_evict(st):
    keep, B, Hkv = st["keep"], st["B"], st["Hkv"]
    scores = torch.zeros(B, Hkv, keep, dtype=torch.float64)
    sc = st["scores"].double().cpu().numpy()
    for b in range(B):
        L = st["plen"][b]
        for h in range(Hkv):
            rank = sorted(range(L), key=lambda j: (not (j < st["sink"] or j >= L - st["recent"]), -sc[b, h, j], j))
            kept = sorted(rank[:keep])
            scores[b, h, :len(kept)] = torch.from_numpy(sc[b, h, kept])
    return {"k": None, "v": None, "index": None, "scores": scores.cuda(), "len": None}


def _exact_logits(st):
    B, D, M, V = (st[n] for n in ("B", "D", "M", "V"))
    R = B * D * M
    conf = torch.zeros(R, dtype=torch.float64, device="cuda")
    lse = torch.full((R,), -math.inf, dtype=torch.float64, device="cuda")
    shift = torch.arange(V, device="cuda") % 32
    word = torch.arange(V, device="cuda") // 32
    for n in range(B * D):
        b = n // D
        text = torch.cat([st["hist"][b, :st["hlen"][b]], st["dtok"][n][st["dmask"][n] == 0]]).long()
        count = torch.bincount(text, minlength=V).double()
        for i in range(M):
            r = n * M + i
            x = st["lg"][r].double()
            used = count > 0
            x[used] = torch.where(x[used] > 0, x[used] / st["repetition"], x[used] * st["repetition"])
            x[used] -= st["presence"] + st["frequency"] * count[used]
            x += st["bias"].double()
            x = x[(st["allow"][r][word].long() >> shift) & 1 == 1]
            if x.numel():
                lse[r] = torch.logsumexp(x, 0)
                conf[r] = torch.exp(x.max() - lse[r])
    return {"tok": None, "conf": conf, "lse": lse}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    e = 4 if case["dtype"] == "fp32" else 2
    if op in ("attention", "weights"):
        B, D, M, Hq, Hkv, Dh, P = (case[n] for n in ("B", "D", "M", "Hq", "Hkv", "Dh", "P"))
        keys = 0.6 * P * B if case["ragged"] else P * B          # prefix keys of all sequences (mean of the lengths)
        rows = D * M * Hq
        q = B * rows * Dh * e
        if op == "weights":
            return {"bytes": q + 4 * B * rows + keys * Hkv * (Dh * e + 8), "flops": 2.0 * rows * keys * Dh}
        S = case["S"] * (0.6 if case["ragged"] and M == 1 else 1.0)
        own_keys = B * D * S
        return {"bytes": 2 * q + 4 * B * rows + 2 * (keys + own_keys) * Hkv * Dh * e,
                "flops": 4.0 * rows * Dh * keys + 4.0 * M * Hq * Dh * own_keys}
    if op == "evict":
        B, Hkv, Dh, P, keep = (case[n] for n in ("B", "Hkv", "Dh", "P", "keep"))
        keys = 0.6 * P if case["ragged"] else P
        n = B * Hkv * min(keep, keys)
        return {"bytes": 4 * B * Hkv * keys + n * (4 * Dh * e + 8), "flops": B * Hkv * keys}
    R, V = case["B"] * case["D"] * case["M"], case["V"]
    return {"bytes": R * V * e + R * V / 8 + 4 * V + 4 * case["B"] * case["T"] + 12 * R, "flops": 4.0 * R * V}

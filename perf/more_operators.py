"""Timed cases of the operators that serve a step in 8 bits, and of the rotation ahead of them: norms of queries and keys
with their position rotation, the 8-bit forms of the prefix's cache and of matrix rows, attention of the drafts over an
8-bit prefix, and the confidence pass over an 8-bit LM head.

A case is a dict of plain values; ``prepare`` makes what a user's program holds before the call, ``run`` is one
pass (with ``own`` the library's call, otherwise the same mathematics in elementary torch operations).  Codes are 8-bit
integers from -127 to 127 that stand for code * scale; what a pass leaves in codes is returned as the values it stands for.
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
_PER_CODE = float(torch.tensor(1.0, dtype=torch.float32) / 127)     # fp32(1 / 127)
_TINY = 2.0 ** -126


# ---- cases ---------------------------------------------------------------------------------------------------------

def listed():
    return [
        # 16 sequences decoded token by token: 32 query and 8 key heads of 128, normed and rotated, filed in the cache
        dict(name="rotate_single_tokens", op="rotate", T=16, Hq=32, Hkv=8, Dh=128, rotary=128, interleaved=False, norm=True,
             far=8192, dtype="bf16"),
        # the batched serving step (64 sequences, 4 drafts, blocks of 32) of a layer that rotates half of each head, far positions
        dict(name="rotate_batched_serving", op="rotate", T=8192, Hq=32, Hkv=8, Dh=128, rotary=64, interleaved=True, norm=True,
             far=1000000, dtype="bf16"),
        # hidden rows of one request's verification batch
        dict(name="rows_single_request", op="rows", R=128, H=4096, dtype="bf16"),
        # an LM head of 126464 x 4096, laid out in 8 bits when a model is loaded
        dict(name="rows_lm_head", op="rows", R=126464, H=4096, dtype="bf16"),
        # a finished block of 32 tokens joins the cache of each of 16 sequences
        dict(name="prefix_block", op="prefix", B=16, P=512, Hkv=8, Dh=128, block=32, add=32, ragged=True, dtype="bf16"),
        # whole prompts of up to 16384 tokens
        dict(name="prefix_prompts", op="prefix", B=8, P=16384, Hkv=8, Dh=128, block=64, add=16384, ragged=True, dtype="bf16"),
        # single request, hidden 4096 as 32 heads, four drafts of a block of 32 behind a prompt of 2000
        dict(name="attn8_single_request", op="attention", B=1, D=4, M=32, Hq=32, Hkv=8, Dh=128, P=2000, S=32, block=32,
             causal=False, ragged=False, dtype="bf16"),
        # 64 sequences served token by token, each with a few dozen 16-bit tokens behind its 8-bit prefix
        dict(name="attn8_single_tokens", op="attention", B=64, D=1, M=1, Hq=32, Hkv=8, Dh=128, P=16384, S=64, block=64,
             causal=True, ragged=True, dtype="fp16"),
        # the deep speculation sweep: 16 sequences, 8 drafts of 64 slots, long prefixes
        dict(name="attn8_deep_sweep", op="attention", B=16, D=8, M=64, Hq=32, Hkv=8, Dh=128, P=8192, S=64, block=64,
             causal=False, ragged=True, dtype="bf16"),
        # the smallest benchmark shape (hidden 256, vocabulary 1024): latency of a call
        dict(name="head8_tiny", op="head", R=128, H=256, V=1024, dtype="bf16"),
        # single request: one pass over the LM head's codes
        dict(name="head8_single_request", op="head", R=128, H=4096, V=126464, dtype="bf16"),
        # the batched serving step: 8192 rows
        dict(name="head8_batched_serving", op="head", R=8192, H=4096, V=126464, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "rows", "prefix", "attention", "attention", "head"])
    top = {}
    for c in listed():
        top[c["op"]] = max(top.get(c["op"], 0), _cost(c))
    while True:
        hq, hkv = rng.choice([(4, 4), (8, 1), (12, 4), (16, 2), (28, 4), (32, 8), (32, 32), (40, 8)])
        dh, dt = rng.choice([64, 80, 96, 128, 128]), rng.choice(["bf16", "bf16", "fp16"])
        if op == "rotate":
            c = dict(op=op, T=_log(rng, 1, 16384), Hq=hq, Hkv=hkv, Dh=dh, rotary=rng.choice([dh, dh, dh // 2, dh // 4]),
                     interleaved=rng.random() < 0.5, norm=rng.random() < 0.6, far=_log(rng, 64, 4000000), dtype=dt)
        elif op == "rows":
            c = dict(op=op, R=_log(rng, 1, 126464), H=16 * _log(rng, 4, 1024), dtype=dt)
        elif op == "prefix":
            P = _log(rng, 33, 16384)
            c = dict(op=op, B=_log(rng, 1, 32), P=P, Hkv=hkv, Dh=dh, block=rng.choice([16, 32, 32, 64, 128]),
                     add=rng.choice([P, P, min(P, _log(rng, 1, 512))]), ragged=rng.random() < 0.6, dtype=dt)
        elif op == "attention":
            one = rng.random() < 0.4
            M = 1 if one else _log(rng, 2, 64)
            c = dict(op=op, B=_log(rng, 1, 64), D=_log(rng, 1, 8), M=M, Hq=hq, Hkv=hkv, Dh=dh, P=_log(rng, 1, 16384),
                     block=rng.choice([16, 32, 32, 64, 128]), ragged=rng.random() < 0.6, causal=one or rng.random() < 0.3, dtype=dt)
            c["S"] = _log(rng, 1, 200) if one else M + (_log(rng, 1, 64) if c["causal"] else 0)
        else:
            c = dict(op=op, R=_log(rng, 1, 8192), H=64 * _log(rng, 2, 72), V=rng.choice([1024, 32000, 50257, 126464, 152064]),
                     dtype=dt)
        if _cost(c) <= top[op]:
            return c


def _cost(c):
    w = work(c)
    return w["bytes"] / 6.5e12 + w["flops"] / 1.6e15


# ---- inputs -------------------------------------------------------------------------------------------------------------------

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


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _codes(x, dims):
    """fp32 values -> (codes as fp32 whole numbers, scale): one scale over `dims`, fp32 operations rounded one by one.  A
    NaN or an infinity makes the scale NaN."""
    top = x.abs().amax(dims, keepdim=True)
    fine = torch.isfinite(top)
    scale = torch.where(fine, (top * _PER_CODE).clamp_min(_TINY), math.nan)
    return torch.where(fine, torch.round(x * torch.reciprocal(scale)), 0.0), scale


def prepare(case, seed):
    return {"rotate": _prepare_rotate, "rows": _prepare_rows, "prefix": _prepare_prefix, "attention": _prepare_attention,
            "head": _prepare_head}[case["op"]](case, seed)


def _prepare_rotate(case, seed):
    T, Hq, Hkv, Dh, R, dt = (case[n] for n in ("T", "Hq", "Hkv", "Dh", "rotary", "dtype"))
    g, dt = _gen(seed), _DT[dt]
    # one projection's output, of which queries, keys and values are views
    qkv = torch.randn(T, Hq + 2 * Hkv, Dh, generator=g, device="cuda").to(dt)
    weight = lambda: (1.0 + 0.2 * torch.randn(Dh, generator=g, device="cuda")).to(dt)  # noqa: E731
    # the sequences' tokens stand in the cache in another order, with room for half as many again
    slots = T + T // 2 + 1
    st = dict(case, q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], q_norm=weight() if case["norm"] else None,
              k_norm=weight() if case["norm"] else None, eps=1e-6,
              position=torch.randint(0, case["far"], (T,), generator=g, device="cuda", dtype=torch.int32),
              slot=torch.randperm(slots, generator=g, device="cuda")[:T].to(torch.int32),
              # a context stretched by 8: positions count an eighth, sines and cosines a little more than one
              frequency=10000.0 ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R) / 8.0,
              gain=1.0 + 0.1 * math.log(8.0),
              q_out=torch.zeros(T, Hq, Dh, device="cuda", dtype=dt),
              k_out=torch.zeros(slots, Hkv, Dh, device="cuda", dtype=dt), v_out=torch.zeros(slots, Hkv, Dh, device="cuda", dtype=dt))
    return st


def _prepare_rows(case, seed):
    g = _gen(seed)
    # rows of different size, a few large values among them as trained weights and hidden states have
    x = torch.empty(case["R"], case["H"], device="cuda", dtype=_DT[case["dtype"]])
    for r in range(0, case["R"], 8192):      # piecewise: the fp32 draw of all rows at once would be large
        n = min(8192, case["R"] - r)
        x[r:r + n] = torch.randn(n, case["H"], generator=g, device="cuda") * (0.02 + 0.1 * torch.rand(n, 1, generator=g, device="cuda"))
    x[:, ::97] *= 3
    return dict(case, x=x, codes=torch.empty(case["R"], case["H"], device="cuda", dtype=torch.int8),
                scale=torch.empty(case["R"], device="cuda"))


def _prepare_prefix(case, seed):
    B, P, Hkv, Dh, T, add = (case[n] for n in ("B", "P", "Hkv", "Dh", "block", "add"))
    g, dt, nb = _gen(seed), _DT[case["dtype"]], -(-case["P"] // case["block"])
    end = _lens(B, P, case["ragged"], seed + 1)
    begin = [max(0, e - add) for e in end]
    k, v = (torch.randn(B, P, Hkv, Dh, generator=g, device="cuda").to(dt) for _ in "kv")
    k[:, :, :, ::17] *= 3                    # a few channels of the keys are larger, as trained ones are
    past = torch.arange(P, device="cuda")[None, :] >= _i32(end)[:, None]
    k[past] = math.nan                       # memory that nobody wrote
    v[past] = math.nan
    old = lambda *s: torch.randint(-127, 128, s, generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    st = dict(case, k=k, v=v, begin=_i32(begin), end=_i32(end), add=max(1, add), k_codes=old(B, P, Hkv, Dh), v_codes=old(B, P, Hkv, Dh),
              k_scale=torch.rand(B, Hkv, nb, generator=g, device="cuda"), v_scale=torch.rand(B, Hkv, nb, generator=g, device="cuda"))
    # for returning codes as values: the scale of each token (a view that repeats each block's)
    st["of_token"] = torch.arange(P, device="cuda") // T
    return st


def _prepare_attention(case, seed):
    B, D, M, Hq, Hkv, Dh, P, S, T = (case[n] for n in ("B", "D", "M", "Hq", "Hkv", "Dh", "P", "S", "block"))
    g, dt, N, nb = _gen(seed), _DT[case["dtype"]], case["B"] * case["D"], -(-case["P"] // case["block"])
    plen = _lens(B, P, case["ragged"], seed + 1)
    olen = _lens(N, S, case["ragged"] and M == 1, seed + 2)
    st = dict(case, q=(torch.randn(N, M, Hq, Dh, generator=g, device="cuda") + 0.3).to(dt), scale=1.0 / math.sqrt(Dh),
              plen=_i32(plen), olen=_i32(olen), plen_host=plen, olen_host=olen)
    past = torch.arange(nb * T, device="cuda")[None, :] >= st["plen"][:, None]
    for name in "kv":
        # unit normal keys and values, the first few keys along a direction that queries share, in 8 bits; what lies past a
        # sequence's end is memory nobody wrote
        x = torch.randn(B, nb * T, Hkv, Dh, generator=g, device="cuda")
        if name == "k":
            x[:, :4] += 0.6
        x[past] = 0
        codes, scale = _codes(x.to(dt).float().view(B, nb, T, Hkv, Dh), (2, 4))
        codes = codes.view(B, nb * T, Hkv, Dh).to(torch.int8)
        codes[past] = 119
        scale = scale.view(B, nb, Hkv).transpose(1, 2).contiguous()
        scale[(torch.arange(nb, device="cuda")[None, :] * T >= st["plen"][:, None])[:, None, :].expand(B, Hkv, nb)] = math.nan
        st[name + "_codes"], st[name + "_scale"] = codes[:, :P].contiguous(), scale
        o = torch.randn(N, S, Hkv, Dh, generator=g, device="cuda").to(dt)
        o[torch.arange(S, device="cuda")[None, :] >= st["olen"][:, None]] = math.nan
        st[name + "_own"] = o
    st.update(out=torch.empty_like(st["q"]), lse=torch.empty(N, M, Hq, device="cuda"))
    return st


def _prepare_head(case, seed):
    R, H, V = case["R"], case["H"], case["V"]
    g, dt = _gen(seed), _DT[case["dtype"]]
    codes, scale = torch.empty(V, H, device="cuda", dtype=torch.int8), torch.empty(V, device="cuda")
    hidden = torch.randn(R, H, generator=g, device="cuda")
    peak = torch.randint(0, V, (R,), generator=g, device="cuda")
    gain = (math.log(V) + 8.0 * torch.rand(R, 1, generator=g, device="cuda") - 3.0) / (H * 0.02 ** 2)
    for v in range(0, V, 8192):
        w = 0.02 * torch.randn(min(8192, V - v), H, generator=g, device="cuda")
        here = (peak >= v) & (peak < v + w.shape[0])
        # two rows in five lean towards one row of the head, so that confidences spread from 1 / V to 1
        hidden += torch.where(here[:, None], gain * w[(peak - v).clamp(0, w.shape[0] - 1)], 0.0) * (torch.arange(R, device="cuda") % 5 < 2)[:, None]
        c, s = _codes(w.to(torch.bfloat16).float(), (1,))
        codes[v:v + w.shape[0]], scale[v:v + w.shape[0]] = c.to(torch.int8), s[:, 0]
    return dict(case, hidden=hidden.to(dt), w_codes=codes, w_scale=scale, tok=torch.empty(R, device="cuda", dtype=torch.int32),
                conf=torch.empty(R, device="cuda"), lse=torch.empty(R, device="cuda"))


# ---- one pass -----------------------------------------------------------------------------------------------------------------

def run(st):
    if own:
        return {"rotate": _own_rotate, "rows": _own_rows, "prefix": _own_prefix, "attention": _own_attention,
                "head": _own_head}[st["op"]](st)
    return {"rotate": _plain_rotate, "rows": _plain_rows, "prefix": _plain_prefix, "attention": _plain_attention,
            "head": _plain_head}[st["op"]](st)


def _own_rotate(st):
    import paper_2605_15609_b200 as psd
    psd.psd_rotate_qk(st["q"], st["k"], st["q_out"], st["k_out"], st["position"], st["frequency"], v=st["v"], v_out=st["v_out"],
                      slot=st["slot"], q_norm=st["q_norm"], k_norm=st["k_norm"], eps=st["eps"], interleaved=st["interleaved"],
                      gain=st["gain"])
    return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}


def _own_rows(st):
    import paper_2605_15609_b200 as psd
    psd.psd_quantize_rows(st["x"], st["codes"], st["scale"])
    return {"values": torch.mul(st["codes"], st["scale"][:, None]), "scale": st["scale"]}


def _own_prefix(st):
    import paper_2605_15609_b200 as psd
    psd.psd_prefix_quantize(st["k"], st["v"], st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"], block=st["block"],
                            begin=st["begin"], end=st["end"], span=st["add"])
    return {"k": _values(st, "k"), "v": _values(st, "v"), "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _values(st, name):
    return torch.mul(st[name + "_codes"], st[name + "_scale"].transpose(1, 2)[:, st["of_token"]][..., None])


def _own_attention(st):
    import paper_2605_15609_b200 as psd
    if "ws" not in st:
        n = psd.psd_attention_q8_workspace_bytes(st["B"], st["D"], st["M"], st["Hq"], st["Hkv"], st["Dh"], st["P"], st["S"])
        st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    psd.psd_draft_attention_q8(st["q"], st["k_codes"], st["v_codes"], st["k_scale"], st["v_scale"], st["out"], st["lse"],
                               st["k_own"], st["v_own"], block=st["block"], prefix_len=st["plen"], own_len=st["olen"],
                               scale=st["scale"], causal=st["causal"], workspace=st["ws"])
    return {"out": st["out"], "lse": st["lse"]}


def _own_head(st):
    import paper_2605_15609_b200 as psd
    if "ws" not in st:
        st["ws"] = torch.empty(psd.psd_confidence_q8_workspace_bytes(st["R"], st["H"], st["V"]), dtype=torch.uint8, device="cuda")
    psd.psd_confidence_q8(st["hidden"], st["w_codes"], st["w_scale"], st["tok"], st["conf"], st["lse"], workspace=st["ws"])
    return {"tok": st["tok"], "conf": st["conf"], "lse": st["lse"]}


def _plain_rotate(st):
    R = st["rotary"]
    turn = st["position"].double()[:, None] * st["frequency"]          # far positions: angles in 64 bits
    cos, sin = (torch.cos(turn) * st["gain"]).float()[:, None], (torch.sin(turn) * st["gain"]).float()[:, None]

    def one(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + st["eps"]) * weight.float()
        y = x.clone()
        first, second = (slice(0, R, 2), slice(1, R, 2)) if st["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        y[..., first] = x[..., first] * cos - x[..., second] * sin
        y[..., second] = x[..., second] * cos + x[..., first] * sin
        return y.to(st["q"].dtype)

    k_out, v_out, at = st["k_out"], st["v_out"], st["slot"].long()
    k_out[at] = one(st["k"], st["k_norm"])
    v_out[at] = st["v"]
    return {"q": one(st["q"], st["q_norm"]), "k": k_out, "v": v_out}


def _plain_rows(st):
    codes, scale = _codes(st["x"].float(), (1,))
    return {"values": codes * scale, "scale": scale[:, 0]}


def _plain_prefix(st):
    B, P, Hkv, Dh, T = (st[n] for n in ("B", "P", "Hkv", "Dh", "block"))
    nb, got = -(-P // T), {}
    at = torch.arange(P, device="cuda")[None, :]
    start = st["begin"][:, None] // T * T                             # from the begun block's first token on
    new = (at >= start) & (at < st["end"][:, None]) & (st["begin"] < st["end"])[:, None]
    for name in "kv":
        x = torch.zeros(B, nb * T, Hkv, Dh, device="cuda")
        x[:, :P] = torch.where(new[..., None, None], st[name].float(), 0.0)
        codes, scale = _codes(x.view(B, nb, T, Hkv, Dh), (2, 4))
        touched = torch.nn.functional.pad(new, (0, nb * T - P)).view(B, nb, T).any(2)
        scale = torch.where(touched[:, None, :], scale.view(B, nb, Hkv).transpose(1, 2), st[name + "_scale"])
        codes = torch.where(new[..., None, None], codes.view(B, nb * T, Hkv, Dh)[:, :P], st[name + "_codes"].float())
        got[name] = codes * scale.transpose(1, 2)[:, st["of_token"]][..., None]
        got[name + "_scale"] = scale
    return got


def _plain_attention(st):
    B, D, M, Hq, Hkv, Dh, P, S, T = (st[n] for n in ("B", "D", "M", "Hq", "Hkv", "Dh", "P", "S", "block"))
    G, of_token = Hq // Hkv, torch.arange(P, device="cuda") // T
    q = st["q"].float().view(B, D, M, Hkv, G, Dh).permute(0, 3, 1, 2, 4, 5).reshape(B, Hkv, D * M * G, Dh)
    there = torch.arange(P, device="cuda")[None, :] < st["plen"][:, None]
    kp, vp = (torch.where(there[:, None, :, None], st[n + "_codes"].permute(0, 2, 1, 3) * st[n + "_scale"][..., of_token, None], 0.0)
              for n in "kv")
    sp = (q @ kp.transpose(2, 3)) * st["scale"]
    sp = sp.masked_fill_(~there[:, None, None, :], -math.inf)
    # own keys: slot s of node d counts where s < its length, and, causally, s <= length - M + i for query i
    slot, olen = torch.arange(S, device="cuda"), st["olen"].view(B, D)
    own_there = slot < olen[..., None]
    ko, vo = (torch.where(own_there[..., None, None], st[n + "_own"].float().view(B, D, S, Hkv, Dh), 0.0).permute(0, 3, 1, 2, 4) for n in "kv")
    limit = olen[..., None].expand(B, D, M)
    if st["causal"]:
        limit = limit - M + 1 + torch.arange(M, device="cuda")
    seen = (slot < limit[..., None]).repeat_interleave(G, 2)
    so = torch.where(seen[:, None], (q.view(B, Hkv, D, M * G, Dh) @ ko.transpose(3, 4)) * st["scale"], -math.inf)
    m = torch.maximum(sp.amax(-1, keepdim=True), so.amax(-1).view(B, Hkv, -1, 1))
    m = torch.where(m == -math.inf, 0.0, m)
    pp, po = torch.exp_(sp.sub_(m)), torch.exp(so - m.view(B, Hkv, D, M * G, 1))
    l = pp.sum(-1, keepdim=True) + po.sum(-1).view(B, Hkv, -1, 1)
    o = pp @ vp + (po @ vo).reshape(B, Hkv, D * M * G, Dh)
    o = torch.where(l > 0, o / l, 0.0)
    back = lambda x, w: x.view(B, Hkv, D, M, G, w).permute(0, 2, 3, 1, 4, 5).reshape(B * D, M, Hq, w)  # noqa: E731
    return {"out": back(o, Dh).to(st["q"].dtype), "lse": back(m + torch.log(l), 1)[..., 0]}


def _plain_head(st):
    codes, scale = _codes(st["hidden"].float(), (1,))
    # sums of products of codes go past 2^24: in 64 bits they are exact
    x = (codes.double() @ st["w_codes"].t().double()).float() * st["w_scale"] * scale
    m = x.amax(-1, keepdim=True)
    first = torch.where(x == m, torch.arange(st["V"], device="cuda", dtype=torch.int32), st["V"]).amin(-1)
    s = torch.exp_(x.sub_(m)).sum(-1)
    return {"tok": first.to(torch.int32), "conf": 1.0 / s, "lse": m[:, 0] + torch.log(s)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------

def exact(case, seed):
    """What run() returns for these inputs, in fp64; scales and codes are the numbers that fp32 operations in the stated
    order give."""
    st = prepare(case, seed)
    return {"rotate": _exact_rotate, "rows": _exact_rows, "prefix": _exact_prefix, "attention": _exact_attention,
            "head": _exact_head}[case["op"]](st)


def _exact_codes(x):
    """Codes and scale of each row of a matrix of 16-bit numbers."""
    scale = torch.clamp((x.double().abs().amax(1) * _PER_CODE).float(), min=_TINY)
    inverse = (1.0 / scale.double()).float()
    return torch.round((x.double() * inverse.double()[:, None]).float()).double(), scale.double()


def _exact_rotate(st):
    T, R = st["T"], st["rotary"]
    angle = st["position"].double()[:, None, None] * st["frequency"]
    turn = torch.polar(torch.full_like(angle, st["gain"]), angle)

    def one(x, weight):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / st["Dh"] + st["eps"]) * weight.double()
        head, rest = x[..., :R], x[..., R:]
        pairs = head.reshape(T, -1, R // 2, 2) if st["interleaved"] else head.reshape(T, -1, 2, R // 2).transpose(2, 3)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z.reshape(T, -1, R) if st["interleaved"] else z.transpose(2, 3).reshape(T, -1, R)
        return torch.cat([z, rest], -1)

    k, v = st["k_out"].double(), st["v_out"].double()
    k[st["slot"].long()] = one(st["k"], st["k_norm"])
    v[st["slot"].long()] = st["v"].double()
    return {"q": one(st["q"], st["q_norm"]), "k": k, "v": v}


def _exact_rows(st):
    codes, scale = _exact_codes(st["x"])
    return {"values": codes.mul_(scale[:, None]), "scale": scale}


def _exact_prefix(st):
    B, P, Hkv, Dh, T = (st[n] for n in ("B", "P", "Hkv", "Dh", "block"))
    got = {}
    begin, end = st["begin"].tolist(), st["end"].tolist()
    for name in "kv":
        scale = st[name + "_scale"].double()
        val = st[name + "_codes"].double() * scale.transpose(1, 2)[:, st["of_token"]][..., None]
        for b in range(B):
            for j in range(begin[b] // T, -(-end[b] // T)) if begin[b] < end[b] else ():
                x = st[name][b, j * T:min(end[b], (j + 1) * T)].transpose(0, 1).reshape(Hkv, -1)
                c, s = _exact_codes(x)
                # (the block's room behind the last token keeps its codes)
                val[b, j * T:(j + 1) * T] = st[name + "_codes"][b, j * T:(j + 1) * T].double() * s[:, None]
                val[b, j * T:min(end[b], (j + 1) * T)] = (c * s[:, None]).view(Hkv, -1, Dh).transpose(0, 1)
                scale[b, :, j] = s
        got[name], got[name + "_scale"] = val, scale
    return got


def _exact_attention(st):
    N, M, Hq, Dh = st["q"].shape
    G, D, T = Hq // st["Hkv"], st["D"], st["block"]
    out = torch.zeros(N, M, Hq, Dh, dtype=torch.float64, device="cuda")
    lse = torch.full((N, M, Hq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(st["B"]):
        L = st["plen_host"][b]
        at = torch.arange(L, device="cuda") // T
        for h in range(st["Hkv"]):
            hq = slice(h * G, (h + 1) * G)
            kp, vp = (st[n + "_codes"][b, :L, h].double() * st[n + "_scale"][b, h, at].double()[:, None] for n in "kv")
            for n in range(b * D, (b + 1) * D):
                o = st["olen_host"][n]
                k, v = torch.cat([kp, st["k_own"][n, :o, h].double()]), torch.cat([vp, st["v_own"][n, :o, h].double()])
                if k.shape[0] == 0:
                    continue
                s = torch.einsum("igd,kd->igk", st["q"][n, :, hq].double(), k) * st["scale"]
                if st["causal"] and M > 1:
                    for i in range(M):
                        s[i, :, max(L, L + o - M + 1 + i):] = -math.inf
                z = torch.logsumexp(s, -1)
                lse[n, :, hq] = z
                dead = torch.isinf(z)
                out[n, :, hq] = torch.einsum("igk,kd->igd", torch.exp(s - torch.where(dead, 0.0, z)[..., None]), v)
    return {"out": out, "lse": lse}


def _exact_head(st):
    codes, scale = _exact_codes(st["hidden"])
    conf, lse = torch.empty(2, st["R"], dtype=torch.float64, device="cuda")
    w = st["w_codes"].double() * st["w_scale"].double()[:, None]
    for r in range(0, st["R"], 1024):
        x = (codes[r:r + 1024] * scale[r:r + 1024, None]) @ w.t()
        lse[r:r + 1024] = torch.logsumexp(x, 1)
        conf[r:r + 1024] = torch.exp(x.amax(1) - lse[r:r + 1024])
    return {"tok": None, "conf": conf, "lse": lse}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "rotate":
        T, heads, R = case["T"], case["Hq"] + 2 * case["Hkv"], case["rotary"]
        return {"bytes": T * heads * case["Dh"] * 4 + 8 * T + 4 * R, "flops": T * (case["Hq"] + case["Hkv"]) * (3.0 * R + 4.0 * case["Dh"])}
    if op == "rows":
        return {"bytes": case["R"] * (3 * case["H"] + 4), "flops": 3.0 * case["R"] * case["H"]}
    if op == "prefix":
        B, P, Hkv, Dh, T = (case[n] for n in ("B", "P", "Hkv", "Dh", "block"))
        tokens = B * min(case["add"] + T / 2, 0.6 * P if case["ragged"] else P)
        return {"bytes": 2 * tokens * Hkv * (3 * Dh + 4 / T), "flops": 6.0 * tokens * Hkv * Dh}
    if op == "attention":
        B, D, M, Hq, Hkv, Dh, P, T = (case[n] for n in ("B", "D", "M", "Hq", "Hkv", "Dh", "P", "block"))
        keys = 0.6 * P * B if case["ragged"] else P * B          # prefix keys of all sequences (mean of the lengths)
        rows = D * M * Hq
        own_keys = B * D * case["S"] * (0.6 if case["ragged"] and M == 1 else 1.0)
        return {"bytes": 4 * B * rows * Dh + 4 * B * rows + 2 * keys * Hkv * (Dh + 4 / T) + 4 * own_keys * Hkv * Dh,
                "flops": 4.0 * rows * Dh * keys + 4.0 * M * Hq * Dh * own_keys}
    R, H, V = case["R"], case["H"], case["V"]
    return {"bytes": V * (H + 4) + 2 * R * H + 12 * R, "flops": 2.0 * R * H * V}

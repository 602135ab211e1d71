"""The operators around the step from their definitions in 64 bits, batched on the GPU: for shapes at which the row-by-row versions
of ops_plain.py take too long."""
import torch


def draft_attention(q, kp, vp, plen, ko, vo, olen, scale, causal):
    """out, lse, sum_j p_j |v_j| and the largest sum_d |q_d k_d| * scale, as ops_plain.draft_attention (tensors, float64)."""
    N, M, Hq, Dh = q.shape
    B, Hkv = kp.shape[0], kp.shape[2]
    D, G = N // B, Hq // Hkv
    out, absv = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full((N, M, Hq), -float("inf"), dtype=torch.float64, device=q.device)
    big = 0.0
    for n in range(N):
        L, o = plen[n // D], olen[n] if ko is not None else 0
        k, v = kp[n // D, :L].double(), vp[n // D, :L].double()
        if o:
            k, v = torch.cat([k, ko[n, :o].double()]), torch.cat([v, vo[n, :o].double()])
        if L + o == 0:
            continue
        x = q[n].double().view(M, Hkv, G, Dh)
        s = torch.einsum("mhgd,jhd->mhgj", x, k) * scale
        big = max(big, float(torch.einsum("mhgd,jhd->mhgj", x.abs(), k.abs()).max()) * scale)
        if causal and o:
            seen = o - M + torch.arange(M, device=q.device)[:, None] >= torch.arange(o, device=q.device)[None]
            s[..., L:].masked_fill_(~seen[:, None, None], -float("inf"))
        top = s.amax(-1, keepdim=True)
        none = top == -float("inf")
        p = torch.exp(s - torch.where(none, 0.0, top))
        total = p.sum(-1, keepdim=True)
        lse[n] = (top + torch.log(total)).squeeze(-1).reshape(M, Hq)
        p = torch.where(none, 0.0, p / total)
        out[n] = torch.einsum("mhgj,jhd->mhgd", p, v).reshape(M, Hq, Dh)
        absv[n] = torch.einsum("mhgj,jhd->mhgd", p, v.abs()).reshape(M, Hq, Dh)
    return out, lse, absv, big


def prefix_weights(q, kp, plen, lse, scale, beta, acc_in):
    """The sums, and the largest sum_d |q_d k_d| * scale."""
    N, M, Hq, Dh = q.shape
    B, P, Hkv, _ = kp.shape
    D, G = N // B, Hq // Hkv
    acc, big = torch.zeros(B, Hkv, P, dtype=torch.float64, device=q.device), 0.0
    for b in range(B):
        L = plen[b]
        if L == 0:
            continue
        x = q[b * D:(b + 1) * D].double().reshape(D * M, Hkv, G, Dh)
        k = kp[b, :L].double()
        big = max(big, float(torch.einsum("thgd,jhd->thgj", x.abs(), k.abs()).max()) * scale)
        at = lse[b * D:(b + 1) * D].double().reshape(D * M, Hkv, G, 1)
        w = torch.exp(torch.einsum("thgd,jhd->thgj", x, k) * scale - torch.where(at == -float("inf"), 0.0, at))
        w = torch.where(at == -float("inf"), 0.0, w)
        acc[b, :, :L] = w.sum((0, 2))
        if acc_in is not None:
            acc[b, :, :L] += beta * acc_in[b, :, :L].double()
    return acc, big


def confidences(lg, D, M, history, history_len, draft_tokens, draft_mask, rep, pres, freq, bias, allow):
    """token, conf, lse of edited rows: edits in float32, each operation rounded on its own, then 64 bits."""
    R, V = lg.shape
    N = R // M
    count = torch.zeros(N, V, dtype=torch.int32, device=lg.device)

    def note(node, ids, use):
        ok = use & (ids >= 0) & (ids < V)
        count[node].index_add_(0, ids[ok].long(), torch.ones_like(ids[ok]))
    for n in range(N):
        if history is not None:
            h = history[n // D]
            note(n, h, torch.arange(len(h), device=lg.device) < (len(h) if history_len is None else int(history_len[n // D])))
        if draft_tokens is not None:
            note(n, draft_tokens[n], draft_mask[n] == 0)
    x = lg.float()
    c = count.repeat_interleave(M, 0)
    y = torch.where(x > 0, x / rep, x * rep)
    x = torch.where(c > 0, y - (c.float() * torch.tensor(freq, device=lg.device) + torch.tensor(pres, device=lg.device)), x)
    if bias is not None:
        b = bias.view(-1, V)
        x = x + b.repeat_interleave(R // len(b), 0)
    if allow is not None:
        bits = (allow[:, :, None] >> torch.arange(32, dtype=torch.int32, device=lg.device)) & 1
        bits = bits.reshape(len(allow), -1)[:, :V].repeat_interleave(R // len(allow), 0)
        x = torch.where(bits == 0, -float("inf"), x)
    bad = torch.isnan(x).any(1) | (x == float("inf")).any(1)
    none = ~bad & (x == -float("inf")).all(1)
    x = x.double()
    top = x.amax(1)
    s = torch.exp(x - torch.where(none, 0.0, top)[:, None]).sum(1)
    first = (x == top[:, None]).int().argmax(1).int()
    tok = torch.where(none, -1, first)
    conf, lse = torch.where(none, 0.0, 1 / s), torch.where(none, -float("inf"), top + torch.log(s))
    nan = float("nan")
    return tok, torch.where(bad, nan, conf), torch.where(bad, nan, lse), bad

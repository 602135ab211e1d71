"""Plain 64-bit implementations of the operators around the step, one row at a time (numpy on the CPU)."""
import numpy as np


def draft_attention(q, kp, vp, plen, ko, vo, olen, scale, causal):
    """q [N, M, Hq, Dh], kp/vp [B, P, Hkv, Dh], ko/vo [N, S, Hkv, Dh] (all float64) -> out, lse, sum_j p_j |v_j| and the
    largest sum_d |q_d k_d| * scale of any score (for error bounds)."""
    N, M, Hq, Dh = q.shape
    B, Hkv = kp.shape[0], kp.shape[2]
    D, G = N // B, Hq // Hkv
    out, absv = np.zeros_like(q), np.zeros_like(q)
    lse = np.full((N, M, Hq), -np.inf)
    big = 0.0
    for n in range(N):
        L, o = plen[n // D], olen[n]
        for h in range(Hq):
            for i in range(M):
                seen = min(o, max(0, o - M + 1 + i)) if causal else o
                k = np.concatenate([kp[n // D, :L, h // G], ko[n, :seen, h // G]])
                v = np.concatenate([vp[n // D, :L, h // G], vo[n, :seen, h // G]])
                if len(k) == 0:
                    continue
                s = (k @ q[n, i, h]) * scale
                big = max(big, float((np.abs(k) @ np.abs(q[n, i, h])).max() * scale))
                m = s.max()
                p = np.exp(s - m)
                lse[n, i, h] = m + np.log(p.sum())
                p /= p.sum()
                out[n, i, h] = p @ v
                absv[n, i, h] = p @ np.abs(v)
    return out, lse, absv, big


def prefix_weights(q, kp, plen, lse, scale, beta, acc_in):
    N, M, Hq, Dh = q.shape
    B, P, Hkv, _ = kp.shape
    D, G = N // B, Hq // Hkv
    acc = np.zeros((B, Hkv, P))
    for b in range(B):
        L = plen[b]
        for h in range(Hkv):
            if acc_in is not None:
                acc[b, h, :L] = beta * acc_in[b, h, :L]
            for n in range(b * D, (b + 1) * D):
                for g in range(h * G, (h + 1) * G):
                    for i in range(M):
                        if lse[n, i, g] > -np.inf:
                            acc[b, h, :L] += np.exp((kp[b, :L, h] @ q[n, i, g]) * scale - lse[n, i, g])
    return acc


def prefix_evict(scores, plen, keep, n_sink, n_recent):
    """Kept positions per (b, h), ascending."""
    B, Hkv, _ = scores.shape
    kept = []
    for b in range(B):
        L, row = plen[b], []
        for h in range(Hkv):
            def rank(j):
                s = scores[b, h, j]
                forced = j < n_sink or j >= L - n_recent
                return (not forced, bool(np.isnan(s)), 0.0 if np.isnan(s) else -s, j)
            row.append(sorted(sorted(range(L), key=rank)[:keep]))
        kept.append(row)
    return kept


def edited_logits(logits, D, M, history, hist_len, draft_tokens, draft_mask, rep, pres, freq, bias, allow):
    """The edited rows as the operator defines them (float32, each operation rounded on its own), -inf where forbidden;
    logits float32 [R, V]."""
    R, V = logits.shape
    f = np.float32
    x = logits.astype(f).copy()
    for r in range(R):
        node, b = r // M, r // (M * D)
        text = []
        if history is not None:
            text += [int(t) for t in history[b, :hist_len[b] if hist_len is not None else history.shape[1]]]
        if draft_tokens is not None:
            text += [int(draft_tokens[node, i]) for i in range(M) if draft_mask[node, i] == 0]
        for v in set(t for t in text if 0 <= t < V):
            c = f(text.count(v))
            y = f(x[r, v] / f(rep)) if x[r, v] > 0 else f(x[r, v] * f(rep))
            x[r, v] = f(y - f(f(f(freq) * c) + f(pres)))
        if bias is not None:
            x[r] = x[r] + bias[r // (R // bias.shape[0])]
        if allow is not None:
            w = allow[r // (R // allow.shape[0])].view(np.uint32)
            bit = (w[np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1
            x[r][bit == 0] = -np.inf
    return x


def confidence(x):
    """token, conf, lse of edited rows, in 64 bits."""
    R = x.shape[0]
    tok, conf, lse = np.full(R, -1, np.int32), np.zeros(R), np.full(R, -np.inf)
    for r in range(R):
        y = x[r].astype(np.float64)
        if np.isnan(y).any() or (y == np.inf).any():
            conf[r] = lse[r] = np.nan
            continue
        m = y.max()
        if m == -np.inf:
            continue
        tok[r] = int(np.argmax(y))          # the first of equal maxima
        s = np.exp(y - m).sum()
        conf[r], lse[r] = 1.0 / s, m + np.log(s)
    return tok, conf, lse

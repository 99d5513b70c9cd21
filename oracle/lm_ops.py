"""Plain NumPy forms, in 64 bits, of the operators that stand next to the transformer's layers: scaled embedding
lookup and its gradients, dropout from a counter-based generator, linear attention with a decay per head, log
probabilities of tokens with their gradient, distillation from a teacher's top logits.  Written from the formulas; no
chunks, no sorting, no segments."""
import numpy as np


def embed_fwd(ids, table, pos, scale):
    """h[r] = scale * table[ids[r]] + pos[r mod T] (pos may be None); ids are clamped into the table."""
    h = scale * table[np.clip(ids, 0, len(table) - 1)]
    return h if pos is None else h + pos[np.arange(len(ids)) % len(pos)]


def embed_bwd(ids, dh, vocab, seq_len, scale):
    dtable = np.zeros((vocab, dh.shape[1]))
    for r, t in enumerate(np.clip(ids, 0, vocab - 1)):
        dtable[t] += dh[r]
    dpos = None
    if seq_len:
        dpos = np.zeros((seq_len, dh.shape[1]))
        for r in range(len(ids)):
            dpos[r % seq_len] += dh[r]
    return scale * dtable, dpos


def philox4x32(counter, key, rounds=10):
    """Philox4x32 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011).  counter: four
    integers or arrays, key: two integers; returns four uint64 arrays of 32-bit words."""
    m32 = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, dtype=np.uint64) & m32 for x in counter]
    k = [int(key[0]), int(key[1])]
    s = np.uint64(32)
    for _ in range(rounds):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> s) ^ c[1] ^ np.uint64(k[0]), p1 & m32, (p0 >> s) ^ c[3] ^ np.uint64(k[1]), p0 & m32]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_keep(n, p, seed, offset=0, w2=0, w3=0):
    """Which of n elements stay: word i mod 4 of the counter offset + i div 4, against floor(p 2^32)."""
    with np.errstate(over="ignore"):
        ctr = np.arange((n + 3) // 4, dtype=np.uint64) + np.uint64(offset % (1 << 64))
    w = philox4x32([ctr, ctr >> np.uint64(32), np.full_like(ctr, w2), np.full_like(ctr, w3)],
                   (seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF))
    return np.stack(w, 1).reshape(-1)[:n] >= np.uint64(int(np.floor(p * 2.0 ** 32)))


def dropout(x, resid, p, seed, offset=0, w2=0, w3=0):
    keep = dropout_keep(x.size, p, seed, offset, w2, w3).reshape(x.shape)
    y = np.where(keep, x / (1.0 - p), 0.0)
    return y if resid is None else y + resid


def linear_attention_fwd(q, k, v, log_decay, scale, state=None, lengths=None):
    """S_t = l S_{t-1} + k_t v_t^T, o_t = scale q_t S_t, token by token.  q, k, v: [B, T, H, 64]; returns o (zero behind
    a sequence's end) and the last states [B, H, 64, 64]."""
    B, T, H, D = q.shape
    S = np.zeros((B, H, D, D)) if state is None else state.astype(np.float64).copy()
    o = np.zeros((B, T, H, D))
    l = np.exp(np.asarray(log_decay, dtype=np.float64))[:, None, None]
    for b in range(B):
        for t in range(T if lengths is None else int(np.clip(lengths[b], 0, T))):
            S[b] = l * S[b] + k[b, t][:, :, None] * v[b, t][:, None, :]
            o[b, t] = scale * np.einsum("hk,hkv->hv", q[b, t], S[b])
    return o, S


def linear_attention_bwd(q, k, v, do, log_decay, scale, state=None, dstate=None, lengths=None):
    """Gradients of sum(o * do) + sum(S_last * dstate) with respect to q, k, v and the incoming state."""
    B, T, H, D = q.shape
    l = np.exp(np.asarray(log_decay, dtype=np.float64))[:, None, None]
    dq, dk, dv = (np.zeros((B, T, H, D)) for _ in range(3))
    R = np.zeros((B, H, D, D)) if dstate is None else dstate.astype(np.float64).copy()
    for b in range(B):
        n = T if lengths is None else int(np.clip(lengths[b], 0, T))
        S = np.zeros((H, D, D)) if state is None else state[b].astype(np.float64).copy()
        for t in range(n):
            S = l * S + k[b, t][:, :, None] * v[b, t][:, None, :]
            dq[b, t] = scale * np.einsum("hkv,hv->hk", S, do[b, t])
        for t in reversed(range(n)):               # R: gradient of S_t through everything behind token t
            R[b] = R[b] + scale * q[b, t][:, :, None] * do[b, t][:, None, :]
            dk[b, t] = np.einsum("hkv,hv->hk", R[b], v[b, t])
            dv[b, t] = np.einsum("hkv,hk->hv", R[b], k[b, t])
            R[b] = l * R[b]
    return dq, dk, dv, R


def log_softmax(x, temperature):
    """Log probabilities of one row and its log-sum-exp; -infinity throughout where every logit is -infinity."""
    z = np.asarray(x, dtype=np.float64) / temperature
    m = z.max()
    if m == -np.inf:
        return np.full_like(z, -np.inf), -np.inf
    if not m < np.inf:                              # NaN or +infinity in the row
        return np.full_like(z, np.nan), np.nan
    log_s = np.log(np.exp(z - m).sum())
    return z - m - log_s, m + log_s                 # rows of huge values keep their digits


def token_logprobs(x, tokens, temperature=1.0, top_k=0):
    """logp, entropy, lse [rows], top ids and their log probabilities [rows, top_k]; token ids outside [0, vocab) are none."""
    rows, n = x.shape
    logp, ent, lses = np.zeros(rows), np.zeros(rows), np.zeros(rows)
    ids, tops = np.zeros((rows, top_k), dtype=np.int64), np.zeros((rows, top_k))
    for r in range(rows):
        l, lses[r] = log_softmax(x[r], temperature)
        p = np.exp(l)
        ent[r] = -np.sum(p[p != 0] * l[p != 0])     # a NaN stays in
        if tokens is not None and 0 <= tokens[r] < n:
            logp[r] = l[tokens[r]]
        order = sorted(range(n), key=lambda j: (bool(np.isnan(x[r, j])), 0.0 if np.isnan(x[r, j]) else -float(x[r, j]), j)) if top_k else []
        ids[r] = order[:top_k]
        tops[r] = l[ids[r]]
    return logp, ent, lses, ids, tops


def token_logprobs_bwd(x, tokens, dlogp=None, dentropy=None, dlse=None, temperature=1.0):
    dx = np.zeros(x.shape)
    for r in range(len(x)):
        has = dlogp is not None and 0 <= tokens[r] < x.shape[1]
        a, b, c = (dlogp[r] if has else 0.0), (0.0 if dentropy is None else dentropy[r]), (0.0 if dlse is None else dlse[r])
        l, lse = log_softmax(x[r], temperature)
        if (a == 0 and b == 0 and c == 0) or lse == -np.inf:
            continue
        p = np.exp(l)
        pl = np.where(p == 0, 0.0, p * np.where(p == 0, 0.0, l))
        dx[r] = (c - a) * p - b * (pl - p * pl.sum())
        if has:
            dx[r, tokens[r]] += a
    return dx / temperature


def distill(x, ids, teacher, rest, temperature=1.0, scale=1.0, dloss=None):
    """loss [rows] = scale * KL(teacher || student) and its gradient with respect to the logits, times dloss."""
    rows, n = x.shape
    loss, dx = np.zeros(rows), np.zeros(x.shape)
    for r in range(rows):
        entries = [(int(i), float(t)) for i, t in zip(ids[r], teacher[r]) if 0 <= i < n]
        t = np.array([e[1] for e in entries])
        if not len(t) or (t == -np.inf).all():
            continue
        if rest:
            q = np.exp(t)
            qr = 1.0 - q.sum()
            qr = qr if qr > 2.0 ** -20 else 0.0
        else:
            q = np.exp((t - t.max()) / temperature)
            q, qr = q / q.sum(), 0.0
        l, lse = log_softmax(x[r], temperature)
        p = np.exp(l)
        outside = np.ones(n, dtype=bool)
        outside[[e[0] for e in entries]] = False
        lo = l[outside]
        log_rest = -np.inf if not len(lo) or lo.max() == -np.inf else lo.max() + np.log(np.exp(lo - lo.max()).sum())
        zo = x[r][outside] / temperature                # the rest's shares by itself: beside far larger logits l has lost their digits
        eo = np.exp(zo - zo.max()) if log_rest != -np.inf else np.zeros(len(zo))
        kl = sum(qj * (np.log(qj) - l[i]) for (i, _), qj in zip(entries, q) if qj != 0)
        if qr > 0:
            kl += qr * (np.log(qr) - log_rest)
        loss[r] = scale * kl
        if lse == -np.inf:
            continue
        d = (q.sum() + qr) * p
        for (i, _), qj in zip(entries, q):
            d[i] -= qj
        if qr > 0 and log_rest != -np.inf:
            d[outside] -= qr * eo / eo.sum()
        f = (1.0 if dloss is None else dloss[r]) * scale / temperature
        dx[r] = d * f if f != 0 else 0.0
    return loss, dx

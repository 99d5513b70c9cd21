"""Workloads of the language-model operators: scaled embedding lookup and its gradient by sorted tokens, dropout
from a counter-based generator, linear attention with a decay per head (prompt, backward and single-token form).

``own`` selects the path: False runs each operator as elementary torch operations in 32 bits, True calls the
library.  ``listed()`` names the fixed cases, ``draw(rng)`` makes further ones over the same ranges.
"""
import math

import numpy as np
import torch

own = False

D = 64   # width of a head, as in the framework's attention
DEV = "cuda"


def _lp():
    from paper_2012_03837_b200 import binding
    return binding


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one new token for each of 64 sequences being answered: latency
        dict(name="embed_fwd_few", op="embed_fwd", dtype="fp32", rows=64, vocab=8192, d=512, T=0, scale=math.sqrt(512.0),
             zipf=False),
        # the input of the 24-block transformer: 16 x 512 tokens, 32768 tokens in the vocabulary, positions added
        dict(name="embed_fwd_train", op="embed_fwd", dtype="bf16", rows=8192, vocab=32768, d=1024, T=512, scale=1.0,
             zipf=False),
        # the 8-block transformer's table gradient: uniform tokens
        dict(name="embed_bwd_uniform", op="embed_bwd", dtype="bf16", rows=8192, vocab=8192, d=512, T=256, scale=1.0,
             zipf=False),
        # the large table under a minibatch of natural text: a few tokens make up much of it
        dict(name="embed_bwd_zipf", op="embed_bwd", dtype="bf16", rows=65536, vocab=32768, d=1024, T=512, scale=32.0,
             zipf=True),
        # a small fp32 activation (64 rows, an odd tail): latency
        dict(name="dropout_small", op="dropout", dtype="fp32", n=64 * 256 + 3, p=0.1, resid=False, offset=7),
        # a transformer branch joining the residual stream, 32768 positions of 1024 channels
        dict(name="dropout_residual", op="dropout", dtype="bf16", n=32768 * 1024, p=0.1, resid=True, offset=1 << 33),
        # training forward of the 8-block transformer's shape, q, k and v packed in one tensor
        dict(name="linattn_fwd_packed", op="la_fwd", batch=32, seq=256, heads=8, packed=True, state=False, ragged=False),
        # four prompts of unequal length, each continuing from a state and leaving one for the answer
        dict(name="linattn_fwd_prompts", op="la_fwd", batch=4, seq=8191, heads=16, packed=False, state=True, ragged=True),
        # training backward of the 24-block transformer's shape
        dict(name="linattn_bwd_train", op="la_bwd", batch=16, seq=512, heads=16, packed=False, state=False, ragged=False),
        # backward through long sequences cut into pieces: gradients enter and leave through the state
        dict(name="linattn_bwd_long", op="la_bwd", batch=2, seq=4097, heads=16, packed=False, state=True, ragged=False),
        # one sequence answering: latency
        dict(name="linattn_step_one", op="la_step", batch=1, heads=16, idle=False),
        # many sequences answering, some of the slots idle
        dict(name="linattn_step_many", op="la_step", batch=256, heads=16, idle=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed_fwd", "embed_bwd", "dropout", "la_fwd", "la_bwd", "la_step"])
    if op in ("embed_fwd", "embed_bwd"):
        d = rng.choice([_log(rng, 8, 1024), 8 * _log(rng, 1, 128)])
        rows = _log(rng, 1, 65536)
        vocab = _log(rng, 2, 32768)
        T = rng.choice([0, _log(rng, 1, 1024)])
        return dict(op=op, dtype=rng.choice(["bf16", "fp32"]) if d * rows <= 1 << 25 else "bf16", rows=rows, vocab=vocab,
                    d=d, T=T, scale=rng.choice([1.0, math.sqrt(d), rng.uniform(0.1, 3.0)]), zipf=rng.random() < 0.5)
    if op == "dropout":
        dtype = rng.choice(["bf16", "fp32"])
        return dict(op=op, dtype=dtype, n=_log(rng, 1, (1 << 25) if dtype == "bf16" else (1 << 24)),
                    p=rng.choice([0.0, 0.1, 0.5, rng.uniform(0.01, 0.9)]), resid=rng.random() < 0.5,
                    offset=rng.choice([0, rng.randrange(1 << 20), rng.randrange(1 << 48)]))
    heads = rng.randint(1, 16)
    if op == "la_step":
        return dict(op=op, batch=_log(rng, 1, 256), heads=heads, idle=rng.random() < 0.5)
    budget = 4 * 8191 * 16 if op == "la_fwd" else 2 * 4097 * 16
    seq = _log(rng, 1, 8191)
    batch = max(1, min(64, _log(rng, 1, 64), budget // (seq * heads)))
    return dict(op=op, batch=batch, seq=seq, heads=heads, packed=rng.random() < 0.5, state=rng.random() < 0.5,
                ragged=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _dt(case):
    return torch.bfloat16 if case.get("dtype", "bf16") == "bf16" else torch.float32


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _tokens(case, g):
    rows, vocab = case["rows"], case["vocab"]
    if not case["zipf"]:
        return torch.randint(0, vocab, (rows,), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
    w = 1.0 / torch.arange(1, vocab + 1, device=DEV, dtype=torch.float64)   # frequency of the k-th commonest token ~ 1/k
    cdf = torch.cumsum(w, 0) / w.sum()
    u = torch.rand(rows, generator=g, device=DEV, dtype=torch.float64)
    return torch.searchsorted(cdf, u).clamp_(max=vocab - 1).to(torch.int32)


def _log_decay(case, seed):
    """Per-head log decay: from forgetting within a dozen tokens to keeping everything (one head in eight)."""
    r = np.random.default_rng(seed + 77)
    h = case["heads"]
    e = r.uniform(3.0, 12.0, h)
    g = np.log1p(-2.0 ** -e)
    g[r.random(h) < 0.125] = 0.0
    return torch.from_numpy(g.astype(np.float32)).to(DEV)


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    rn = lambda *s, dtype=torch.float32: torch.randn(*s, generator=g, device=DEV, dtype=torch.float32).to(dtype)
    st = dict(case=case, seed=seed)
    if op in ("embed_fwd", "embed_bwd"):
        rows, vocab, d, T, dt = case["rows"], case["vocab"], case["d"], case["T"], _dt(case)
        st["ids"] = _tokens(case, g)
        if op == "embed_fwd":
            st["table"] = (0.02 * rn(vocab, d)).to(dt)
            st["pos"] = (0.02 * rn(T, d)).to(dt) if T else None
            st["out"] = torch.zeros(rows, d, dtype=dt, device=DEV)
        else:
            st["dout"] = (1e-3 * rn(rows, d)).to(dt)
            st["dtable"] = torch.zeros(vocab, d, device=DEV)
            st["dpos"] = torch.zeros(T, d, device=DEV) if T else None
            if own:
                st["ws"] = torch.empty(_lp().lp_embed_workspace_bytes(rows, vocab, d), dtype=torch.uint8, device=DEV)
    elif op == "dropout":
        st["x"] = rn(case["n"], dtype=_dt(case))
        st["resid"] = rn(case["n"], dtype=_dt(case)) if case["resid"] else None
        st["y"] = torch.zeros(case["n"], dtype=_dt(case), device=DEV)
        st["key"] = int(np.random.default_rng(seed).integers(0, 1 << 63))
    else:
        B, H, T = case["batch"], case["heads"], case.get("seq", 1)
        bf = torch.bfloat16
        if case.get("packed"):
            qkv = rn(B, T, 3, H, D, dtype=bf)
            st["q"], st["k"], st["v"] = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
        else:
            st["q"], st["k"], st["v"] = (rn(B, T, H, D, dtype=bf) for _ in range(3))
        st["g"] = _log_decay(case, seed)
        st["scale"] = 0.125
        with_state = op == "la_step" or case["state"]
        st["s_in"] = rn(B, H, D, D) if with_state else None
        st["s_out"] = torch.zeros(B, H, D, D, device=DEV) if with_state else None
        st["lengths"] = None
        if case.get("ragged"):
            r = np.random.default_rng(seed + 5)
            L = r.integers(max(0, T // 2), T + 1, B).astype(np.int32)
            L[0] = T
            st["lengths"] = torch.from_numpy(L).to(DEV)
        if case.get("idle"):
            r = np.random.default_rng(seed + 6)
            st["lengths"] = torch.from_numpy((r.random(B) < 0.9).astype(np.int32)).to(DEV)
        fill = lambda: torch.full((B, T, H, D), 0.5, dtype=bf, device=DEV)   # what rows behind a sequence's end keep
        if op == "la_bwd":
            st["do"] = rn(B, T, H, D, dtype=bf)
            if case.get("packed"):
                dqkv = torch.full((B, T, 3, H, D), 0.5, dtype=bf, device=DEV)
                st["dq"], st["dk"], st["dv"] = dqkv[:, :, 0], dqkv[:, :, 1], dqkv[:, :, 2]
            else:
                st["dq"], st["dk"], st["dv"] = fill(), fill(), fill()
            st["ds_out"] = rn(B, H, D, D) if with_state else None
            st["ds_in"] = torch.zeros(B, H, D, D, device=DEV) if with_state else None
        else:
            st["o"] = fill()
        if own:
            lp = _lp()
            form = {"la_fwd": lp.LP_LINATTN_FORWARD, "la_bwd": lp.LP_LINATTN_BACKWARD, "la_step": lp.LP_LINATTN_STEP}[op]
            st["ws"] = torch.empty(lp.lp_linear_attention_workspace_bytes(form, B, T, H), dtype=torch.uint8, device=DEV)
    return st


# ------------------------------------------------------------------------------------------------ plain forms
_M32 = 0xFFFFFFFF


def _philox_words(n, key, offset):
    """The first n words of Philox4x32-10 (Salmon et al., SC 2011) under `key`, counters offset, offset + 1, ..."""
    nc = (n + 3) // 4
    c = torch.arange(nc, device=DEV, dtype=torch.int64) + offset      # offsets here stay below 2^63
    x = [c & _M32, (c >> 32) & _M32, torch.zeros_like(c), torch.zeros_like(c)]
    k0, k1 = key & _M32, (key >> 32) & _M32

    def mul(a, m):   # high and low word of a 32 x 32-bit product, within 63 bits: the multiplier in two 16-bit halves
        lo, hi = a * (m & 0xFFFF), a * (m >> 16)
        t = (lo >> 16) + hi
        return (t >> 16) & _M32, ((t & 0xFFFF) << 16) | (lo & 0xFFFF)

    for _ in range(10):
        h0, l0 = mul(x[0], 0xD2511F53)
        h1, l1 = mul(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ k0, l1, h0 ^ x[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return torch.stack(x, 1).reshape(-1)[:n]


def _plain_embed_fwd(st):
    c = st["case"]
    h = st["table"].float()[st["ids"].long()] * c["scale"] if c["vocab"] <= 4 * c["rows"] else \
        st["table"][st["ids"].long()].float() * c["scale"]
    if c["T"]:
        h = h + st["pos"].float()[torch.arange(c["rows"], device=DEV) % c["T"]]
    return h.to(_dt(c))


def _plain_embed_bwd(st):
    c = st["case"]
    dh = st["dout"].float()
    out = [torch.zeros(c["vocab"], c["d"], device=DEV).index_add_(0, st["ids"].long(), dh) * c["scale"]]
    if c["T"]:
        at = torch.arange(c["rows"], device=DEV) % c["T"]
        out.append(torch.zeros(c["T"], c["d"], device=DEV).index_add_(0, at, dh))
    return out


def _plain_dropout(st):
    c = st["case"]
    keep = _philox_words(c["n"], st["key"], c["offset"]) >= int(math.floor(c["p"] * 2.0 ** 32))
    y = torch.where(keep, st["x"].float() * (1.0 / (1.0 - c["p"])), 0.0)
    if c["resid"]:
        y = y + st["resid"].float()
    return y.to(_dt(c))


def _scan(a, b, c, g, s, lens):
    """y_t = sum_{s<=t} l^(t-s) (a_t . b_s) c_s + l^(t+1) a_t S, chunk by chunk in 32 bits; returns y and the last state.
    a, b, c: [B, H, T, 64] fp32; s: [B, H, 64, 64]; lens: [B] valid positions."""
    B, H, T, _ = a.shape
    C = min(64, T)
    i = torch.arange(C, device=DEV)
    y = torch.empty_like(a)
    lg = g.double()[None, :, None, None]
    rel = (i[:, None] - i[None, :]).double()
    mask = torch.where(rel >= 0, torch.exp(lg * rel.clamp(min=0)), 0.0).float()   # [1, H, C, C]
    for t0 in range(0, T, C):
        n = min(C, T - t0)
        av, bv, cv = (x[:, :, t0:t0 + n] for x in (a, b, c))
        valid = (lens - t0).clamp(0, n)                                             # [B]
        inside = (i[:n][None] < valid[:, None])[:, None, :, None]                   # [B, 1, n, 1]
        left = valid[:, None] - 1 - i[:n][None]                                     # decay steps to the chunk's end
        ga = torch.exp(lg * (i[:n] + 1)[None, None, :, None].double()).float()
        gl = torch.exp(lg * left[:, None, :, None].clamp(min=0).double()).float()
        bm = torch.where(inside, bv, 0.0)
        y[:, :, t0:t0 + n] = torch.matmul(torch.matmul(av, bm.transpose(-1, -2)) * mask[:, :, :n, :n], cv) \
            + torch.matmul(av, s) * ga
        s = s * torch.exp(lg * valid[:, None, None, None].double()).float() + torch.matmul((bm * gl).transpose(-1, -2), cv)
    return y, s


def _heads_first(x):
    return x.float().transpose(1, 2)


def _plain_linattn(st):
    c = st["case"]
    B, H, T = c["batch"], c["heads"], c.get("seq", 1)
    q, k, v = (_heads_first(st[n]) for n in "qkv")
    lens = st["lengths"].long() if st["lengths"] is not None else torch.full((B,), T, device=DEV)
    zero = torch.zeros(B, H, D, D, device=DEV)
    s_in = st["s_in"] if st["s_in"] is not None else zero
    ok = (torch.arange(T, device=DEV)[None] < lens[:, None])[:, :, None, None]
    put = lambda y, buf: torch.where(ok, y.transpose(1, 2).to(torch.bfloat16), buf)
    if c["op"] != "la_bwd":
        y, s = _scan(q * st["scale"], k, v, st["g"], s_in, lens)
        out = [put(y, st["o"])]
        return out + [s] if st["s_out"] is not None else out
    do = _heads_first(st["do"]) * st["scale"]
    ds = st["ds_out"] if st["ds_out"] is not None else zero
    dq, _ = _scan(do, v, k, st["g"], s_in.transpose(-1, -2), lens)
    dk, dv, r = _reverse_pair(q, k, v, do, st["g"], ds, lens)
    out = [put(dq, st["dq"]), put(dk, st["dk"]), put(dv, st["dv"])]
    return out + [r] if st["ds_in"] is not None else out


def _reverse_pair(q, k, v, do, g, ds, lens):
    """dk_s = R_s v_s, dv_s = R_s^T k_s with R_s = l R_{s+1} + q_s do_s^T, R behind the end = dS_out / l; and l R_0."""
    B, H, T, _ = q.shape
    C = min(64, T)
    i = torch.arange(C, device=DEV)
    lg = g.double()[None, :, None, None]
    rel = (i[None, :] - i[:, None]).double()                   # reader s in rows, source t >= s in columns
    mask = torch.where(rel >= 0, torch.exp(lg * rel.clamp(min=0)), 0.0).float()
    dk, dv = torch.empty_like(k), torch.empty_like(v)
    s = ds                                                     # gradient of the state behind the chunk's last token
    for t0 in reversed(range(0, T, C)):
        n = min(C, T - t0)
        valid = (lens - t0).clamp(0, n)
        inside = (i[:n][None] < valid[:, None])[:, None, :, None]
        gb = torch.exp(lg * (valid[:, None] - 1 - i[:n][None]).clamp(min=0)[:, None, :, None].double()).float()
        ga = torch.exp(lg * (i[:n][None] + 1)[:, None, :, None].double()).float()
        qm, dm = torch.where(inside, q[:, :, t0:t0 + n], 0.0), torch.where(inside, do[:, :, t0:t0 + n], 0.0)
        kc, vc = k[:, :, t0:t0 + n], v[:, :, t0:t0 + n]
        m = mask[:, :, :n, :n]
        dk[:, :, t0:t0 + n] = torch.matmul(torch.matmul(vc, dm.transpose(-1, -2)) * m, qm) \
            + torch.matmul(vc, s.transpose(-1, -2)) * gb
        dv[:, :, t0:t0 + n] = torch.matmul(torch.matmul(kc, qm.transpose(-1, -2)) * m, dm) + torch.matmul(kc, s) * gb
        s = s * torch.exp(lg * valid[:, None, None, None].double()).float() + torch.matmul((qm * ga).transpose(-1, -2), dm)
    return dk, dv, s


# ------------------------------------------------------------------------------------------------ one pass
def _own(st):
    lp, c = _lp(), st["case"]
    op = c["op"]
    stream = torch.cuda.current_stream().cuda_stream
    dt = lp.LP_BF16 if c.get("dtype", "bf16") == "bf16" else lp.LP_FP32
    if op == "embed_fwd":
        lp.lp_embed_forward(dt, st["ids"], st["table"], st["pos"], st["out"], c["rows"], c["vocab"], c["d"], c["T"],
                            c["scale"], None, stream)
        return st["out"]
    if op == "embed_bwd":
        lp.lp_embed_backward(dt, st["ids"], st["dout"], st["dtable"], st["dpos"], c["rows"], c["vocab"], c["d"], c["T"],
                             c["scale"], None, st["ws"], st["ws"].numel(), stream)
        return [st["dtable"], st["dpos"]] if c["T"] else [st["dtable"]]
    if op == "dropout":
        lp.lp_dropout(dt, st["x"], st["resid"], st["y"], c["n"], c["p"], st["key"], c["offset"], None, stream)
        return st["y"]
    desc = dict(q=st["q"], k=st["k"], v=st["v"], log_decay=st["g"], scale=st["scale"], state_in=st["s_in"],
                lengths=st["lengths"])
    if op == "la_bwd":
        desc.update(dout=st["do"], dq=st["dq"], dk=st["dk"], dv=st["dv"], dstate_out=st["ds_out"], dstate_in=st["ds_in"])
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, desc, st["ws"], stream)
        out = [st["dq"], st["dk"], st["dv"]]
        return out + [st["ds_in"]] if st["ds_in"] is not None else out
    desc.update(o=st["o"], state_out=st["s_out"])
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_STEP if op == "la_step" else lp.LP_LINATTN_FORWARD, desc, st["ws"], stream)
    return [st["o"], st["s_out"]] if st["s_out"] is not None else [st["o"]]


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "embed_fwd":
        return _plain_embed_fwd(state)
    if op == "embed_bwd":
        return _plain_embed_bwd(state)
    if op == "dropout":
        return _plain_dropout(state)
    return _plain_linattn(state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    es = 2 if case.get("dtype", "bf16") == "bf16" else 4
    if op == "embed_fwd":   # the rows gathered (a distinct row once), the positions, the rows written
        rows, d = case["rows"], case["d"]
        return dict(bytes=rows * 4 + (min(rows, case["vocab"]) + case["T"] + rows) * d * es, flops=2 * rows * d)
    if op == "embed_bwd":   # the incoming gradient, and the whole table's gradient written
        rows, d = case["rows"], case["d"]
        return dict(bytes=rows * 4 + rows * d * es + (case["vocab"] + case["T"]) * d * 4,
                    flops=rows * d * (2 if case["T"] else 1))
    if op == "dropout":
        return dict(bytes=case["n"] * es * (3 if case["resid"] else 2), flops=2 * case["n"])
    B, H, T = case["batch"], case["heads"], case.get("seq", 1)
    tok, states = B * T * H, B * H * D * D * 4
    if op == "la_step":
        return dict(bytes=tok * D * 2 * 4 + 2 * states, flops=tok * 4 * D * D)
    # the recurrence itself: the state's update and one product with it (forward); three products and two states (backward)
    if op == "la_fwd":
        return dict(bytes=tok * D * 2 * 4 + (2 * states if case["state"] else 0), flops=tok * 4 * D * D)
    return dict(bytes=tok * D * 2 * 7 + (3 * states if case["state"] else 0), flops=tok * 10 * D * D)


# ------------------------------------------------------------------------------------------------ 64-bit values
def _np_keep(n, key, offset, p):
    c = np.arange((n + 3) // 4, dtype=np.uint64) + np.uint64(offset)
    m32 = np.uint64(_M32)
    w = [c & m32, c >> np.uint64(32), np.zeros_like(c), np.zeros_like(c)]
    for r in range(10):
        k0 = np.uint64((key + r * 0x9E3779B9) & _M32)
        k1 = np.uint64(((key >> 32) + r * 0xBB67AE85) & _M32)
        a, b = w[0] * np.uint64(0xD2511F53), w[2] * np.uint64(0xCD9E8D57)
        w = [(b >> np.uint64(32)) ^ w[1] ^ k0, b & m32, (a >> np.uint64(32)) ^ w[3] ^ k1, a & m32]
    return np.stack(w, 1).reshape(-1)[:n] >= np.uint64(int(p * 4294967296.0))


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "embed_fwd":
        h = torch.nn.functional.embedding(st["ids"].long(), st["table"]).double() * case["scale"]
        if case["T"]:
            reps = -(-case["rows"] // case["T"])
            h += st["pos"].double().repeat(reps, 1)[:case["rows"]]
        return h
    if op == "embed_bwd":
        # sort, then sum every run of equal tokens as a difference-free segment reduction in 64 bits
        tok, order = torch.sort(st["ids"].long(), stable=True)
        seg = torch.bincount(tok, minlength=case["vocab"])
        dh = st["dout"].double()
        out = [torch.segment_reduce(dh[order], "sum", lengths=seg, axis=0, initial=0.0) * case["scale"]]
        if case["T"]:
            T = case["T"]
            pad = torch.zeros(-(-case["rows"] // T) * T, case["d"], dtype=torch.float64, device=DEV)
            pad[:case["rows"]] = dh
            out.append(pad.view(-1, T, case["d"]).sum(0))
        return out
    if op == "dropout":
        keep = torch.from_numpy(_np_keep(case["n"], st["key"], case["offset"], case["p"])).to(DEV)
        y = st["x"].double() / (1.0 - case["p"])
        y[~keep] = 0.0
        return y + st["resid"].double() if case["resid"] else y
    B, H, T = case["batch"], case["heads"], case.get("seq", 1)
    if B * H * T * T > 3e10:
        return None
    lens = st["lengths"].tolist() if st["lengths"] is not None else [T] * B
    back = op == "la_bwd"
    outs = [st[n].double().clone() for n in (("dq", "dk", "dv") if back else ("o",))]
    state = (st["ds_in"] if back else st["s_out"])
    state = state.double().clone() if state is not None else None
    R = 1024                                          # the T x T weights, some rows of them at a time
    for b in range(B):
        n = lens[b]
        if n == 0:
            if state is not None:
                state[b] = (st["ds_out"] if back else st["s_in"])[b].double()
            continue
        q, k, v = (st[x][b, :n].double().transpose(0, 1) for x in "qkv")         # [H, n, 64]
        lg = st["g"].double()[:, None, None]
        t = torch.arange(n, device=DEV, dtype=torch.float64)
        s_in = st["s_in"][b].double() if st["s_in"] is not None else None
        since = torch.exp(lg * (t + 1)[None, :, None])                           # decay from the incoming state
        until = torch.exp(lg * (n - 1 - t)[None, :, None])                       # decay to the outgoing state
        sc = st["scale"]
        if back:
            do = st["do"][b, :n].double().transpose(0, 1)
            dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
        else:
            o = torch.zeros_like(q)
        for r0 in range(0, n, R):
            r1 = min(n, r0 + R)
            age = t[r0:r1, None] - t[None, :r1]
            w = torch.where(age >= 0, torch.exp(lg * age.clamp(min=0)), 0.0) * sc  # [H, rows, columns]
            p = (q[:, r0:r1] @ k[:, :r1].transpose(1, 2)) * w
            if not back:
                o[:, r0:r1] = p @ v[:, :r1]
            else:
                dv[:, :r1] += p.transpose(1, 2) @ do[:, r0:r1]
                dp = (do[:, r0:r1] @ v[:, :r1].transpose(1, 2)) * w
                dq[:, r0:r1] = dp @ k[:, :r1]
                dk[:, :r1] += dp.transpose(1, 2) @ q[:, r0:r1]
        if not back:
            if s_in is not None:
                o += sc * since * (q @ s_in)
            if state is not None:
                state[b] = torch.exp(lg * n) * s_in + (k * until).transpose(1, 2) @ v
            outs[0][b, :n] = o.transpose(0, 1)
        else:
            if s_in is not None:
                dq += sc * since * (do @ s_in.transpose(1, 2))
            if state is not None:
                ds = st["ds_out"][b].double()
                dk += until * (v @ ds.transpose(1, 2))
                dv += until * (k @ ds)
                state[b] = torch.exp(lg * n) * ds + sc * (q * since).transpose(1, 2) @ do
            for buf, y in zip(outs, (dq, dk, dv)):
                buf[b, :n] = y.transpose(0, 1)
    return outs + [state] if state is not None else outs

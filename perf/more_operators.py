"""Workloads of the operators that read a model's logits: log probabilities of given tokens with entropy and top
alternatives, their gradient, and distillation from a teacher's top logits.

``own`` selects the path: False runs each operator as elementary torch operations in 32 bits, True calls the
library.  ``listed()`` names the fixed cases, ``draw(rng)`` makes further ones over the same ranges.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
SMALLEST_REST = 2.0 ** -20    # a teacher's rest below this is rounding of its listed probabilities, and counts as none


def _lp():
    from paper_2012_03837_b200 import binding
    return binding


# ------------------------------------------------------------------------------------------------ cases
# op "logprobs": want = which of l(og probability), e(ntropy), s (log-sum-exp); top = how many alternatives
# op "logprobs_bwd": want = which of them carry a gradient
# op "distill": top = teacher's entries per row, rest = the teacher's remaining mass counts, grad = dlogits wanted
# pad: elements between the end of a row and the start of the next; masked: share of the vocabulary at -infinity
def listed():
    return [
        # one sequence answering: the alternatives of its next token
        dict(name="logprobs_one_row", op="logprobs", dtype="bf16", rows=1, vocab=32768, top=8, want="le", temp=1.0, pad=0, masked=0.0),
        # 64 sequences answering with the 8-block transformer's vocabulary in fp32
        dict(name="logprobs_slots", op="logprobs", dtype="fp32", rows=64, vocab=8192, top=20, want="les", temp=0.75, pad=0, masked=0.0),
        # scoring a minibatch of the 24-block transformer (16 x 512 tokens): log probabilities alone
        dict(name="logprobs_score", op="logprobs", dtype="bf16", rows=8192, vocab=32768, top=0, want="l", temp=1.0, pad=0, masked=0.0),
        # the same minibatch read by a teacher, which hands on its 64 best at temperature 2
        dict(name="logprobs_teacher", op="logprobs", dtype="bf16", rows=8192, vocab=32768, top=64, want="les", temp=2.0, pad=0, masked=0.0),
        # an odd vocabulary in padded rows, fp32
        dict(name="logprobs_odd_fp32", op="logprobs", dtype="fp32", rows=1031, vocab=50021, top=5, want="le", temp=1.0, pad=27, masked=0.0),
        # a large odd vocabulary of which a grammar allows a tenth
        dict(name="logprobs_masked_large", op="logprobs", dtype="bf16", rows=300, vocab=151001, top=16, want="les", temp=1.0, pad=0,
             masked=0.9),
        # training by rewards with an entropy bonus, the 24-block transformer's minibatch
        dict(name="logprobs_bwd_policy", op="logprobs_bwd", dtype="bf16", rows=8192, vocab=32768, want="le", temp=1.0, pad=0, masked=0.0),
        # a small minibatch of the 8-block transformer in fp32, log probabilities alone
        dict(name="logprobs_bwd_small", op="logprobs_bwd", dtype="fp32", rows=256, vocab=8192, want="l", temp=1.0, pad=0, masked=0.0),
        # a student's loss on held-out rows
        dict(name="distill_loss", op="distill", dtype="bf16", rows=2048, vocab=32768, top=32, rest=True, grad=False, temp=1.0, pad=0,
             masked=0.0),
        # the 24-block transformer's minibatch taught from 64 entries a row: loss and gradient
        dict(name="distill_train", op="distill", dtype="bf16", rows=8192, vocab=32768, top=64, rest=False, grad=True, temp=2.0, pad=0,
             masked=0.0),
        # a large odd vocabulary taught with the teacher's remaining mass, many entries
        dict(name="distill_train_rest_large", op="distill", dtype="bf16", rows=1000, vocab=131071, top=128, rest=True, grad=True,
             temp=1.0, pad=1, masked=0.0),
        # a few rows in fp32: latency
        dict(name="distill_few", op="distill", dtype="fp32", rows=16, vocab=8192, top=8, rest=True, grad=True, temp=1.0, pad=0,
             masked=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "logprobs_bwd", "distill", "distill"])
    dtype = rng.choice(["bf16", "fp32"])
    vocab = rng.choice([_log(rng, 300, 160000), 64 * _log(rng, 5, 2500)])
    rows = min(_log(rng, 1, 16384), (1 << 28 if dtype == "bf16" else 1 << 27) // (vocab + 64))
    case = dict(op=op, dtype=dtype, rows=max(1, rows), vocab=vocab, temp=rng.choice([1.0, 1.0, 0.75, 2.0, rng.randint(8, 96) / 32]),
                pad=rng.choice([0, 0, rng.randint(1, 63)]), masked=rng.choice([0.0, 0.0, 0.5]))
    if op == "logprobs":
        case.update(top=rng.choice([0, 1, _log(rng, 1, 128)]), want=rng.choice(["l", "le", "les", "e", "s"]))
    elif op == "logprobs_bwd":
        case.update(want=rng.choice(["l", "le", "les", "e"]))
    else:
        case.update(top=_log(rng, 1, 128), rest=rng.random() < 0.5, grad=rng.random() < 0.75)
    return case


# ------------------------------------------------------------------------------------------------ inputs
def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _blocks(rows, vocab):
    """Pieces of the rows of about 2^25 logits."""
    step = max(1, (1 << 25) // vocab)
    return [slice(r, min(rows, r + step)) for r in range(0, rows, step)]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rows, vocab, dt = case["rows"], case["vocab"], _dt(case)
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV)
    ru = lambda *s: torch.rand(*s, generator=g, device=DEV)
    st = dict(case=case)
    strided = lambda fill: torch.full((rows, vocab + case["pad"]), fill, dtype=dt, device=DEV)[:, :vocab]
    x = st["logits"] = strided(float("nan"))              # what lies between the rows is not to be read
    teaching = case["op"] == "distill"
    if teaching:
        k = case["top"]
        st["ids"], st["teacher"] = torch.empty(rows, k, dtype=torch.int32, device=DEV), torch.empty(rows, k, device=DEV)
    else:
        st["tokens"] = torch.empty(rows, dtype=torch.int32, device=DEV)
    common = 2.0 * rn(vocab)                              # some tokens are likelier than others everywhere
    for b in _blocks(rows, vocab):
        n = b.stop - b.start
        z = common + 2.0 * rn(n, vocab)
        z[torch.arange(n, device=DEV), torch.randint(0, vocab, (n,), generator=g, device=DEV)] += 8.0 * ru(n)
        if case["masked"]:
            z.masked_fill_(ru(n, vocab) < case["masked"], -math.inf)
        x[b] = z.to(dt)
        if teaching:                                      # a teacher that mostly agrees
            t = (z + 0.7 * rn(n, vocab)) / case["temp"]
            lse = torch.logsumexp(t, 1, keepdim=True)
            v, i = torch.topk(t, k, dim=1)
            st["ids"][b], st["teacher"][b] = i.to(torch.int32), v - lse if case["rest"] else v * case["temp"]
        else:                                             # a token drawn from the model itself
            noise = -torch.log(-torch.log(ru(n, vocab).clamp_(1e-7, 1 - 1e-7)))
            st["tokens"][b] = (x[b].float() / case["temp"] + noise).argmax(1).to(torch.int32)
    absent = ru(rows) < 0.05                              # padding behind the ends of sequences
    f32 = lambda *s: torch.zeros(*s, device=DEV)
    if case["op"] == "logprobs":
        st["tokens"][absent] = -1
        st["out"] = {n: f32(rows) for n, c in (("logp", "l"), ("entropy", "e"), ("lse", "s")) if c in case["want"]}
        if case["top"]:
            st["out"].update(top_ids=torch.zeros(rows, case["top"], dtype=torch.int32, device=DEV), top_logp=f32(rows, case["top"]))
    elif case["op"] == "logprobs_bwd":
        st["tokens"][absent] = -1
        st["grads"] = {n: rn(rows) * s / rows for n, c, s in (("dlogp", "l", 1.0), ("dentropy", "e", 0.01), ("dlse", "s", 0.01))
                       if c in case["want"]}
        for t in st["grads"].values():
            t[absent] = 0.0
        st["dlogits"] = strided(0.0)
    else:
        st["ids"][ru(rows, k) < 0.02] = -1                # entries that are not there
        st["dloss"] = torch.where(absent, 0.0, (0.5 + ru(rows)) / rows)
        st["loss"] = f32(rows)
        st["dlogits"] = strided(0.0) if case["grad"] else None
    return st


# ------------------------------------------------------------------------------------------------ plain forms
def _softmax_parts(z):
    """log p and p of z / 1 in 32 bits; p = 0 where z is -infinity."""
    m = z.max(1, keepdim=True).values
    d = z - m
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    return d, e, s, m


def _plain_logprobs(st):
    c = st["case"]
    d, e, s, m = _softmax_parts(st["logits"].float() * (1.0 / c["temp"]))
    logs = torch.log(s)
    out = []
    if "l" in c["want"]:
        tok = st["tokens"].long()
        lp = torch.gather(d, 1, tok.clamp(min=0)[:, None])[:, 0] - logs[:, 0]
        out.append(torch.where(tok >= 0, lp, 0.0))
    if "e" in c["want"]:
        out.append(logs[:, 0] - (torch.where(e > 0, e * d, 0.0).sum(1) / s[:, 0]))
    if "s" in c["want"]:
        out.append((m + logs)[:, 0])
    if c["top"]:
        # equal logits go by index: one whole number from the logit's order and the place
        bits = st["logits"].float().contiguous().view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 18) - torch.arange(c["vocab"], device=DEV)
        ids = torch.topk(key, c["top"], dim=1).indices
        out += [ids.to(torch.int32), torch.gather(d, 1, ids) - logs]
    return out


def _plain_logprobs_bwd(st):
    c, g = st["case"], st["grads"]
    tok = st["tokens"].long()
    d, e, s, _ = _softmax_parts(st["logits"].float() * (1.0 / c["temp"]))
    p = e / s
    lp = d - torch.log(s)
    coef = torch.zeros(c["rows"], 1, device=DEV)
    if "l" in c["want"]:
        coef = coef - torch.where(tok >= 0, g["dlogp"], 0.0)[:, None]
    if "s" in c["want"]:
        coef = coef + g["dlse"][:, None]
    dz = p * coef
    if "e" in c["want"]:
        plp = torch.where(p > 0, p * lp, 0.0)
        dz = dz - g["dentropy"][:, None] * (plp - p * plp.sum(1, keepdim=True))
    if "l" in c["want"]:
        dz.scatter_add_(1, tok.clamp(min=0)[:, None], torch.where(tok >= 0, g["dlogp"], 0.0)[:, None])
    return [(dz * (1.0 / c["temp"])).to(_dt(c))]


def _plain_distill(st):
    c, T = st["case"], st["case"]["temp"]
    ids, there = st["ids"].long().clamp(min=0), st["ids"] >= 0
    z = st["logits"].float() * (1.0 / T)
    m = z.max(1, keepdim=True).values
    e = torch.exp(z - m)
    t = torch.where(there, st["teacher"].double(), -math.inf)
    if c["rest"]:
        q = torch.exp(t)
        qr = 1.0 - q.sum(1, keepdim=True)
        qr = torch.where(qr > SMALLEST_REST, qr, 0.0)
    else:
        q = torch.exp((t - t.max(1, keepdim=True).values.clamp(min=-1e300)) / T)
        q = q / q.sum(1, keepdim=True).clamp(min=1e-300)
        qr = torch.zeros(c["rows"], 1, device=DEV, dtype=torch.float64)
    q, qr = torch.where((q > 0).any(1, keepdim=True), q, 0.0), torch.where((q > 0).any(1, keepdim=True), qr, 0.0)
    Q = q.sum(1, keepdim=True) + qr
    elsewhere = torch.where(there, ids, c["vocab"])
    listed_ = torch.zeros(c["rows"], c["vocab"] + 1, dtype=torch.bool, device=DEV).scatter_(1, elsewhere, True)[:, :-1]
    er = torch.where(listed_, 0.0, e)
    sr = er.sum(1, keepdim=True)
    s = sr + torch.where(listed_, e, 0.0).sum(1, keepdim=True)
    lp = torch.gather(z, 1, ids) - m - torch.log(s)
    loss = torch.where(q > 0, q * (torch.log(q.clamp(min=1e-300)) - lp.double()), 0.0).sum(1)
    loss = loss + torch.where(qr > 0, qr * (torch.log(qr.clamp(min=1e-300)) - torch.log(sr / s).double()), 0.0)[:, 0]
    scale = T * T
    out = [(scale * loss).float()]
    if c["grad"]:
        w = st["dloss"][:, None] * (scale / T)
        dz = e * (Q.float() / s) - er * torch.where(qr > 0, qr.float() / sr, 0.0)
        dz.scatter_add_(1, ids, -torch.where(there, q.float(), 0.0))
        out.append((dz * w).to(_dt(c)))
    return out


# ------------------------------------------------------------------------------------------------ one pass
def _own(st):
    lp, c = _lp(), st["case"]
    stream = torch.cuda.current_stream().cuda_stream
    if c["op"] == "logprobs":
        o = st["out"]
        lp.lp_token_logprobs(st["logits"], st["tokens"] if "l" in c["want"] else None, temperature=c["temp"], stream=stream, **o)
        return list(o.values())
    if c["op"] == "logprobs_bwd":
        lp.lp_token_logprobs_backward(st["logits"], st["tokens"] if "l" in c["want"] else None, dlogits=st["dlogits"],
                                      temperature=c["temp"], stream=stream, **st["grads"])
        return [st["dlogits"]]
    lp.lp_distill(lp.LP_DISTILL_REST if c["rest"] else lp.LP_DISTILL_TOP, st["logits"], st["ids"], st["teacher"], loss=st["loss"],
                  dloss=st["dloss"] if c["grad"] else None, dlogits=st["dlogits"], temperature=c["temp"], scale=c["temp"] * c["temp"],
                  stream=stream)
    return [st["loss"], st["dlogits"]] if c["grad"] else [st["loss"]]


def run(state):
    if own:
        return _own(state)
    return {"logprobs": _plain_logprobs, "logprobs_bwd": _plain_logprobs_bwd, "distill": _plain_distill}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    rows, n, es = case["rows"], case["rows"] * case["vocab"], 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "logprobs":      # the logits once; per logit a difference, an exponential, a sum and, for the entropy, two more
        outs = len(case["want"]) + ("l" in case["want"]) + 2 * case["top"]
        return dict(bytes=n * es + rows * 4 * outs, flops=n * (5 if "e" in case["want"] else 3))
    if case["op"] == "logprobs_bwd":
        return dict(bytes=2 * n * es + rows * 4 * (len(case["want"]) + ("l" in case["want"])), flops=n * (9 if "e" in case["want"] else 6))
    return dict(bytes=(2 if case["grad"] else 1) * n * es + rows * 4 * (2 * case["top"] + 1 + case["grad"]),
                flops=n * (6 if case["grad"] else 3))


# ------------------------------------------------------------------------------------------------ 64-bit values
def exact(case, seed):
    st = prepare(case, seed)
    rows, vocab, T = case["rows"], case["vocab"], case["temp"]
    parts = []
    for b in _blocks(rows, 4 * vocab):
        x = st["logits"][b].double() / T
        lse = torch.logsumexp(x, dim=1)
        logp = x - lse[:, None]
        p = logp.exp()
        rr = torch.arange(x.shape[0], device=DEV)
        out = []
        if case["op"] != "distill":
            tok = st["tokens"][b].long()
            has = tok >= 0
            ent = -torch.special.xlogy(p, p).sum(1)
        if case["op"] == "logprobs":
            if "l" in case["want"]:
                v = torch.zeros_like(lse)
                v[has] = logp[rr[has], tok[has]]
                out.append(v)
            if "e" in case["want"]:
                out.append(ent)
            if "s" in case["want"]:
                out.append(lse)
            if case["top"]:
                order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
                out += [order.to(torch.int32), logp.gather(1, order)]
        elif case["op"] == "logprobs_bwd":
            dz = torch.zeros_like(p)
            g = {n: t[b].double() for n, t in st["grads"].items()}
            if "dlogp" in g:
                a = g["dlogp"] * has
                dz -= a[:, None] * p
                dz[rr[has], tok[has]] += a[has]
            if "dentropy" in g:
                dz -= g["dentropy"][:, None] * (torch.special.xlogy(p, p) + p * ent[:, None])
            if "dlse" in g:
                dz += g["dlse"][:, None] * p
            out.append(dz / T)
        else:
            # the teacher's distribution laid out over the whole vocabulary
            ids, t = st["ids"][b].long(), st["teacher"][b].double()
            q = torch.zeros_like(p)
            inside = torch.zeros_like(p, dtype=torch.bool)
            for j in range(case["top"]):
                ok = ids[:, j] >= 0
                inside[rr[ok], ids[ok, j]] = True
                q[rr[ok], ids[ok, j]] = (t[ok, j] if case["rest"] else t[ok, j] / T)
            q = torch.where(inside, q, -math.inf)
            q = q.exp() if case["rest"] else torch.softmax(q, 1).nan_to_num(0.0)
            mass = q.sum(1)
            rest = torch.where((1.0 - mass > SMALLEST_REST) & (mass > 0), 1.0 - mass, 0.0) if case["rest"] else torch.zeros_like(mass)
            out_p = torch.where(inside, -math.inf, x)
            log_out = torch.logsumexp(out_p, 1) - lse
            kl = torch.where(q > 0, torch.special.xlogy(q, q) - q * logp, 0.0).sum(1)
            kl = kl + torch.where(rest > 0, torch.special.xlogy(rest, rest) - rest * log_out, 0.0)
            out.append(T * T * kl)
            if case["grad"]:
                dz = p * (mass + rest)[:, None] - q
                share = torch.where(inside, 0.0, (logp - log_out[:, None]).exp()).nan_to_num(0.0)
                dz -= rest[:, None] * share
                out.append(dz * (st["dloss"][b].double() * T)[:, None])
        parts.append(out)
    return [torch.cat(o) for o in zip(*parts)]

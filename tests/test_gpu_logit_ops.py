"""Log probabilities of tokens with entropy and top alternatives, their gradient, and distillation from a teacher's top
logits on the GPU against their plain 64-bit forms (oracle/lm_ops.py), at the sizes, strides and masks where they can go wrong.

Tolerances.  u = 2^-24 is the largest relative error of a rounding to fp32 (2^-8 to bf16).  With y = (x - max) / T every
exponential is off by at most 3 u |y| (difference, factor, product) + 2^-21 (the function) of itself; in a row's sum no term
passes more than vocab / 256 + 64 additions.  What follows from these is written out in `errors`."""
import numpy as np
import pytest
import torch

from oracle import lm_ops as O
from paper_2012_03837_b200 import binding as lp

pytestmark = pytest.mark.gpu
DT = {"fp32": (torch.float32, 2.0 ** -24), "bf16": (torch.bfloat16, 2.0 ** -8)}
U, EXP, TINY = 2.0 ** -24, 2.0 ** -21, 2.0 ** -120
INF = float("inf")


def np64(t):
    return t.double().cpu().numpy()


def cu(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def matrix(rows, vocab, dtype, pad=0, off=0, fill=float("nan")):
    """[rows, vocab] with `pad` elements between rows, `off` elements behind an aligned address."""
    ld = vocab + pad
    return torch.full((rows * ld + off,), fill, dtype=dtype, device="cuda")[off:].view(rows, ld)[:, :vocab]


def between(t):
    """What lies in t's storage outside its rows."""
    whole = torch.ones(t.untyped_storage().nbytes() // t.element_size(), dtype=torch.bool, device="cuda")
    whole.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(False)
    return torch.empty(0, dtype=t.dtype, device="cuda").set_(t.untyped_storage())[whole]


def values(g, rows, vocab, kind):
    x = 3.0 * g.standard_normal((rows, vocab))
    if kind == "masked":
        x[g.random(x.shape) < 0.9] = -np.inf
        x[0] = -np.inf                                       # a row without any token
        if rows > 1:
            x[1] = -np.inf
            x[1, vocab // 2] = 1.5                           # and one with a single token
    elif kind == "lowmask":                                  # masked by the type's lowest value
        x[g.random(x.shape) < 0.9] = -3.3895314e38
    elif kind == "peaked":
        x[np.arange(rows), g.integers(0, vocab, rows)] += 60.0
    elif kind == "ties":
        x = g.integers(-2, 3, x.shape).astype(np.float64)
        x[x == 0] *= np.where(g.random((x == 0).sum()) < 0.5, -1.0, 1.0)     # -0 and 0 are equal
    elif kind == "constant":
        x[:] = 0.25
    elif kind == "lowest":
        x[:] = -3.0e38
        x[:, ::3] = -np.inf
        x[-1] = np.where(np.arange(vocab) % 2, -3.3e38, -3.0e38)
    elif kind == "highest":
        x = 1e37 * g.standard_normal(x.shape)
        x[:, ::5] = -np.inf
    elif kind == "far":
        x += 2e4
    elif kind == "descending":
        x = np.sort(x, axis=1)[:, ::-1]
    elif kind == "ascending":
        x = np.sort(x, axis=1)
    return x


def put(x, dtype, pad=0, off=0):
    t = matrix(*x.shape, dtype, pad, off)
    with np.errstate(over="ignore"):
        t.copy_(cu(x.astype(np.float32)).to(dtype))
    return t


def errors(x, T, n):
    """Per row: parts of the distribution in 64 bits and how far fp32 may be off in log S, lse and the entropy."""
    with np.errstate(all="ignore"):
        m = x.max(1, keepdims=True)
        m = np.where(np.isfinite(m), m, 0.0)
        y = (x - m) / T
        e = np.exp(y)
        S = e.sum(1, keepdims=True)
        logs = np.where(S > 0, np.log(S), 0.0)
        l = np.where(S > 0, y - logs, -np.inf)
        p = np.exp(l)
        ay = np.where(p > 0, -y, 0.0)
        py, pyy = (p * ay).sum(1, keepdims=True), (p * ay * ay).sum(1, keepdims=True)
        d = (n / 256 + 64) * U + EXP
        e_logs = d + 3 * U * py + 2 * U * np.abs(logs)
        H = -np.where(p > 0, p * l, 0.0).sum(1, keepdims=True)
        e_h = e_logs + (2 * d + 8 * U) * py + 3 * U * (pyy + py * py) + 2 * U * H
        e_lse = e_logs + 2 * U * np.abs(m / T) + U * np.abs(m / T + logs)
        # of a log probability, which is finite where the probability itself may be too small for any type
        e_l = np.where(np.isfinite(l), e_logs + 3 * U * np.abs(y) + U * np.abs(l), 0.0)
        rel = np.where(p > 0, e_logs + 3 * U * ay + EXP + 4 * U, 0.0)         # of a probability
    return dict(p=p, l=l, H=H, e_logs=e_logs, e_h=e_h, e_lse=e_lse, e_l=e_l, rel=rel)


def close(got, want, tol, what=""):
    """Equal where not finite (values beyond fp32's range are infinite: -3e38 / 0.75), within tol elsewhere."""
    got, want, tol = np.broadcast_arrays(got, want, tol)
    with np.errstate(over="ignore", invalid="ignore"):
        want = np.where(np.isinf(want.astype(np.float32)), np.sign(want) * INF, want)
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True), what
    bad = ~(np.abs(got[fin] - want[fin]) <= tol[fin])
    assert not bad.any(), (what, got[fin][bad][:5], want[fin][bad][:5], tol[fin][bad][:5])


SIZES = [  # rows, vocab, pad, offset, top_k
    (1, 1, 0, 0, 1), (3, 2, 0, 1, 2), (5, 7, 2, 0, 7), (2, 31, 1, 3, 20), (9, 64, 0, 0, 64), (700, 33, 0, 0, 3), (4, 255, 0, 1, 128), (3, 1000, 24, 0, 1),
    (160, 515, 5, 7, 9), (2, 2049, 0, 0, 128), (1, 8192, 0, 0, 64), (6, 8200, 3, 5, 30), (300, 4096, 0, 0, 5), (2, 32768, 0, 0, 128),
    (3, 50021, 6, 1, 17), (330, 32771, 1, 0, 2), (1, 131071, 0, 1, 100), (2, 150001, 7, 2, 128), (1, 262144, 0, 0, 50), (149, 100003, 0, 0, 4),
]
KINDS = ["normal", "masked", "lowmask", "peaked", "ties", "constant", "lowest", "highest", "far", "descending", "ascending"]
# every size with plain values, every kind of values at three sizes
CASES = [(*s, "normal") for s in SIZES] + [(*s, k) for s in [(3, 700, 1, 1, 40), (4, 20011, 0, 0, 128), (2, 200000, 0, 3, 33)] for k in KINDS[1:]]


def make(rows, vocab, pad, off, kind, dt, seed=0):
    g = np.random.default_rng(rows * 7 + vocab + seed)
    t = put(values(g, rows, vocab, kind), DT[dt][0], pad, off)
    return g, t, np64(t)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,off,k,kind", CASES)
def test_log_probabilities(rows, vocab, pad, off, k, kind, dt):
    g, t, x = make(rows, vocab, pad, off, kind, dt)
    T = float(np.float32(g.choice([1.0, 0.75, 2.0])))
    tok = g.integers(0, vocab, rows).astype(np.int32)
    tok[::7] = -1
    tok[1::11] = vocab + 3
    tok[:1] = x[0].argmax()
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    f = lambda *s: torch.full(s, 7.0, device="cuda")
    o = dict(logp=f(rows), entropy=f(rows), lse=f(rows), top_ids=torch.full((rows, k), -9, dtype=torch.int32, device="cuda"), top_logp=f(rows, k))
    lp.lp_token_logprobs(t, cu(tok, torch.int32), temperature=T, out_of_range=flag, **o)
    # the oracle in full for a few rows, the same expressions in one go for all
    some = list(range(min(rows, 2))) + [rows - 1]
    logp, ent, lse, ids, tops = O.token_logprobs(x[some], tok[some], T, k)
    E = errors(x, T, vocab)
    close(np64(o["logp"])[some], logp, np.array([E["e_l"][r, tok[r]] if 0 <= tok[r] < vocab else 0.0 for r in some]), "logp")
    close(np64(o["entropy"])[some], ent, E["e_h"][some, 0], "entropy")
    close(np64(o["lse"])[some], lse, E["e_lse"][some, 0], "lse")
    assert np.array_equal(o["top_ids"].cpu().numpy()[some], ids)
    close(np64(o["top_logp"])[some], tops, np.take_along_axis(E["e_l"][some], ids, 1), "top_logp")
    assert flag.item() == int((tok >= vocab).any())
    ok = (tok >= 0) & (tok < vocab)
    at = np.where(ok, tok, 0)[:, None]
    close(np64(o["logp"]), np.where(ok, np.take_along_axis(E["l"], at, 1)[:, 0], 0.0), np.take_along_axis(E["e_l"], at, 1)[:, 0], "logp of all rows")
    close(np64(o["entropy"]), E["H"][:, 0], E["e_h"][:, 0], "entropy of all rows")
    order = np.argsort(-x, axis=1, kind="stable")[:, :k]
    assert np.array_equal(o["top_ids"].cpu().numpy(), order)
    close(np64(o["top_logp"]), np.take_along_axis(E["l"], order, 1), np.take_along_axis(E["e_l"], order, 1), "top_logp of all rows")
    # again, and each output alone, the same bits; a row is cut otherwise where alternatives are asked for, and its sums round otherwise
    t_tok = cu(tok, torch.int32)
    again = {n: torch.zeros_like(v) for n, v in o.items()}
    lp.lp_token_logprobs(t, t_tok, temperature=T, **again)
    assert all(torch.equal(v, o[n]) for n, v in again.items())
    tops = {n: torch.zeros_like(v) for n, v in o.items() if n.startswith("top")}
    lp.lp_token_logprobs(t, temperature=T, **tops)
    assert all(torch.equal(v, o[n]) for n, v in tops.items())
    rest = {n: torch.zeros_like(v) for n, v in o.items() if n not in tops}
    lp.lp_token_logprobs(t, t_tok, temperature=T, **rest)
    close(np64(rest["lse"])[some], lse, E["e_lse"][some, 0], "lse without alternatives")
    close(np64(rest["entropy"])[some], ent, E["e_h"][some, 0], "entropy without alternatives")
    for name, v in rest.items():
        alone = {name: torch.zeros_like(v)}
        lp.lp_token_logprobs(t, t_tok if name == "logp" else None, temperature=T, **alone)
        assert torch.equal(alone[name], v), name


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,off,k,kind", CASES)
def test_gradient_of_log_probabilities(rows, vocab, pad, off, k, kind, dt):
    g, t, x = make(rows, vocab, pad, off, kind, dt, 1)
    td, us = DT[dt]
    T = float(np.float32(g.choice([1.0, 0.75, 2.0])))
    tok = g.integers(0, vocab, rows).astype(np.int32)
    tok[::5] = -1
    tok[1::6] = vocab
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    E = errors(x, T, vocab)
    has = (tok >= 0) & (tok < vocab)
    for which in ("a", "b", "abc", "c"):
        a, b, c = (np.float32(g.standard_normal(rows)) if n in which else None for n in "abc")
        for v in (a, b, c):
            if v is not None:
                v[::4] = 0.0
        dev = {n: cu(v) for n, v in (("dlogp", a), ("dentropy", b), ("dlse", c)) if v is not None}
        # a gradient of its own layout; then in the logits' place
        dx = matrix(rows, vocab, td, 3 if which == "b" else pad, off, 5.0)
        lp.lp_token_logprobs_backward(t, cu(tok, torch.int32) if a is not None else None, dlogits=dx, temperature=T, out_of_range=flag, **dev)
        assert flag.item() == int(a is not None and (tok >= vocab).any())
        flag.zero_()
        some = list(range(min(rows, 6))) + [rows - 1]
        want = O.token_logprobs_bwd(x[some], tok[some], *(v[some].astype(np.float64) if v is not None else None for v in (a, b, c)), T)
        a0 = np.where(has, a, 0.0)[:, None] if a is not None else np.zeros((rows, 1))
        b0, c0 = ((v[:, None] if v is not None else np.zeros((rows, 1))) for v in (b, c))
        with np.errstate(all="ignore"):
            lz = np.where(E["p"] > 0, E["l"], 0.0)
            k0 = np.abs(c0) + np.abs(a0) + np.abs(b0) * E["H"]
            tol = E["p"] * (E["rel"] * (k0 + np.abs(b0 * lz)) + np.abs(b0) * (np.where(E["p"] > 0, E["e_l"], 0.0) + E["e_h"]) + 6 * U * k0)
            tol = tol + TINY * (k0 + np.abs(b0) * 200)
            tol[np.arange(rows), np.where(has, tok, 0)] += 8 * U * (np.abs(a0[:, 0]) + k0[:, 0])
            tol = tol[some] / T + us * np.abs(want) * (1 + us)
        close(np64(dx)[some], want, tol, which)
        assert (between(dx) == 5.0).all()
        zero = (a0 == 0) & (b0 == 0) & (c0 == 0)
        assert (np64(dx)[zero[:, 0]] == 0).all()
        y = t.clone() if pad == 0 and off == 0 else put(x, td, pad, off)
        lp.lp_token_logprobs_backward(y, cu(tok, torch.int32) if a is not None else None, dlogits=y, temperature=T, **dev)
        assert torch.equal(y, dx), which
        assert torch.isnan(between(y)).all()


def teacher_of(g, x, k, T, rest, dup):
    """Entries of a teacher near the student: the best ones mostly, some missing, some at -infinity, some twice."""
    rows, vocab = x.shape
    near = np.where(np.isfinite(x), x, -30.0) + g.standard_normal(x.shape)
    near = np.clip(near - near.max(1, keepdims=True), -60, 0) / T
    l = near - np.log(np.exp(near).sum(1, keepdims=True))
    ids = np.argsort(-near, axis=1)[:, :min(k, vocab)]
    if ids.shape[1] < k:
        ids = np.concatenate([ids, g.integers(0, vocab, (rows, k - ids.shape[1]))], 1)
    t = np.take_along_axis(l, ids, 1)
    if not rest:
        t = t * T + 3.0                                      # logits: any constant
    if dup and k > 3:
        ids[:, 3], t[:, 3] = ids[:, 1], t[:, 1] - 2.0
        ids[:, k - 1] = -1
        t[:, 2] = -np.inf
        if rows > 2:
            ids[2] = -1
        if rows > 3:
            ids[3, 0] = vocab
            t[3, 1:] = -np.inf
    return ids.astype(np.int32), t.astype(np.float32)


def distill_bounds(x, E, ids, t, rest, T, scale, dl):
    """Tolerances of loss and gradient; the terms of `oracle.lm_ops.distill` with the errors of each."""
    rows, n = x.shape
    k = ids.shape[1]
    tl, tg = np.zeros(rows), np.zeros(x.shape)
    for r in range(rows):
        ok = (ids[r] >= 0) & (ids[r] < n)
        i, tt = ids[r][ok], t[r][ok].astype(np.float64)
        if not len(i) or (tt == -np.inf).all() or not np.isfinite(E["e_logs"][r, 0]):
            continue
        with np.errstate(all="ignore"):
            if rest:
                q, rq, e_q = np.exp(tt), np.full(len(tt), EXP), 0.0
                qr = 1 - q.sum()
                qr = qr if qr > 2.0 ** -20 else 0.0
            else:
                s = (tt - tt.max()) / T
                q = np.exp(s) / np.exp(s).sum()
                rq, qr = EXP + 4 * U * np.where(q > 0, np.abs(s), 0) + (k + 8) * U + 3 * U * (q * np.where(q > 0, np.abs(s), 0)).sum() + EXP, 0.0
            lq = np.where(q > 0, np.log(q), 0.0)
            e_lq = rq + 4 * U * np.abs(lq) + 4 * U * np.where(q > 0, np.abs(tt - tt.max()) / T, 0)
            e_mass = (q * rq).sum() + (k + 8) * U * max(q.sum(), 1.0)         # of q's sum, of Q and of the rest
            outside = np.ones(n, dtype=bool)
            outside[i] = False
            p, l = E["p"][r], E["l"][r]
            pr = p[outside].sum()
            # sums over the tokens not listed: terms relative to their own maximum, which is closer than the row's
            e_ls = 2 * E["e_logs"][r, 0] + 6 * U * np.abs(l[np.isfinite(l)]).max(initial=0.0)
            li = np.where(np.isfinite(l[i]), l[i], 0.0)
            tl[r] = (q * (rq * np.abs(lq - li) + e_lq + e_ls + 4 * U * np.abs(li))).sum() + 20 * U * (q * (np.abs(lq) + np.abs(li))).sum()
            if qr > 0 and pr > 0:
                tl[r] += e_mass * (np.abs(np.log(qr) - np.log(pr)) + 2) + qr * (e_ls + 8 * U * (np.abs(np.log(qr)) + np.abs(np.log(pr)))) + 20 * U
            tl[r] *= abs(scale)
            Q = q.sum() + qr
            rel = E["rel"][r] + e_ls + 8 * U
            f = abs(scale / T) * (1.0 if dl is None else abs(float(dl[r])))
            w = np.where(outside & (pr > 0), p / max(pr, 1e-300), 0.0)
            tg[r] = f * (p * Q * rel + e_mass * p + (qr * rel + e_mass) * w * (qr > 0) + TINY * (Q + 1 / max(pr, 1e-30) * qr))
            np.add.at(tg[r], i, f * q * (rq + 8 * U))
    return tl, tg


DISTILL = [(1, 1, 0, 0, 1), (2, 3, 0, 1, 5), (5, 7, 2, 0, 7), (9, 64, 0, 0, 128), (700, 33, 0, 0, 4), (5, 255, 0, 1, 128), (160, 515, 5, 7, 9), (4, 2049, 0, 0, 64),
           (1, 8192, 0, 0, 64), (6, 8200, 3, 5, 30), (4, 32768, 0, 0, 128), (5, 50021, 6, 1, 17), (40, 32771, 1, 0, 5), (1, 131071, 0, 1, 100),
           (2, 150001, 7, 2, 128), (1, 262144, 0, 0, 50)]
DISTILL_CASES = [(*s, "normal") for s in DISTILL] + [(*s, kind) for s in [(5, 700, 1, 1, 40), (4, 20011, 0, 0, 128), (4, 140000, 0, 3, 9)]
                                                     for kind in ("masked", "lowmask", "peaked", "ties", "constant", "far")]


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,off,k,kind", DISTILL_CASES)
def test_distillation(rows, vocab, pad, off, k, kind, dt, rest):
    g, s, x = make(rows, vocab, pad, off, kind, dt, 2)
    td, us = DT[dt]
    T = float(np.float32(g.choice([1.0, 0.75, 2.0])))
    scale = 1.75
    ids, t = teacher_of(g, x, k, T, rest, dup=vocab > 8)
    dl = np.float32(g.standard_normal(rows))
    dl[4::5] = 0.0
    E = errors(x, T, vocab)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    form = lp.LP_DISTILL_REST if rest else lp.LP_DISTILL_TOP
    args = (form, s, cu(ids, torch.int32), cu(t))
    loss, dx = torch.full((rows,), 9.0, device="cuda"), matrix(rows, vocab, td, pad, off, 5.0)
    lp.lp_distill(*args, loss=loss, dloss=cu(dl), dlogits=dx, temperature=T, scale=scale, out_of_range=flag)
    assert flag.item() == int((ids >= vocab).any())
    some = sorted({*range(min(rows, 8)), rows - 1})
    with np.errstate(all="ignore"):
        w_loss, w_dx = O.distill(x[some], ids[some], t[some].astype(np.float64), rest, T, scale, dl[some].astype(np.float64))
    tl, tg = distill_bounds(x[some], {n: v[some] for n, v in E.items()}, ids[some], t[some], rest, T, scale, dl[some])
    close(np64(loss)[some], w_loss, tl, "loss")
    close(np64(dx)[some], w_dx, tg + us * np.abs(w_dx) * (1 + us), "gradient")
    assert (between(dx) == 5.0).all()
    assert (np64(dx)[dl == 0] == 0).all()
    # the loss alone, the gradient alone, in the logits' place, with another stride: the same bits
    alone = torch.zeros(rows, device="cuda")
    lp.lp_distill(*args, loss=alone, temperature=T, scale=scale)
    assert torch.equal(alone, loss)
    other = matrix(rows, vocab, td, pad + 1, off + 1, 5.0)
    lp.lp_distill(*args, dloss=cu(dl), dlogits=other, temperature=T, scale=scale)
    assert torch.equal(other, dx) and (between(other) == 5.0).all()
    y = put(x, td, pad, off)
    lp.lp_distill(form, y, *args[2:], loss=alone, dloss=cu(dl), dlogits=y, temperature=T, scale=scale)
    assert torch.equal(y, dx) and torch.equal(alone, loss) and torch.isnan(between(y)).all()


MANY = [(1400, 1, 0, 0), (2000, 3, 0, 1), (1300, 17, 2, 0), (5000, 50, 0, 1), (3001, 1000, 1, 3), (2500, 4099, 0, 0), (1500, 9000, 7, 0), (1300, 33001, 0, 1), (640, 70003, 1, 0), (300, 140001, 0, 0)]


def many_rows(rows, vocab, pad, off, dt, seed):
    """Rows enough that every block takes several, of all kinds in turn."""
    g = np.random.default_rng(seed)
    kinds = ["normal", "masked", "peaked", "ties", "lowest", "normal", "constant", "lowmask", "descending", "highest"]
    t = matrix(rows, vocab, DT[dt][0], pad, off)
    for i, k in enumerate(kinds):
        if len(range(i, rows, len(kinds))):
            t[i::len(kinds)] = cu(values(g, len(range(i, rows, len(kinds))), vocab, k).astype(np.float32)).to(t.dtype)
    return g, t


def many_reference(t, T):
    """log p, p and the bound of a probability's relative error, in 64 bits on the GPU; rows without any token: p = 0."""
    x = t.double()
    m = x.max(1, keepdim=True).values
    y = torch.where(m > -INF, (x - m) / T, -INF)
    s = y.exp().sum(1, keepdim=True)
    l = torch.where(m > -INF, y - s.log(), -INF)
    far = torch.where(l.exp() > 0, -y, 0.0)
    rel = (t.shape[1] / 256 + 64) * U + 2 * EXP + 8 * U + 3 * U * (far + (l.exp() * far).sum(1, keepdim=True)) + 2 * U * s.log().clamp(min=0)
    return l, l.exp(), rel


def same(got, want, tol, what):
    fin = torch.isfinite(want) & torch.isfinite(want.float())
    assert torch.equal(torch.where(fin, 0.0, got.double()), torch.where(fin, 0.0, want.float().double())), what
    gap = torch.where(fin, (got.double() - want).abs() - tol, -1.0)
    assert (gap <= 0).all(), (what, gap.max(), (gap > 0).nonzero()[:5])


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,off", MANY)
def test_many_rows(rows, vocab, pad, off, dt):
    g, t = many_rows(rows, vocab, pad, off, dt, rows)
    us, T = DT[dt][1], 1.25
    l, p, rel = many_reference(t, T)
    tok = cu(g.integers(-1, vocab, rows), torch.int32)
    has, at = tok >= 0, tok.long().clamp(min=0)[:, None]
    f = lambda *s: torch.full(s, 7.0, device="cuda")
    for k in (0, 1, min(40, vocab)):
        o = dict(logp=f(rows), entropy=f(rows), lse=f(rows))
        if k:
            o.update(top_ids=torch.zeros(rows, k, dtype=torch.int32, device="cuda"), top_logp=f(rows, k))
        lp.lp_token_logprobs(t, tok, temperature=T, **o)
        lz = torch.where(torch.isfinite(l), l, 0.0)
        plain = torch.where(p > 0, l, 0.0)
        # a log probability: that of log S, the difference's, the difference itself rounded three times
        e_l = rel + 4 * U * lz.abs()
        same(o["logp"], torch.where(has, l.gather(1, at)[:, 0], 0.0), e_l.gather(1, at)[:, 0], "logp")
        H = -(p * plain).sum(1)
        same(o["entropy"], H, (p * (rel * (1 + plain.abs()) + 8 * U * plain.abs())).sum(1) * 2 + 2 * U * H, "entropy")
        if k:
            order = torch.sort(t.float(), dim=1, descending=True, stable=True).indices[:, :k]
            assert torch.equal(o["top_ids"].long(), order)
            same(o["top_logp"], l.gather(1, order), e_l.gather(1, order), "top_logp")
    for which in ("a", "ab"):
        a, b = cu(g.standard_normal(rows)), cu(g.standard_normal(rows)) * 0.5
        a[3::7], b[3::7] = 0.0, 0.0                               # rows of zeros among the others
        a0 = torch.where(has, a, 0.0).double()[:, None]
        b0 = b.double()[:, None] if "b" in which else torch.zeros_like(a0)
        pl = p * plain
        want = -a0 * p - b0 * (pl - p * pl.sum(1, keepdim=True))
        want.scatter_add_(1, at, a0)
        size = a0.abs() + b0.abs() * (plain.abs() - pl.sum(1, keepdim=True))
        tol = p * (2 * rel * size + b0.abs() * 2 * rel) + TINY * (1 + size)
        tol.scatter_add_(1, at, 16 * U * a0.abs())
        want, tol = want / T, tol / T
        want[~(p > 0).any(1)] = 0.0                               # no token at all
        dx = matrix(rows, vocab, t.dtype, pad, off, 5.0)
        lp.lp_token_logprobs_backward(t, tok, dlogp=a, dentropy=b if "b" in which else None, dlogits=dx, temperature=T)
        same(dx, want, tol + us * want.abs() * (1 + us), which)
        assert (between(dx) == 5.0).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,off", MANY)
def test_distillation_of_many_rows(rows, vocab, pad, off, dt, rest):
    g, t = many_rows(rows, vocab, pad, off, dt, rows + 1)
    us, T, k = DT[dt][1], 1.25, 20
    l, p, rel = many_reference(t, T)
    # the teacher's entries: among the student's best, a token often twice, some missing
    ids = torch.sort(t.float(), dim=1, descending=True, stable=True).indices[:, :15]
    ids = torch.cat([ids, cu(g.integers(0, vocab, (rows, k - ids.shape[1])), torch.int64)], 1)
    q = cu(g.random((rows, k))) + 0.01
    te = (q / q.sum(1, keepdim=True) * 0.8).log()
    ids[cu(g.random((rows, k))) < 0.1] = -1
    ids[5::11] = -1                                               # rows without entries
    dl = cu(g.standard_normal(rows))
    dl[2::9] = 0.0
    there = ids >= 0
    at = ids.clamp(min=0)
    v = torch.where(there, te.double(), -INF)
    any_ = there.any(1, keepdim=True)
    if rest:
        q = v.exp()
        qr = 1 - q.sum(1, keepdim=True)
        qr = torch.where(any_ & (qr > 2.0 ** -20), qr, 0.0)
    else:
        q = torch.softmax(v / T, 1).nan_to_num(0.0)
        qr = torch.zeros(rows, 1, dtype=torch.float64, device="cuda")
    q = torch.where(any_, q, 0.0)
    inside = torch.zeros(rows, vocab + 1, dtype=torch.bool, device="cuda").scatter_(1, torch.where(there, ids, vocab), True)[:, :-1]
    out = torch.where(inside, -INF, l)
    lr = torch.logsumexp(out, 1, keepdim=True)
    lj = l.gather(1, at)
    zl = lambda a: torch.where(torch.isfinite(a), a, 0.0)
    want = torch.where(q > 0, q * (q.clamp(min=1e-300).log() - lj), 0.0).sum(1) + torch.where(qr > 0, qr * (qr.clamp(min=1e-300).log() - lr), 0.0)[:, 0]
    e_q = (k + 8) * U + 2 * EXP
    e_j = rel.gather(1, at) + 8 * U * zl(lj).abs() + 8 * U * 12 + e_q * 2
    e_rest = (rel * p).sum(1, keepdim=True) + 6 * U * zl(lr).abs() + (vocab / 256 + 64) * U + 40 * U + 4 * EXP     # of log of the rest's sum, against its own maximum
    tol = (q * (e_j + e_q * (12 + zl(lj).abs()))).sum(1) + (qr * e_rest + e_q * (zl(lr).abs() + 12) * (qr > 0))[:, 0]
    loss, dx = torch.full((rows,), 9.0, device="cuda"), matrix(rows, vocab, t.dtype, pad, off, 5.0)
    form = lp.LP_DISTILL_REST if rest else lp.LP_DISTILL_TOP
    args = (form, t, ids.to(torch.int32), te.float())
    lp.lp_distill(*args, loss=loss, dloss=dl, dlogits=dx, temperature=T, scale=2.0)
    same(loss, 2 * want, 2 * tol, "loss")
    Q = q.sum(1, keepdim=True) + qr
    w = torch.softmax(out, 1).nan_to_num(0.0)                     # against the rest's own maximum: it may be the type's lowest value
    grad = Q * p - qr * w
    grad.scatter_add_(1, at, -torch.where(there, q, 0.0))
    # the rest's share is formed against the rest's own maximum: as many roundings of its own
    y = torch.where(w > 0, -(l - l.masked_fill(inside, -INF).max(1, keepdim=True).values), 0.0).nan_to_num(0.0, posinf=0.0, neginf=0.0).abs()
    tolg = Q * p * (rel + e_rest + e_q) + (w * qr) * (rel + e_rest + 3 * U * y) + w * e_q * (qr > 0) + TINY * (Q + qr)
    tolg.scatter_add_(1, at, torch.where(there, q * (e_q + 3 * U * 12), 0.0))
    f = (dl.double() * 2.0 / T)[:, None]
    grad = torch.where((p > 0).any(1, keepdim=True), grad, 0.0) * f
    same(dx, grad, tolg * f.abs() + us * grad.abs() * (1 + us), "gradient")
    assert (between(dx) == 5.0).all()
    alone = torch.zeros(rows, device="cuda")
    lp.lp_distill(*args, loss=alone, temperature=T, scale=2.0)
    assert torch.equal(alone, loss)
    lp.lp_distill(form, t, *args[2:], dloss=dl, dlogits=t, temperature=T, scale=2.0)       # in the logits' place
    assert torch.equal(t, dx)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [50, 40001])
def test_rows_with_nan_and_infinity(vocab, dt):
    """A NaN or +infinity spoils its own row and no other; the order puts a NaN last."""
    g = np.random.default_rng(5)
    x = values(g, 8, vocab, "normal")
    x[1, vocab - 1], x[2, 0], x[3, 7], x[4, :] = np.nan, np.inf, np.nan, np.nan
    x[5] = -np.inf
    x[5, 9] = np.nan                                         # nothing but a NaN among the masked
    x[6, 3] = np.inf
    x[6, 8] = np.nan
    t = put(x, DT[dt][0])
    tok = torch.arange(8, dtype=torch.int32, device="cuda")
    f = lambda *s: torch.zeros(*s, device="cuda")
    o = dict(logp=f(8), entropy=f(8), lse=f(8), top_ids=torch.zeros(8, 12, dtype=torch.int32, device="cuda"), top_logp=f(8, 12))
    lp.lp_token_logprobs(t, tok, **o)
    spoilt = torch.tensor([False, True, True, True, True, True, True, False])
    for n in ("logp", "entropy", "lse"):
        assert torch.equal(torch.isnan(o[n]).cpu(), spoilt), n
    assert torch.equal(torch.isnan(o["top_logp"]).all(1).cpu(), spoilt) and torch.equal(torch.isnan(o["top_logp"]).any(1).cpu(), spoilt)
    want = O.token_logprobs(np64(t), None, 1.0, 12)[3]
    assert np.array_equal(o["top_ids"].cpu().numpy(), want)
    one = torch.ones(8, device="cuda")
    for kw in (dict(dlogp=one), dict(dentropy=one), dict(dlse=one), dict(dlogp=one, dentropy=one, dlse=one)):
        dx = torch.zeros_like(t)
        lp.lp_token_logprobs_backward(t, tok, dlogits=dx, **kw)
        assert torch.equal(torch.isnan(dx).all(1).cpu(), spoilt) and torch.equal(torch.isnan(dx).any(1).cpu(), spoilt), kw
    dx = torch.ones_like(t)
    lp.lp_token_logprobs_backward(t, tok, dlse=f(8), dlogits=dx)     # nothing comes in: the logits do not matter
    assert (dx == 0).all()
    ids, te = torch.tensor([[3, 1, 9]] * 8, dtype=torch.int32, device="cuda"), torch.log(torch.tensor([[0.5, 0.2, 0.1]] * 8, device="cuda"))
    for form in (lp.LP_DISTILL_TOP, lp.LP_DISTILL_REST):
        loss, dx = f(8), torch.zeros_like(t)
        lp.lp_distill(form, t, ids, te, loss=loss, dlogits=dx)
        assert torch.equal(torch.isnan(loss).cpu(), spoilt) and torch.equal(torch.isnan(dx).all(1).cpu(), spoilt)
        assert torch.equal(torch.isnan(dx).any(1).cpu(), spoilt)
        lp.lp_distill(form, t, -ids, te, loss=loss, dlogits=dx)      # no entries: the logits do not matter
        assert (loss == 0).all() and (dx == 0).all()
    te[0, 1] = float("nan")                                          # a teacher's NaN
    for form in (lp.LP_DISTILL_TOP, lp.LP_DISTILL_REST):
        lp.lp_distill(form, t, ids, te, loss=loss, dlogits=dx)
        assert torch.isnan(loss[0]) and torch.isfinite(loss[7]) and torch.isfinite(dx[7].float()).all()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
def test_impossible_tokens_and_an_impossible_rest(dt):
    """The student excludes what the teacher holds: an infinite loss, finite gradients where the formula has them."""
    vocab = 9000
    x = np.zeros((4, vocab))
    x[0, 5] = -np.inf
    x[1, 10:] = -np.inf
    x[2, 1] = 300.0                                          # a rest of exp(-300): its loss and gradient stay finite
    x[3] = -np.inf
    t = put(x, DT[dt][0])
    ids = np.array([[5, 6], [0, 1], [1, 2], [0, 1]], dtype=np.int32)
    te = np.log(np.array([[0.5, 0.25], [0.5, 0.5], [0.5, 0.25], [0.5, 0.25]])).astype(np.float32)
    ids[1, 0] = 3
    for rest in (False, True):
        if rest:
            te[1] = np.log([0.5, 0.25])
        x1 = np64(t)
        if rest:
            x1[1, :10] = np.where(np.isin(np.arange(10), ids[1]), 0.0, -np.inf)
            t = put(x1, DT[dt][0])
        with np.errstate(all="ignore"):
            want, w_dx = O.distill(x1, ids, te.astype(np.float64), rest)
        loss, dx = torch.zeros(4, device="cuda"), torch.zeros_like(t)
        lp.lp_distill(lp.LP_DISTILL_REST if rest else lp.LP_DISTILL_TOP, t, cu(ids, torch.int32), cu(te), loss=loss, dlogits=dx)
        assert np.isinf(want[[0, 3]]).all() and np.isinf(want[1]) == rest and np.isfinite(w_dx).all()
        close(np64(loss), want, 1e-5 * np.abs(np.where(np.isfinite(want), want, 0.0)) + 1e-5)
        close(np64(dx), w_dx, 2e-5 + DT[dt][1] * np.abs(w_dx) * 1.01)
        assert (np64(dx)[3] == 0).all()


@pytest.mark.parametrize("T", [2.0 ** -20, 2.0 ** -8, 2.0 ** 8, 2.0 ** 20])
@pytest.mark.parametrize("rows,vocab,dt", [(5, 3001, "fp32"), (3, 40000, "bf16")])
def test_extreme_temperatures(rows, vocab, dt, T):
    g, t, x = make(rows, vocab, 1, 0, "normal", dt, 7)
    k = 9
    tok = x.argmax(1).astype(np.int32)
    tok[0] = 5
    E = errors(x, T, vocab)
    f = lambda *s: torch.zeros(*s, device="cuda")
    o = dict(logp=f(rows), entropy=f(rows), lse=f(rows), top_ids=torch.zeros(rows, k, dtype=torch.int32, device="cuda"), top_logp=f(rows, k))
    lp.lp_token_logprobs(t, cu(tok, torch.int32), temperature=T, **o)
    logp, ent, lse, ids, tops = O.token_logprobs(x, tok, T, k)
    close(np64(o["logp"]), logp, np.take_along_axis(E["e_l"], tok[:, None], 1)[:, 0], "logp")
    close(np64(o["entropy"]), ent, E["e_h"][:, 0], "entropy")
    close(np64(o["lse"]), lse, E["e_lse"][:, 0], "lse")
    assert np.array_equal(o["top_ids"].cpu().numpy(), ids)
    close(np64(o["top_logp"]), tops, np.take_along_axis(E["e_l"], ids, 1), "top_logp")
    one = np.ones(rows, dtype=np.float32)
    dx = torch.zeros_like(t)
    lp.lp_token_logprobs_backward(t, cu(tok, torch.int32), dlogp=cu(one), dlogits=dx, temperature=T)
    want = O.token_logprobs_bwd(x, tok, one, None, None, T)
    close(np64(dx) * T, want * T, E["p"] * (E["rel"] + 8 * U) + DT[dt][1] * np.abs(want * T) * 1.01 + 16 * U * (np.arange(vocab) == tok[:, None]) + TINY, "gradient")
    te = tops.astype(np.float32)
    for rest in (False, True):
        use = te if rest else te * np.float32(T)
        w_loss, w_dx = O.distill(x, ids, use.astype(np.float64), rest, T)
        loss = f(rows)
        lp.lp_distill(int(rest), t, cu(ids.astype(np.int32), torch.int32), cu(use), loss=loss, dlogits=dx, temperature=T)
        # te, use: each rounded once to fp32
        tl, tg = distill_bounds(x, E, ids, use, rest, T, 1.0, None)
        close(np64(loss), w_loss, tl + 1e-6, "loss")
        close(np64(dx) * T, w_dx * T, tg * T + DT[dt][1] * np.abs(w_dx * T) * 1.01 + 1e-6, "gradient of the loss")


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("vocab", [90, 5003, 70000])
def test_one_token_in_every_entry(vocab, rest):
    """128 entries of a single token, and of two in turn, beside rows of other sizes of the same."""
    g = np.random.default_rng(vocab)
    rows, k = 4, 128
    t = put(values(g, rows, vocab, "normal"), torch.float32)
    x = np64(t)
    ids = np.full((rows, k), vocab - 1, dtype=np.int32)
    ids[1, ::2] = 0
    ids[2] = np.arange(k) % 7
    te = np.log(g.random((rows, k)) / k * 0.9).astype(np.float32)
    want, w_dx = O.distill(x, ids, te.astype(np.float64), rest, 1.0)
    E = errors(x, 1.0, vocab)
    tl, tg = distill_bounds(x, E, ids, te, rest, 1.0, 1.0, None)
    runs = []
    for _ in range(3):
        loss, dx = torch.zeros(rows, device="cuda"), torch.zeros_like(t)
        lp.lp_distill(int(rest), t, cu(ids, torch.int32), cu(te), loss=loss, dlogits=dx)
        runs.append((loss, dx))
    close(np64(loss), want, tl, "loss")
    close(np64(dx), w_dx, tg + U * np.abs(w_dx) * (1 + U), "gradient")
    assert all(torch.equal(a, loss) and torch.equal(b, dx) for a, b in runs)


def test_strides_beyond_two_to_the_31_elements():
    ld = (1 << 31) + 40
    store = torch.empty(ld + 1000, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((2, 1000), (ld, 1))
    x.copy_(torch.randn(2, 1000, device="cuda"))
    near = x.contiguous()
    tok = torch.tensor([3, 999], dtype=torch.int32, device="cuda")
    f = lambda: torch.zeros(2, device="cuda")
    a, b, g = f(), f(), torch.ones(2, device="cuda")
    lp.lp_token_logprobs(x, tok, logp=a)
    lp.lp_token_logprobs(near, tok, logp=b)
    assert torch.equal(a, b)
    want = torch.empty_like(near)
    lp.lp_token_logprobs_backward(near, tok, dlogp=g, dlogits=want)
    lp.lp_token_logprobs_backward(x, tok, dlogp=g, dlogits=x)
    assert torch.equal(x, want)
    ids, te = torch.tensor([[3, 1], [999, 0]], dtype=torch.int32, device="cuda"), torch.zeros(2, 2, device="cuda")
    lp.lp_distill(0, near, ids, te, loss=a, dlogits=want)
    x.copy_(near)
    lp.lp_distill(0, x, ids, te, loss=b, dlogits=x)
    assert torch.equal(x, want) and torch.equal(a, b)


def chain(x, tok, st, s):
    """A teacher's alternatives, the student taught from them, and the gradient of its own log probabilities."""
    lp.lp_token_logprobs(x, tok, st["logp"], st["ent"], None, st["ids"], st["tops"], 2.0, None, s)
    lp.lp_distill(lp.LP_DISTILL_REST, st["y"], st["ids"], st["tops"], st["loss"], st["ent"], st["dy"], 2.0, 4.0, None, s)
    lp.lp_token_logprobs_backward(st["y"], tok, st["logp"], st["ent"], st["loss"], st["dz"], 1.0, None, s)


@pytest.mark.parametrize("rows,vocab", [(3, 1000), (40, 9001), (2, 131072)])
def test_calls_on_side_streams_and_replayed_from_a_graph(rows, vocab):
    def fresh(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
        f = lambda *s: torch.zeros(*s, device="cuda")
        x = r(rows, vocab)
        st = dict(y=r(rows, vocab), logp=f(rows), ent=f(rows), loss=f(rows), tops=f(rows, 16), dy=torch.zeros_like(x), dz=torch.zeros_like(x),
                  ids=torch.zeros(rows, 16, dtype=torch.int32, device="cuda"))
        return x, torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32), st

    sets = [fresh(s) for s in (1, 2)]
    for x, tok, st in sets:
        chain(x, tok, st, None)
    torch.cuda.synchronize()
    want = [{n: v.clone() for n, v in st.items()} for _, _, st in sets]
    clear = lambda: [v.zero_() for _, _, st in sets for n, v in st.items() if n != "y"]
    same = lambda: all(torch.equal(w[n], st[n]) for w, (_, _, st) in zip(want, sets) for n in w)
    side = [torch.cuda.Stream() for _ in sets]
    clear()
    torch.cuda.synchronize()
    for _ in range(3):                                       # two streams at once
        for (x, tok, st), s in zip(sets, side):
            chain(x, tok, st, s.cuda_stream)
    torch.cuda.synchronize()
    assert same()
    graphs = []
    for (x, tok, st), s in zip(sets, side):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            chain(x, tok, st, s.cuda_stream)
    clear()
    for gr in graphs:
        gr.replay()
    torch.cuda.synchronize()
    assert same()


FIRST_CALLS = """
import sys
sys.path.insert(0, sys.argv[1])
import torch
from tests.test_gpu_logit_ops import chain
x, y = (torch.randn(5, 70001, device="cuda").bfloat16() for _ in range(2))
f = lambda *s: torch.zeros(*s, device="cuda")
st = dict(y=y, logp=f(5), ent=f(5), loss=f(5), tops=f(5, 16), dy=torch.zeros_like(x), dz=torch.zeros_like(x),
          ids=torch.zeros(5, 16, dtype=torch.int32, device="cuda"))
tok = torch.arange(5, dtype=torch.int32, device="cuda")
stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=stream):
    chain(x, tok, st, stream.cuda_stream)
graph.replay()
torch.cuda.synchronize()
first = {n: v.clone() for n, v in st.items()}
chain(x, tok, st, torch.cuda.current_stream().cuda_stream)
torch.cuda.synchronize()
assert all(torch.equal(first[n], v) for n, v in st.items()) and st["dy"].float().abs().sum() > 0 and st["dz"].float().abs().sum() > 0
print("equal")
"""


def test_the_very_first_calls_may_be_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS, root], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "equal" in r.stdout, r.stdout + r.stderr


def test_memory_of_the_host_is_refused():
    x, host = torch.zeros(2, 64, device="cuda"), np.zeros(64, dtype=np.float32)
    out = torch.zeros(2, device="cuda")
    for kw in (dict(entropy=host.ctypes.data), dict(lse=out, out_of_range=host.ctypes.data)):
        with pytest.raises(lp.LpError) as e:
            lp.lp_token_logprobs(x, **kw)
        assert e.value.code == -1
    torch.cuda.synchronize()


def test_a_student_model_is_taught_by_a_larger_one():
    """The operators as they are used: two transformers' logits, the teacher's alternatives, the student's loss and the
    gradient of its head's weights, against automatic differentiation in 64 bits."""
    import lp_synth
    from tests import lp_testlib as H
    base = dict(batch=2, seq_len=64, vocab=1000, d_ffn=256, blocks_per_chunk=[1, 1], schedule="sync")
    teacher = H.GpuModel(lp_synth.config("c3", d_model=256, n_heads=4, **base))
    student = H.GpuModel(lp_synth.config("c3", d_model=128, n_heads=2, **base))
    tok, lab = lp_synth.minibatch(teacher.cfg, 0)
    rows, vocab, k, T = 128, 1000, 24, 2.0
    logits = {}
    for name, m in (("teacher", teacher), ("student", student)):
        z, _ = m.forward(tok, lab)
        logits[name] = cu(z).bfloat16().view(rows, vocab)
    nxt = cu(np.asarray(lab).reshape(-1), torch.int32)       # -1 at the end of each sequence
    f = lambda *s: torch.zeros(*s, device="cuda")
    ids, tops, loss, dz = torch.zeros(rows, k, dtype=torch.int32, device="cuda"), f(rows, k), f(rows), torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    lp.lp_token_logprobs(logits["teacher"], top_ids=ids, top_logp=tops, temperature=T)
    weight = (nxt >= 0).float() / (nxt >= 0).sum()
    lp.lp_distill(lp.LP_DISTILL_REST, logits["student"], ids, tops, loss=loss, dloss=weight, dlogits=dz, temperature=T, scale=T * T)
    hidden = torch.randn(rows, 128, device="cuda").bfloat16()
    dW = f(vocab, 128)
    lp.lp_gemm_bf16([dict(A=dz, B=hidden, C=dW, M=vocab, N=128, K=rows, a_ms=1, a_ks=vocab, b_ns=1, b_ks=128, ldc=128, out_f32=1)], 0)
    z = logits["student"].double().cpu().requires_grad_()
    q = torch.log_softmax(logits["teacher"].double().cpu() / T, 1)
    l = torch.log_softmax(z / T, 1)
    at = ids.long().cpu()
    inside = torch.zeros_like(q, dtype=torch.bool).scatter_(1, at, True)
    tail = lambda a: torch.logsumexp(a.masked_fill(inside, -INF), 1)
    ql, ll = q.gather(1, at), l.gather(1, at)
    kl = (ql.exp() * (ql - ll)).sum(1) + tail(q).exp() * (tail(q) - tail(l))
    total = (weight.cpu().double() * T * T * kl).sum()
    total.backward()
    assert ((loss.cpu().double() - T * T * kl.detach()).abs() <= 1e-4 * (1 + kl.detach())).all()
    gap = (dz.cpu().double() - z.grad).abs()
    assert (gap <= 2.0 ** -8 * z.grad.abs() + 1e-5 * z.grad.abs().max()).all()
    ref = z.grad.t() @ hidden.cpu().double()
    assert (dW.cpu().double() - ref).norm() <= 2.0 ** -8 * ref.norm()
    # the student's own tokens: log probabilities against its cross-entropy, and their gradient
    logp = f(rows)
    lp.lp_token_logprobs(logits["student"], nxt, logp=logp)
    ce = torch.nn.functional.cross_entropy(logits["student"].double().cpu(), nxt.long().cpu(), ignore_index=-1, reduction="none")
    assert ((logp.cpu().double() + ce).abs() <= 1e-4).all()
    teacher.close(), student.close()

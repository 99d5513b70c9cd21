"""The operators on logits over the whole range of values: rows far below and far above 0, masks of any finite size, the
border at which differences are taken before the factor.  Every row against 64 bits.

Tolerances go beyond those of test_gpu_logit_ops by what the place of a row's reference costs: powers are taken against
a rounded multiple of the maximum, off by at most 2 (3 with margin), which log S and the mean of y then hold on both
sides of a difference.  y: rounded constant, difference or product, and the factor ln 2 with its product, 5 u at most."""
import numpy as np
import pytest
import torch

from oracle import lm_ops as O
from paper_2012_03837_b200 import binding as lp
from tests.test_gpu_logit_ops import DT, EXP, INF, U, close, cu, errors, np64, put

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -118                     # powers below 2^-126 are 0, against a reference off by up to 2^3, with margin


def bounds(x, T):
    n = x.shape[1]
    E = errors(x, T, n)
    d = (n / 256 + 64) * U + EXP
    with np.errstate(all="ignore"):
        y = np.where(E["l"] > -np.inf, np.abs(x - np.where(np.isfinite(x.max(1, keepdims=True)), x.max(1, keepdims=True), 0.0)) / T, 0.0)
        E["e_logs"] = E["e_logs"] + 6 * U
        E["e_l"] = np.where(np.isfinite(E["l"]), E["e_logs"] + 5 * U * y + 2 * U * np.abs(E["l"]), 0.0)
        E["e_h"] = E["e_h"] + 4 * d + 12 * U
        E["e_lse"] = E["e_lse"] + 6 * U
        E["rel"] = np.where(E["p"] > 0, E["e_logs"] + 5 * U * y + EXP + 8 * U, 0.0)
    return E


def check_log_probabilities(t, T, g, k=9, E=None):
    x = np64(t)
    rows, n = x.shape
    E = E or bounds(x, T)
    k = min(k, n)
    tok = g.integers(0, n, rows).astype(np.int32)
    tok[::2] = x.argmax(1)[::2]
    f = lambda *s: torch.full(s, 7.0, device="cuda")
    for top in (0, k):
        o = dict(logp=f(rows), entropy=f(rows), lse=f(rows))
        if top:
            o.update(top_ids=torch.zeros(rows, k, dtype=torch.int32, device="cuda"), top_logp=f(rows, k))
        lp.lp_token_logprobs(t, cu(tok, torch.int32), temperature=T, **o)
        m = x.max(1)
        with np.errstate(all="ignore"):
            lse = np.where(m > -np.inf, m / T + np.log(np.exp((x - np.where(m > -np.inf, m, 0.0)[:, None]) / T).sum(1)), -np.inf)
        close(np64(o["logp"]), E["l"][np.arange(rows), tok], E["e_l"][np.arange(rows), tok], "logp")
        close(np64(o["entropy"]), E["H"][:, 0], E["e_h"][:, 0], "entropy")
        close(np64(o["lse"]), lse, E["e_lse"][:, 0], "lse")
        if top:
            order = np.argsort(-x, axis=1, kind="stable")[:, :k]
            assert np.array_equal(o["top_ids"].cpu().numpy(), order)
            close(np64(o["top_logp"]), np.take_along_axis(E["l"], order, 1), np.take_along_axis(E["e_l"], order, 1), "top_logp")
        alone = f(rows)                                    # sums without the entropy's
        lp.lp_token_logprobs(t, cu(tok, torch.int32), logp=alone, temperature=T)
        close(np64(alone), E["l"][np.arange(rows), tok], E["e_l"][np.arange(rows), tok], "logp alone")


def check_gradient(t, T, g, E=None):
    x = np64(t)
    rows, n = x.shape
    us = DT["bf16" if t.dtype is torch.bfloat16 else "fp32"][1]
    E = E or bounds(x, T)
    tok = g.integers(0, n, rows).astype(np.int32)
    tok[::2] = x.argmax(1)[::2]
    a, b, c = (np.float32(v) for v in g.standard_normal((3, rows)))
    for which in ("a", "abc"):
        b0, c0 = (v if len(which) > 1 else None for v in (b, c))
        dx = torch.full_like(t, 5.0)
        lp.lp_token_logprobs_backward(t, cu(tok, torch.int32), dlogp=cu(a), dentropy=None if b0 is None else cu(b0), dlse=None if c0 is None else cu(c0),
                                      dlogits=dx, temperature=T)
        want = O.token_logprobs_bwd(x, tok, *(None if v is None else v.astype(np.float64) for v in (a, b0, c0)), T)
        a1, b1, c1 = (np.zeros((rows, 1)) if v is None else np.abs(v[:, None]).astype(np.float64) for v in (a, b0, c0))
        lz = np.where(E["p"] > 0, np.abs(E["l"]), 0.0)
        k0 = a1 + c1 + b1 * (E["H"] + 3.0)                 # the mean of y, which holds the reference's 3
        with np.errstate(all="ignore"):
            tol = E["p"] * (E["rel"] * (k0 + b1 * (lz + 3.0)) + b1 * (E["e_l"] * (E["p"] > 0) + E["e_h"]) + 8 * U * k0) + TINY * (k0 + 200 * b1)
        tol[np.arange(rows), tok] += 8 * U * (a1 + k0)[:, 0]
        with np.errstate(over="ignore"):
            close(np64(dx), want, tol / T + us * np.abs(want) * (1 + us), which)


def distill_bounds(x, E, ids, te, rest, T, scale):
    """As in test_gpu_logit_ops, with the tokens not listed against their own maximum, and nothing that grows with a
    masked token's value unless it is listed."""
    rows, n = x.shape
    k = ids.shape[1]
    tl, tg = np.zeros(rows), np.zeros(x.shape)
    for r in range(rows):
        i, tt = ids[r], te[r].astype(np.float64)
        xo = x[r:r + 1].copy()
        xo[0, i] = -np.inf
        Eo = bounds(xo, T)
        s = tt - tt.max()
        if rest:
            q, rq = np.exp(tt), np.full(k, EXP)
            qr = 1 - q.sum()
            qr = qr if qr > 2.0 ** -20 else 0.0
        else:
            q = np.exp(s / T) / np.exp(s / T).sum()
            rq, qr = 2 * EXP + 4 * U * np.abs(s / T) + (k + 8) * U + 3 * U * (q * np.abs(s / T)).sum(), 0.0
        lq = np.log(np.where(q > 0, q, 1.0))
        e_mass = (q * rq).sum() + (k + 8) * U * max(q.sum(), 1.0)
        l = E["l"][r]
        li = np.where(np.isfinite(l[i]), l[i], 0.0)
        e_lq = rq + 4 * U * np.abs(lq) + 4 * U * (np.abs(s) / T if not rest else 0.0)
        tl[r] = (q * (rq * np.abs(lq - li) + e_lq + E["e_l"][r, i] + 20 * U * (np.abs(lq) + np.abs(li)))).sum()
        pr = 0.0
        with np.errstate(all="ignore"):
            mo, m = xo.max(), x[r].max()
            log_pr = (mo - m) / T + np.log(np.exp((xo - mo) / T).sum()) - np.log(np.exp((x[r] - m) / T).sum()) if mo > -np.inf else -np.inf
        e_pr = Eo["e_logs"][0, 0] + E["e_logs"][r, 0]
        if qr > 0 and log_pr > -np.inf:
            e_pr += 6 * U * np.abs(log_pr) + 5 * U * (m - mo) / T
            tl[r] += e_mass * (np.abs(np.log(qr) - log_pr) + 2) + qr * (e_pr + 8 * U * np.abs(np.log(qr))) + 20 * U
        Q = q.sum() + qr
        p, w = E["p"][r], Eo["p"][0]
        # of p outside: its power against the others' maximum, and that one's against the row's
        rel = E["rel"][r] + Eo["rel"][0] + e_pr + (5 * U * (m - mo) / T if np.isfinite(mo) else 0.0) + 8 * U
        f = abs(scale) / T
        tg[r] = f * (p * Q * np.where(p > 0, rel, 0.0) + e_mass * p + (qr * (Eo["rel"][0] + Eo["e_logs"][0, 0] + 8 * U) + e_mass) * w * (qr > 0) + TINY * (1 + Q))
        np.add.at(tg[r], i, f * q * (rq + 8 * U))
    return tl * abs(scale), tg


def check_distillation(t, T, g, listed=None, k=7, E=None):
    """Entries of any ids, or `listed` of every row; the teacher's values have nothing to do with the student's."""
    x = np64(t)
    rows, n = x.shape
    us = DT["bf16" if t.dtype is torch.bfloat16 else "fp32"][1]
    E = E or bounds(x, T)
    ids = np.stack([g.permutation(n)[:min(k, n)] for _ in range(rows)]) if listed is None else listed
    ids = ids.astype(np.int32)
    for rest in (False, True):
        q = g.random(ids.shape) + 0.05
        te = np.log(q / q.sum(1, keepdims=True) * 0.75).astype(np.float32)
        if not rest:
            te = (te * np.float32(T) + np.float32(1)).astype(np.float32)
        loss, dx = torch.full((rows,), 9.0, device="cuda"), torch.full_like(t, 5.0)
        form = lp.LP_DISTILL_REST if rest else lp.LP_DISTILL_TOP
        lp.lp_distill(form, t, cu(ids, torch.int32), cu(te), loss=loss, dlogits=dx, temperature=T, scale=1.5)
        with np.errstate(all="ignore"):
            w_loss, w_dx = O.distill(x, ids, te.astype(np.float64), rest, T, 1.5)
            tl, tg = distill_bounds(x, E, ids, te, rest, T, 1.5)
        close(np64(loss), w_loss, tl, ("loss", rest))
        close(np64(dx), w_dx, tg + us * np.abs(w_dx) * (1 + us), ("gradient", rest))
        alone = torch.full((rows,), 9.0, device="cuda")
        lp.lp_distill(form, t, cu(ids, torch.int32), cu(te), loss=alone, temperature=T, scale=1.5)
        assert torch.equal(alone, loss)


def check(t, T, g, **kw):
    E = bounds(np64(t), T)
    check_log_probabilities(t, T, g, E=E)
    check_gradient(t, T, g, E=E)
    check_distillation(t, T, g, E=E, **kw)


# ------------------------------------------------------------------------------------------------ warps without a token
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 7, 64, 515, 3000, 9001, 40010])
@pytest.mark.parametrize("level", [-100.0, -1000.0, -1e5])
def test_rows_below_zero_of_which_warps_hold_no_token(level, vocab, dt):
    """A warp without a token says that its sum is 0, whatever the row's reference: 2^(0 - reference) has no place in it."""
    g = np.random.default_rng(vocab)
    x = level + 3.0 * g.standard_normal((5, vocab))
    x[1, : vocab // 2] = -np.inf
    x[2, vocab // 2 + 1:] = -np.inf
    x[3] = np.where(np.arange(vocab) < 5, x[3], -np.inf)
    x[4] = np.where(np.arange(vocab) >= vocab - 3, x[4], -np.inf)
    for T in (1.0, 0.5):
        check(put(x, DT[dt][0]), T, g)


# ------------------------------------------------------------------------------------------------ losses near the type's end
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
def test_a_loss_is_finite_where_a_log_probability_is_not(dt):
    """A listed token of the type's lowest values: log p may be below fp32's range, a small weight times it is not."""
    x = np.zeros((4, 500))
    x[0, 7], x[1, 7], x[2, 7], x[3, 7] = -3.0e38, -3.3e38, -2.0e38, -INF
    t = put(x, DT[dt][0])
    x = np64(t)
    ids = np.array([[7, 3]] * 4, dtype=np.int32)
    q = np.array([[0.05, 0.6], [0.2, 0.7], [1e-30, 0.5], [1e-42, 0.5]])      # the last: a weight below the normal numbers, no probability
    te = np.log(q).astype(np.float32)
    for T in (0.75, 0.25):
        for rest in (False, True):
            use = te if rest else (te * np.float32(T)).astype(np.float32)
            loss = torch.zeros(4, device="cuda")
            lp.lp_distill(int(rest), t, cu(ids, torch.int32), cu(use), loss=loss, temperature=T)
            with np.errstate(all="ignore"):
                want, _ = O.distill(x, ids, use.astype(np.float64), rest, T)
            assert np.isfinite(want[:3].astype(np.float32)).all() and np.isinf(want[3])
            # of a weight: its exponential of an argument up to 70, in the first form a quotient; of a distance: three roundings
            close(np64(loss), want, np.abs(np.where(np.isfinite(want), want, 0.0)) * (2 * EXP + 3 * U * 70 + 16 * U) + 72 * U + 4 * EXP, (T, rest))

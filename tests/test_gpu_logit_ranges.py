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
from tests.test_gpu_logit_ops import DT, EXP, INF, MANY, U, between, close, cu, errors, many_rows, matrix, np64, put, same

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


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
def test_a_loss_is_finite_where_the_rests_log_probability_is_not(dt):
    """All but the listed tokens at the type's lowest values: log p of the rest is below fp32's range, its weight times it is not."""
    g = np.random.default_rng(4)
    x = np.full((3, 600), -3.3e38)
    x[1] = -2.0e38
    ids = np.stack([g.permutation(600)[:3] for _ in range(3)]).astype(np.int32)
    np.put_along_axis(x, ids, g.standard_normal((3, 3)), 1)
    np.put_along_axis(x[2:], ids[2:], np.array([[1e37, 0.5e37, -1e37]]), 1)
    t = put(x, DT[dt][0])
    x = np64(t)
    te = np.log([[0.5, 0.3, 0.15], [0.3, 0.2, 0.2], [0.4, 0.2, 0.35]]).astype(np.float32)
    for T in (0.75, 0.5, 0.25):
        loss, dx = torch.zeros(3, device="cuda"), torch.zeros_like(t)
        lp.lp_distill(lp.LP_DISTILL_REST, t, cu(ids, torch.int32), cu(te), loss=loss, dlogits=dx, temperature=T)
        want, w_dx = O.distill(x, ids, te.astype(np.float64), True, T)
        fits = want < 3.0e38
        assert fits[:2].all() or T == 0.25
        # the rest: 64 bits rounded once; the listed tokens' distances, three roundings each; c, one
        close(np64(loss)[fits], want[fits], want[fits] * 32 * U)
        # the others' sum, 600 equal terms, their shares and p of the listed ones: orders of one
        close(np64(dx), w_dx, (np.abs(w_dx) + (w_dx != 0) * 1e-3) * (72 * U + 4 * EXP) + DT[dt][1] * np.abs(w_dx) * 1.01, T)


# ------------------------------------------------------------------------------------------------ values of any size
TEMPERATURES = [0.5, 0.699999988079071, 0.75, 1.0, 1.5, 2.0]


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("left", ["half", "tenth", "five"])
@pytest.mark.parametrize("mask", [-1e7, -1e8, -1e9, -1e10, -1e12, -1e15, -1e18, -1e22])
def test_masks_of_a_finite_value(mask, left, dt):
    g = np.random.default_rng(int(7 * np.log10(-mask)))
    for i, T in enumerate(TEMPERATURES):
        rows, vocab = [(3, 1003), (2, 9011), (4, 250)][i % 3]
        x = 3.0 * g.standard_normal((rows, vocab))
        allowed = None
        if left == "five":
            allowed = np.stack([g.permutation(vocab)[:5] for _ in range(rows)])
            y = np.full_like(x, mask)
            np.put_along_axis(y, allowed, np.take_along_axis(x, allowed, 1), 1)
            x = y
        else:
            x[g.random(x.shape) < (0.5 if left == "half" else 0.9)] = mask
        x[-1, g.integers(0, vocab, 3)] = -np.inf            # beside the other kind of mask
        t = put(x, DT[dt][0], 1, 1)
        check(t, T, g)
        if allowed is not None:                             # the teacher's rest is nothing but masked tokens
            check_distillation(t, T, g, listed=allowed)


LARGEST = [1e5, 1e6, 1e7, 2.3e7, 4.6e7, 4.7e7, 9e7, 1e8, 1e9, 5e9, 1e10, 1e11, 5e11, 1e12, 1e13, 1e20, 1e30]


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("vocab", [77, 4100])
def test_largest_logits_of_any_size(vocab, sign, dt):
    """Rows whose other logits are at most a few steps of the type lower, and rows with ordinary ones beside the largest."""
    g = np.random.default_rng(vocab + sign)
    for unit in (1.0, 8.0):                                 # the largest and the temperature, together: more rows about the border
        x = np.zeros((2 * len(LARGEST), vocab))
        for i, M in enumerate(LARGEST):
            top = float(torch.tensor(sign * M * unit).to(DT[dt][0]))
            step = abs(top) * 2 * DT[dt][1]
            x[2 * i] = top - step * g.integers(0, 5, vocab)
            x[2 * i, g.integers(0, vocab)] = top
            x[2 * i + 1] = (3.0 if sign > 0 else 2 * top) + g.standard_normal(vocab)
            x[2 * i + 1, g.integers(0, vocab)] = top
        for T in (unit, 3.0 * unit):
            check(put(x, DT[dt][0], 3, 0), T, g)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
def test_small_temperatures(dt):
    g = np.random.default_rng(11)
    for T, sizes in ((2.0 ** -20, [1.0, 10.0, 22.0, 30.0, 43.0, 45.0, 60.0, 3008.0, 19968.0, 3e4, 1e5]), (2.0 ** -14, [13.0, 2800.0, 3000.0, 3e5]),
                     (1e-4, [4000.0, 5000.0, 1e6])):
        x = np.zeros((2 * len(sizes), 2050))
        for i, M in enumerate(sizes):
            for j, s in enumerate((M, -M)):
                top = float(torch.tensor(s).to(DT[dt][0]))
                x[2 * i + j] = top - abs(top) * 2 * DT[dt][1] * g.integers(0, 3, 2050) - T * g.integers(0, 9, 2050)
        check(put(x, DT[dt][0]), float(np.float32(T)), g)


@pytest.mark.parametrize("T", [1.0, 2.0, 16.0, 2.0 ** 20])
@pytest.mark.parametrize("vocab", [60, 1500])
def test_listed_tokens_and_the_rest_on_both_sides_of_the_border(vocab, T):
    """Where a row's references stop being rounded multiples of its maximum, above 0 and below: the listed tokens' largest
    logit, the others', both or none beyond it, a few steps of the type apart."""
    g = np.random.default_rng(vocab)
    x, ids = [], []
    for power in range(24, 32):                             # of two, in units of ln 2 T
        for sign in (1, -1):
            border = np.float32(sign * 2.0 ** power * np.log(2.0) * T)
            step = float(np.spacing(np.abs(border)))
            for up in (-2, -1, 0, 1, 2):
                for gap in (-1, 0, 1):
                    listed = g.permutation(vocab)[:7]
                    r = float(border) + step * (up - g.integers(0, 3, vocab))
                    r[listed] += gap * step
                    x.append(r)
                    ids.append(listed)
    x, ids = np.stack(x), np.stack(ids)
    check_distillation(put(x, torch.float32), T, g, listed=ids)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(1500, 700), (700, 33000), (5, 200003)])
def test_many_rows_with_masks_and_levels_of_all_kinds(rows, vocab, dt):
    """Rows of all sizes of values after one another in the same blocks, and long ones over clusters of blocks: against the
    same expressions in 64 bits on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    T, us = 0.75, DT[dt][1]
    x = 2.0 * torch.randn(rows, vocab, generator=g, device="cuda")
    levels = torch.tensor([0.0, -200.0, 3e4, -1e6, 3.4e7, -3.6e7, 1e9, -1e10, 4e11, 0.0], device="cuda")
    x += levels[torch.arange(rows, device="cuda") % 10][:, None]
    masks = torch.tensor([-1e10, -INF, -1e12, -1e18, -3e38, -1e9, -INF], device="cuda")
    hidden = torch.rand(rows, vocab, generator=g, device="cuda") < 0.9
    hidden[3::4] = False
    t = torch.where(hidden, masks[torch.arange(rows, device="cuda") % 7][:, None], x).to(DT[dt][0])
    z = t.double()
    m = z.max(1, keepdim=True).values
    y = (z - m) / T
    s = y.exp().sum(1, keepdim=True)
    l, d = y - s.log(), (vocab / 256 + 64) * U + EXP
    p = l.exp()
    far = torch.where(p > 0, -y, 0.0)
    mean = (p * far).sum(1, keepdim=True)
    e_logs = d + 5 * U * mean + 8 * U + 2 * U * s.log()
    e_l = e_logs + 5 * U * y.abs() + 2 * U * l.abs()
    rel = e_logs + 5 * U * far + EXP + 8 * U
    H = -(p * torch.where(p > 0, l, 0.0)).sum(1, keepdim=True)
    e_h = e_logs + (6 * d + 8 * U) * (1 + mean) + 5 * U * ((p * far * far).sum(1, keepdim=True) + mean * mean) + 12 * U + 2 * U * H
    lse, e_lse = m / T + s.log(), e_logs + 3 * U * (m / T).abs() + U * (m / T + s.log()).abs()
    f32 = lambda *n: torch.full(n, 7.0, device="cuda")
    tok = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    tok[::3] = z.argmax(1)[::3]
    at, tok = tok[:, None], tok.int()

    def near(got, want, tol, what):
        over = want.float().isinf()
        assert torch.equal(torch.where(over, got.float(), 0.0), torch.where(over, want.float(), 0.0)), what
        gap = torch.where(over, -1.0, (got.double() - want).abs() - tol)
        assert (gap <= 0).all(), (what, gap.max(), (gap > 0).nonzero()[:5])

    for k in (0, 12):
        o = dict(logp=f32(rows), entropy=f32(rows), lse=f32(rows))
        if k:
            o.update(top_ids=torch.zeros(rows, k, dtype=torch.int32, device="cuda"), top_logp=f32(rows, k))
        lp.lp_token_logprobs(t, tok, temperature=T, **o)
        near(o["logp"], l.gather(1, at)[:, 0], e_l.gather(1, at)[:, 0], "logp")
        near(o["entropy"], H[:, 0], e_h[:, 0], "entropy")
        near(o["lse"], lse[:, 0], e_lse[:, 0], "lse")
        if k:
            order = torch.sort(t.float(), dim=1, descending=True, stable=True).indices[:, :k]
            assert torch.equal(o["top_ids"].long(), order)
            near(o["top_logp"], l.gather(1, order), e_l.gather(1, order), "top_logp")
    a, b = torch.randn(rows, generator=g, device="cuda"), torch.randn(rows, generator=g, device="cuda")
    for with_b in (False, True):
        b1 = b.double()[:, None] if with_b else torch.zeros(rows, 1, dtype=torch.float64, device="cuda")
        a1 = a.double()[:, None]
        lz = torch.where(p > 0, l, 0.0)
        want = -a1 * p - b1 * p * (lz + H)
        want.scatter_add_(1, at, a1)
        k0 = a1.abs() + b1.abs() * (H + 3)
        tol = p * (rel * (k0 + b1.abs() * (lz.abs() + 3)) + b1.abs() * (torch.where(p > 0, e_l, 0.0) + e_h) + 8 * U * k0) + TINY * (k0 + 200 * b1.abs())
        tol.scatter_add_(1, at, 8 * U * (a1.abs() + k0))
        dx = torch.full_like(t, 5.0)
        lp.lp_token_logprobs_backward(t, tok, dlogp=a, dentropy=b if with_b else None, dlogits=dx, temperature=T)
        near(dx, want / T, tol / T + us * (want / T).abs() * (1 + us), ("gradient", with_b))
    some = slice(0, min(rows, 70))                          # of distillation the first rows, seven of each kind
    ids = torch.rand(rows, vocab, generator=g, device="cuda").topk(5).indices
    te = (torch.rand(rows, 5, generator=g, device="cuda") * 0.15 + 0.01).log()
    for rest in (False, True):
        loss, dx = f32(rows), torch.full_like(t, 5.0)
        lp.lp_distill(int(rest), t, ids.int(), te, loss=loss, dlogits=dx, temperature=T)
        xs, i, v = np64(t[some]), ids[some].int().cpu().numpy(), te[some].cpu().numpy()
        with np.errstate(all="ignore"):
            w_loss, w_dx = O.distill(xs, i, v.astype(np.float64), rest, T)
            tl, tg = distill_bounds(xs, bounds(xs, T), i, v, rest, T, 1.0)
        close(np64(loss)[some], w_loss, tl, ("loss", rest))
        close(np64(dx)[some], w_dx, tg + us * np.abs(w_dx) * (1 + us), ("gradient", rest))
        assert torch.isfinite(dx.float()).all()
        again = f32(rows)
        lp.lp_distill(int(rest), t, ids.int(), te, loss=again, temperature=T)
        assert torch.equal(again, loss) and not torch.isnan(loss).any()


# ------------------------------------------------------------------------------------------------ what lacks of 1
@pytest.mark.parametrize("rest", [3e-6, 1e-4, 0.02])
@pytest.mark.parametrize("k", [1, 40, 128])
def test_a_small_rest_keeps_its_digits(k, rest):
    """A teacher's rest is what its entries lack of 1.  Its entries' exponentials and their sum are in 64 bits, so that of the
    rest only the rounding to 32 bits is left; where the student has next to no probability elsewhere, the gradient there is
    the teacher's rest shared by the student's odds."""
    g = np.random.default_rng(k)
    rows, vocab, T = 6, 700, 1.0
    x = g.standard_normal((rows, vocab))
    ids = np.stack([g.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)
    np.put_along_axis(x, ids, 40.0 + g.standard_normal((rows, k)), 1)
    t = put(x, torch.float32)
    x = np64(t)
    q = g.random((rows, k)) + 0.01
    q *= (1.0 - rest) / q.sum(1, keepdims=True)
    te = np.log(q).astype(np.float32)
    lack = 1.0 - np.exp(te.astype(np.float64)).sum(1)       # of the rounded entries
    loss, dx = torch.zeros(rows, device="cuda"), torch.zeros_like(t)
    lp.lp_distill(lp.LP_DISTILL_REST, t, cu(ids, torch.int32), cu(te), loss=loss, dlogits=dx, temperature=T)
    want, w_dx = O.distill(x, ids, te.astype(np.float64), True, T)
    xo = x.copy()
    np.put_along_axis(xo, ids, -np.inf, 1)
    E = bounds(xo, T)
    # the rest rounded, the others' sum, the power, the factor of both and its product; p elsewhere, at most 1e-12, is in full
    tol = lack[:, None] * E["p"] * (E["rel"] + E["e_logs"] + 8 * U) + 1e-12 * E["p"]
    got = np64(dx)
    outside = np.isfinite(xo)
    assert (np.abs(got - w_dx) <= tol)[outside].all(), (np.abs(got / w_dx - 1) * outside).max()
    assert (lack > 2.0 ** -20).all() and np.isfinite(want).all()


# ------------------------------------------------------------------------------------------------ tokens in several entries
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab", [(3000, 300), (1300, 9000)])
def test_tokens_in_several_entries_of_many_rows(rows, vocab, rest):
    """Every block finds the doubles of row after row with the same table of claims, rows of doubles beside rows of none."""
    g = np.random.default_rng(vocab)
    k = 128
    x = g.standard_normal((rows, vocab)).astype(np.float32)
    ids = np.stack([g.permutation(vocab)[:k] for _ in range(rows)]).astype(np.int32)
    for r in range(rows):
        if r % 3:
            ids[r] = ids[r, g.integers(0, (1, 3, 60)[r % 3], k)]
    q = g.random((rows, k)) + 0.01
    te = np.log(q / q.sum(1, keepdims=True) * 0.8).astype(np.float32)
    t = cu(x)
    runs = []
    for _ in range(3):
        loss, dx = torch.zeros(rows, device="cuda"), torch.zeros_like(t)
        lp.lp_distill(int(rest), t, cu(ids, torch.int32), cu(te), loss=loss, dlogits=dx)
        runs.append((loss, dx))
    assert all(torch.equal(a, loss) and torch.equal(b, dx) for a, b in runs)
    # the doubles' weights together: rows in 64 bits
    z, at, v = t.double(), cu(ids, torch.int64), cu(te).double()
    w = v.exp() if rest else torch.softmax(v, 1)
    mass = torch.zeros_like(z).scatter_add_(1, at, w)
    inside = torch.zeros_like(z, dtype=torch.bool).scatter_(1, at, True)
    share = torch.softmax(z.masked_fill(inside, -INF), 1)
    lack = (1 - w.sum(1, keepdim=True)) if rest else torch.zeros(rows, 1, dtype=torch.float64, device="cuda")
    want = (w.sum(1, keepdim=True) + lack) * torch.softmax(z, 1) - mass - lack * share
    # p and a share: their sums' terms and powers of |y| < 10; a weight: its power of |y| < 12, its quotient, 128 additions
    d = (vocab / 256 + 64) * U + 2 * EXP + 3 * U * 24 + 16 * U
    tol = (torch.softmax(z, 1) + lack * share) * d + mass * (2 * EXP + 3 * U * 12 + 140 * U)
    assert ((dx.double() - want).abs() <= tol).all()


# ------------------------------------------------------------------------------------------------ every row of many
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,off", MANY)
def test_log_sum_exp_of_every_row_and_its_gradient(rows, vocab, pad, off, dt):
    """Rows that a block takes after its first, of all kinds in turn."""
    g, t = many_rows(rows, vocab, pad, off, dt, rows + 2)
    us, T = DT[dt][1], 1.25
    z = t.double()
    m = z.max(1, keepdim=True).values
    some = m > -INF
    y = torch.where(some, (z - m) / T, -INF)
    p = torch.softmax(y, 1).nan_to_num(0.0)
    log_s = torch.logsumexp(y, 1, keepdim=True)
    want = torch.where(some, m / T + log_s, -INF)[:, 0]
    far = torch.where(p > 0, -y, 0.0)
    mean = (p * far).sum(1, keepdim=True)
    e_logs = (vocab / 256 + 64) * U + EXP + 5 * U * mean + 8 * U + 2 * U * log_s.abs().nan_to_num(0.0, posinf=0.0)
    e_lse = (e_logs + 3 * U * (m / T).abs())[:, 0] + U * want.abs()
    for k in (0, min(5, vocab)):
        lse, o = torch.full((rows,), 7.0, device="cuda"), {}
        if k:
            o = dict(top_ids=torch.zeros(rows, k, dtype=torch.int32, device="cuda"), top_logp=torch.zeros(rows, k, device="cuda"))
        lp.lp_token_logprobs(t, lse=lse, temperature=T, **o)
        same(lse, want, torch.where(torch.isfinite(want), e_lse, 0.0), ("lse", k))
    a, b, c = (cu(g.standard_normal(rows)) for _ in range(3))
    tok = cu(g.integers(0, vocab, rows), torch.int32)
    at = tok.long()[:, None]
    l = torch.where(p > 0, y - log_s, 0.0)
    H = -(p * l).sum(1, keepdim=True)
    rel = e_logs + 5 * U * far + EXP + 8 * U
    e_h = e_logs + (6 * EXP + 6 * (vocab / 256 + 64) * U + 8 * U) * (1 + mean) + 5 * U * ((p * far * far).sum(1, keepdim=True) + mean * mean) + 12 * U + 2 * U * H
    for which in ("c", "abc"):
        a1, b1, c1 = (v.double()[:, None] if n in which else torch.zeros(rows, 1, dtype=torch.float64, device="cuda") for n, v in zip("abc", (a, b, c)))
        grad = (c1 - a1) * p - b1 * p * (l + H)
        grad.scatter_add_(1, at, a1)
        k0 = a1.abs() + c1.abs() + b1.abs() * (H + 3)
        tol = p * (rel * (k0 + b1.abs() * (l.abs() + 3)) + b1.abs() * (e_logs + 5 * U * far + 2 * U * l.abs() + e_h) + 8 * U * k0) + TINY * (k0 + 200 * b1.abs())
        tol.scatter_add_(1, at, 8 * U * (a1.abs() + k0))
        grad, tol = torch.where(some, grad, 0.0) / T, tol / T
        dx = matrix(rows, vocab, t.dtype, pad, off, 5.0)
        kw = dict(dlogp=a, dentropy=b) if which == "abc" else {}
        lp.lp_token_logprobs_backward(t, tok if kw else None, dlse=c, dlogits=dx, temperature=T, **kw)
        same(dx, grad, tol + us * grad.abs() * (1 + us), which)
        assert (between(dx) == 5.0).all()


# ------------------------------------------------------------------------------------------------ gradients that are no numbers
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("value", [INF, -INF, float("nan")])
def test_an_incoming_gradient_that_is_no_number_spoils_its_whole_row(value, dt):
    """0 times infinity is NaN for a masked token too, wherever in the row it stands and however the row is aligned."""
    g = np.random.default_rng(8)
    rows, vocab = 6, 77
    x = g.standard_normal((rows, vocab))
    x[:, g.random(vocab) < 0.4] = -np.inf
    x[:, [0, 40, 76]], x[:, 1] = -np.inf, 0.5
    x[4] = np.where(np.isinf(x[4]), -np.inf, -3.0e38)       # a far row
    x[5] = -np.inf                                          # no token: nothing comes of it
    tok = np.full(rows, 1, dtype=np.int32)
    f = lambda *v: cu(np.array(v, dtype=np.float32))
    dlogp, other, dloss = f(1, value, 2, 1, value, value), f(1, 0, value, 1, 0, 0), f(1, value, 0, 1, value, value)
    for off in range(4):
        t = put(x, DT[dt][0], 1, off)
        dx = matrix(rows, vocab, DT[dt][0], 2, off, 5.0)
        for kw, rows_spoilt in ((dict(dlogp=dlogp), (1, 4)), (dict(dlse=other), (2,)), (dict(dlogp=dlogp, dentropy=other), (1, 2, 4)),
                                (dict(dlogp=dlogp, dentropy=other, dlse=other), (1, 2, 4))):
            lp.lp_token_logprobs_backward(t, cu(tok, torch.int32), dlogits=dx, **kw)
            got = np64(dx)
            masked = np.isinf(x)
            for r in range(rows):
                bad = ~np.isfinite(got[r])
                assert bad.all() if r in rows_spoilt else not bad.any(), (off, r, tuple(kw))
                if r in rows_spoilt:
                    assert np.isnan(got[r][masked[r]]).all(), (off, r, tuple(kw))
            assert (got[5] == 0).all()
        ids, te = cu(np.array([[3, 1]] * rows), torch.int32), cu(np.log(np.full((rows, 2), 0.25)))
        for form in (lp.LP_DISTILL_TOP, lp.LP_DISTILL_REST):
            lp.lp_distill(form, t, ids, te, dlogits=dx, dloss=dloss)
            got = np64(dx)
            for r in (0, 2, 3, 5):
                assert np.isfinite(got[r]).all()
            assert np.isnan(got[1][np.isinf(x[1]) & (np.arange(vocab) != 3)]).all() and not np.isfinite(got[1]).any()


# ------------------------------------------------------------------------------------------------ few tokens to choose from
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,vocab,k", [(2000, 300, 32), (7, 9000, 128), (3, 131071, 16), (20, 200003, 128)])
def test_more_alternatives_asked_for_than_tokens_left(rows, vocab, k, dt):
    """A grammar's few tokens first, then the masked ones by ascending id, in one block and over several, whatever the mask."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(rows, vocab, generator=g, device="cuda")
    keep = torch.zeros(rows, vocab, dtype=torch.bool, device="cuda")
    for r in range(rows):
        n = (0, 1, 5, 100, 5)[r % 5]
        at = torch.randint(0, vocab, (n,), generator=g, device="cuda") if r % 5 < 3 else torch.arange(n, device="cuda") + vocab // 3
        keep[r, at.clamp(max=vocab - 1)] = True
    for mask in (-INF, -1e10, 0.0):
        t = put(np.zeros((rows, vocab)), DT[dt][0], 1, 1)
        t.copy_(torch.where(keep, x, mask))
        ids, tops = torch.zeros(rows, k, dtype=torch.int32, device="cuda"), torch.zeros(rows, k, device="cuda")
        lp.lp_token_logprobs(t, top_ids=ids, top_logp=tops)
        want = torch.sort(t.float(), dim=1, descending=True, stable=True).indices[:, :k]
        assert torch.equal(ids.long(), want), mask
        none = torch.isinf(torch.gather(t, 1, want))
        assert (tops[none] == -INF).all() and torch.isfinite(tops[~none]).all()

"""Embedding and its gradient by sorted tokens, dropout, and linear attention on the GPU against their plain 64-bit
forms (oracle/lm_ops.py), at the sizes, strides, masks and lengths where they can go wrong.

Tolerances.  u(t) = finfo(t).eps / 2 is the largest relative error of one rounding: 2^-8 for bf16, 2^-24 for fp32.  A sum
of n terms in fp32 is off by at most n * 2^-24 * sum |terms|; a stored bf16 value adds 2^-8 of itself."""
import numpy as np
import pytest
import torch

from oracle import lm_ops as O
from paper_2012_03837_b200 import binding as lp

pytestmark = pytest.mark.gpu
DT = {"fp32": (lp.LP_FP32, torch.float32, 2.0 ** -24), "bf16": (lp.LP_BF16, torch.bfloat16, 2.0 ** -8)}
U16, U32 = 2.0 ** -8, 2.0 ** -24


def cu(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype)


def np64(t):
    return t.double().cpu().numpy()


def shifted(shape, dtype, off, fill=float("nan")):
    """A tensor whose first element lies `off` elements behind an aligned address."""
    n = int(np.prod(shape))
    return torch.full((n + off,), fill, dtype=dtype, device="cuda")[off:off + n].view(shape)


# ------------------------------------------------------------------------------------------------ embedding
EMBED = [  # rows, vocab, d, T, tokens
    (1, 2, 8, 0, "uniform"), (1, 1, 1, 1, "uniform"), (7, 5, 64, 3, "uniform"), (64, 500, 520, 0, "uniform"),
    (300, 40, 33, 7, "uniform"), (513, 1000, 96, 512, "zipf"), (1000, 3, 24, 1, "uniform"), (700, 90, 1032, 50, "same"),
    (33000, 129, 8, 100, "zipf"), (2049, 200000, 16, 0, "uniform"), (33000, 7, 40, 2, "same"), (17, 30, 2056, 4, "runs"),
    (4000, 60, 12, 66, "runs"),
]


def make_ids(g, rows, vocab, kind):
    if kind == "same":
        return np.full(rows, vocab - 1, dtype=np.int32)
    if kind == "runs":                              # counts 15, 16, 17, 32, 33: around the length of a stretch
        runs = np.repeat(np.arange(5 * 40) % vocab, np.tile([15, 16, 17, 32, 33], 40))
        return np.resize(runs, rows).astype(np.int32)
    if kind == "zipf":
        w = 1.0 / np.arange(1, vocab + 1)
        return g.choice(vocab, rows, p=w / w.sum()).astype(np.int32)
    return g.integers(0, vocab, rows).astype(np.int32)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("rows,vocab,d,T,kind", EMBED)
def test_embedding_forward_and_gradient(rows, vocab, d, T, kind, off, dt):
    code, td, u = DT[dt]
    g = np.random.default_rng(rows + d)
    ids = make_ids(g, rows, vocab, kind)
    scale = 1.7
    table, pos, dout = (shifted(s, td, off) for s in ((vocab, d), (max(T, 1), d), (rows, d)))
    for x in (table, pos, dout):
        x.copy_(cu(g.standard_normal(x.shape)).to(td))
    t_ids = cu(ids, torch.int32)
    out = shifted((rows, d), td, off)
    lp.lp_embed_forward(code, t_ids, table, pos if T else None, out, rows, vocab, d, T, scale)
    p64 = np64(pos) if T else None
    want = O.embed_fwd(ids, np64(table), p64, scale)
    mag = scale * np.abs(np64(table)[ids]) + (np.abs(p64[np.arange(rows) % T]) if T else 0)
    # scale itself rounds to fp32 once, the product and sum at most once each, the store once
    assert (np.abs(np64(out) - want) <= 3 * U32 * mag + u * np.abs(want) * (1 + u)).all()

    dtab, dpos = shifted((vocab, d), torch.float32, off), shifted((max(T, 1), d), torch.float32, off)
    ws = torch.full((lp.lp_embed_workspace_bytes(rows, vocab, d),), 255, dtype=torch.uint8, device="cuda")
    args = (code, t_ids, dout, dtab, dpos if T else None, rows, vocab, d, T, scale, None, ws, ws.numel())
    lp.lp_embed_backward(*args)
    x64 = np64(dout)
    w_tab, w_pos = O.embed_bwd(ids, x64, vocab, T, scale)
    m_tab, m_pos = O.embed_bwd(ids, np.abs(x64), vocab, T, scale)
    n_tab = np.bincount(ids, minlength=vocab)[:, None]
    got = np64(dtab)
    assert (np.abs(got - w_tab) <= (n_tab + 2) * U32 * m_tab).all()
    assert (got[n_tab[:, 0] == 0] == 0).all()
    if T:
        assert (np.abs(np64(dpos) - w_pos) <= (rows / T + 2) * U32 * m_pos).all()
    first = dtab.clone(), dpos.clone()
    dtab.fill_(float("nan"))
    lp.lp_embed_backward(*args)                     # a used workspace; the same bits
    assert torch.equal(dtab, first[0]) and (not T or torch.equal(dpos, first[1]))


def test_embedding_ids_out_of_range_are_clamped_and_flagged():
    ids = cu(np.array([0, -1, 9, 4, 2 ** 31 - 1, -2 ** 31]), torch.int32)
    table = cu(np.arange(10.0).reshape(5, 2))
    out, flag = torch.empty(6, 2, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    lp.lp_embed_forward(lp.LP_FP32, ids, table, None, out, 6, 5, 2, 0, 1.0, flag)
    assert flag.item() == 1 and out[:, 0].tolist() == [0, 0, 8, 8, 8, 0]
    flag.zero_()
    dtab, ws = torch.empty(5, 2, device="cuda"), torch.empty(lp.lp_embed_workspace_bytes(6, 5, 2), dtype=torch.uint8, device="cuda")
    lp.lp_embed_backward(lp.LP_FP32, ids, torch.ones(6, 2, device="cuda"), dtab, None, 6, 5, 2, 0, 1.0, flag, ws, ws.numel())
    assert flag.item() == 1 and dtab[:, 0].tolist() == [3, 0, 0, 0, 3]
    flag.zero_()
    lp.lp_embed_forward(lp.LP_FP32, ids[:1], table, None, out, 1, 5, 2, 0, 1.0, flag)
    assert flag.item() == 0


@pytest.mark.parametrize("rows,vocab,d,T,dt,kind,off", [
    (70001, 1000, 512, 333, "bf16", "zipf", 0), (70001, 130, 512, 64, "bf16", "zipf", 1), (66000, 150000, 8, 0, "fp32", "uniform", 0),
    (66000, 131072, 8, 5, "fp32", "zipf", 3), (33333, 6, 520, 1000, "fp32", "uniform", 0), (270000, 3, 16, 700, "bf16", "same", 0),
])
def test_embedding_gradient_of_many_rows(rows, vocab, d, T, dt, kind, off):
    """Rows enough for whole batches of ids in every warp and for a gradient beyond the cache (its position sums then run
    beside the sort); ids from an unaligned address, some of them out of range; equal bits on a second call."""
    code, td, _ = DT[dt]
    g = np.random.default_rng(rows + vocab)
    ids = make_ids(g, rows, vocab, kind)
    ids[g.integers(0, rows, 9)] = -5
    ids[rows - 1] = vocab
    t_ids = shifted((rows,), torch.int32, off, 0)
    t_ids.copy_(cu(ids, torch.int32))
    dout = torch.randn(rows, d, device="cuda").to(td)
    ws = torch.full((lp.lp_embed_workspace_bytes(rows, vocab, d),), 255, dtype=torch.uint8, device="cuda")
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    runs = []
    for _ in range(2):
        dtab, dpos = torch.full((vocab, d), float("nan"), device="cuda"), torch.full((max(T, 1), d), float("nan"), device="cuda")
        lp.lp_embed_backward(code, t_ids, dout, dtab, dpos if T else None, rows, vocab, d, T, 0.5, flag, ws, ws.numel())
        runs.append((dtab, dpos))
    assert flag.item() == 1
    assert torch.equal(runs[0][0], runs[1][0]) and (not T or torch.equal(runs[0][1], runs[1][1]))
    x, at = dout.double(), t_ids.long().clamp(0, vocab - 1)
    count = torch.bincount(at, minlength=vocab)[:, None]
    zeros = lambda n: torch.zeros(n, d, dtype=torch.float64, device="cuda")
    want, mag = zeros(vocab).index_add_(0, at, x), zeros(vocab).index_add_(0, at, x.abs())
    assert ((dtab.double() - 0.5 * want).abs() <= 0.5 * (count + 2) * U32 * mag).all()
    if T:
        at = torch.arange(rows, device="cuda") % T
        want, mag = zeros(T).index_add_(0, at, x), zeros(T).index_add_(0, at, x.abs())
        assert ((dpos.double() - want).abs() <= (rows / T + 2) * U32 * mag).all()


# ------------------------------------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("n,p,resid,off,offset", [
    (1, 0.5, False, 0, 0), (3, 0.1, True, 0, 2 ** 32 - 1), (8, 0.0, True, 0, 5), (1027, 0.9, False, 1, 2 ** 33 + 7),
    (4096, 0.1, True, 0, 2 ** 64 - 3), (100003, 0.25, True, 3, 11), (700001, 0.37, False, 0, 123456789012),
    (1 << 20, 0.1, True, 8, 0)])
def test_dropout_matches_the_generator(n, p, resid, off, offset, dt):
    code, td, u = DT[dt]
    g = np.random.default_rng(n)
    seed = 0x9E3779B97F4A7C15
    x, y = shifted((n,), td, off), shifted((n,), td, off)
    x.copy_(cu(g.standard_normal(n)).to(td))
    r = cu(g.standard_normal(n)).to(td) if resid else None
    keep = O.dropout_keep(n, p, seed, offset)
    if n > 8:
        x[cu(np.flatnonzero(~keep)[:5], torch.int64)] = float("nan")      # dropped: must not reach y
    lp.lp_dropout(code, x, r, y, n, p, seed, offset)
    x64 = np.where(keep, np64(x), 0.0)
    r64 = np64(r) if resid else np.zeros(n)
    want = x64 / (1.0 - p) + r64
    mag = np.abs(x64) / (1.0 - p) + np.abs(r64)
    assert (np.abs(np64(y) - want) <= 3 * U32 * mag + u * np.abs(want) * (1 + u)).all()
    if not resid:                                   # whole mask, exactly
        assert np.array_equal(np64(y) != 0, keep & (x64 != 0))
    half = torch.tensor([offset // 2 if offset < 2 ** 63 else 17], dtype=torch.int64, device="cuda")
    y2 = x.clone() if not resid else r.clone()      # in place on x or on resid, the offset partly on the device
    lp.lp_dropout(code, x if resid else y2, y2 if resid else None, y2, n, p, seed, (offset - int(half)) % 2 ** 64, half)
    assert torch.equal(y, y2)


def test_dropout_gradient_uses_the_forward_mask():
    n, p = 5000, 0.3
    x, dy = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    lp.lp_dropout(lp.LP_FP32, x, None, y, n, p, 42, 9)
    lp.lp_dropout(lp.LP_FP32, dy, None, dx, n, p, 42, 9)
    assert torch.equal(y != 0, dx != 0)
    h = 2.0 ** -6                                   # y is linear in x: the difference quotient is exact up to rounding
    y2 = torch.empty_like(x)
    lp.lp_dropout(lp.LP_FP32, x + h * dy, None, y2, n, p, 42, 9)
    assert ((y2 - y).double() / h - dx.double()).abs().max() <= 4 * U32 * (x.abs() + dy.abs()).max().item() / (1 - p) / h


# ------------------------------------------------------------------------------------------------ linear attention
def la_inputs(B, T, H, seed, packed=False, pad=0):
    g = np.random.default_rng(seed)
    t = {}
    if packed:
        base = cu(g.standard_normal((B, T, 3, H, 64)), torch.bfloat16)
        t["q"], t["k"], t["v"] = base[:, :, 0], base[:, :, 1], base[:, :, 2]
    else:
        for n in ("q", "k", "v"):
            t[n] = cu(g.standard_normal((B, T + pad, H, 64)), torch.bfloat16)[:, :T]
    t["dout"] = cu(g.standard_normal((B, T, H, 64)), torch.bfloat16)
    lg = np.log1p(-2.0 ** -g.uniform(1.0, 10.0, H))
    lg[0] = 0.0 if seed % 2 else lg[0]
    if H > 1:
        lg[1] = -40.0 if seed % 3 else -np.inf      # powers underflow inside a chunk
    t["log_decay"] = cu(lg)
    s = cu(g.standard_normal((2, B, H, 64, 64)))
    t["state_in"], t["dstate_out"] = s[0], s[1]
    return t


def la_workspace(form, B, T, H):
    n = lp.lp_linear_attention_workspace_bytes(form, B, T, H)
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda")


def check_tokens(name, got, want, mag, lens, fill, decayed_state):
    """|error| <= 2^-8 of the output, plus 2^-8 per rounded operand of the terms it adds up: one (the scores) or two
    (the decayed k and the state), plus fp32 sums of at most 128 terms a chunk and 64 per product."""
    got = np64(got)
    for b, n in enumerate(lens):
        err = np.abs(got[b, :n] - want[b, :n])
        assert (err <= U16 * np.abs(want[b, :n]) + (2 * U16 + U16 * U16 + 2.0 ** -14) * mag[b, :n] + 1e-30).all(), (name, b, err.max())
        # the roundings are independent: in norm the error stays near one rounding's (2^-8 / sqrt(3) at most each, three of them)
        assert np.linalg.norm(err) <= U16 * np.linalg.norm(want[b, :n]) * np.sqrt(3) + 1e-30, (name, b)
        assert (got[b, n:] == fill).all(), (name, b)


LA = [  # B, T, H, packed, with states, lengths
    (1, 2, 1, False, False, None), (2, 15, 2, False, True, [15, 0]), (1, 16, 1, True, False, None), (1, 17, 2, False, True, None),
    (3, 63, 2, True, True, [63, 1, 40]), (1, 64, 3, False, False, None), (2, 65, 1, False, True, None), (1, 128, 2, True, False, None),
    (2, 130, 2, False, True, [129, 64]), (1, 700, 2, False, True, None), (1, 1030, 1, True, False, None),
    (2, 777, 3, False, True, [777, 300]), (150, 70, 2, False, False, None),
]


@pytest.mark.parametrize("B,T,H,packed,states,lengths", LA)
def test_linear_attention_forward_and_backward(B, T, H, packed, states, lengths):
    seed = B + T + H
    t = la_inputs(B, T, H, seed, packed, pad=3)
    lens = [T] * B if lengths is None else lengths
    t_len = None if lengths is None else cu(np.array(lengths), torch.int32)
    if lengths is not None:                          # what lies behind a sequence must not matter
        for b, n in enumerate(lengths):
            for x in ("q", "k", "v", "dout"):
                t[x][b, n:] = float("nan")
    q, k, v, do = (np.nan_to_num(np64(t[n])) for n in ("q", "k", "v", "dout"))
    lg, s0, ds = np64(t["log_decay"]), np64(t["state_in"]), np64(t["dstate_out"])
    scale = 0.125
    sin, dsout = (s0, ds) if states else (None, None)
    o_ref, S_ref = O.linear_attention_fwd(q, k, v, lg, scale, sin, lens)
    o_mag, S_mag = O.linear_attention_fwd(abs(q), abs(k), abs(v), lg, scale, None if sin is None else abs(sin), lens)
    o = torch.full((B, T, H, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    s_out = torch.full((B, H, 64, 64), float("nan"), device="cuda") if states else None
    desc = dict(q=t["q"], k=t["k"], v=t["v"], o=o, log_decay=t["log_decay"], scale=scale, lengths=t_len,
                state_in=t["state_in"] if states else None, state_out=s_out)
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, desc, la_workspace(lp.LP_LINATTN_FORWARD, B, T, H))
    check_tokens("o", o, o_ref, o_mag, lens, 7.0, True)
    if states:                                       # two bf16 terms: 2^-8 * 2^-8; fp32 sums over the chunks and segments
        tol = (2.0 ** -16 + (T / 64 + 70) * U32) * S_mag
        assert (np.abs(np64(s_out) - S_ref) <= tol + 1e-30).all()
        inplace = t["state_in"].clone()              # the state may be updated in place
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(desc, state_in=inplace, state_out=inplace),
                                    la_workspace(lp.LP_LINATTN_FORWARD, B, T, H))
        assert torch.equal(inplace, s_out)

    refs = O.linear_attention_bwd(q, k, v, do, lg, scale, sin, dsout, lens)
    mags = O.linear_attention_bwd(abs(q), abs(k), abs(v), abs(do), lg, scale, None if sin is None else abs(sin),
                                  None if dsout is None else abs(dsout), lens)
    if packed:
        g = torch.full((B, T, 3, H, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        grads = [g[:, :, i] for i in range(3)]
    else:
        grads = [torch.full((B, T, H, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    ds_in = torch.full((B, H, 64, 64), float("nan"), device="cuda") if states else None
    bdesc = dict(q=t["q"], k=t["k"], v=t["v"], dout=t["dout"], dq=grads[0], dk=grads[1], dv=grads[2], log_decay=t["log_decay"],
                 scale=scale, lengths=t_len, state_in=desc["state_in"], dstate_out=t["dstate_out"] if states else None, dstate_in=ds_in)
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, bdesc, la_workspace(lp.LP_LINATTN_BACKWARD, B, T, H))
    for name, got, want, mag in zip(("dq", "dk", "dv"), grads, refs, mags):
        check_tokens(name, got, want, mag, lens, 7.0, True)
    if states:
        assert (np.abs(np64(ds_in) - refs[3]) <= (2.0 ** -16 + (T / 64 + 70) * U32) * mags[3] + 1e-30).all()


@pytest.mark.parametrize("B,H,idle", [(1, 1, False), (5, 3, True), (40, 16, True)])
def test_linear_attention_step(B, H, idle):
    t = la_inputs(B, 1, H, 4 + B)
    lens = None if not idle else (np.arange(B) % 3 != 1).astype(np.int32)
    o = torch.full((B, 1, H, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    s_out = torch.full((B, H, 64, 64), float("nan"), device="cuda")
    desc = dict(q=t["q"], k=t["k"], v=t["v"], o=o, log_decay=t["log_decay"], scale=0.3, state_in=t["state_in"], state_out=s_out,
                lengths=None if lens is None else cu(lens, torch.int32))
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_STEP, desc)
    args = [np64(t[n]) for n in ("q", "k", "v")]
    lg, s0 = np64(t["log_decay"]), np64(t["state_in"])
    o_ref, S_ref = O.linear_attention_fwd(*args, lg, 0.3, s0, lens)
    o_mag, S_mag = O.linear_attention_fwd(*[abs(a) for a in args], lg, 0.3, abs(s0), lens)
    assert (np.abs(np64(s_out) - S_ref) <= 4 * U32 * S_mag + 1e-30).all()
    live = np.ones(B, bool) if lens is None else lens > 0
    err = np.abs(np64(o) - o_ref)[live]
    assert (err <= U16 * np.abs(o_ref[live]) * (1 + U16) + 70 * U32 * o_mag[live] + 1e-30).all()
    assert (np64(o)[~live] == 7.0).all()
    inplace = t["state_in"].clone()
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_STEP, dict(desc, state_in=inplace, state_out=inplace))
    assert torch.equal(inplace, s_out)
    o2 = torch.full_like(o, 7.0)                     # one token through the prompt's form: the same kernel
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(desc, o=o2, state_out=None))
    assert torch.equal(o, o2)


def test_linear_attention_later_tokens_do_not_matter():
    B, T, H = 1, 300, 2
    t = la_inputs(B, T, H, 8)
    run = lambda: [lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(q=t["q"], k=t["k"], v=t["v"], o=o, log_decay=t["log_decay"],
                   scale=0.125), la_workspace(0, B, T, H)) or o for o in [torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda")]][0]
    a = run()
    for n in ("q", "k", "v"):
        t[n][:, 150:] *= -3
    b = run()
    assert torch.equal(a[:, :150], b[:, :150]) and not torch.equal(a[:, 150:], b[:, 150:])


def test_a_prompt_then_single_tokens_equals_the_whole_sequence():
    """The operators as a model uses them: embed, drop nothing, attend over the prompt, then answer token by token from
    the state; against one pass over all tokens."""
    B, T, P, H, V = 3, 90, 77, 2, 50
    d = 64 * H
    g = np.random.default_rng(3)
    ids = cu(g.integers(0, V, (B, T)), torch.int32)
    table = cu(g.standard_normal((V, d)), torch.bfloat16)
    x = torch.empty(B, T, d, dtype=torch.bfloat16, device="cuda")
    lp.lp_embed_forward(lp.LP_BF16, ids, table, None, x, B * T, V, d, 0, 1.0)
    y = torch.empty_like(x)
    lp.lp_dropout(lp.LP_BF16, x, None, y, x.numel(), 0.0, 1)
    h = y.view(B, T, H, 64)
    lg = cu(np.log([0.97, 0.8]))
    whole, s_whole = torch.empty_like(h), torch.empty(B, H, 64, 64, device="cuda")
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(q=h, k=h, v=h, o=whole, log_decay=lg, scale=0.125, state_out=s_whole),
                                la_workspace(0, B, T, H))
    parts, state = torch.empty_like(h), torch.empty(B, H, 64, 64, device="cuda")
    pre = h[:, :P]
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(q=pre, k=pre, v=pre, o=parts[:, :P], log_decay=lg, scale=0.125, state_out=state),
                                la_workspace(0, B, P, H))
    for i in range(P, T):
        one = h[:, i:i + 1]
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_STEP, dict(q=one, k=one, v=one, o=parts[:, i:i + 1], log_decay=lg, scale=0.125,
                                                             state_in=state, state_out=state))
    x64 = np64(h)
    ref, s_ref = O.linear_attention_fwd(x64, x64, x64, np64(lg), 0.125)
    mag, s_mag = O.linear_attention_fwd(abs(x64), abs(x64), abs(x64), np64(lg), 0.125)
    for o, s in ((whole, s_whole), (parts, state)):
        check_tokens("o", o, ref, mag, [T] * B, None, True)
        assert (np.abs(np64(s) - s_ref) <= (2.0 ** -16 + 90 * U32) * s_mag).all()


# ------------------------------------------------------------------------------------------------ streams and graphs
def test_calls_on_a_side_stream_and_replayed_from_a_graph():
    B, T, H = 2, 600, 2
    d, rows, V = 64 * H, B * T, 300
    t = la_inputs(B, T, H, 12)
    ids = torch.randint(0, V, (rows,), device="cuda", dtype=torch.int32)
    out = dict(o=torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda"), dtab=torch.zeros(V, d, device="cuda"),
               y=torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda"))
    grads = {n: torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda") for n in ("dq", "dk", "dv")}
    ws = [la_workspace(0, B, T, H), la_workspace(1, B, T, H),
          torch.empty(lp.lp_embed_workspace_bytes(rows, V, d), dtype=torch.uint8, device="cuda")]
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    base = dict(q=t["q"], k=t["k"], v=t["v"], log_decay=t["log_decay"], scale=0.125)

    def chain(s):
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(base, o=out["o"]), ws[0], s)
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(base, dout=out["o"], **grads), ws[1], s)
        lp.lp_dropout(lp.LP_BF16, grads["dq"], grads["dk"], out["y"], rows * d, 0.2, 5, 0, counter, s)
        lp.lp_embed_backward(lp.LP_BF16, ids, out["y"], out["dtab"], None, rows, V, d, 0, 1.0, None, ws[2], ws[2].numel(), s)

    chain(None)
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in {**out, **grads}.items()}
    side = torch.cuda.Stream()
    for x in {**out, **grads}.values():
        x.zero_()
    side.wait_stream(torch.cuda.current_stream())
    chain(side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(want[k], v) for k, v in {**out, **grads}.items())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        chain(side.cuda_stream)
    for x in {**out, **grads}.values():
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(want[k], v) for k, v in {**out, **grads}.items())
    counter += (rows * d + 3) // 4                   # other words at the next replay
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(want["o"], out["o"]) and not torch.equal(want["y"], out["y"])


def test_host_memory_is_refused():
    x = torch.zeros(64, device="cuda")
    host = np.zeros(64, dtype=np.float32)
    with pytest.raises(lp.LpError) as e:
        lp.lp_dropout(lp.LP_FP32, x, None, host.ctypes.data, 64, 0.1, 1)
    assert e.value.code == -1
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ sizes beyond 32 bits
def test_dropout_beyond_two_to_the_31_elements():
    n, p, seed, tail = 2 ** 31 + 19, 0.25, 7, 4096
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    lp.lp_dropout(lp.LP_BF16, x, None, x, n, p, seed, 3)
    first = (n - tail) // 4 * 4                      # a whole counter
    keep = O.dropout_keep(n - first, p, seed, 3 + first // 4)
    assert np.array_equal(np64(x[first:]) != 0, keep)
    assert np.array_equal(np64(x[:tail]) != 0, O.dropout_keep(tail, p, seed, 3))


def test_embedding_tables_beyond_two_to_the_31_elements():
    V, d, rows = 2 ** 22 + 5, 520, 40                # 2.2e9 elements
    table = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    g = np.random.default_rng(0)
    ids = np.concatenate([[0, V - 1, V - 1, 5, V - 2], g.integers(V - 1000, V, rows - 5)]).astype(np.int32)
    t_ids = cu(ids, torch.int32)
    used = torch.unique(t_ids).long()
    table[used] = torch.randn(len(used), d, device="cuda").to(torch.bfloat16)
    out = torch.empty(rows, d, dtype=torch.bfloat16, device="cuda")
    lp.lp_embed_forward(lp.LP_BF16, t_ids, table, None, out, rows, V, d, 0, 1.0)
    assert torch.equal(out, table[t_ids.long()])
    del table
    dtab = torch.full((V, d), float("nan"), device="cuda")
    ws = torch.empty(lp.lp_embed_workspace_bytes(rows, V, d), dtype=torch.uint8, device="cuda")
    lp.lp_embed_backward(lp.LP_BF16, t_ids, out, dtab, None, rows, V, d, 0, 1.0, None, ws, ws.numel())
    want = torch.zeros(len(used), d, device="cuda", dtype=torch.float64)
    want.index_add_(0, torch.searchsorted(used, t_ids.long()), out.double())
    assert ((dtab[used].double() - want).abs() <= 1e-6 * want.abs() + 1e-6).all()
    assert not torch.isnan(dtab).any() and int((dtab != 0).any(dim=1).sum()) == len(used)


def test_linear_attention_strides_beyond_two_to_the_31_elements():
    T, H, ts = 100, 1, 2 ** 25                       # the last token lies 3.3e9 elements behind the first
    t = la_inputs(1, T, H, 21)
    big = torch.empty(T * ts, dtype=torch.bfloat16, device="cuda").view(1, T, ts)
    far = {}
    for i, n in enumerate(("q", "k", "v", "dout", "o", "dq", "dk", "dv")):
        far[n] = big[:, :, 64 * i:64 * i + 64].view(1, T, 1, 64)
        if n in t:
            far[n].copy_(t[n])
    near = {n: torch.empty(1, T, H, 64, dtype=torch.bfloat16, device="cuda") for n in ("o", "dq", "dk", "dv")}
    for src, outs in ((far, far), (t, near)):
        base = dict(q=src["q"], k=src["k"], v=src["v"], log_decay=t["log_decay"], scale=0.125)
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(base, o=outs["o"]), la_workspace(0, 1, T, H))
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(base, dout=src["dout"], dq=outs["dq"], dk=outs["dk"], dv=outs["dv"]),
                                    la_workspace(1, 1, T, H))
    for n in near:
        assert torch.equal(far[n], near[n]), n


# ------------------------------------------------------------------------------------------------ two calls at once, layouts
def test_two_streams_with_workspaces_of_their_own():
    B, T, H, rows, V, d = 1, 3000, 2, 9000, 700, 136
    t = la_inputs(B, T, H, 30)
    ids = torch.randint(0, V, (rows,), device="cuda", dtype=torch.int32)
    dh = torch.randn(rows, d, device="cuda").to(torch.bfloat16)
    res = []
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s in streams:
        o, st = torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, H, 64, 64, device="cuda")
        dtab = torch.zeros(V, d, device="cuda")
        res.append((o, st, dtab, la_workspace(0, B, T, H), torch.empty(lp.lp_embed_workspace_bytes(rows, V, d), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (o, st, dtab, w1, w2) in zip(streams, res):
            lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(q=t["q"], k=t["k"], v=t["v"], o=o, state_out=st, log_decay=t["log_decay"],
                                        scale=0.125), w1, s.cuda_stream)
            lp.lp_embed_backward(lp.LP_BF16, ids, dh, dtab, None, rows, V, d, 0, 1.0, None, w2, w2.numel(), s.cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(res[0][:3], res[1][:3]):
        assert torch.equal(a, b) and a.abs().sum() > 0


def test_linear_attention_on_sequence_first_tensors():
    """[seq_len, batch, n_heads, 64] storage: the batch stride is smaller than a token's."""
    B, T, H = 3, 150, 2
    t = la_inputs(B, T, H, 5)
    seq = {n: t[n].transpose(0, 1).contiguous().transpose(0, 1) for n in ("q", "k", "v")}
    o1 = torch.zeros(T, B, H, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    o2 = torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda")
    for src, o in ((seq, o1), (t, o2)):
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(q=src["q"], k=src["k"], v=src["v"], o=o, log_decay=t["log_decay"], scale=0.1),
                                    la_workspace(0, B, T, H))
    assert torch.equal(o1, o2)


def test_a_state_updated_in_place_through_segments_and_a_backward_in_a_graph():
    """Long prompts of few heads are cut into segments; the state is read and written in place, and the gradient with
    respect to the incoming state overwrites the outgoing one's, in a captured call that is replayed."""
    B, T, H = 1, 2100, 2
    t = la_inputs(B, T, H, 17)
    state, grad = t["state_in"].clone(), t["dstate_out"].clone()
    o = torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda")
    g = {n: torch.zeros_like(o) for n in ("dq", "dk", "dv")}
    ws = la_workspace(0, B, T, H), la_workspace(1, B, T, H)
    assert ws[0].numel() > 0 and ws[1].numel() > 0
    base = dict(q=t["q"], k=t["k"], v=t["v"], log_decay=t["log_decay"], scale=0.125)
    keep = state.clone()

    def calls(s):
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(base, dout=t["dout"], state_in=state, dstate_out=grad, dstate_in=grad, **g), ws[1], s)
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(base, o=o, state_in=state, state_out=state), ws[0], s)

    q, k, v, do = (np64(t[n]) for n in ("q", "k", "v", "dout"))
    lg = np64(t["log_decay"])
    refs = O.linear_attention_bwd(q, k, v, do, lg, 0.125, np64(state), np64(grad))
    mags = O.linear_attention_bwd(abs(q), abs(k), abs(v), abs(do), lg, 0.125, abs(np64(state)), abs(np64(grad)))
    s_ref = O.linear_attention_fwd(q, k, v, lg, 0.125, np64(state))[1]
    s_mag = O.linear_attention_fwd(abs(q), abs(k), abs(v), lg, 0.125, abs(np64(state)))[1]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        calls(stream.cuda_stream)
    for _ in range(2):
        state.copy_(keep)
        grad.copy_(t["dstate_out"])
        graph.replay()
    torch.cuda.synchronize()
    assert (np.abs(np64(grad) - refs[3]) <= (2.0 ** -16 + (T / 64 + 70) * U32) * mags[3] + 1e-30).all()
    assert (np.abs(np64(state) - s_ref) <= (2.0 ** -16 + (T / 64 + 70) * U32) * s_mag + 1e-30).all()
    for n, r, m in zip(("dq", "dk", "dv"), refs, mags):
        check_tokens(n, g[n], r, m, [T], None, True)


def test_linear_attention_does_not_depend_on_what_shared_memory_held():
    """Backwards in time the last chunk of a length that is no multiple of 64 has absent tokens; their weights come from a
    table, and what an earlier kernel left in shared memory must not pass for one."""
    a = torch.full((4096, 4096), float("nan"), device="cuda")
    for B, T, H in ((2, 70, 2), (1, 1029, 1), (2, 2, 1)):
        t = la_inputs(B, T, H, 3)
        outs = []
        for dirty in (False, True):
            if dirty:
                torch.matmul(a, a)
                torch.softmax(a, dim=1)
                torch.matmul(a.to(torch.bfloat16), a.to(torch.bfloat16))
            g = [torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
            ds = torch.zeros(B, H, 64, 64, device="cuda")
            lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(q=t["q"], k=t["k"], v=t["v"], dout=t["dout"], dq=g[0], dk=g[1], dv=g[2],
                                        log_decay=t["log_decay"], scale=0.125, state_in=t["state_in"], dstate_out=t["dstate_out"], dstate_in=ds),
                                        la_workspace(1, B, T, H))
            outs.append(g + [ds])
        assert all(torch.equal(x, y) and torch.isfinite(x).all() for x, y in zip(*outs))


@pytest.mark.parametrize("T", [1, 9, 64, 70, 130, 512])
def test_the_states_gradient_may_overwrite_the_one_it_came_from(T):
    """dstate_in in dstate_out's buffer, for sequences that are not cut into segments: dk's scans still read the gradient of
    the outgoing state, whatever dv's scans have written by then.  The same bits as from a buffer of its own, many times."""
    B, H = 20, 16
    t = la_inputs(B, T, H, 40 + T)
    lens = np.array([T if b % 3 else (b * 7) % (T + 1) for b in range(B)], dtype=np.int32)
    assert lp.lp_linear_attention_workspace_bytes(lp.LP_LINATTN_BACKWARD, B, T, H) == 0
    base = dict(q=t["q"], k=t["k"], v=t["v"], dout=t["dout"], log_decay=t["log_decay"], scale=0.125, state_in=t["state_in"],
                lengths=cu(lens, torch.int32))
    grads = lambda: {n: torch.full((B, T, H, 64), 7.0, dtype=torch.bfloat16, device="cuda") for n in ("dq", "dk", "dv")}
    want, s_want = grads(), torch.full((B, H, 64, 64), float("nan"), device="cuda")
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(base, dstate_out=t["dstate_out"], dstate_in=s_want, **want))
    for _ in range(8):
        got, s = grads(), t["dstate_out"].clone()
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(base, dstate_out=s, dstate_in=s, **got))
        assert torch.equal(s, s_want)
        for n in want:
            assert torch.equal(got[n], want[n]), n
    if T == 9:                                       # and the buffers of their own hold the formula's values
        q, k, v, do = (np64(t[n]) for n in ("q", "k", "v", "dout"))
        args = np64(t["log_decay"]), 0.125
        refs = O.linear_attention_bwd(q, k, v, do, *args, np64(t["state_in"]), np64(t["dstate_out"]), lens)
        mags = O.linear_attention_bwd(abs(q), abs(k), abs(v), abs(do), *args, abs(np64(t["state_in"])), abs(np64(t["dstate_out"])), lens)
        for i, n in enumerate(("dq", "dk", "dv")):
            check_tokens(n, got[n], refs[i], mags[i], lens, 7.0, True)


@pytest.mark.parametrize("lg", [float(np.finfo(np.float32).min), -1e37, -2e36, -200.0])
@pytest.mark.parametrize("B,T,H", [(2, 9, 2), (1, 64, 1), (3, 130, 2), (20, 1100, 6), (1, 2100, 1)])
def test_decays_whose_powers_overflow_their_exponent(B, T, H, lg):
    """exp of anything below -104 is 0 in fp32, so such a decay is one of minus infinity, bit for bit, also where a multiple of
    it is no finite number any more; in one chunk, in several, in segments."""
    t = la_inputs(B, T, H, 90 + T)
    outs = []
    for value in (lg, -np.inf):
        o = {n: torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda") for n in ("o", "dq", "dk", "dv")}
        s, ds = torch.zeros(B, H, 64, 64, device="cuda"), torch.zeros(B, H, 64, 64, device="cuda")
        base = dict(q=t["q"], k=t["k"], v=t["v"], scale=0.125, state_in=t["state_in"], log_decay=torch.full((H,), value, device="cuda"))
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(base, o=o["o"], state_out=s), la_workspace(0, B, T, H))
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(base, dout=t["dout"], dq=o["dq"], dk=o["dk"], dv=o["dv"],
                                    dstate_out=t["dstate_out"], dstate_in=ds), la_workspace(1, B, T, H))
        outs.append([*o.values(), s, ds])
    for a, b in zip(*outs):
        assert torch.isfinite(a).all() and torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ states handed out, fp32
def two_terms(x):
    """x as the sum of two bf16 numbers, which is how operands are split where no state leaves."""
    hi = torch.tensor(x, dtype=torch.float32).to(torch.bfloat16).float()
    return (hi + (torch.tensor(x, dtype=torch.float32) - hi).to(torch.bfloat16).float()).item()


@pytest.mark.parametrize("B,T,H", [(1, 20, 1), (2, 70, 1), (10, 1100, 12), (1, 2100, 1)])
def test_states_handed_out_are_exact_to_fp32(B, T, H):
    """One chunk, several, many, segments.  The factors are chosen so that two bf16 terms would be off by 2^-17: an exact
    16 * scale (all ones in 16 tokens, no decay: every partial sum has at most 22 bits), and one power of the decay, where
    expf is off by 2 units in the last place at most (2^-22) and its correction by one rounding."""
    scale = 1.0 + 2.0 ** -9 + 2.0 ** -17
    assert abs(two_terms(scale) - scale) == 2.0 ** -17
    tok = lambda: torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda")
    state = lambda: torch.full((B, H, 64, 64), float("nan"), device="cuda")
    ones, s = tok(), state()
    ones[:, 2:18] = 1
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(q=ones, k=ones, v=ones, dout=ones, dq=tok(), dk=tok(), dv=tok(),
                                log_decay=torch.zeros(H, device="cuda"), scale=scale, dstate_in=s), la_workspace(1, B, T, H))
    assert (s == 16 * scale).all()
    lg = torch.tensor(np.log(0.5 * scale), dtype=torch.float32).item()
    l = float(np.exp(np.float64(lg)))
    assert abs(two_terms(l) - l) > 2.0 ** -18 * l
    one, s = tok(), state()
    one[:, T - 2] = 1
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(q=one, k=one, v=one, o=tok(), log_decay=torch.full((H,), lg, device="cuda"),
                                scale=1.0, state_out=s), la_workspace(0, B, T, H))
    assert (np.abs(np64(s) - l) <= 2.0 ** -21 * l).all()


# ------------------------------------------------------------------------------------------------ position sums beside the sort
def test_position_sums_beside_the_sort_on_side_streams_and_in_graphs():
    """More than 64 MiB of incoming gradient: the position sums start while the sort runs.  They come behind what wrote the
    gradient and before what reads theirs, on two side streams at once and in replays of a graph, where another branch joins
    in front of them."""
    rows, vocab, d, T = 70001, 1000, 512, 333
    g = np.random.default_rng(1)
    ids = cu(make_ids(g, rows, vocab, "zipf"), torch.int32)
    x = torch.randn(rows, d, device="cuda").to(torch.bfloat16)
    n = rows * d

    def call(b, s):                                  # writes b's gradient, sums it, takes the sums on
        lp.lp_dropout(lp.LP_BF16, x, None, b["dh"], n, 0.3, 8, 0, b["word"], s)
        lp.lp_embed_backward(lp.LP_BF16, ids, b["dh"], b["dtab"], b["dpos"], rows, vocab, d, T, 0.5, None, b["ws"], b["ws"].numel(), s)
        lp.lp_dropout(lp.LP_FP32, b["dpos"], None, b["pos_out"], T * d, 0.0, 1, 0, None, s)
        lp.lp_dropout(lp.LP_FP32, b["dtab"], None, b["tab_out"], vocab * d, 0.0, 1, 0, None, s)

    def buffers():
        f = lambda *shape: torch.full(shape, float("nan"), device="cuda")
        return dict(dh=torch.full((rows, d), float("nan"), dtype=torch.bfloat16, device="cuda"), dtab=f(vocab, d), dpos=f(T, d), tab_out=f(vocab, d),
                    pos_out=f(T, d), word=torch.zeros(1, dtype=torch.int64, device="cuda"),
                    ws=torch.full((lp.lp_embed_workspace_bytes(rows, vocab, d),), 255, dtype=torch.uint8, device="cuda"))

    def want(word):
        b = buffers()
        b["word"] += word
        call(b, None)
        torch.cuda.synchronize()
        at = torch.arange(rows, device="cuda") % T
        ref = torch.zeros(T, d, dtype=torch.float64, device="cuda").index_add_(0, at, b["dh"].double())
        mag = torch.zeros(T, d, dtype=torch.float64, device="cuda").index_add_(0, at, b["dh"].double().abs())
        assert ((b["pos_out"].double() - ref).abs() <= (rows / T + 2) * U32 * mag).all()
        return b["pos_out"], b["tab_out"]

    first, second = want(0), want(999)
    assert not torch.equal(first[0], second[0])
    streams, sets = [torch.cuda.Stream(), torch.cuda.Stream()], [buffers(), buffers()]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, b in zip(streams, sets):
            call(b, s.cuda_stream)
    torch.cuda.synchronize()
    for b in sets:
        assert torch.equal(b["pos_out"], first[0]) and torch.equal(b["tab_out"], first[1])
    b, graph, other = sets[0], torch.cuda.CUDAGraph(), streams[1]
    with torch.cuda.graph(graph, stream=streams[0]):
        other.wait_stream(streams[0])
        with torch.cuda.stream(other):
            b["word"] += 999
        streams[0].wait_stream(other)
        call(b, streams[0].cuda_stream)
    for k in ("dh", "dtab", "dpos", "pos_out", "tab_out"):
        b[k].fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(b["pos_out"], second[0]) and torch.equal(b["tab_out"], second[1])
    b["word"].fill_(-999)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(b["pos_out"], first[0]) and torch.equal(b["tab_out"], first[1])


def test_a_state_gradient_overwritten_in_a_replayed_graph():
    B, T, H = 8, 70, 16
    t = la_inputs(B, T, H, 77)
    g = [torch.zeros(B, T, H, 64, dtype=torch.bfloat16, device="cuda") for _ in range(6)]
    ds, inplace = torch.zeros(B, H, 64, 64, device="cuda"), t["dstate_out"].clone()
    base = dict(q=t["q"], k=t["k"], v=t["v"], dout=t["dout"], log_decay=t["log_decay"], scale=0.125, state_in=t["state_in"])
    lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(base, dq=g[0], dk=g[1], dv=g[2], dstate_out=t["dstate_out"], dstate_in=ds))
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        lp.lp_linear_attention_bf16(lp.LP_LINATTN_BACKWARD, dict(base, dq=g[3], dk=g[4], dv=g[5], dstate_out=inplace, dstate_in=inplace), None,
                                    stream.cuda_stream)
    for _ in range(3):
        inplace.copy_(t["dstate_out"])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(inplace, ds)
        for a, b in zip(g[:3], g[3:]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("rows,vocab,d,T,dt,kind", [
    (66001, 500, 513, 7, "bf16", "zipf"), (40003, 300, 421, 333, "fp32", "uniform"), (40003, 300, 421, 2, "fp32", "same"),
    (4300001, 3, 8, 1, "bf16", "zipf"), (17000000, 40, 1, 100, "fp32", "uniform")])
def test_position_sums_beside_the_sort_of_odd_and_narrow_widths(rows, vocab, d, T, dt, kind):
    """Widths that take one element at a time, few lanes a row, a single position."""
    code, td, _ = DT[dt]
    ids = cu(make_ids(np.random.default_rng(rows), rows, vocab, kind), torch.int32)
    dout = torch.randn(rows, d, device="cuda").to(td)
    ws = torch.full((lp.lp_embed_workspace_bytes(rows, vocab, d),), 255, dtype=torch.uint8, device="cuda")
    runs = []
    for _ in range(2):
        dtab, dpos = torch.full((vocab, d), float("nan"), device="cuda"), torch.full((T, d), float("nan"), device="cuda")
        lp.lp_embed_backward(code, ids, dout, dtab, dpos, rows, vocab, d, T, 0.5, None, ws, ws.numel())
        runs.append((dtab, dpos))
    assert torch.equal(runs[0][0], runs[1][0]) and torch.equal(runs[0][1], runs[1][1])
    x = dout.double()
    for got, at, n, scale in ((dtab, ids.long(), vocab, 0.5), (dpos, torch.arange(rows, device="cuda") % T, T, 1.0)):
        count = torch.bincount(at, minlength=n)[:, None]
        want = torch.zeros(n, d, dtype=torch.float64, device="cuda").index_add_(0, at, x)
        mag = torch.zeros(n, d, dtype=torch.float64, device="cuda").index_add_(0, at, x.abs())
        assert ((got.double() - scale * want).abs() <= scale * (count + 2) * U32 * mag).all()


FIRST_CALLS = """
import sys
sys.path.insert(0, sys.argv[1])
import torch
from paper_2012_03837_b200 import binding as lp
B, T, H, V = 2, 2100, 2, 300
rows, d = B * T, 64 * H
bf = dict(dtype=torch.bfloat16, device="cuda")
x, g, o = torch.randn(B, T, H, 64, **bf), [torch.zeros(B, T, H, 64, **bf) for _ in range(4)], torch.zeros(rows, d, **bf)
ids, table, dtab = torch.randint(0, V, (rows,), device="cuda", dtype=torch.int32), torch.randn(V, d, **bf), torch.zeros(V, d, device="cuda")
state, lg = torch.zeros(B, H, 64, 64, device="cuda"), torch.full((H,), -0.01, device="cuda")
ws = [torch.empty(max(256, n), dtype=torch.uint8, device="cuda") for n in (
    lp.lp_linear_attention_workspace_bytes(0, B, T, H), lp.lp_linear_attention_workspace_bytes(1, B, T, H), lp.lp_embed_workspace_bytes(rows, V, d))]

def calls(s):
    lp.lp_embed_forward(lp.LP_BF16, ids, table, None, o, rows, V, d, 0, 1.5, None, s)
    lp.lp_linear_attention_bf16(0, dict(q=x, k=x, v=x, o=g[0], log_decay=lg, state_out=state), ws[0], s)
    lp.lp_linear_attention_bf16(1, dict(q=x, k=x, v=x, dout=g[0], dq=g[1], dk=g[2], dv=g[3], log_decay=lg), ws[1], s)
    lp.lp_dropout(lp.LP_BF16, g[1], o, o, rows * d, 0.1, 3, 0, None, s)
    lp.lp_embed_backward(lp.LP_BF16, ids, o, dtab, None, rows, V, d, 0, 1.0, None, ws[2], ws[2].numel(), s)

stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=stream):
    calls(stream.cuda_stream)
graph.replay()
torch.cuda.synchronize()
first = [t.clone() for t in g + [o, dtab, state]]
calls(torch.cuda.current_stream().cuda_stream)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(first, g + [o, dtab, state])) and dtab.abs().sum() > 0
print("equal")
"""


def test_the_very_first_calls_may_be_captured():
    """A process whose first calls of the operators are captured ones: kernels are loaded and limits raised meanwhile."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS, root], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "equal" in r.stdout, r.stdout + r.stderr

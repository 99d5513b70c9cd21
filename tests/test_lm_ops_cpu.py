"""The operators next to the transformer's layers without a GPU: their plain forms pinned by known answers, finite
differences and identities, and the refusals of the library's entry points."""
import ctypes as C

import numpy as np
import pytest

from oracle import lm_ops as O
from paper_2012_03837_b200 import binding as lp

ERR = {v: k for k, v in lp.LP_ERR.items()}


def test_philox_known_answers():
    """The published test vectors of Philox4x32-10."""
    f = 0xFFFFFFFF
    for ctr, key, want in [
            ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((f, f, f, f), (f, f), (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
             (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]:
        assert tuple(int(x) for x in O.philox4x32(ctr, key)) == want


def test_dropout_mask_is_a_function_of_the_counter():
    a = O.dropout_keep(1000, 0.3, 99, 5)
    assert np.array_equal(a[40:], O.dropout_keep(960, 0.3, 99, 15))             # ten counters on
    assert np.array_equal(O.dropout_keep(37, 0.3, 99, 5), a[:37])
    assert O.dropout_keep(1000, 0.0, 1).all()
    assert np.array_equal(O.dropout_keep(64, 0.5, 3, 2 ** 64 - 2)[8:], O.dropout_keep(56, 0.5, 3, 0))   # wraps
    n, p = 200000, 0.1
    kept = O.dropout_keep(n, p, 12345).mean()
    assert abs(kept - 0.9) < 6 * np.sqrt(p * (1 - p) / n)


def test_embedding_gradient_is_the_transpose_of_the_lookup():
    g = np.random.default_rng(0)
    ids = np.array([3, 0, 3, -2, 9, 3, 1])                                      # -2 and 9 are clamped into five tokens
    table, pos, dh = g.standard_normal((5, 4)), g.standard_normal((3, 4)), g.standard_normal((7, 4))
    dt, dp = O.embed_bwd(ids, dh, 5, 3, 0.7)
    f = lambda t, p: (O.embed_fwd(ids, t, p, 0.7) * dh).sum()
    dx, dy = g.standard_normal(table.shape), g.standard_normal(pos.shape)
    assert np.isclose(f(table + dx, pos + dy) - f(table, pos), (dt * dx).sum() + (dp * dy).sum())


@pytest.mark.parametrize("lengths", [None, [3, 0]])
def test_linear_attention_gradients_match_differences(lengths):
    g = np.random.default_rng(1)
    B, T, H = 2, 5, 2
    x = {n: g.standard_normal((B, T, H, 64)) for n in ("q", "k", "v", "do")}
    s0, ds = g.standard_normal((B, H, 64, 64)), g.standard_normal((B, H, 64, 64))
    lg = np.array([-0.3, 0.0])

    def f(q, k, v, s):
        o, S = O.linear_attention_fwd(q, k, v, lg, 0.125, s, lengths)
        return (o * x["do"]).sum() + (S * ds).sum()

    grads = O.linear_attention_bwd(x["q"], x["k"], x["v"], x["do"], lg, 0.125, s0, ds, lengths)
    args = [x["q"], x["k"], x["v"], s0]
    for i, gr in enumerate(grads):
        d = g.standard_normal(args[i].shape)
        h = 1e-4
        up = [a + (h * d if j == i else 0) for j, a in enumerate(args)]
        dn = [a - (h * d if j == i else 0) for j, a in enumerate(args)]
        num = (f(*up) - f(*dn)) / (2 * h)
        assert abs(num - (gr * d).sum()) <= 1e-6 * max(1.0, abs(num)), i


def test_linear_attention_without_decay_is_unnormalised_attention():
    g = np.random.default_rng(2)
    q, k, v = (g.standard_normal((1, 9, 1, 64)) for _ in range(3))
    o, S = O.linear_attention_fwd(q, k, v, [0.0], 0.5)
    w = np.tril(q[0, :, 0] @ k[0, :, 0].T) * 0.5
    assert np.allclose(o[0, :, 0], w @ v[0, :, 0]) and np.allclose(S[0, 0], k[0, :, 0].T @ v[0, :, 0])
    o, _ = O.linear_attention_fwd(q, k, v, [-np.inf], 0.5)                      # a token sees itself only
    assert np.allclose(o[0, :, 0], np.diag(np.diag(w)) @ v[0, :, 0])


# ---- refusals: answered before anything touches a GPU
ONE = C.c_void_p(256)
ODD = C.c_void_p(257)


def test_embedding_entries_check_their_arguments():
    L = lp._lib
    fwd = lambda dt=1, ids=ONE, tab=ONE, pos=None, out=ONE, rows=4, vocab=8, d=16, T=0: \
        L.lp_embed_forward(dt, ids, tab, pos, out, rows, vocab, d, T, 1.0, None, None)
    assert fwd(dt=2) == ERR["INVALID_ARG"]
    assert fwd(ids=None) == fwd(tab=None) == fwd(out=None) == ERR["INVALID_ARG"]
    assert fwd(rows=0) == fwd(vocab=0) == fwd(d=0) == fwd(pos=ONE, T=0) == fwd(rows=(1 << 30) + 1) == ERR["SHAPE"]
    assert fwd(out=ODD) == fwd(ids=C.c_void_p(258)) == fwd(dt=0, tab=C.c_void_p(258)) == ERR["UNSUPPORTED"]
    need = lp.lp_embed_workspace_bytes(4, 8, 16)
    assert need > 0 and lp.lp_embed_workspace_bytes(0, 8, 16) == lp.lp_embed_workspace_bytes(4, -1, 16) == 0
    bwd = lambda dt=1, ids=ONE, dout=ONE, dtab=ONE, dpos=None, rows=4, T=0, ws=ONE, n=need: \
        L.lp_embed_backward(dt, ids, dout, dtab, dpos, rows, 8, 16, T, 1.0, None, ws, n, None)
    assert bwd(dt=-1) == bwd(ids=None) == bwd(dout=None) == bwd(dtab=None) == bwd(ws=None) == bwd(n=need - 1) == ERR["INVALID_ARG"]
    assert b"workspace" in L.lp_last_error(None)
    assert bwd(rows=-3) == bwd(dpos=ONE, T=0) == ERR["SHAPE"]
    assert bwd(dtab=ODD) == bwd(ws=C.c_void_p(128)) == ERR["UNSUPPORTED"]


def test_dropout_entry_checks_its_arguments():
    L = lp._lib
    call = lambda dt=1, x=ONE, r=None, y=ONE, n=8, p=0.1, od=None: L.lp_dropout(dt, x, r, y, n, p, 1, 0, od, None)
    assert call(dt=3) == call(x=None) == call(y=None) == ERR["INVALID_ARG"]
    for p in (-0.1, 1.0, 2.0, float("nan")):
        assert call(p=p) == ERR["INVALID_ARG"], p
    assert call(n=-1) == ERR["SHAPE"] and call(n=0) == lp.LP_OK
    assert call(x=ODD) == call(r=ODD) == call(od=C.c_void_p(260)) == ERR["UNSUPPORTED"]


def linattn(form=0, ws=None, nbytes=0, **kw):
    d = lp.lp_linattn_desc()
    at = dict(q=0x1000, k=0x2000, v=0x3000, o=0x4000, dout=0x5000, dq=0x6000, dk=0x7000, dv=0x8000)
    at.update({k: kw.pop(k) for k in list(kw) if k in at})
    H = kw.get("n_heads", 2)
    for name, p in at.items():
        t = getattr(d, name)
        t.p, t.batch_stride, t.token_stride = p, kw.pop(name + "_bs", 64 * H * 8), kw.pop(name + "_ts", 64 * H)
    base = dict(log_decay=0x9000, batch=2, seq_len=8, n_heads=2, scale=0.125)
    base.update(kw)
    for k, v in base.items():
        setattr(d, k, v)
    return lp._lib.lp_linear_attention_bf16(form, C.byref(d), ws, nbytes, None)


def test_linear_attention_entry_checks_its_arguments():
    F, B, S = lp.LP_LINATTN_FORWARD, lp.LP_LINATTN_BACKWARD, lp.LP_LINATTN_STEP
    assert lp._lib.lp_linear_attention_bf16(F, None, None, 0, None) == ERR["INVALID_ARG"]
    assert linattn(3) == linattn(-1) == ERR["INVALID_ARG"]
    for name in ("q", "k", "v", "o", "log_decay"):
        assert linattn(F, **{name: None}) == ERR["INVALID_ARG"], name
    for name in ("dout", "dq", "dk", "dv"):
        assert linattn(B, **{name: None}) == ERR["INVALID_ARG"], name
    assert linattn(F, batch=0) == linattn(F, seq_len=0) == linattn(F, n_heads=-1) == linattn(S) == ERR["SHAPE"]
    assert linattn(F, batch=1 << 20) == linattn(F, q_ts=64) == linattn(F, o_bs=64) == linattn(F, k_bs=-128) == ERR["SHAPE"]
    assert linattn(F, q=0x1008) == linattn(F, v_ts=132) == linattn(F, o_bs=1025) == linattn(F, state_in=0xa008) == ERR["UNSUPPORTED"]
    assert linattn(B, dstate_in=0xa004) == ERR["UNSUPPORTED"]
    assert linattn(F, o=0x1000) == linattn(B, dq=0x5000) == linattn(B, dk=0x6000) == ERR["INVALID_ARG"]
    assert linattn(B, state_in=0xa000, dstate_in=0xa000) == linattn(F, scale=float("nan")) == ERR["INVALID_ARG"]
    # long sequences of few heads are cut into segments whose states need room
    need = lp.lp_linear_attention_workspace_bytes(F, 1, 8192, 2)
    assert need > 0 and lp.lp_linear_attention_workspace_bytes(B, 1, 8192, 2) >= need
    assert lp.lp_linear_attention_workspace_bytes(S, 1, 1, 2) == lp.lp_linear_attention_workspace_bytes(F, 0, 8, 2) == 0
    assert linattn(F, batch=1, seq_len=8192) == ERR["INVALID_ARG"]
    assert linattn(F, ws=ONE, nbytes=need - 1, batch=1, seq_len=8192) == ERR["INVALID_ARG"]
    assert linattn(F, ws=C.c_void_p(16), nbytes=need, batch=1, seq_len=8192) == ERR["UNSUPPORTED"]


def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    x = torch.zeros(8)
    with pytest.raises(lp.LpError) as e:
        lp.lp_dropout(lp.LP_FP32, x, None, x, 8, 0.1, 1)
    assert e.value.code == ERR["INVALID_ARG"]
    t = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
    for bad in (t[:, :, :, :32], t.float(), t[:, :2]):
        with pytest.raises(lp.LpError) as e:
            lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, dict(q=t, k=bad, v=t, o=t, scale=1.0))
        assert e.value.code in (ERR["SHAPE"], ERR["INVALID_ARG"])


def test_binding_refuses_wrong_types_and_names():
    """Tensors of another type would be read as what they are not."""
    import torch
    t = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
    good = dict(q=t, k=t, v=t, o=t, log_decay=torch.zeros(2))
    for change in (dict(log_decay=torch.zeros(2, dtype=torch.int32)), dict(log_decay=torch.zeros(1)), dict(lengths=torch.zeros(2)),
                   dict(lengths=torch.zeros(2, dtype=torch.int64)), dict(state_in=torch.zeros(2, 2, 64, 64, dtype=torch.int32)),
                   dict(state_out=torch.zeros(2, 64, 2, 64).transpose(1, 2)), dict(q=None), dict(q=t[0]), dict(mask=t)):
        with pytest.raises(lp.LpError) as e:
            lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, {**good, **change})
        assert e.value.code in (ERR["SHAPE"], ERR["INVALID_ARG"])
        assert "CUDA" not in str(e.value) and "device" not in str(e.value)


# ---- the training step with dropout: the oracle's gradients against differences, and its refusals
def test_oracle_gradients_with_dropout_match_differences():
    import lp_synth
    from oracle.local_step import LocalUpdateOracle
    cfg = lp_synth.config("c3", batch=2, seq_len=5, vocab=11, d_model=8, n_heads=2, d_ffn=12, blocks_per_chunk=[1, 2], dropout=0.4,
                          dropout_seed=77, embed_scale=2.5)
    g = np.random.default_rng(9)
    params = {n: a.astype(np.float64) + 0.3 * g.standard_normal(a.shape) for n, a in lp_synth.init_params(dict(cfg, dtype="fp32")).items()}
    x, y = lp_synth.minibatch(cfg, 0)
    orc = LocalUpdateOracle(cfg, params, dtype=np.float64)
    orc.drop_step = 3
    inp = x
    dropped = 0
    for k in range(2):
        loss, h, grads = orc.local_grads(k, inp, y)
        for n in orc.names_of_chunk[k]:
            flat = orc.p[n].reshape(-1)
            for idx in g.choice(flat.size, size=min(4, flat.size), replace=False):
                old, eps = flat[idx], 1e-6
                flat[idx] = old + eps
                up = orc.local_grads(k, inp, y)[0]
                flat[idx] = old - eps
                dn = orc.local_grads(k, inp, y)[0]
                flat[idx] = old
                num = (up - dn) / (2 * eps)
                assert abs(num - grads[n].reshape(-1)[idx]) <= 1e-5 * max(1.0, abs(num)), (n, idx)
        dropped += sum(int((f == 0).sum()) for b in orc._last_cache["blocks"] for f in b[-2:])
        inp = h
    assert dropped > 0
    a = orc.local_grads(0, x, y)[0]
    orc.drop_step = 4
    assert orc.local_grads(0, x, y)[0] != a                     # another step, another mask
    orc.drop_step = None
    assert LocalUpdateOracle(dict(cfg, dropout=0.0), params, dtype=np.float64).local_grads(0, x, y)[0] == orc.local_grads(0, x, y)[0]


def test_create_refuses_bad_dropout():
    import lp_synth
    for kw in (dict(dropout=1.0), dict(dropout=-0.1), dict(dropout=float("nan")), dict(embed_scale=float("inf"))):
        m, K, hd, op = lp.specs_from_config(lp_synth.config("c3", **kw))
        with pytest.raises(lp.LpError) as e:
            lp.lp_create(m, K, hd, op)
        assert lp.LP_ERR[e.value.code] == "INVALID_ARG", kw


class OnDevice:
    """What the binding looks at of a tensor on a GPU, here without one; its address is never read."""

    def __init__(self, shape, dtype, stride=None):
        import torch
        t = torch.empty(shape, dtype=dtype, device="meta")
        if stride is not None:
            t = t.as_strided(shape, stride)
        self.t, self.is_cuda, self.dtype, self.shape, self.nbytes, self.ndim = t, True, dtype, t.shape, t.nbytes, t.ndim

    def __getattr__(self, name):                    # numel, stride, is_contiguous
        return getattr(self.t, name)

    def data_ptr(self):
        return 256


def refused(code, call, *args, says=""):
    with pytest.raises(lp.LpError) as e:
        call(*args)
    assert e.value.code == ERR[code] and says in str(e.value), str(e.value)


def test_binding_of_the_lookup_checks_types_and_sizes():
    import torch
    i32, i64, f32, b16 = torch.int32, torch.int64, torch.float32, torch.bfloat16
    rows, vocab, d, T = 12, 7, 16, 4
    X = OnDevice
    good = dict(ids=X((3, 4), i32), table=X((vocab, d), b16), pos=X((T, d), b16), out=X((rows, d), b16), flag=X((1,), i32))
    bad = dict(ids=[X((rows,), i64), X((rows - 1,), i32), X((rows,), i32, (2,)), X((rows,), torch.int16)],
               table=[X((vocab, d), f32), X((vocab - 1, d), b16), X((vocab, d), b16, (2 * d, 1)), X((vocab, d), torch.float16)],
               pos=[X((T, d), f32), X((T - 1, d), b16)], out=[X((rows, d), f32), X((rows, d - 1), b16), X((rows, d), b16, (1, rows))],
               flag=[X((1,), i64), X((0,), i32)])
    fwd = lambda ids, table, pos, out, flag: lp.lp_embed_forward(lp.LP_BF16, ids, table, pos, out, rows, vocab, d, T, 1.0, flag)
    for name, cases in bad.items():
        for t in cases:
            refused("SHAPE", lambda: fwd(**{**good, name: t}), says="out_of_range" if name == "flag" else name)
    refused("INVALID_ARG", lambda: lp.lp_embed_forward(7, *[good[n] for n in ("ids", "table", "pos", "out")], rows, vocab, d, T))
    need = lp.lp_embed_workspace_bytes(rows, vocab, d)
    good = dict(ids=X((rows,), i32), dout=X((rows, d), f32), dtable=X((vocab, d), f32), dpos=X((T, d), f32), ws=X((need,), torch.uint8))
    bad = dict(ids=[X((rows,), i64)], dout=[X((rows, d), b16), X((rows - 1, d), f32), X((rows, d), f32, (0, 1))],
               dtable=[X((vocab, d), b16), X((vocab - 1, d), f32)], dpos=[X((T, d), b16), X((T, d - 1), f32)])
    bwd = lambda ids, dout, dtable, dpos, ws: lp.lp_embed_backward(lp.LP_FP32, ids, dout, dtable, dpos, rows, vocab, d, T, 1.0, None, ws, need)
    for name, cases in bad.items():
        for t in cases:
            refused("SHAPE", lambda: bwd(**{**good, name: t}), says=name)
    for ws in (X((need - 1,), torch.uint8), X((need,), torch.uint8, (2,)), X((need // 4 - 1,), f32), torch.zeros(need, dtype=torch.uint8),
               np.zeros(need, dtype=np.uint8)):
        refused("INVALID_ARG", lambda: bwd(**{**good, "ws": ws}))


def test_binding_of_dropout_checks_types_and_sizes():
    import torch
    i64, f32, b16 = torch.int64, torch.float32, torch.bfloat16
    n, X = 40, OnDevice
    good = dict(x=X((5, 8), b16), resid=X((n,), b16), y=X((n + 3,), b16), word=X((1,), i64))
    call = lambda x, resid, y, word: lp.lp_dropout(lp.LP_BF16, x, resid, y, n, 0.1, 1, 0, word)
    bad = dict(x=[X((n,), f32), X((n - 1,), b16), X((5, 8), b16, (1, 5)), X((n,), b16, (2,))], resid=[X((n,), torch.float16)],
               y=[X((n,), f32), X((n - 1,), b16)], word=[X((1,), torch.int32), X((1,), f32), X((0,), i64)])
    for name, cases in bad.items():
        for t in cases:
            refused("SHAPE", lambda: call(**{**good, name: t}), says="offset_dev" if name == "word" else name)
    refused("INVALID_ARG", lambda: lp.lp_dropout(5, good["x"], None, good["y"], n, 0.1, 1))
    refused("INVALID_ARG", lambda: lp.lp_dropout(lp.LP_BF16, np.zeros(n, dtype=np.float32), None, good["y"], n, 0.1, 1), says="host")


def test_binding_of_linear_attention_checks_the_shapes_of_states():
    import torch
    B, T, H = 2, 3, 4
    X = OnDevice
    t = X((B, T, H, 64), torch.bfloat16)
    good = dict(q=t, k=t, v=t, o=t, log_decay=X((H,), torch.float32))
    for change in (dict(state_in=X((H, B, 64, 64), torch.float32)), dict(state_out=X((B * H, 64, 64), torch.float32)),
                   dict(log_decay=X((2, 2), torch.float32)), dict(lengths=X((1, B), torch.int32))):
        refused("SHAPE", lambda: lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, {**good, **change}), says=list(change)[0])
    refused("INVALID_ARG", lambda: lp.lp_linear_attention_bf16(lp.LP_LINATTN_FORWARD, good, X((64,), torch.float32, (2,))), says="workspace")


@pytest.mark.parametrize("workload", ["c1", "c4"])
def test_families_without_dropout_refuse_it(workload):
    import lp_synth
    for p in (0.1, float("nan")):
        refused("INVALID_ARG", lambda: lp.lp_create(*lp.specs_from_config(lp_synth.config(workload, dropout=p))), says="dropout")


def test_linear_attention_refuses_lengths_whose_chunks_leave_32_bits():
    """seq_len may be a capacity far above lengths; counted in chunks and segments it has to stay a positive int."""
    for form in (lp.LP_LINATTN_FORWARD, lp.LP_LINATTN_BACKWARD):
        for T in (2 ** 31 - 1, 2 ** 31 - 64, 2 ** 30 + 1):
            assert lp.lp_linear_attention_workspace_bytes(form, 1, T, 1) == 0, T
            assert linattn(form, ws=ONE, nbytes=1 << 40, batch=1, seq_len=T, lengths=0xb000) == ERR["SHAPE"], T
        assert 0 < lp.lp_linear_attention_workspace_bytes(form, 1, 2 ** 30, 1) < 1 << 28

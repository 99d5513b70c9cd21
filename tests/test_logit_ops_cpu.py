"""The operators on logits without a GPU: their plain forms pinned by differences, identities and known answers, and the
refusals of the library's entry points and of the binding."""
import ctypes as C

import numpy as np
import pytest

from oracle import lm_ops as O
from paper_2012_03837_b200 import binding as lp
from tests.test_lm_ops_cpu import ERR, ODD, ONE, OnDevice, refused


def rng(seed=0):
    return np.random.default_rng(seed)


# ------------------------------------------------------------------------------------------------ plain forms
def test_log_probabilities_of_known_rows():
    x = np.log(np.array([[1.0, 2.0, 5.0], [1.0, 1.0, 1.0]]))
    logp, ent, lse, ids, tops = O.token_logprobs(x, [1, 2], 1.0, 3)
    assert np.allclose(np.exp(logp), [0.25, 1 / 3]) and np.allclose(np.exp(lse), [8.0, 3.0])
    assert np.allclose(ent, [-(0.125 * np.log(0.125) + 0.25 * np.log(0.25) + 0.625 * np.log(0.625)), np.log(3.0)])
    assert ids.tolist() == [[2, 1, 0], [0, 1, 2]] and np.allclose(np.exp(tops[0]), [0.625, 0.25, 0.125])
    assert np.allclose(O.token_logprobs(2.0 * x, [1, 2], 2.0)[0], logp)          # the temperature divides


def test_rows_of_masked_tokens():
    inf = np.inf
    x = np.array([[-inf, 0.0, -inf, 0.0], [-inf] * 4, [0.0, np.nan, 1.0, -inf], [-3e38] * 4])
    logp, ent, lse, ids, tops = O.token_logprobs(x, [0, 1, 2, 3], 1.0, 4)
    assert logp[0] == -inf and np.isclose(ent[0], np.log(2)) and ids[0].tolist() == [1, 3, 0, 2]
    assert logp[1] == lse[1] == -inf and ent[1] == 0 and ids[1].tolist() == [0, 1, 2, 3] and (tops[1] == -inf).all()
    assert np.isnan([logp[2], ent[2], lse[2]]).all() and ids[2].tolist() == [2, 0, 3, 1]      # a NaN comes last
    assert np.isclose(logp[3], -np.log(4)) and np.isclose(ent[3], np.log(4))
    dx = O.token_logprobs_bwd(x[[0, 1, 3]], [1, 1, 1], np.ones(3), np.ones(3), np.ones(3))
    assert (dx[0, [0, 2]] == 0).all() and (dx[1] == 0).all() and np.isfinite(dx).all()


def test_gradient_of_log_probabilities_matches_differences():
    g = rng(1)
    x, tok = g.standard_normal((4, 9)), np.array([3, -1, 8, 12])                 # two rows without a token
    a, b, c = g.standard_normal((3, 4))
    f = lambda y: sum((w * v).sum() for w, v in zip((a, b, c), O.token_logprobs(y, tok, 0.7)))
    dx, h = O.token_logprobs_bwd(x, tok, a, b, c, 0.7), 1e-6
    for _ in range(5):
        d = g.standard_normal(x.shape)
        assert abs((f(x + h * d) - f(x - h * d)) / (2 * h) - (dx * d).sum()) <= 1e-7
    parts = [O.token_logprobs_bwd(x, tok, a, None, None, 0.7), O.token_logprobs_bwd(x, tok, None, b, None, 0.7),
             O.token_logprobs_bwd(x, tok, None, None, c, 0.7)]
    assert np.allclose(sum(parts), dx)
    assert (parts[0][[1, 3]] == 0).all()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("ids", [[[0, 4, 7], [2, 2, 5], [-1, 3, 40], [6, -1, -1]], [[1], [8], [0], [5]]])
def test_gradient_of_distillation_matches_differences(rest, ids):
    g = rng(2)
    ids = np.array(ids)
    x, dl = g.standard_normal((4, 9)), g.standard_normal(4)
    t = np.log(0.3 * g.random(ids.shape) + 0.01)
    f = lambda y: (dl * O.distill(y, ids, t, rest, 1.7, 2.5)[0]).sum()
    _, dx = O.distill(x, ids, t, rest, 1.7, 2.5, dl)
    h = 1e-6
    for _ in range(5):
        d = g.standard_normal(x.shape)
        assert abs((f(x + h * d) - f(x - h * d)) / (2 * h) - (dx * d).sum()) <= 1e-7


def test_distillation_of_a_distribution_into_itself():
    g = rng(3)
    x = g.standard_normal((3, 12))
    for temperature in (1.0, 2.0):
        ids, lp_ = O.token_logprobs(x, None, temperature, 5)[3:]
        loss, dx = O.distill(x, ids, lp_, True, temperature)
        assert np.abs(loss).max() <= 1e-14 and np.abs(dx).max() <= 1e-14
        every = np.tile(np.arange(12), (3, 1))
        for rest, t in ((False, x), (True, O.token_logprobs(x, None, temperature, 0)[2][:, None] * 0 + np.stack([O.log_softmax(r, temperature)[0] for r in x]))):
            loss, dx = O.distill(x, every, t, rest, temperature)                  # the whole vocabulary listed
            assert np.abs(loss).max() <= 1e-14 and np.abs(dx).max() <= 1e-14


def test_distillation_from_everything_is_the_cross_entropy_gradient():
    """One entry of weight one: the loss is -log p of it, the gradient that of softmax cross-entropy."""
    g = rng(4)
    x, tok = g.standard_normal((5, 7)), np.array([0, 6, 3, 3, 1])
    loss, dx = O.distill(x, tok[:, None], np.zeros((5, 1)), True)
    assert np.allclose(loss, -O.token_logprobs(x, tok)[0])
    assert np.allclose(dx, O.token_logprobs_bwd(x, tok, -np.ones(5)))


def test_rows_without_weight_and_impossible_tokens():
    inf = np.inf
    x = np.array([[0.0, 1.0, -inf, 2.0]] * 5 + [[-inf] * 4])
    ids = np.array([[-1, -1], [0, 1], [2, 0], [0, 3], [0, 1], [0, 1]])
    t = np.log(np.array([[0.5, 0.5], [0.0, 0.0], [0.5, 0.5], [0.0, 0.5], [0.5, 0.25], [0.5, 0.5]]))
    loss, dx = O.distill(x, ids, t, True)
    assert loss[0] == loss[1] == 0 and (dx[:2] == 0).all()
    assert loss[2] == inf and np.isfinite(dx[2]).all() and dx[2, 2] == -0.5
    assert np.isfinite(loss[3]) and np.isfinite(loss[4]) and loss[5] == inf and (dx[5] == 0).all()
    y = np.array([[0.0, 1.0, -inf, -inf]])                                       # the rest is impossible
    loss, dx = O.distill(y, np.array([[0, 1]]), np.log([[0.5, 0.25]]), True)
    assert loss[0] == inf and (dx[0, 2:] == 0).all() and np.isfinite(dx).all()


@pytest.mark.parametrize("mask", [-1e9, -1e12, -1e15, -1e18, -1e30])
def test_a_rest_of_equal_masked_tokens_shares_alike(mask):
    """The rest's shares are those of its own softmax, whatever the distance to the listed tokens."""
    x = np.full((2, 12), mask)
    x[:, :3] = [0.5, 1.0, -1.0]
    x[1, 11] += mask * 1e-3
    ids, t = np.array([[0, 1, 2]] * 2), np.log([[0.25, 0.125, 0.125]] * 2)
    loss, dx = O.distill(x, ids, t, True)
    assert np.allclose(dx[0, 3:], -0.5 / 9, rtol=1e-12) and np.allclose(dx[1, 3:11], -0.5 / 8, rtol=1e-12) and abs(dx[1, 11]) <= 1e-12
    assert np.isclose(loss[0], -0.5 * mask, rtol=1e-6) and np.abs(dx.sum(1)).max() <= 1e-12


# ------------------------------------------------------------------------------------------------ refusals
L = lp._lib


def forward(dt=1, x=ONE, ld=16, tok=None, logp=None, ent=ONE, lse=None, ids=None, tops=None, k=0, rows=4, vocab=16, temp=1.0, flag=None):
    return L.lp_token_logprobs(dt, x, ld, tok, logp, ent, lse, ids, tops, k, rows, vocab, temp, flag, None)


def backward(dt=1, x=ONE, ld=16, tok=ONE, a=ONE, b=None, c=None, dx=C.c_void_p(4096), ld_out=16, rows=4, vocab=16, temp=1.0, flag=None):
    return L.lp_token_logprobs_backward(dt, x, ld, tok, a, b, c, dx, ld_out, rows, vocab, temp, flag, None)


def teach(form=0, dt=1, x=ONE, ld=16, ids=ONE, t=ONE, k=3, loss=ONE, dloss=None, dx=None, ld_out=0, rows=4, vocab=16, temp=1.0, scale=1.0,
          flag=None):
    return L.lp_distill(form, dt, x, ld, ids, t, k, loss, dloss, dx, ld_out, rows, vocab, temp, scale, flag, None)


@pytest.mark.parametrize("call", [forward, backward, teach])
def test_entries_check_the_logits(call):
    for dt in (-1, 2):
        assert call(dt=dt) == ERR["INVALID_ARG"]
    assert call(x=None) == ERR["INVALID_ARG"]
    assert call(rows=0) == call(rows=-1) == call(rows=(1 << 27) + 1) == call(vocab=0) == call(vocab=(1 << 18) + 1, ld=1 << 20) == ERR["SHAPE"]
    assert call(ld=15) == call(ld=-16) == call(ld=(1 << 38) + 1) == ERR["SHAPE"]
    for temp in (0.0, -1.0, float("nan"), float("inf"), 2.0 ** -21, 2.0 ** 21):
        assert call(temp=temp) == ERR["INVALID_ARG"], temp
    assert call(x=ODD) == call(dt=0, x=C.c_void_p(258)) == call(flag=C.c_void_p(258)) == ERR["UNSUPPORTED"]


def test_log_probabilities_check_their_arguments():
    assert forward(ent=None) == ERR["INVALID_ARG"] and b"output" in L.lp_last_error(None)
    assert forward(logp=ONE) == ERR["INVALID_ARG"]                              # no tokens
    assert forward(k=129, ids=ONE, tops=ONE, vocab=500, ld=500) == forward(k=17, ids=ONE, tops=ONE) == forward(k=-1) == ERR["SHAPE"]
    assert forward(k=3) == forward(k=3, ids=ONE) == forward(k=3, tops=ONE) == forward(k=0, ids=ONE, tops=ONE) == ERR["INVALID_ARG"]
    for name in ("tok", "logp", "ent", "lse"):
        assert forward(**{"tok": ONE, name: C.c_void_p(258)}) == ERR["UNSUPPORTED"], name
    assert forward(k=3, ids=C.c_void_p(258), tops=ONE) == forward(k=3, ids=ONE, tops=C.c_void_p(257)) == ERR["UNSUPPORTED"]


def test_their_gradient_checks_its_arguments():
    assert backward(dx=None) == backward(a=None) == backward(tok=None) == ERR["INVALID_ARG"]
    assert backward(ld_out=15) == backward(ld_out=(1 << 38) + 1) == ERR["SHAPE"]
    assert backward(dx=ONE, ld_out=17) == ERR["INVALID_ARG"] and b"stride" in L.lp_last_error(None)
    for name in ("tok", "a", "b", "c"):
        assert backward(**{name: C.c_void_p(258)}) == ERR["UNSUPPORTED"], name
    assert backward(dx=C.c_void_p(4097)) == ERR["UNSUPPORTED"]


def test_distillation_checks_its_arguments():
    assert teach(form=2) == teach(form=-1) == teach(ids=None) == teach(t=None) == teach(loss=None) == ERR["INVALID_ARG"]
    assert teach(k=0) == teach(k=129) == teach(dx=C.c_void_p(4096), ld_out=8) == ERR["SHAPE"]
    for scale in (float("nan"), float("inf")):
        assert teach(scale=scale) == ERR["INVALID_ARG"]
    for name in ("ids", "t", "loss", "dloss"):
        assert teach(**{name: C.c_void_p(258)}) == ERR["UNSUPPORTED"], name
    assert teach(dx=ONE, ld_out=32) == ERR["INVALID_ARG"]


def test_binding_checks_types_sizes_and_strides():
    import torch
    i32, i64, f32, b16 = torch.int32, torch.int64, torch.float32, torch.bfloat16
    X = OnDevice
    R, V, k = 4, 40, 3
    x = X((R, V), b16)
    good = dict(tokens=X((R,), i32), logp=X((R,), f32), entropy=X((R,), f32), lse=X((R,), f32), top_ids=X((R, k), i32), top_logp=X((R, k), f32),
                out_of_range=X((1,), i32))
    bad = dict(tokens=[X((R,), i64), X((R - 1,), i32)], logp=[X((R,), b16), X((R - 1,), f32), X((R,), f32, (2,))], entropy=[X((R,), i32)],
               lse=[X((1,), f32)], top_ids=[X((R, k), i64), X((R * k,), i32), X((R - 1, k), i32), X((R, k), i32, (1, R))],
               top_logp=[X((R, k - 1), f32), X((R, k), b16)], out_of_range=[X((1,), i64)])
    for name, cases in bad.items():
        for t in cases:
            refused("SHAPE", lambda: lp.lp_token_logprobs(x, **{**good, name: t}), says=name)
    matrices = [X((R, V), torch.float16), X((R * V,), b16), X((2, 2, V), b16), None, np.zeros((R, V), dtype=np.float32)]
    strided = [X((R, V), b16, (1, R)), X((R, V), b16, (2 * V, 2))]
    for code, cases in (("SHAPE", matrices), ("UNSUPPORTED", strided), ("INVALID_ARG", [torch.zeros(R, V)])):
        for t in cases:
            refused(code, lambda: lp.lp_token_logprobs(t, entropy=good["entropy"]), says="logits")
            refused(code, lambda: lp.lp_token_logprobs_backward(t, dlse=good["lse"], dlogits=x), says="logits")
            refused(code, lambda: lp.lp_distill(lp.LP_DISTILL_TOP, t, good["top_ids"], good["top_logp"], loss=good["logp"]), says="logits")
    for t in (X((R, V), f32), X((R, V + 1), b16), X((R + 1, V), b16), None):
        refused("SHAPE", lambda: lp.lp_token_logprobs_backward(x, dlse=good["lse"], dlogits=t), says="dlogits")
        if t is not None:
            refused("SHAPE", lambda: lp.lp_distill(0, x, good["top_ids"], good["top_logp"], dlogits=t), says="dlogits")
    bad = dict(teacher_ids=[X((R, k), i64), X((R * k,), i32), X((R + 1, k), i32), None], teacher=[X((R, k), b16), X((R, k - 1), f32)],
               loss=[X((R,), b16)], dloss=[X((R - 1,), f32)])
    fine = dict(teacher_ids=good["top_ids"], teacher=good["top_logp"], loss=good["logp"], dloss=good["lse"])
    for name, cases in bad.items():
        for t in cases:
            refused("SHAPE", lambda: lp.lp_distill(lp.LP_DISTILL_TOP, x, **{**fine, name: t}), says=name)
    for name in ("dlogp", "dentropy", "dlse"):
        refused("SHAPE", lambda: lp.lp_token_logprobs_backward(x, good["tokens"], dlogits=x, **{name: X((R - 1,), f32)}), says=name)
    # one row may have any stride, a column of single logits any step
    refused("INVALID_ARG", lambda: lp.lp_token_logprobs(X((1, V), b16, (7, 1))), says="output")
    refused("INVALID_ARG", lambda: lp.lp_token_logprobs(X((R, 1), b16, (5, 5))), says="output")


def test_values_beside_ids_have_their_shape():
    """Values of a wider (longer, turned) matrix than the ids' would belong to other tokens."""
    import torch
    i32, f32, b16 = torch.int32, torch.float32, torch.bfloat16
    X = OnDevice
    R, V, k = 4, 40, 8
    x, ids, out = X((R, V), b16), X((R, k), i32), X((R,), f32)
    for shape in ((R, 32), (R + 1, k), (k, R), (R * k,), (R, k, 1), (2, R, k), (R, k - 1)):
        v = X(shape, f32)
        refused("SHAPE", lambda: lp.lp_token_logprobs(x, top_ids=ids, top_logp=v), says="top_logp")
        refused("SHAPE", lambda: lp.lp_distill(lp.LP_DISTILL_TOP, x, ids, v, loss=out), says="teacher")
    refused("SHAPE", lambda: lp.lp_token_logprobs(x, top_ids=256, top_logp=X((R, k), f32)), says="top_ids")      # an address says no shape
    refused("SHAPE", lambda: lp.lp_distill(lp.LP_DISTILL_TOP, x, 256, X((R, k), f32), loss=out), says="teacher_ids")
    # the first entries of a longer list, as a view: strided
    refused("SHAPE", lambda: lp.lp_distill(lp.LP_DISTILL_TOP, x, ids, X((R, k), f32, (2 * k, 1)), loss=out), says="teacher")
    # as they should be, or an address: the entry's own checks come next
    for v in (X((R, k), f32), 256):
        refused("INVALID_ARG", lambda: lp.lp_token_logprobs(x, top_ids=ids, top_logp=v, temperature=0.0), says="temperature")
        refused("INVALID_ARG", lambda: lp.lp_distill(lp.LP_DISTILL_TOP, x, ids, v, loss=out, temperature=0.0), says="temperature")

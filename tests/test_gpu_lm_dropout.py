"""Training steps of the transformer family with dropout and a scaled embedding against the oracle, which forms the
same masks from the same key and counters; the bounds are those of the steps without dropout."""
import numpy as np
import pytest
import torch

import lp_synth
from paper_2012_03837_b200 import binding as lp
from tests import lp_testlib as T
from tests.test_gpu_parity import check, check_overlap

pytestmark = pytest.mark.gpu


def small(dtype, **kw):
    sizes = dict(batch=2, seq_len=80, vocab=300, d_ffn=192) if dtype == "fp32" else dict(batch=3, seq_len=136, vocab=1000, d_ffn=320)
    return lp_synth.config("c3", dtype=dtype, d_model=128, n_heads=2, blocks_per_chunk=[1, 2, 1],
                           **{**sizes, "dropout": 0.1, "dropout_seed": 0x1234567890ABCDEF, "embed_scale": 1.5, **kw})


@pytest.mark.parametrize("dtype,schedule,backend", [("fp32", "sync", 0), ("fp32", "pipelined", 0), ("bf16", "sync", 0),
                                                    ("bf16", "pipelined", 0), ("bf16", "pipelined", 1)])
def test_lm_steps_with_dropout(dtype, schedule, backend):
    check(small(dtype, schedule=schedule), gemm_backend=backend)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_overlapping_updates_with_dropout(dtype):
    check_overlap(small(dtype), shared_per_boundary=12)


def test_many_equal_tokens_and_heavy_dropout():
    """Most positions hold one token: its table gradient is summed in pieces."""
    cfg = small("fp32", batch=6, dropout=0.6, vocab=40, optim=dict(kind="sgdm", lr=0.01, momentum=0.9, weight_decay=0.0))
    init = lp_synth.init_params(cfg)
    gm = T.GpuModel(cfg, init)
    orc = T.LocalUpdateOracle(cfg, init, dtype=np.float32)
    x, y = lp_synth.minibatch(cfg, 0)
    x[:, ::3] = 7
    x[:, 1::3] = 7
    gl, ol = gm.step(x, y), orc.step(x, y)
    assert np.abs(gl - ol).max() <= 1e-4 * np.abs(ol).max()
    got = gm.get(lp.LP_GRAD)["c0.tok"]
    ref = orc.last_grads["c0.tok"]
    assert np.linalg.norm(got - ref) <= 1e-3 * np.linalg.norm(ref)
    gm.close()


def test_evaluation_drops_nothing():
    cfg = small("bf16")
    a, b = T.GpuModel(cfg), T.GpuModel(dict(cfg, dropout=0.0))
    x, y = lp_synth.minibatch(cfg, 3)
    for u, v in zip(a.forward(x, y), b.forward(x, y)):
        assert np.array_equal(u, v)
    for u, v in zip(T.gpu_evaluate(a, x, y), T.gpu_evaluate(b, x, y)):
        assert np.array_equal(u, v)
    a.close(), b.close()


def test_masks_go_on_behind_a_checkpoint_and_differ_from_step_to_step():
    cfg = small("bf16", schedule="pipelined")
    a = T.GpuModel(cfg)
    batches = [lp_synth.minibatch(cfg, t) for t in range(4)]
    for x, y in batches[:2]:
        a.step(x, y)
    blob = np.empty(lp.lp_state_size(a.h), dtype=np.uint8)
    lp.lp_save_state(a.h, blob)
    rest = [a.step(x, y) for x, y in batches[2:]]
    want = a.get()
    b = T.GpuModel(cfg)
    lp.lp_load_state(b.h, blob)
    again = [b.step(x, y) for x, y in batches[2:]]
    assert np.array_equal(rest, again)
    got = b.get()
    assert all(np.array_equal(want[n], got[n]) for n in want)
    c = T.GpuModel(dict(cfg, dropout_seed=5))
    first = T.GpuModel(cfg).step(*batches[0])
    assert not np.array_equal(first, c.step(*batches[0]))       # another key, other masks
    torch.cuda.synchronize()
    for m in (a, b, c):
        m.close()

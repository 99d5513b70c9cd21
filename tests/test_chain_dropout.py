"""Dropout in a chain of pieces on several GPUs: every block draws the masks that it would draw inside the whole model, so
no two blocks of the chain share one.  On CPU the counter words; on one GPU the ranks emulated in turn, against the oracle's
whole model."""
import pytest

import lp_synth
from paper_2012_03837_b200 import binding as B
from paper_2012_03837_b200 import pipeline as P
from tests.test_chunk_per_gpu import SMALL, run_emulated, run_emulated_ranges


def mask_words(cfg, chunk_of_piece, s):
    """{(block of the whole model, branch): last two counter words} of the masks that a piece's chunk draws at the
    piece's step s, as lp_model_spec documents them."""
    sc, out = cfg, {}
    at = sc.get("first_block", 0) + sum(sc["blocks_per_chunk"][:chunk_of_piece])
    for n in range(at, at + sc["blocks_per_chunk"][chunk_of_piece]):
        for branch in (1, 2):
            out[n, branch] = (branch + 2 * n, sc.get("first_step", 0) + s)
    return out


def test_pieces_of_a_chain_draw_the_masks_of_the_whole_model():
    cfg = dict(SMALL["lm"], blocks_per_chunk=[1, 2, 1, 3], dropout=0.1, dropout_seed=2 ** 40 + 5)
    for ranges in ([(0, 1), (1, 1), (2, 1), (3, 1)], [(0, 2), (2, 2)], [(0, 1), (1, 3)]):
        for t in range(9):
            drawn = {}
            for first, count in ranges:
                sc = P.stage_config(cfg, first, count)
                assert (sc["dropout"], sc["dropout_seed"]) == (cfg["dropout"], cfg["dropout_seed"])
                m, _, _, _ = B.specs_from_config(sc)
                assert (m.first_block, m.first_step) == (sc["first_block"], sc["first_step"])
                for j in range(count):
                    if t >= first + j:                           # busy at iteration t, its piece's step t - first
                        drawn.update(mask_words(sc, j, t - first))
            whole = {}
            for k in range(4):
                if t >= k:
                    whole.update(mask_words(cfg, k, t))
            assert drawn == whole
            assert len(set(drawn.values())) == len(drawn)        # no two branches of the chain share a mask
    # a piece of a piece counts on
    sc = P.stage_config(P.stage_config(cfg, 1, 3), 1, 2)
    assert (sc["first_block"], sc["first_step"]) == (3, 2)
    with pytest.raises(B.LpError) as e:
        B.lp_create(*B.specs_from_config(dict(lp_synth.config("c3"), first_block=-1)))
    assert B.LP_ERR[e.value.code] == "INVALID_ARG"


DROPPING = dict(dropout=0.2, dropout_seed=0x0123456789ABCDEF, embed_scale=1.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_emulated_ranks_lm_with_dropout(dtype):
    run_emulated(lp_synth.config("c3", dtype=dtype, batch=3, seq_len=64, vocab=256, d_model=128, n_heads=2, d_ffn=256,
                                 blocks_per_chunk=[1, 2, 1], **DROPPING), 6)


@pytest.mark.gpu
def test_emulated_ranges_lm_with_dropout_and_drain():
    run_emulated_ranges(lp_synth.config("c3", dtype="fp32", batch=2, seq_len=72, vocab=256, d_model=128, n_heads=2, d_ffn=256,
                                        blocks_per_chunk=[1, 1, 2, 1, 1], **DROPPING), [(0, 3), (3, 2)], 5)

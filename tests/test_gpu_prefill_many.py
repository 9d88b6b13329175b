"""Prompt attention where 128 rows share a workgroup's tiles (bf16; long caches, or tiles enough for every CU), split keys and whole ones: masks, caps,
distances, documents, and what masked places hold."""
import numpy as np
import pytest
import torch

from paper_2506_18226_amd import binding as B

from prompt_common import f64
from test_gpu_prefill import Prompt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")

# a cache of more than 512 slots (keys in two parts), and 260 and more (sequence, head, 128 rows) tiles (keys whole)
SPLIT = dict(lens=[129, 66, 1, 0, 200], past=[0, 37, 300, 5, 390], h=2, cap=600)
WHOLE = dict(lens=[70, 65, 128, 0, 97, 1] * 22, past=[0, 3] * 66, h=2, cap=131)


def make(shape, D, G, **kw):
    return Prompt(shape["lens"], shape["past"], shape["h"], D, "bf16", G, cap=shape["cap"], **kw)


@pytest.mark.parametrize("shape", [SPLIT, WHOLE], ids=["split", "whole"])
@pytest.mark.parametrize("D,G,layout", [(64, 0, "head_major"), (128, 0, "slot_major"), (128, 2, "head_major"), (64, 3, "slot_major")])
@pytest.mark.parametrize("mask", [B.MASK_CAUSAL, B.MASK_PREFIX])
def test_against_the_definition(shape, D, G, layout, mask):
    p = make(shape, D, G, layout=layout, prefix=90)
    p.run(mask=mask)
    p.check(mask=mask)


@pytest.mark.parametrize("shape", [SPLIT, WHOLE], ids=["split", "whole"])
@pytest.mark.parametrize("D,G", [(64, 0), (128, 0), (128, 2)])
@pytest.mark.parametrize("cap,slope,docs", [(5.0, False, False), (0.0, True, False), (0.0, False, True), (20.0, True, True), (20.0, True, False), (0.0, True, True)])
def test_scores_capped_lowered_and_masked_by_document(shape, D, G, cap, slope, docs):
    p = make(shape, D, G, prefix=33, q_scale=4.0)
    mods = dict(mask=B.MASK_PREFIX, softcap=cap)
    if slope:
        p.batch.pos += 1_000_000_000
        mods["slopes"] = torch.tensor([2.0 ** -(i + 1) for i in range(2 * p.G)], device=DEV)
    if docs:                                                 # documents of 13 slots with 4 of padding, whose rows see nothing; some come back later
        slot = torch.arange(p.batch.params.cap + 2)
        doc = torch.where(slot % 13 >= 9, -1 - slot % 2, slot // 13 % 4).to(torch.int32)
        mods["doc"] = doc.repeat(len(p.lens), 1).contiguous().to(DEV)
        for t in (p.K, p.V):                                 # what padding holds is nobody's business
            t[:, :, (doc[:p.batch.params.cap] < 0).to(DEV)] = NAN
    p.run(**mods)
    p.check(**mods)


@pytest.mark.parametrize("shape", [SPLIT, WHOLE], ids=["split", "whole"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("at", [0, 13, 40, 64])
def test_infinities_and_nan_behind_the_mask(shape, D, at):
    """A token whose row holds infinities or NaN changes the rows that see it and no others."""
    p = make(shape, D, 0)
    p.run()
    clean, lse = p.out.clone(), p.lse.clone()
    slot = p.past[0] + at
    p.V[0, 0, slot, 3], p.V[0, 0, slot, D - 1], p.V[0, 1, slot, 5] = float("inf"), NAN, -float("inf")
    p.batch.score.copy_(torch.from_numpy(p.score0))
    p.run()
    assert torch.equal(p.out[:at], clean[:at]) and torch.equal(p.lse, lse)
    rows = slice(at, int(p.lens[0]))
    assert (p.out[rows, 0, 3] == float("inf")).all() and p.out[rows, 0, D - 1].isnan().all() and (p.out[rows, 1, 5] == -float("inf")).all()
    keep = torch.ones(D, dtype=torch.bool, device=DEV)
    keep[[3, D - 1]] = False
    assert torch.equal(p.out[rows, 0][:, keep], clean[rows, 0][:, keep]) and torch.equal(p.out[int(p.lens[0]):], clean[int(p.lens[0]):])
    p.V[0, :, slot] = 0.0
    p.K[0, :, slot] = NAN
    p.run()
    assert torch.equal(p.out[:at], clean[:at]) and torch.equal(p.lse[:at], lse[:at]) and p.out[rows].isnan().all()


@pytest.mark.parametrize("shape", [SPLIT, WHOLE], ids=["split", "whole"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_grow_along_the_keys(shape, D):
    """Every later key scores far above all before it: maxima are followed again and again."""
    p = make(shape, D, 0, q_scale=0.1)
    p.q += 2.0
    ramp = torch.arange(p.batch.params.cap, device=DEV) * 0.05
    p.K += ramp[None, None, :, None].to(p.K.dtype)
    p.run()
    p.check()


def test_records_that_do_not_fit_with_split_keys():
    p = make(SPLIT, 64, 0)
    s = p.batch.read_seqs()
    s["n_res"][0], s["status"][1] = 7, B.SEQ_CACHE_FULL
    p.batch.upload_seqs()
    p.run()
    assert p.batch.read_seqs()["status"].tolist() == [B.SEQ_BAD_STATE, B.SEQ_CACHE_FULL, 0, 0, 0]
    assert not p.out[:195].any() and not p.lse[:195].any() and np.array_equal(f64(p.batch.score)[:2], p.score0[:2])
    p.check(sequences=[2, 4])

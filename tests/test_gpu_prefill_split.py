"""Prompt attention with probabilities of 16 bits (FLAG_SPLIT_P): as exact as adsa_attend under every mask, cap and distance, and what infinities and NaN do.

Bound: as in test_gpu_shared_precision, whose roundings are the same."""
import numpy as np
import pytest
import torch

import test_gpu_prefill
from paper_2506_18226_amd import binding as B
from test_gpu_prefill import LENS, LONG, Prompt
from test_gpu_prefill_many import SPLIT, WHOLE
from test_gpu_shared_precision import attended as attended_whole

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")
SHAPES = [dict(lens=LENS, past=5, h=2), dict(lens=LONG, past=70, h=1), dict(lens=[7, 3], past=[1500, 2011], h=2), SPLIT, dict(WHOLE, lens=WHOLE["lens"][:66], past=WHOLE["past"][:66])]
IDS = ["few", "short", "deep", "split", "whole"]


def attended(q, k, v, scale, *, seen, **kw):
    """(a value that nobody sees may be anything)"""
    return attended_whole(q, k, np.where(seen.any(0)[:, None], v, 0.0) if len(k) else v, scale, seen=seen, **kw)


def check(p, **mods):
    p.run(flags=B.FLAG_SPLIT_P, **mods)
    p.check(**mods)


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("D,G,layout", [(64, 0, "head_major"), (128, 0, "slot_major"), (128, 2, "head_major"), (64, 3, "slot_major")])
@pytest.mark.parametrize("mask", [B.MASK_CAUSAL, B.MASK_PREFIX])
def test_outputs_are_rounded_once(monkeypatch, shape, D, G, layout, mask):
    monkeypatch.setattr(test_gpu_prefill, "attended", attended)
    check(Prompt(D=D, G=G, layout=layout, prefix=50, q_scale=0.7, **shape), mask=mask)


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("D,G", [(64, 0), (128, 2)])
@pytest.mark.parametrize("cap,slope,docs", [(5.0, False, False), (0.0, True, False), (0.0, False, True), (20.0, True, True), (20.0, True, False)])
def test_under_caps_distances_and_documents(monkeypatch, shape, D, G, cap, slope, docs):
    monkeypatch.setattr(test_gpu_prefill, "attended", attended)
    p = Prompt(D=D, G=G, prefix=33, **shape)
    mods = dict(mask=B.MASK_PREFIX, softcap=cap, slopes=torch.tensor([2.0 ** -(i + 4) for i in range(p.h * p.G)], device=DEV) if slope else None)
    if docs:
        slot = torch.arange(p.batch.params.cap)
        doc = torch.where(slot % 13 >= 9, -1 - slot % 2, slot // 13 % 4).to(torch.int32)
        mods["doc"] = doc.repeat(len(p.lens), 1).contiguous().to(DEV)
        for t in (p.K, p.V):
            t[:, :, (doc < 0).to(DEV)] = NAN
    check(p, **mods)


@pytest.mark.parametrize("shape", [dict(lens=[40, 200], past=0, h=2), dict(lens=[20, 3], past=[90, 700], h=2), SPLIT, WHOLE], ids=["short", "deep", "split", "whole"])
@pytest.mark.parametrize("D,G", [(64, 0), (128, 0), (64, 3)])
@pytest.mark.parametrize("slot", [0, 13, 64, "last"])
def test_infinities_and_nan(shape, D, G, slot):
    """In a slot that all rows, some or one of the first sequence see: those rows have them, and no others."""
    p = Prompt(D=D, G=G, **shape)
    p.run(flags=B.FLAG_SPLIT_P)
    clean, lse = p.out.clone(), p.lse.clone()
    at = int(p.keys[0]) - 1 if slot == "last" else min(slot, int(p.keys[0]) - 1)
    p.V[0, 0, at, 3], p.V[0, 0, at, D - 1], p.V[0, 1, at, 5] = INF, NAN, -INF
    p.batch.score.copy_(torch.from_numpy(p.score0))
    p.run(flags=B.FLAG_SPLIT_P)
    want = clean.clone()
    rows = slice(max(0, at - int(p.past[0])), int(p.lens[0]))
    want[rows, :p.G, 3], want[rows, :p.G, D - 1], want[rows, p.G:2 * p.G, 5] = INF, NAN, -INF
    assert torch.equal(torch.nan_to_num(p.out.float(), nan=12345.0), torch.nan_to_num(want.float(), nan=12345.0)) and torch.equal(p.lse, lse)


def test_no_effect_with_an_fp32_cache():
    p = Prompt([5, 90], 3, 2, 64, "f32")
    p.run()
    out, score = p.out.clone(), p.batch.score.clone()
    p.batch.score.copy_(torch.from_numpy(p.score0))
    p.run(flags=B.FLAG_SPLIT_P)
    assert torch.equal(p.out, out) and torch.equal(p.batch.score, score)


@pytest.mark.parametrize("D,G", [(64, 0), (128, 0), (128, 2), (64, 3)])
@pytest.mark.parametrize("lens,past", [([1, 1, 1], [0, 300, 2011]), ([7, 3, 10], [1500, 60, 0])])
def test_few_rows_are_as_exact_without_the_flag(monkeypatch, D, G, lens, past):
    monkeypatch.setattr(test_gpu_prefill, "attended", attended)
    p = Prompt(lens, past, 2, D, "bf16", G, q_scale=0.7)
    p.run()
    p.check()

"""Scores under caps far beyond them: a cap takes from a score what tanh takes, and nothing for being far off.

Bounds, u = 2^-24.  The cap's own error is relative to the capped score: within 16 u of it (constants 4 u, the argument 3, an exponential 3, a reciprocal 2
and three roundings), instead of prompt_common's 8 u of the cap; the rest is as there."""
import numpy as np
import pytest
import torch

import prompt_common
import test_gpu_prefill
import test_gpu_shared
from prompt_common import U
from test_gpu_prefill import Prompt
from test_gpu_prefill_many import SPLIT, WHOLE
from test_gpu_shared import Shared

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def attended(q, k, v, scale, *, seen=None, cap=0.0, slope=0.0, dist=None, bf16=False):
    """prompt_common.attended with the cap's bound as above."""
    n, m = q.shape[0], k.shape[0]
    if m == 0:
        return prompt_common.attended(q, k, v, scale)
    seen = np.ones((n, m), bool) if seen is None else seen
    with np.errstate(invalid="ignore", over="ignore"):
        z = q @ k.T * scale
        d = (q.shape[1] + 4) * U * (np.abs(q) @ np.abs(k).T) * scale
        z = cap * np.tanh(z / cap)
        d = d + 16 * U * np.abs(z)
        if slope:
            z, d = z - slope * np.abs(dist), d + 4 * U * slope * np.abs(dist)
    z, d = np.where(seen, z, -np.inf), np.where(seen, d, 0.0)
    top = z.max(1, keepdims=True)
    e = np.exp(z - np.where(np.isinf(top), 0.0, top))
    l = e.sum(1, keepdims=True)
    p = np.divide(e, l, out=np.zeros_like(e), where=l > 0)
    with np.errstate(divide="ignore"):
        lse = np.where(l[:, 0] > 0, np.where(np.isinf(top[:, 0]), 0.0, top[:, 0]) + np.log(l[:, 0]), -np.inf)
    worst = d.max(1)
    rel = 2 * worst + 32 * U
    vv = np.where(seen.any(0)[:, None], v, 0.0)
    out, size = p @ vv, p @ np.abs(vv)
    tol = (rel[:, None] + (2.0 ** -8 if bf16 else 0.0)) * size + (2.0 ** -8 if bf16 else U) * np.abs(out) + 1e-30
    return out, lse, p, tol, worst + 32 * U * (1 + np.abs(np.where(np.isinf(lse), 0.0, lse))), np.broadcast_to(rel[:, None], p.shape)


@pytest.fixture(autouse=True)
def bounds(monkeypatch):
    monkeypatch.setattr(test_gpu_prefill, "attended", attended)
    monkeypatch.setattr(test_gpu_shared, "attended", attended)


# scores of a few units to some hundred: far below the cap, and up to it (both sides of where the series ends)
CAPS = [(300.0, 60.0), (2000.0, 300.0), (1e6, 2.0), (1e30, 4.0)]


def slopes(on, heads):
    return torch.tensor([2.0 ** -(i + 3) for i in range(heads)], device=DEV) if on else None


@pytest.mark.parametrize("cap,q_scale", CAPS)
@pytest.mark.parametrize("slope", [False, True])
@pytest.mark.parametrize("shape", [dict(lens=[3, 30, 1], past=40, h=2), dict(lens=[150, 40, 77], past=0, h=2), SPLIT, WHOLE], ids=["few", "short", "split", "whole"])
@pytest.mark.parametrize("dtype,D,G", [("bf16", 64, 0), ("bf16", 128, 2), ("f32", 64, 0)])
def test_prompts(cap, q_scale, slope, shape, dtype, D, G):
    if dtype == "f32" and shape in (SPLIT, WHOLE):
        shape = dict(shape, lens=shape["lens"][:6], past=shape["past"][:6])
    p = Prompt(dtype=dtype, D=D, G=G, q_scale=q_scale, **shape)
    mods = dict(softcap=cap, slopes=slopes(slope, 2 * p.G))
    p.run(**mods)
    p.check(**mods)


@pytest.mark.parametrize("cap,q_scale", CAPS)
@pytest.mark.parametrize("slope", [False, True])
@pytest.mark.parametrize("members", [[3, 2], [40, 3]])
@pytest.mark.parametrize("h,D,dtype,G", [(2, 64, "bf16", 0), (1, 128, "bf16", 0), (1, 128, "bf16", 5), (2, 64, "bf16", 3), (2, 64, "f32", 0)])
def test_shared_prompts(cap, q_scale, slope, members, h, D, dtype, G):
    s = Shared(members, [150, 333], [(7 * i + 1) % 65 for i in range(sum(members))], h, D, dtype, G, q_scale=q_scale)
    mods = dict(softcap=cap, slopes=slopes(slope, h * s.G))
    s.run(**mods)
    s.check(**mods)

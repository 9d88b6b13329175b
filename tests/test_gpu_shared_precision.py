"""bf16 decode attention over shared prompts is as exact as adsa_attend: probabilities enter the product with V in 16 bits, the output is rounded once.

Bound: a bf16 value and what it leaves of an fp32 one, as another, are off by half a step of a half step, 2^-16 of it; the output's own rounding is
half a step, 2^-8 of it; scores and sums as in prompt_common."""
import numpy as np
import pytest
import torch

import prompt_common
import test_gpu_shared
from test_gpu_shared import Shared

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def attended(q, k, v, scale, *, bf16=False, **kw):
    out, lse, p, tol, lse_tol, p_tol = prompt_common.attended(q, k, v, scale, bf16=False, **kw)
    if bf16 and len(k):
        tol = tol + 2.0 ** -16 * (p @ np.abs(v)) + 2.0 ** -8 * np.abs(out)
    return out, lse, p, tol, lse_tol, p_tol


@pytest.mark.parametrize("members,prompts,lists", [([3, 2], [150, 20], [70, 1, 33, 300, 200]), ([40, 3], [700, 333], [(37 * i + 1) % 165 for i in range(43)]), ([2], [0], [500, 31])])
@pytest.mark.parametrize("h,D,G", [(2, 64, 0), (1, 128, 0), (1, 128, 8), (2, 64, 3), (1, 64, 16)])
@pytest.mark.parametrize("cap,slope", [(0.0, False), (20.0, False), (0.0, True), (20.0, True)])
def test_outputs_are_rounded_once(monkeypatch, members, prompts, lists, h, D, G, cap, slope):
    monkeypatch.setattr(test_gpu_shared, "attended", attended)
    s = Shared(members, prompts, lists, h, D, "bf16", G, q_scale=0.7)
    mods = dict(softcap=cap, slopes=torch.tensor([2.0 ** -(7 + i % 4) for i in range(h * s.G)], device=DEV) if slope else None)
    s.run(**mods)
    s.check(**mods)

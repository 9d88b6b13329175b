"""Sequences without new tokens in a call of prompt tokens: adsa_append and adsa_prefill leave them alone, whatever else their records and the call say."""
import numpy as np
import pytest
import torch

from paper_2506_18226_amd import binding as B

from prompt_common import f64, randn
from test_gpu_prefill import Prompt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("shape", [dict(lens=[5, 0, 33, 0, 0, 1], past=37, h=2), dict(lens=[150, 0, 0, 40, 200, 0], past=300, h=1, cap=700), dict(lens=[0, 70] * 70, past=3, h=2)],
                         ids=["few", "split", "many"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_idle_sequences_keep_their_records(shape, dtype):
    """One slot0 for all, behind which idle sequences have fewer resident slots (none, some, a count that is no cache's, a hole)."""
    p = Prompt(dtype=dtype, D=64, **shape)
    s = p.batch.read_seqs()
    idle = np.flatnonzero(p.lens == 0)
    s["n_res"][idle] = [0, 2, -7, p.batch.params.cap + 5][: len(idle)] if len(idle) <= 4 else np.arange(len(idle)) % 3
    s["hole"][idle[-1]] = 1
    p.batch.upload_seqs()
    before = p.batch.read_seqs().copy()
    gen = torch.Generator().manual_seed(5)
    k, v = (randn(gen, p.T, p.h, 64, dtype=p.batch.tdtype).to(DEV) for _ in range(2))
    p.batch.append(p.tokens, None, p.q, k, v, torch.empty_like(p.q))
    after_append = p.batch.read_seqs().copy()
    s = p.batch.seqs_host
    s["step"] = 3
    p.batch.upload_seqs()
    p.batch.score.copy_(torch.from_numpy(p.score0))
    p.run(flags=B.FLAG_ADVANCE)
    after = p.batch.read_seqs()
    assert not after_append["status"].any() and not after["status"].any()
    for f in ("n_res", "hole", "pending_slot", "compacted"):
        assert (before[f][idle] == after_append[f][idle]).all() and (before[f][idle] == after[f][idle]).all()
    assert (after["step"] == np.where(p.lens > 0, 4, 3)).all()
    assert np.array_equal(f64(p.batch.score)[idle], p.score0[idle])
    p.check()

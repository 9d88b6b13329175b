"""The attention mass of a document's slots is its own rows' business: NaN among another document's rows, keys or padding does not reach it."""
import numpy as np
import pytest
import torch

from test_gpu_prefill import Prompt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


@pytest.mark.parametrize("dtype,D,G", [("bf16", 64, 0), ("bf16", 128, 2), ("f32", 64, 0), ("f32", 128, 0)])
@pytest.mark.parametrize("lens,past", [([90], 0), ([300], 0), ([40], 200)])
@pytest.mark.parametrize("where", ["query", "key"])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_documents_do_not_spoil_each_other(dtype, D, G, lens, past, where, cap):
    """Documents of 20 slots; a row (the last one among them) or a key of two of them is NaN."""
    p = Prompt(lens, past, 2, D, dtype, G)
    doc = (torch.arange(p.batch.params.cap) // 20).to(torch.int32)[None].contiguous().to(DEV)
    n, a = int(p.keys[0]), int(p.past[0])
    spoilt = [a + 7, n - 1]                                  # slots of new tokens
    p.run(doc=doc, softcap=cap)
    clean, out = p.batch.score.clone(), p.out.clone()
    for s in spoilt:
        if where == "query":
            p.q[s - a] = NAN
        else:
            p.K[0, :, s, 5] = NAN
    p.batch.score.copy_(torch.from_numpy(p.score0))
    p.run(doc=doc, softcap=cap)
    touched = np.isin(np.arange(p.batch.params.cap) // 20, [s // 20 for s in spoilt]) & (np.arange(p.batch.params.cap) < n)
    at = torch.from_numpy(~touched).to(DEV)
    assert torch.equal(p.batch.score[0][:, at], clean[0][:, at])
    rows = torch.from_numpy(~touched[a:n]).to(DEV)
    assert torch.equal(p.out[rows], out[rows])
    for s in spoilt:                                         # and the slots that a spoilt row sees are
        assert p.batch.score[0, :, s // 20 * 20:s + 1].isnan().all()


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 128)])
def test_a_spoilt_prefix_row_spoils_what_it_sees(dtype, D):
    """Without documents: a NaN row in the middle gives NaN to the slots before it and leaves later ones alone."""
    p = Prompt([150], 0, 2, D, dtype)
    p.run()
    clean = p.batch.score.clone()
    p.q[70] = NAN
    p.batch.score.copy_(torch.from_numpy(p.score0))
    p.run()
    assert p.batch.score[0, :, :71].isnan().all() and torch.equal(p.batch.score[0, :, 71:], clean[0, :, 71:])

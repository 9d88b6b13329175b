"""Batches whose records were not uploaded yet: inactive, with their arrays in place."""
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch, ModelBatch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("layout", ["head_major", "slot_major"])
def test_a_dense_batch_without_records_is_inactive(layout):
    """The records' addresses are looked at before anything follows them."""
    p = B.make_params(n_seq=2, n_heads=3, head_dim=64, grid_h=9, grid_w=5, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=64, layout=layout)
    batch = LayerBatch(p, DEV)
    records = batch.read_seqs()
    assert (records["step"] == -1).all() and (records["n_res"] == 0).all() and (records["status"] == 0).all()
    for name, whole in (("k", batch.K), ("v", batch.V), ("pos", batch.pos), ("score", batch.score)):
        assert records[name].tolist() == [whole[b].data_ptr() for b in range(2)], name
    rows = [torch.ones(2, 3, 64, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    batch.out.fill_(7)
    batch.step(*rows)
    torch.cuda.synchronize()
    assert not batch.out.any() and not batch.K.any() and (batch.read_seqs()["n_res"] == 0).all() and (batch.seqs_host["step"] == -1).all()
    begin = torch.tensor([0, 1, 1], dtype=torch.int32, device=DEV)
    batch.append(B.make_tokens(begin, torch.zeros(2, dtype=torch.int32, device=DEV), 1, 1), None, *rows, torch.empty_like(rows[0]), flags=B.FLAG_ADVANCE)
    torch.cuda.synchronize()
    assert batch.read_seqs()["n_res"].tolist() == [1, 0] and not batch.seqs_host["status"].any() and int((batch.K != 0).sum()) == 3 * 64
    model = ModelBatch(p, 2, DEV)
    assert (model.read_seqs()["step"] == -1).all() and (model.seqs_host["pos"] != 0).all()

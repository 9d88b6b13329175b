"""The host's side of caches in pages: what a batch does with its table and its free pages.  (No GPU: the pools are host tensors.)"""
import numpy as np
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import PagedBatch


def host_batch(n_seq=4, cap=64, page=16, n_pages=8, layout="head_major"):
    batch = PagedBatch.__new__(PagedBatch)                   # (without the device's workspace)
    batch.params = B.make_params(n_seq=n_seq, n_heads=2, head_dim=64, grid_h=8, grid_w=8, win_rows_back=1, win_col_radius=2, dtype=B.F32, score_mode=B.SCORE_ATTN_MASS, cap=cap, layout=layout)
    batch.page_size, batch.n_pages, batch.device, batch.tdtype, batch.head_major = page, n_pages, torch.device("cpu"), torch.float32, layout == "head_major"
    batch.seqs_host, batch.vcos_u = np.zeros(n_seq, dtype=B.SEQ_DTYPE), None
    batch.pos, batch.score = torch.zeros(n_seq, cap, dtype=torch.int32), torch.zeros(n_seq, 2, cap)
    batch._allocate_caches()
    batch.table = batch.table.clone()                        # (host tensors of numpy arrays share their memory)
    return batch


def rows(n, value):
    return np.full((n, 2, 64), value, dtype=np.float32)


# ---------------------------------------------------------------------------------------------------- rows of sequences without pages
@pytest.mark.parametrize("layout", ["head_major", "slot_major"])
def test_rows_of_slots_without_a_page_are_refused(layout):
    """A table's -1 is no page: neither written (it would be the last of the pool, somebody else's) nor read."""
    batch = host_batch(layout=layout)
    batch.reserve(1, 64)
    batch.reserve(2, 17)
    batch.table_host[1] = batch.table_host[1][::-1].copy()
    batch.upload_table()
    batch.K.fill_(3.0)
    batch.V.fill_(4.0)
    call = dict(pos=np.arange(20), score=None, step=1, grid_origin=20)
    record = batch.seqs_host.copy()
    for b, n in ((0, 20), (0, 1), (2, 33)):                  # no page at all; one slot more than the pages have
        with pytest.raises(ValueError, match="page"):
            batch.set_sequence(b, k=rows(n, 9.0), v=rows(n, 9.0), **{**call, "pos": np.arange(n)})
        with pytest.raises(ValueError, match="page"):
            batch.cache_rows(batch.K, b, n)
    batch.reserve(3, 16)                                     # not in the device's table yet
    with pytest.raises(ValueError, match="upload_table"):
        batch.set_sequence(3, k=rows(5, 9.0), v=rows(5, 9.0), **{**call, "pos": np.arange(5)})
    batch.table[0, 0] = batch.n_pages                        # beyond the pool
    with pytest.raises(ValueError, match="page"):
        batch._put_rows(0, torch.zeros(2, 2, 64), torch.zeros(2, 2, 64))
    assert (batch.K == 3.0).all() and (batch.V == 4.0).all() and (batch.seqs_host == record).all() and not batch.pos.any()
    batch.upload_table()
    batch.set_sequence(3, k=rows(5, 9.0), v=rows(5, 8.0), **{**call, "pos": np.arange(5)})
    batch.set_sequence(0, k=rows(0, 9.0), v=rows(0, 8.0), **{**call, "pos": np.arange(0)})           # (no row, no page)
    assert (batch.cache_rows(batch.K, 3, 5) == 9.0).all() and (batch.cache_rows(batch.V, 3, 5) == 8.0).all() and int((batch.K != 3.0).sum()) == 5 * 2 * 64
    assert batch.cache_rows(batch.K, 0, 0).shape[0] == 0

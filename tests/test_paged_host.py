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


# ---------------------------------------------------------------------------------------------------- pages of several sequences
def in_use(batch):
    return set(batch.table_host[batch.table_host >= 0].tolist())


def all_there(batch, lost=()):
    """Every page is free, once, or in the table."""
    assert len(set(batch.free_pages)) == len(batch.free_pages) and not in_use(batch) & set(batch.free_pages)
    assert in_use(batch) | set(batch.free_pages) | set(lost) == set(range(batch.n_pages))


def test_a_shared_page_is_free_when_the_last_of_its_sequences_gives_it_back():
    batch = host_batch(n_pages=9)
    batch.reserve(0, 64)
    batch.share(1, 0, 40)                                    # two whole pages
    batch.reserve(1, 64)
    assert list(batch.table_host[1, :2]) == list(batch.table_host[0, :2]) and not set(batch.table_host[1, 2:]) & set(batch.table_host[0]) and len(batch.free_pages) == 3
    all_there(batch)
    prompt = set(batch.table_host[0, :2].tolist())
    batch.release(0)
    assert len(batch.free_pages) == 5 and not prompt & set(batch.free_pages)
    batch.reserve(2, 64)                                     # none of the pages that 1 still has
    assert not set(batch.table_host[2].tolist()) & set(batch.table_host[1].tolist())
    all_there(batch)
    batch.release(1, 32)
    all_there(batch)
    batch.release(1)
    batch.release(1)
    all_there(batch)
    assert prompt <= set(batch.free_pages)
    batch.release(2, 17)
    all_there(batch)
    batch.reserve(3, 64)
    with pytest.raises(MemoryError):
        batch.reserve(0, 64)
    assert (batch.table_host[0] == -1).all()
    all_there(batch)


def test_pages_that_sharing_replaces_are_free():
    batch = host_batch(n_pages=9)
    for b in (0, 1):
        batch.reserve(b, 64)
    own = set(batch.table_host[1, :3].tolist())
    batch.share(1, 0, 48)
    assert own <= set(batch.free_pages)
    batch.share(1, 0, 48)                                    # once more: as it is
    batch.share(0, 0, 64)
    all_there(batch)
    for what in ((2, 3, 16), (2, 0, 65), (2, 0, -1)):        # who has no page; no such slots
        with pytest.raises(ValueError):
            batch.share(*what)
    batch.share(2, 0, 15)                                    # no whole page
    assert (batch.table_host[2] == -1).all()
    all_there(batch)


def test_rows_written_by_hand():
    """Numbers that a program writes into the table: a page in two rows is given back once, one that is taken is not given again, what is no page is forgotten."""
    batch = host_batch(n_pages=9)
    batch.reserve(0, 32)
    batch.table_host[1, :2] = batch.table_host[0, :2]
    batch.table_host[2, :2] = batch.free_pages[-1], 0x7FFFFFFF
    hand = batch.free_pages[-1]
    batch.reserve(3, 64)
    assert hand not in batch.table_host[3] and hand not in batch.free_pages
    all_there(type("without", (), dict(table_host=np.where(batch.table_host == 0x7FFFFFFF, -1, batch.table_host), free_pages=batch.free_pages, n_pages=9)))
    with pytest.raises(ValueError):
        batch.share(0, 2, 32)                                # one of them is no page
    batch.reserve(2, 32)                                     # gets one in its place
    assert 0 <= batch.table_host[2, 1] < 9 and batch.table_host[2, 0] == hand
    for b in range(4):
        batch.release(b)
    assert sorted(batch.free_pages) == list(range(9)) and (batch.table_host == -1).all()


def test_batches_that_take_their_pages_from_one_list():
    a, b = host_batch(n_seq=2, n_pages=8), host_batch(n_seq=2, n_pages=8)
    b.free_pages = a.free_pages
    a.reserve(0, 64)
    b.reserve(0, 48)
    a.reserve(1, 16)
    assert not b.free_pages and b.free_pages is a.free_pages and sorted(in_use(a) | in_use(b)) == list(range(8))
    with pytest.raises(MemoryError):
        b.reserve(1, 16)
    a.release(0, 20)
    b.reserve(1, 32)
    assert not a.free_pages and sorted(in_use(a) | in_use(b)) == list(range(8))


def test_layers_that_go_by_one_table():
    first, second = host_batch(n_pages=8), host_batch(n_pages=8)
    second.reserve(0, 16)
    second.use_table(first)
    assert second.pages.table == first.table.data_ptr() and second.pages.k == second.K.data_ptr() != first.K.data_ptr()
    first.reserve(1, 40)
    second.share(2, 1, 32)
    second.upload_table()
    for value, batch in ((2.0, first), (5.0, second)):
        batch.set_sequence(1, k=rows(40, value), v=rows(40, value), pos=np.arange(40), score=None, step=1, grid_origin=40)
    assert (first.cache_rows(first.K, 2, 32) == 2.0).all() and (second.cache_rows(second.K, 2, 32) == 5.0).all()
    first.release(1)
    second.release(2)
    assert len(first.free_pages) == 8 and second.free_pages is first.free_pages
    for other in (host_batch(n_pages=9), host_batch(page=32), host_batch(n_seq=3), host_batch(cap=65)):
        with pytest.raises(ValueError):
            second.use_table(other)

"""The same cache rows in pages: pools whose pages lie in any order, with NaN in pages and slots that are nobody's."""
import numpy as np
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import PagedBatch

DEV = "cuda:0"


def paged_twin(dense, page, *, layout="head_major", spare=3, seed=3, resident=None, interleaved=False, far=False):
    """A PagedBatch with the records, positions, scores and rows of a LayerBatch.  resident: slots that have a page (all of cap if None); far: pages so far
    apart that a pool spans more than 4 GiB."""
    p = dense.params
    params = B.make_params(n_seq=p.n_seq, n_heads=p.n_heads, head_dim=p.head_dim, grid_h=p.grid_h, grid_w=p.grid_w, win_rows_back=p.win_rows_back,
                           win_col_radius=p.win_col_radius, dtype=p.dtype, score_mode=p.score_mode, cap=p.cap, sel_cap=p.sel_cap, layout=layout,
                           softmax_scale=p.softmax_scale, win_recent_m=p.win_recent_m, evict_policy=p.evict_policy, q_per_kv=p.q_per_kv)
    resident = [p.cap] * p.n_seq if resident is None else [int(x) for x in resident]
    need = [-(-n // page) for n in resident]
    paged = PagedBatch(params, n_pages=sum(need) + spare, page_size=page, device=DEV)
    order = np.random.default_rng(seed).permutation(paged.n_pages)
    at = 0
    for b, n in enumerate(need):
        paged.table_host[b, :n] = order[at:at + n]
        paged.table_host[b, n:] = np.random.default_rng(seed + b).choice([-1, -7, paged.n_pages, 0x7FFFFFFF], paged.table_host.shape[1] - n)
        at += n
    paged.upload_table()
    if interleaved:                                          # K and V of a page side by side in one pool
        both = torch.empty((2, *paged.K.shape), dtype=paged.tdtype, device=DEV).transpose(0, 1).contiguous()
        paged.K, paged.V = both[:, 0], both[:, 1]
        paged.pages = B.make_pages(paged.K, paged.V, paged.table, page_size=page, layout=layout)
    if far:
        stride = max((1 << 32) // paged.K.element_size() // paged.n_pages, paged.K.stride(0)) // 64 * 64 + 64
        paged.K, paged.V = (torch.empty(paged.n_pages * stride, dtype=paged.tdtype, device=DEV).as_strided(paged.K.shape, (stride, *paged.K.stride()[1:])) for _ in range(2))
        paged.pages = B.make_pages(paged.K, paged.V, paged.table, page_size=page, layout=layout)
    paged.K.fill_(float("nan"))
    paged.V.fill_(float("nan"))
    K, V = (t if dense.head_major else t.transpose(1, 2) for t in (dense.K, dense.V))          # [n][h][cap][D]
    for b, n in enumerate(resident):
        if n:
            paged._put_rows(b, K[b, :, :n].transpose(0, 1), V[b, :, :n].transpose(0, 1))
    paged.pos.copy_(dense.pos)
    paged.score.copy_(dense.score)
    paged.sel_idx.copy_(dense.sel_idx)
    paged.sel_cnt.copy_(dense.sel_cnt)
    host = dense.read_seqs().copy()
    for name in ("n_res", "step", "grid_origin", "n_keep_prefix", "budget", "budget_num", "budget_den", "status", "compacted", "pending_slot", "hole"):
        paged.seqs_host[name] = host[name]
    assert (paged.seqs_host["k"] == 0).all()
    paged.upload_seqs()
    return paged


def same_bits(a, b):
    """Equal, a NaN being equal to a NaN."""
    a, b = a.contiguous(), b.contiguous()
    kind = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return a.shape == b.shape and (torch.equal(a.view(kind), b.view(kind)) or torch.equal(torch.nan_to_num(a.float(), 7e30), torch.nan_to_num(b.float(), 7e30)))


def records(batch):
    """What a record says of its sequence, the addresses apart."""
    s = batch.read_seqs()
    return {name: s[name].copy() for name in ("n_res", "step", "grid_origin", "n_keep_prefix", "budget", "status", "compacted", "pending_slot", "hole")}


def same_records(a, b):
    x, y = records(a), records(b)
    for name in x:
        assert np.array_equal(x[name], y[name]), (name, x[name], y[name])

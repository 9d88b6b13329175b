"""Layers of a model over pages, by one table for all of them, against layers with tables of their own; prefixes given by share()."""
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import PagedBatch

from paged_common import same_bits, same_records
from prompt_common import randn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("G,layout", [(0, "head_major"), (4, "slot_major")])
def test_one_table_for_all_layers(G, layout):
    n, h, D, W, P, layers = 3, 2, 64, 6, 32, 3
    cap, gen = P + 8 + 3 * W, torch.Generator().manual_seed(6)
    kw = dict(n_seq=n, n_heads=h, head_dim=D, grid_h=9, grid_w=W, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=cap, q_per_kv=G, layout=layout)
    own, one = ([PagedBatch(B.make_params(**kw), n_pages=16, page_size=16, device=DEV) for _ in range(layers)] for _ in range(2))
    for batch in one[1:]:
        batch.use_table(one[0])
    rows = [randn(gen, P, h, D, dtype=torch.bfloat16).to(DEV) for _ in range(layers)]
    for batch in own + one:
        s = batch.seqs_host
        s["grid_origin"] = s["n_keep_prefix"] = s["n_res"] = P
        s["budget"], s["step"] = 8, 1
        batch.upload_seqs()
        batch.pos[:] = torch.arange(cap, dtype=torch.int32, device=DEV)
    for batch in own + one[:1]:
        batch.reserve(0, cap)
        for b in (1, 2):
            if batch is one[0]:
                batch.share(b, 0, P)
            batch.reserve(b, cap)
        batch.upload_table()
    for batches in (own, one):
        for batch, x in zip(batches, rows):
            for b in range(n):
                batch._put_rows(b, x, x * 2)
    hq = h * max(G, 1)
    for t in range(3 * W + 1):
        for i in range(layers):
            q, k, v = (randn(gen, n, heads, D, dtype=torch.bfloat16).to(DEV) for heads in (hq, h, h))
            for batch in (own[i], one[i]):
                batch.step(q, k, v)
            torch.cuda.synchronize()
            same_records(own[i], one[i])
            assert same_bits(own[i].out, one[i].out) and same_bits(own[i].lse, one[i].lse), (t, i)
        n_res = one[0].read_seqs()["n_res"]
        for b in range(n):                                   # what evictions have left empty, and the next token's
            one[0].release(b, int(n_res[b]))
            one[0].reserve(b, min(int(n_res[b]) + 1, cap))
        one[0].upload_table()
    assert not any(batch.read_seqs()["status"].any() for batch in own + one)
    assert all(same_bits(batch.cache_rows(batch.K, b, P), x) for batch, x in zip(one, rows) for b in range(n))
    for b in range(n):
        one[0].release(b)
    assert sorted(one[2].free_pages) == list(range(16))

"""Caches of as many slots as there may be, in the smallest pages: a table's row of 512 entries, all of which are used.  Against the dense calls' bits."""
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch, PagedBatch, Sampler

from common import plan_of
from paged_common import paged_twin, same_bits, same_records
from prompt_common import randn
from test_gpu_paged import DEV, Decode
from test_gpu_prefill import Prompt

pytestmark = pytest.mark.gpu
CAP = B.MAX_CAP


@pytest.mark.parametrize("G,D,dtype", [(0, 64, "bf16"), (0, 128, "f32"), (4, 64, "bf16"), (4, 128, "bf16")])
@pytest.mark.parametrize("far", [False, True])
def test_single_tokens(G, D, dtype, far):
    d = Decode([CAP, 1, 5000], CAP, 1, D, dtype, G, cap=CAP)
    assert plan_of(d.batch.params).chunks > 1
    paged = paged_twin(d.batch, 16, resident=d.resident, far=far)
    assert paged.table.shape[1] == 512 and (paged.table_host[0] >= 0).all()
    k, v = d.rows(False)
    for batch in (d.batch, paged):
        batch.attend(d.q, B.FLAG_APPEND | B.FLAG_ADVANCE, k, v)
    torch.cuda.synchronize()
    same_records(d.batch, paged)
    assert same_bits(d.batch.out, paged.out) and same_bits(d.batch.lse, paged.lse) and same_bits(d.batch.score, paged.score)
    last = paged.cache_rows(paged.K, 0, CAP)[-1]
    assert same_bits(last, k[0])
    paged.table[0, 511] = paged.n_pages                      # the last entry is looked at, too
    paged.attend(d.q, B.FLAG_APPEND, k, v)
    torch.cuda.synchronize()
    assert list(paged.read_seqs()["status"]) == [B.SEQ_BAD_STATE, 0, 0] and not paged.out[0].any() and same_bits(d.batch.out[1:], paged.out[1:])


@pytest.mark.parametrize("lens", [[3, 2], [200, 64]])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 64), ("bf16", 128)])
def test_prompts(lens, dtype, D):
    p = Prompt(lens, [CAP - x for x in lens], 1, D, dtype, cap=CAP)
    paged = paged_twin(p.batch, 16, resident=p.keys)
    p.run()
    want = [t.clone() for t in (p.out, p.lse, p.batch.score)]
    paged.prefill(p.tokens, p.q, p.out, p.lse)
    torch.cuda.synchronize()
    assert all(same_bits(a, b) for a, b in zip((p.out, p.lse, paged.score), want)) and not paged.read_seqs()["status"].any()
    paged.table[1, 511] = -1
    paged.prefill(p.tokens, p.q, p.out, p.lse)
    torch.cuda.synchronize()
    x = int(p.begin[1])
    assert list(paged.read_seqs()["status"]) == [0, B.SEQ_BAD_STATE] and same_bits(p.out[:x], want[0][:x]) and not p.out[x:].any()


def test_the_whole_cache_enters_at_once():
    n, h, D = 2, 2, 64
    p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=91, grid_w=91, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=CAP)
    dense, paged = LayerBatch(p, DEV), PagedBatch(p, n_pages=1024, page_size=16, device=DEV)
    for b in range(n):
        paged.reserve(b, CAP)
    paged.upload_table()
    assert not paged.free_pages
    for batch in (dense, paged):
        batch.seqs_host["step"] = 0
        batch.upload_seqs()
    gen = torch.Generator().manual_seed(3)
    k, v = (randn(gen, n * CAP, h, D, dtype=torch.bfloat16).to(DEV) for _ in range(2))
    tokens = B.make_tokens(torch.tensor([0, CAP, 2 * CAP], dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV), n * CAP, CAP)
    for batch in (dense, paged):
        batch.append(tokens, None, None, k, v, None)
    torch.cuda.synchronize()
    same_records(dense, paged)
    assert (paged.seqs_host["n_res"] == CAP).all() and same_bits(paged.cache_rows(paged.K, 1, CAP), k[CAP:]) and same_bits(paged.cache_rows(paged.V, 0, CAP), v[:CAP])


def test_the_most_rows_of_logits():
    """2^20 rows of three: the first of the largest, and where a random number falls among all of them."""
    n = 1 << 20
    logits = torch.randint(-3, 4, (n, 3), generator=torch.Generator().manual_seed(1)).float().to(DEV)
    u = torch.rand(n, generator=torch.Generator().manual_seed(2)).to(DEV)
    s = Sampler(n, 3, B.F32, temperature=0.0, device=DEV)
    s.sample(logits, u)
    first = (logits == logits.max(1, keepdim=True)[0]).int().argmax(1).int()
    assert torch.equal(s.token, first)
    s = Sampler(n, 3, B.F32, device=DEV)
    s.sample(logits, u)
    p = torch.softmax(logits.double(), 1)
    sums = torch.cumsum(p, 1)
    want = (sums <= u.double()[:, None]).sum(1).clamp(max=2).int()
    near = ((sums - u.double()[:, None]).abs() < 2.0 ** -40).any(1)          # (a sum of three whole numbers of 2^-44, and the reference's own roundings)
    assert torch.equal(s.token[~near], want[~near]) and int(near.sum()) < 10
    assert ((s.logprob.double() - torch.log(p.gather(1, s.token.long()[:, None])[:, 0])).abs() <= 2.0 ** -21).all()

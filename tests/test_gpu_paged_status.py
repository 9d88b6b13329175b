"""Single tokens over pages of sequences that have a status before the call, with a list of their own: skipped, whichever way the launch goes."""
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import PagedBatch

from common import plan_of
from paged_common import paged_twin, same_bits
from test_gpu_paged import DEV, Decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", [0, 4])
@pytest.mark.parametrize("lists,resident,split", [([30, 40, 50], 60, False), ([2900, 2950, 2800], 3000, True), ([1, 1, 1], 3000, True)])
@pytest.mark.parametrize("status", [B.SEQ_CACHE_FULL, B.SEQ_BAD_STATE, B.SEQ_SEL_OVERFLOW, 7])
def test_single_tokens_of_a_sequence_with_a_status(G, lists, resident, split, status):
    d = Decode(lists, resident, 2, 64, "bf16", G, cap=resident + 40, sel_cap=max(max(lists), 2950 if split else 1))
    assert (plan_of(d.batch.params).chunks > 1) == split
    good, paged = (paged_twin(d.batch, 16, resident=d.resident) for _ in range(2))
    k, v = d.rows(False)
    good.attend(d.q, B.FLAG_APPEND | B.FLAG_ADVANCE, k, v)
    paged.seqs_host["status"][1] = status
    paged.upload_seqs()
    paged.workspace.fill_(0x7F)                              # whatever partial sums are left over there
    paged.out.fill_(3.0)
    paged.lse.fill_(3.0)
    K, V, score = paged.K.clone(), paged.V.clone(), paged.score.clone()
    for _ in range(2):                                       # the second call finds the partial sums of the first
        paged.attend(d.q, B.FLAG_APPEND, k, v)
    torch.cuda.synchronize()
    assert not paged.out[1].any() and not paged.lse[1].any() and same_bits(paged.score[1], score[1])
    assert same_bits(paged.out[0], good.out[0]) and same_bits(paged.out[2], good.out[2]) and same_bits(paged.lse[0], good.lse[0])
    paged.attend(d.q, B.FLAG_APPEND | B.FLAG_ADVANCE, k, v)
    torch.cuda.synchronize()
    r = paged.read_seqs()
    assert list(r["status"]) == [0, status, 0] and list(r["step"]) == [5, 4, 5] and (r["n_res"] == resident).all()
    mine = torch.from_numpy(paged.table_host[1, :-(-resident // 16)]).long().to(paged.device)
    assert same_bits(paged.K[mine], K[mine]) and same_bits(paged.V[mine], V[mine])
    paged.seqs_host["status"][1] = 0                         # cleared: attended as the others were
    paged.upload_seqs()
    paged.attend(d.q, B.FLAG_APPEND | B.FLAG_NO_ACCUMULATE | B.FLAG_ADVANCE, k, v)
    torch.cuda.synchronize()
    assert same_bits(paged.out, good.out) and same_bits(paged.lse, good.lse)
    assert list(paged.read_seqs()["step"]) == [6, 5, 6]


@pytest.mark.parametrize("G,D", [(0, 64), (0, 128), (8, 64), (8, 128)])
@pytest.mark.parametrize("length,entry", [(40, 250), (300, 131), (300, 0), (300, 255)])
def test_workgroups_that_start_after_a_sequence_got_its_status(G, D, length, entry):
    """More workgroups than the card holds at once, of which the first find that an entry is no page: the later ones, some of whose waves see the status, skip their sequences all the same."""
    n, h, resident = 24, 32 if G else 96, 4090              # 256 pages a sequence: every thread has some, and the bad one is some thread's alone
    p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=90, grid_w=90, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=4096, sel_cap=length, q_per_kv=G)
    paged = PagedBatch(p, n_pages=64, page_size=16, device=DEV)
    assert plan_of(p).chunks == 1
    paged.table.copy_(torch.randint(0, 64, tuple(paged.table.shape), generator=torch.Generator().manual_seed(3)).to(torch.int32))          # (any pages of the pool will do)
    paged.table[::2, entry] = 64
    paged.K.fill_(0.5)
    paged.V.fill_(0.5)
    paged.sel_idx.copy_(torch.arange(length, dtype=torch.int32) * 13)
    paged.sel_cnt.fill_(length)
    paged.seqs_host["n_res"], paged.seqs_host["step"] = resident, 4
    paged.upload_seqs()
    q = torch.ones(n, h * max(G, 1), D, dtype=torch.bfloat16, device=DEV)
    paged.out.fill_(3.0)
    paged.lse.fill_(3.0)
    score = paged.score.clone()
    paged.attend(q, 0)
    torch.cuda.synchronize()
    assert list(paged.read_seqs()["status"]) == [B.SEQ_BAD_STATE, 0] * (n // 2)
    assert not paged.out[::2].any() and not paged.lse[::2].any() and same_bits(paged.score[::2], score[::2])
    assert (paged.out[1::2] == 0.5).all() and torch.isfinite(paged.lse[1::2]).all()


@pytest.mark.parametrize("dtype,D,G", [(B.BF16, 64, 0), (B.BF16, 128, 4), (B.F32, 64, 0), (B.F32, 128, 0)])
@pytest.mark.parametrize("tokens,h", [(2, 32), (200, 32)])
@pytest.mark.parametrize("entry", [0, 63, 250])
def test_prompts_whose_workgroups_start_after_a_sequence_got_its_status(dtype, D, G, tokens, h, entry):
    """As above, for chunks of new tokens behind some 4000 slots, few rows and many."""
    n, resident = 12, 4090
    p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=90, grid_w=90, win_rows_back=1, win_col_radius=2, dtype=dtype, score_mode=B.SCORE_ATTN_MASS, cap=4096, q_per_kv=G)
    paged = PagedBatch(p, n_pages=64, page_size=16, device=DEV)
    paged.table.copy_(torch.randint(0, 64, tuple(paged.table.shape), generator=torch.Generator().manual_seed(3)).to(torch.int32))
    paged.table[::2, entry] = -1
    paged.K.fill_(0.5)
    paged.V.fill_(0.5)
    paged.seqs_host["n_res"], paged.seqs_host["step"] = resident, 4
    paged.upload_seqs()
    hq, T = h * max(G, 1), n * tokens
    begin = torch.arange(n + 1, dtype=torch.int32, device=DEV) * tokens
    new = B.make_tokens(begin, torch.full((n,), resident - tokens, dtype=torch.int32, device=DEV), T, tokens)
    q = torch.ones(T, hq, D, dtype=paged.tdtype, device=DEV)
    out, lse = torch.full((T, hq, D), 3.0, dtype=paged.tdtype, device=DEV), torch.full((T, hq), 3.0, device=DEV)
    paged.prefill(new, q, out, lse)
    torch.cuda.synchronize()
    assert list(paged.read_seqs()["status"]) == [B.SEQ_BAD_STATE, 0] * (n // 2)
    out, lse = out.view(n, tokens, hq, D), lse.view(n, tokens, hq)
    assert not out[::2].any() and not lse[::2].any() and not paged.score[::2].any()
    # a mean of halves, whose probabilities and sum are off by 2^-8 at most, and a rounding
    assert ((out[1::2].float() - 0.5).abs() <= 0.5 * 2.0 ** -7).all() and torch.isfinite(lse[1::2]).all()
    mass = paged.score[1::2].double().sum(-1)                # every row gives 1 in all: tokens * G a cache head, each share off by some 2^-16
    assert ((mass - tokens * max(G, 1)).abs() <= tokens * max(G, 1) * 2.0 ** -7).all()

"""Single tokens over pages of sequences that have a status before the call, with a list of their own: skipped, whichever way the launch goes."""
import pytest
import torch

from paper_2506_18226_amd import binding as B

from common import plan_of
from paged_common import paged_twin, same_bits
from test_gpu_paged import Decode

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

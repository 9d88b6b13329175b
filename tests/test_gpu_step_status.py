"""adsa_step of few pairs, whose workgroups each rank for themselves: a record that only some slots show to be unfit is refused by all of them alike, and its status written
when none of them reads it any more."""
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch

from common import plan_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype,D,cap,at", [(B.BF16, 64, 250, 240), (B.BF16, 64, 700, 255), (B.BF16, 64, 700, 690), (B.BF16, 64, 1000, 3), (B.BF16, 64, 1000, 980), (B.BF16, 128, 700, 600),
                                            (B.F32, 64, 250, 70), (B.F32, 64, 700, 511)])
@pytest.mark.parametrize("what", ["newer", "long"])
def test_records_that_one_wave_finds_unfit(dtype, D, cap, at, what):
    n, h, W = 3, 31, 20
    p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=60, grid_w=W, win_rows_back=1, win_col_radius=2, dtype=dtype, score_mode=B.SCORE_ATTN_MASS, cap=cap, sel_cap=cap - 5)
    assert plan_of(p).eviction == 2
    batch = LayerBatch(p, DEV)
    gen = torch.Generator().manual_seed(1)
    rows = [torch.randn(n, h, D, generator=gen).to(batch.tdtype).to(DEV) for _ in range(3)]
    resident, prefix = cap - 2, cap - 80
    for trial in range(8):
        batch.K.fill_(0.25)
        batch.V.fill_(0.25)
        batch.score.uniform_()
        batch.pos.copy_(torch.arange(cap, dtype=torch.int32))
        s = batch.seqs_host
        s["n_res"], s["step"], s["status"], s["grid_origin"], s["n_keep_prefix"], s["budget"] = resident, resident - prefix + 1, 0, prefix, prefix, 0
        if what == "newer":                                  # a position behind the query token's
            batch.pos[1, at] = cap + 7
        else:                                                # all are pinned, more than a list holds
            s["grid_origin"][1] = s["n_keep_prefix"][1] = resident
            s["step"][1] = 1
        batch.upload_seqs()
        batch.out.fill_(3.0)
        batch.lse.fill_(3.0)
        K, score, pos = batch.K.clone(), batch.score.clone(), batch.pos.clone()
        batch.step(*rows)
        torch.cuda.synchronize()
        r = batch.read_seqs()
        assert list(r["status"]) == [0, B.SEQ_BAD_STATE if what == "newer" else B.SEQ_SEL_OVERFLOW, 0], trial
        assert r["n_res"][1] == resident and r["step"][1] == (resident - prefix + 1 if what == "newer" else 1) and r["pending_slot"][1] == -1
        assert not batch.out[1].any() and not batch.lse[1].any() and torch.equal(batch.score[1], score[1]) and torch.equal(batch.pos[1], pos[1])
        assert torch.equal(batch.K[1], K[1]) and batch.out[0].any() and batch.out[2].any()
        batch.step(*rows)                                    # with a status: skipped
        torch.cuda.synchronize()
        assert list(batch.read_seqs()["status"]) == [0, int(r["status"][1]), 0] and not batch.out[1].any() and torch.equal(batch.score[1], score[1])

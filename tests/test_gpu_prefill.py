"""Attention of prompts over their caches, against 64-bit sums on the host: masks, caps, distances, odd sizes, split keys, what masked
places hold, and the attention mass."""
import numpy as np
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch

from prompt_common import attended, close, f64, randn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


class Prompt:
    def __init__(self, lens, past, h, D, dtype="bf16", G=0, layout="head_major", cap=None, prefix=0, seed=1, q_scale=1.5, score_mode=B.SCORE_ATTN_MASS):
        self.lens, self.past = np.asarray(lens), np.broadcast_to(np.asarray(past), (len(lens),)).copy()
        n, self.h, self.D, self.G = len(lens), h, D, max(G, 1)
        self.keys = self.past + self.lens
        cap = int(self.keys.max()) + 3 if cap is None else cap
        p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=200, grid_w=200, win_rows_back=1, win_col_radius=2, dtype=B.F32 if dtype == "f32" else B.BF16,
                          score_mode=score_mode, cap=cap, layout=layout, q_per_kv=G)
        self.batch = LayerBatch(p, DEV)
        gen = torch.Generator().manual_seed(seed)
        dt = self.batch.tdtype
        self.bf16 = dt == torch.bfloat16
        rows = (lambda t: t) if layout == "head_major" else (lambda t: t.transpose(1, 2))
        self.K, self.V = rows(self.batch.K), rows(self.batch.V)
        for t in (self.K, self.V):
            t.copy_(randn(gen, n, h, cap, D, dtype=dt))
            for b in range(n):                               # rows that hold no token yet
                t[b, :, self.keys[b]:] = NAN
        self.T = int(self.lens.sum())
        self.begin = np.concatenate([[0], np.cumsum(self.lens)])
        self.q = randn(gen, self.T, h * self.G, D, dtype=dt, scale=q_scale).to(DEV)
        self.batch.pos[:] = 2 * torch.arange(cap, dtype=torch.int32, device=DEV) + 5
        s = self.batch.seqs_host
        s["n_res"], s["n_keep_prefix"], s["step"] = self.keys, prefix, 3
        self.prefix = prefix
        self.batch.upload_seqs()
        self.batch.score.uniform_(generator=torch.Generator(device=DEV).manual_seed(seed))
        self.score0 = f64(self.batch.score)
        self.tokens = B.make_tokens(torch.tensor(self.begin, dtype=torch.int32, device=DEV), torch.tensor(self.past, dtype=torch.int32, device=DEV), self.T,
                                    int(self.lens.max()))
        self.out = torch.full((self.T, h * self.G, D), 7.0, dtype=dt, device=DEV)
        self.lse = torch.full((self.T, h * self.G), 7.0, device=DEV)

    def run(self, flags=0, **mods):
        self.batch.prefill(self.tokens, self.q, self.out, self.lse, mods=B.make_mods(**mods) if mods else None, flags=flags)
        torch.cuda.synchronize()

    def check(self, mask=B.MASK_CAUSAL, softcap=0.0, slopes=None, doc=None, mass=True, sequences=None):
        K, V, q, out, lse, score = (f64(x) for x in (self.K, self.V, self.q, self.out, self.lse, self.batch.score))
        docs = None if doc is None else doc.cpu().numpy()
        want_score, tol_score = self.score0.copy(), 4 * 2.0 ** -24 * np.abs(self.score0)
        for b in range(len(self.lens)) if sequences is None else sequences:
            m, a, x, y = self.keys[b], self.past[b], self.begin[b], self.begin[b + 1]
            qs, ks = np.arange(a, m)[:, None], np.arange(m)[None]
            seen = ks <= qs
            if mask == B.MASK_PREFIX:
                seen = seen | ((qs < self.prefix) & (ks < self.prefix))
            if docs is not None:
                seen = seen & (docs[b, a:m, None] == docs[b, None, :m]) & (docs[b, None, :m] >= 0)
            for j in range(self.h * self.G):
                hd = j // self.G
                o, s, p, ot, st, pt = attended(q[x:y, j], K[b, hd, :m], V[b, hd, :m], self.D ** -0.5, seen=seen, cap=softcap,
                                               slope=0.0 if slopes is None else float(slopes[j]), dist=2 * (qs - ks), bf16=self.bf16)
                close(out[x:y, j], o, ot, f"out of sequence {b}, head {j}")
                close(lse[x:y, j], s, st, f"lse of sequence {b}, head {j}")
                if not mass:
                    continue
                want_score[b, hd, :m] += p.sum(0)
                tol_score[b, hd, :m] += (p * pt).sum(0) + 2.0 ** -22 * (1 + want_score[b, hd, :m])
        if sequences is None:
            if mass:
                close(score, want_score, tol_score, "mass")
            else:
                assert np.array_equal(score, self.score0)


LENS = [1, 2, 33, 0, 31, 64, 65, 5]
LONG = [129, 1, 200, 64, 0, 127]


@pytest.mark.parametrize("lens,past,h,D,dtype,G,layout", [
    (LENS, 0, 2, 64, "bf16", 0, "head_major"), (LONG, 0, 3, 128, "bf16", 0, "slot_major"), (LENS, 37, 2, 64, "f32", 0, "slot_major"), (LONG, 3, 1, 128, "f32", 0, "head_major"),
    (LENS, 5, 2, 128, "bf16", 3, "head_major"), (LONG, 70, 2, 64, "bf16", 8, "slot_major"), ([1], 0, 1, 64, "bf16", 0, "head_major"), ([1, 1, 1], [0, 300, 31], 2, 128, "bf16", 16, "head_major"),
    ([1, 4, 2], [700, 1000, 3], 2, 64, "f32", 0, "head_major"), ([7, 3], [1500, 2011], 3, 64, "bf16", 0, "slot_major"), ([90, 130], [900, 41], 1, 128, "bf16", 0, "head_major")])
@pytest.mark.parametrize("mask", [B.MASK_CAUSAL, B.MASK_PREFIX])
def test_against_the_definition(lens, past, h, D, dtype, G, layout, mask):
    p = Prompt(lens, past, h, D, dtype, G, layout, prefix=50)
    p.run(mask=mask)
    p.check(mask=mask)
    assert not p.batch.read_seqs()["status"].any() and (p.batch.seqs_host["step"] == 3).all()


@pytest.mark.parametrize("dtype,D,G", [("bf16", 64, 0), ("bf16", 128, 2), ("f32", 64, 0), ("f32", 128, 0)])
@pytest.mark.parametrize("lens,past", [([3, 30, 1], 40), ([150, 40, 77], 0)])
@pytest.mark.parametrize("cap,slope,docs", [(5.0, False, False), (0.0, True, False), (0.0, False, True), (20.0, True, True)])
def test_scores_capped_lowered_and_masked_by_document(dtype, D, G, lens, past, cap, slope, docs):
    p = Prompt(lens, past, 2, D, dtype, G, prefix=33, q_scale=4.0)
    mods = dict(mask=B.MASK_PREFIX, softcap=cap)
    if slope:
        mods["slopes"] = torch.tensor([2.0 ** -(i + 1) for i in range(2 * p.G)], device=DEV)
    if docs:                                                 # documents of 13 slots with 4 of padding, whose rows see nothing; some come back later
        slot = torch.arange(p.batch.params.cap + 2)
        doc = torch.where(slot % 13 >= 9, -1 - slot % 2, slot // 13 % 4).to(torch.int32)
        mods["doc"] = doc.repeat(len(lens), 1).contiguous().to(DEV)
        for t in (p.K, p.V):                                 # what padding holds is nobody's business
            t[:, :, (doc[:p.batch.params.cap] < 0).to(DEV)] = NAN
    p.run(**mods)
    p.check(**mods)
    if docs:
        empty = torch.isinf(p.lse)
        assert empty.any() and not p.out[empty].any()


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("lens,past", [([40, 200], 0), ([20], 90)])
def test_infinities_and_nan_behind_the_mask(dtype, D, lens, past):
    """A token whose row holds infinities or NaN changes the rows that see it and no others."""
    p = Prompt(lens, past, 2, D, dtype)
    p.run()
    clean, lse = p.out.clone(), p.lse.clone()
    at = 13                                                  # new token number
    slot = p.past[0] + at
    p.V[0, 0, slot, 3], p.V[0, 0, slot, D - 1], p.V[0, 1, slot, 5] = float("inf"), NAN, -float("inf")
    p.batch.score.copy_(torch.from_numpy(p.score0))
    p.run()
    assert torch.equal(p.out[:at], clean[:at]) and torch.equal(p.lse, lse)
    rows = slice(at, int(p.lens[0]))
    assert (p.out[rows, 0, 3] == float("inf")).all() and p.out[rows, 0, D - 1].isnan().all() and (p.out[rows, 1, 5] == -float("inf")).all()
    keep = torch.ones(D, dtype=torch.bool, device=DEV)
    keep[[3, D - 1]] = False
    assert torch.equal(p.out[rows, 0][:, keep], clean[rows, 0][:, keep]) and torch.equal(p.out[int(p.lens[0]):], clean[int(p.lens[0]):])
    p.V[0, :, slot] = 0.0
    p.K[0, :, slot] = NAN
    p.run()
    assert torch.equal(p.out[:at], clean[:at]) and torch.equal(p.lse[:at], lse[:at]) and p.out[rows].isnan().all()


@pytest.mark.parametrize("dtype,D,G", [("bf16", 64, 0), ("bf16", 128, 2), ("f32", 64, 0), ("f32", 128, 0)])
@pytest.mark.parametrize("lens,past", [([3, 30, 1], 40), ([150, 40, 300], 0)])
def test_distances_between_far_positions(dtype, D, G, lens, past):
    """Positions that fp32 does not hold (it counts in steps of 64 there) lie as far apart as near ones."""
    p = Prompt(lens, past, 2, D, dtype, G)
    p.batch.pos += 1_000_000_000
    mods = dict(slopes=torch.tensor([2.0 ** -(i + 1) for i in range(2 * p.G)], device=DEV))
    p.run(**mods)
    p.check(**mods)


def test_mass_is_left_alone_where_it_is_not_wanted_and_steps_advance():
    p = Prompt([5, 0, 70], [0, 9, 4], 2, 64)
    p.run(flags=B.FLAG_NO_ACCUMULATE | B.FLAG_ADVANCE)
    p.check(mass=False)
    assert p.batch.read_seqs()["step"].tolist() == [4, 3, 4]
    p = Prompt([5, 70], 0, 2, 64, score_mode=B.SCORE_EXT_LARGEST)
    p.run()
    p.check(mass=False)


def test_records_that_do_not_fit():
    p = Prompt([5, 90, 7, 4], [3, 0, 2, 8], 2, 64)
    s = p.batch.read_seqs()
    s["n_res"][0], s["status"][2], s["n_res"][1] = 7, B.SEQ_CACHE_FULL, p.batch.params.cap + 1
    p.batch.upload_seqs()
    p.run()
    assert p.batch.read_seqs()["status"].tolist() == [B.SEQ_BAD_STATE, B.SEQ_BAD_STATE, B.SEQ_CACHE_FULL, 0]
    assert not p.out[:102].any() and not p.lse[:102].any()
    p.check(sequences=[3])
    assert np.array_equal(f64(p.batch.score)[:3], p.score0[:3])


def test_results_repeat_bit_by_bit_and_split_keys_agree():
    p = Prompt([200, 150, 31], [60, 900, 1000], 2, 128, "bf16", 2, prefix=100)
    p.run()
    first = p.out.clone(), p.lse.clone(), p.batch.score.clone()
    for _ in range(3):
        p.batch.score.copy_(torch.from_numpy(p.score0))
        p.out.fill_(1.0)
        p.run()
        assert all(torch.equal(a, b) for a, b in zip(first, (p.out, p.lse, p.batch.score)))
    p.check()


def test_wide_strides():
    """Rows far apart: a cache of 6 GiB, whose later rows 32 bits do not reach."""
    h, D, cap, n = 2, 64, 100, 1
    slot_stride = 1 << 25                                    # 64 MiB a slot: offsets pass 32 bits
    buf = torch.zeros(cap * slot_stride, dtype=torch.bfloat16, device=DEV)
    p = Prompt([100], 0, h, D, cap=cap)
    params = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=200, grid_w=200, win_rows_back=1, win_col_radius=2, dtype=B.BF16,
                           score_mode=B.SCORE_ATTN_MASS, cap=cap, kv_slot_stride=slot_stride, kv_head_stride=D)
    view = buf.view(cap, slot_stride)
    for i, x in enumerate((p.K, p.V)):
        for hd in range(h):
            view[:, (i * h + hd) * D:(i * h + hd + 1) * D] = x[0, hd]
    s = p.batch.read_seqs()
    s["k"], s["v"] = buf.data_ptr(), buf.data_ptr() + h * D * 2
    p.batch.upload_seqs()
    p.batch.params = params
    p.run()
    p.check()


def test_a_workspace_that_grows_on_another_stream():
    """Calls on a stream of their own, each needing more workspace than the last, leave results that no later use of that memory changes."""
    want, got = [], []
    for side in (False, True):
        stream = torch.cuda.Stream() if side else None
        batch = None
        for lens, past in (([2, 1], [700, 900]), ([20, 31], [900, 1400]), ([140, 90], [2000, 1500])):
            p = Prompt(lens, past, 2, 64, cap=2200)
            if batch is not None:
                p.batch.prompt_workspace = batch.prompt_workspace
            batch = p.batch
            torch.cuda.synchronize()
            batch.prefill(p.tokens, p.q, p.out, p.lse, stream=stream)
            torch.full((batch.prompt_workspace.numel(),), 255, dtype=torch.uint8, device=DEV)
            torch.cuda.synchronize()
            (got if side else want).append((p.out, p.lse, batch.score))
    assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))

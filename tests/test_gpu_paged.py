"""Caches in pages: each call against its definition in 64 bits, and against the dense call on the same rows, which it has to repeat bit by bit (the same
sums in the same order, from other places)."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch, PagedBatch

from paged_common import paged_twin, same_bits, same_records
from prompt_common import attended, close, f64, randn, turned
from test_gpu_prefill import LENS, LONG, Prompt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# ---------------------------------------------------------------------------------------------------- prompts
def twin_of(p, page, layout, **kw):
    return paged_twin(p.batch, page, layout=layout, resident=p.keys, **kw)


def prefill_both(p, page, layout, check=True, flags=0, twin=None, **mods):
    """The dense call, then the paged one, which is compared with it and with the definition."""
    paged = twin_of(p, page, layout) if twin is None else twin
    p.run(flags=flags, **mods)
    dense = [t.clone() for t in (p.out, p.lse, p.batch.score)]
    p.out.fill_(3.0)
    p.lse.fill_(3.0)
    before = paged.K.clone()
    paged.prefill(p.tokens, p.q, p.out, p.lse, mods=B.make_mods(**mods) if mods else None, flags=flags)
    torch.cuda.synchronize()
    p.batch.score.copy_(paged.score)
    for got, want, name in zip((p.out, p.lse, p.batch.score), dense, ("out", "lse", "mass")):
        assert same_bits(got, want), name
    assert same_bits(paged.K, before)
    same_records(paged, p.batch)
    if check:
        p.check(**{k: v for k, v in mods.items()})
    return paged


@pytest.mark.parametrize("lens,past,h,D,dtype,G,page,layout", [
    ([1], 0, 1, 64, "bf16", 0, 16, "head_major"), (LENS, 0, 2, 64, "bf16", 0, 16, "head_major"), (LENS, 37, 2, 64, "f32", 0, 32, "slot_major"), (LENS, 5, 2, 128, "bf16", 3, 64, "head_major"),
    ([1, 1, 1], [0, 300, 31], 2, 128, "bf16", 16, 128, "slot_major"), ([1, 4, 2], [700, 1000, 3], 2, 64, "f32", 0, 16, "head_major"), ([7, 3], [1500, 2011], 3, 64, "bf16", 0, 16, "slot_major"),
    ([1, 4, 2], [33, 100, 3], 1, 128, "f32", 0, 16, "slot_major"), (LONG, 3, 1, 128, "f32", 0, 64, "head_major"),
    (LONG, 0, 3, 128, "bf16", 0, 16, "slot_major"), (LONG, 70, 2, 64, "bf16", 8, 32, "slot_major"), ([90, 130], [900, 41], 1, 128, "bf16", 0, 64, "head_major"),
    ([300, 1, 64], [17, 600, 0], 2, 64, "bf16", 0, 128, "head_major"), ([200], [1000], 2, 64, "bf16", 2, 8192, "head_major"), ([70, 33], [0, 95], 2, 128, "bf16", 4, 16, "head_major")])
@pytest.mark.parametrize("mask", [B.MASK_CAUSAL, B.MASK_PREFIX])
def test_prompts_against_the_definition_and_dense_caches(lens, past, h, D, dtype, G, page, layout, mask):
    p = Prompt(lens, past, h, D, dtype, G, prefix=50)
    prefill_both(p, page, layout, mask=mask)
    p.batch.score.copy_(torch.from_numpy(p.score0).float())
    prefill_both(p, page, layout, twin=twin_of(p, page, layout, far=True), check=False, mask=mask)


@pytest.mark.parametrize("dtype,D,G", [("bf16", 64, 0), ("bf16", 128, 2), ("f32", 64, 0), ("f32", 128, 0)])
@pytest.mark.parametrize("lens,past", [([3, 30, 1], 40), ([150, 40, 77], 0)])
@pytest.mark.parametrize("cap,slope,docs", [(5.0, False, False), (0.0, True, False), (0.0, False, True), (20.0, True, True), (900.0, False, False)])
def test_prompts_capped_lowered_and_masked_by_document(dtype, D, G, lens, past, cap, slope, docs):
    p = Prompt(lens, past, 2, D, dtype, G, prefix=33, q_scale=4.0)
    mods = dict(mask=B.MASK_PREFIX, softcap=cap)
    if slope:
        mods["slopes"] = torch.tensor([2.0 ** -(i + 1) for i in range(2 * p.G)], device=DEV)
    if docs:                                                 # documents of 13 slots with 4 of padding, whose rows see nothing; some come back later
        slot = torch.arange(p.batch.params.cap + 2)
        doc = torch.where(slot % 13 >= 9, -1 - slot % 2, slot // 13 % 4).to(torch.int32)
        mods["doc"] = doc.repeat(len(lens), 1).contiguous().to(DEV)
    prefill_both(p, 16, "head_major", check=cap != 900.0, **mods)


@pytest.mark.parametrize("flags", [B.FLAG_SPLIT_P, B.FLAG_NO_ACCUMULATE | B.FLAG_ADVANCE])
def test_prompt_flags(flags):
    p = Prompt([150, 40, 0, 77], 21, 2, 64, "bf16", 2)
    prefill_both(p, 32, "slot_major", check=False, flags=flags)
    p.check(mass=not flags & B.FLAG_NO_ACCUMULATE)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dtype,D,lens", [("bf16", 64, [200, 20]), ("bf16", 128, [150, 9]), ("f32", 64, [40, 20]), ("f32", 128, [40, 3])])
def test_infinities_in_pages_reach_who_sees_them(dtype, D, lens, page):
    """A value of infinity or NaN in V at a late slot: rows before it are as if it were not there."""
    p = Prompt(lens, 33, 2, D, dtype)
    for b, x in ((0, float("inf")), (1, float("nan"))):
        p.V[b, 0, p.keys[b] - 2, 5] = x
    paged = twin_of(p, page, "head_major")
    prefill_both(p, page, "head_major", check=False, twin=paged)
    out = f64(p.out)
    for b in range(2):
        rows = out[p.begin[b]:p.begin[b + 1] - 2, 0]
        assert np.isfinite(rows).all() and not np.isfinite(out[p.begin[b + 1] - 2, 0, 5])


def test_prompt_records_that_do_not_fit():
    p = Prompt([5, 6, 7, 8], 10, 2, 64, "bf16", 0)
    paged = twin_of(p, 16, "head_major")
    paged.seqs_host["status"][0] = B.SEQ_CACHE_FULL
    paged.seqs_host["n_res"][1] = 12                         # fewer than slot0 + tokens
    paged.upload_seqs()
    paged.table[2, 0] = paged.n_pages                        # no page of the pool, under slots that are resident already
    score = paged.score.clone()
    paged.prefill(p.tokens, p.q, p.out, p.lse)
    torch.cuda.synchronize()
    status = paged.read_seqs()["status"]
    assert list(status) == [B.SEQ_CACHE_FULL, B.SEQ_BAD_STATE, B.SEQ_BAD_STATE, 0]
    x = int(p.begin[3])
    assert not p.out[:x].any() and not p.lse[:x].any() and p.out[x:].abs().sum() > 0
    assert same_bits(paged.score[:3], score[:3]) and not same_bits(paged.score[3:], score[3:])


@pytest.mark.parametrize("bad", [-1, 1000, -(1 << 31), (1 << 31) - 1])
@pytest.mark.parametrize("lens,past", [([3, 2], 40), ([150, 140], 300), ([2, 2], 1500)])
def test_entries_that_are_no_pages_spoil_their_sequence_alone(bad, lens, past):
    p = Prompt(lens, past, 2, 64, "bf16", 0)
    p.run()
    want = [t.clone() for t in (p.out, p.lse)]
    paged = twin_of(p, 16, "head_major")
    paged.score.copy_(torch.from_numpy(p.score0).float())
    paged.table[0, (p.keys[0] - 1) // 16] = bad
    paged.prefill(p.tokens, p.q, p.out, p.lse)
    torch.cuda.synchronize()
    x = int(p.begin[1])
    assert list(paged.read_seqs()["status"]) == [B.SEQ_BAD_STATE, 0]
    assert not p.out[:x].any() and not p.lse[:x].any()
    assert same_bits(p.out[x:], want[0][x:]) and same_bits(p.lse[x:], want[1][x:])


# ---------------------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("page,layout", [(16, "head_major"), (64, "slot_major"), (32, "head_major")])
@pytest.mark.parametrize("dtype,D,G,in_f32,pairing", [("bf16", 64, 0, False, "halves"), ("bf16", 128, 3, True, "neighbours"), ("f32", 64, 0, False, "neighbours"), ("f32", 128, 0, False, "halves")])
@pytest.mark.parametrize("lens,past", [([1], [0]), ([5, 0, 33, 1, 90], [0, 7, 31, 64, 16]), ([300, 200], [3, 0])])
def test_append(page, layout, dtype, D, G, in_f32, pairing, lens, past):
    h, n = 2, len(lens)
    hq, T, cap = h * max(G, 1), sum(lens), max(a + b for a, b in zip(lens, past)) + 5
    p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=30, grid_w=30, win_rows_back=1, win_col_radius=2, dtype=B.F32 if dtype == "f32" else B.BF16, score_mode=B.SCORE_ATTN_MASS,
                      cap=cap, q_per_kv=G)
    dense = LayerBatch(p, DEV)
    gen = torch.Generator().manual_seed(5)
    for t in (dense.K, dense.V):
        t.copy_(randn(gen, *t.shape, dtype=dense.tdtype))
    dense.pos[:] = torch.arange(cap, dtype=torch.int32, device=DEV)
    dense.score.uniform_()
    s = dense.seqs_host
    s["n_res"], s["grid_origin"], s["n_keep_prefix"], s["step"] = past, 20, 20, 0
    dense.upload_seqs()
    keys = [a + b for a, b in zip(lens, past)]
    paged = paged_twin(dense, page, layout=layout, resident=keys, far=page == 32)
    it = torch.float32 if in_f32 else dense.tdtype
    q, k, v = (randn(gen, T, heads * D, dtype=it).to(DEV) for heads in (hq, h, h))
    freq = torch.rand(2, D // 2, generator=torch.Generator().manual_seed(6), dtype=torch.float64).to(DEV)
    rope = B.make_rope(freq, pairing=pairing, text=(1, 1), origin=(1, 1), row=(1, 0), col=(0, 1))
    begin = np.concatenate([[0], np.cumsum(lens)])
    tokens = B.make_tokens(torch.tensor(begin, dtype=torch.int32, device=DEV), torch.tensor(past, dtype=torch.int32, device=DEV), T, max(lens))
    flags = (B.FLAG_NEW_F32 if in_f32 else 0) | B.FLAG_ADVANCE
    outs = [torch.full((T, hq, D), 9.0, dtype=dense.tdtype, device=DEV) for _ in range(2)]
    before = paged.K.clone(), paged.V.clone()
    for _ in range(2):                                       # (the same call may be made again)
        dense.append(tokens, rope, q, k, v, outs[0], flags=flags)
        paged.append(tokens, rope, q, k, v, outs[1], flags=flags)
    torch.cuda.synchronize()
    assert same_bits(*outs) and same_bits(paged.pos, dense.pos) and same_bits(paged.score, dense.score)
    same_records(paged, dense)
    for b in range(n):
        for pool, cache in ((paged.K, dense.K), (paged.V, dense.V)):
            if keys[b]:
                assert same_bits(paged.cache_rows(pool, b, keys[b]).transpose(0, 1), cache[b, :, :keys[b]]), b
    # nothing else was written: put back what was there under the new slots
    for pool, old in zip((paged.K, paged.V), before):
        for b in range(n):
            page_of, place = paged._slots(b, keys[b]) if keys[b] else (None, None)
            if keys[b]:
                new = slice(past[b], keys[b])
                if paged.head_major:
                    pool[page_of[new], :, place[new]] = old[page_of[new], :, place[new]]
                else:
                    pool[page_of[new], place[new]] = old[page_of[new], place[new]]
        assert same_bits(pool, old)
    # against the definition
    p0 = np.concatenate([np.arange(a, a + m) for a, m in zip(past, lens)])
    i = p0 - 20
    c = np.stack([np.where(i < 0, p0, 20 + i // 30), np.where(i < 0, p0, 20 + i % 30)], 1).astype(np.float64)
    want, tol = turned(f64(q).reshape(T, hq, D), c @ freq.cpu().numpy(), pairing)
    close(outs[1], want, tol + (torch.finfo(dense.tdtype).eps / 2) * np.abs(want) * (1 + 2 ** -20) + 1e-30, "q")


def test_append_without_pages():
    p = B.make_params(n_seq=4, n_heads=2, head_dim=64, grid_h=30, grid_w=30, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=100)
    batch = PagedBatch(p, n_pages=14, page_size=16, device=DEV)
    for b, slots in enumerate((40, 32, 100, 16)):
        batch.reserve(b, slots)
    batch.upload_table()
    batch.table[2, 1] = batch.n_pages                            # among the new slots' pages
    s = batch.seqs_host
    s["n_res"], s["step"] = [0, 0, 0, 16], 0
    batch.upload_seqs()
    lens = [40, 33, 90, 5]                                   # the second and the last have a page less than they need
    T = sum(lens)
    gen = torch.Generator().manual_seed(1)
    q, k, v = (randn(gen, T, 128, dtype=torch.bfloat16).to(DEV) for _ in range(3))
    begin = torch.tensor([0, 40, 73, 163, 168], dtype=torch.int32, device=DEV)
    tokens = B.make_tokens(begin, torch.tensor([0, 0, 0, 16], dtype=torch.int32, device=DEV), T, max(lens))
    out = torch.full((T, 2, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    batch.append(tokens, None, q, k, v, out)
    torch.cuda.synchronize()
    r = batch.read_seqs()
    assert list(r["status"]) == [0, B.SEQ_CACHE_FULL, B.SEQ_CACHE_FULL, B.SEQ_CACHE_FULL] and list(r["n_res"]) == [40, 0, 0, 16]
    assert same_bits(out[:40], q[:40].view(40, 2, 64)) and not out[40:].any()
    assert same_bits(batch.cache_rows(batch.K, 0, 40), k[:40].view(40, 2, 64))
    others = [i for i in range(batch.n_pages) if i not in batch.table_host[0]]
    assert not batch.K[others].any() and not batch.V[others].any()


# ---------------------------------------------------------------------------------------------------- single tokens
class Decode:
    def __init__(self, lists, resident, h, D, dtype="bf16", G=0, seed=1, cap=None, sel_cap=None, mass=True, q_scale=1.5, with_new=True):
        n, self.h, self.D, self.G = len(lists), h, D, max(G, 1)
        self.lists, self.resident = lists, np.broadcast_to(np.asarray(resident), (n,)).copy()
        cap = int(self.resident.max()) + 3 if cap is None else cap
        p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=90, grid_w=90, win_rows_back=1, win_col_radius=2, dtype=B.F32 if dtype == "f32" else B.BF16,
                          score_mode=B.SCORE_ATTN_MASS if mass else B.SCORE_EXT_LARGEST, cap=cap, sel_cap=max(max(lists), 1) if sel_cap is None else sel_cap, q_per_kv=G)
        self.batch = LayerBatch(p, DEV)
        gen = torch.Generator().manual_seed(seed)
        dt = self.batch.tdtype
        self.bf16 = dt == torch.bfloat16
        for t in (self.batch.K, self.batch.V):
            t.copy_(randn(gen, *t.shape, dtype=dt))
        self.batch.pos[:] = torch.arange(cap, dtype=torch.int32, device=DEV)
        self.batch.score.uniform_(generator=torch.Generator(device=DEV).manual_seed(seed))
        rng = np.random.default_rng(seed)
        self.idx = []
        for b, m in enumerate(lists):
            r = int(self.resident[b])
            slots = np.sort(rng.permutation(r - 1)[:m - 1]) if m else np.zeros(0, int)
            self.idx.append(np.concatenate([slots, [r - 1]]).astype(np.int32) if m else slots.astype(np.int32))
            self.batch.sel_idx[b, :m] = torch.from_numpy(self.idx[b]).to(DEV)
        self.batch.sel_idx_host = self.batch.sel_idx.clone()
        self.batch.sel_cnt.copy_(torch.tensor(lists, dtype=torch.int32))
        s = self.batch.seqs_host
        s["n_res"], s["step"], s["pending_slot"] = self.resident, 4, self.resident - 1 if with_new else -1
        self.batch.upload_seqs()
        self.q = randn(gen, n, h * self.G, D, dtype=dt, scale=q_scale).to(DEV)
        self.k_new, self.v_new = (randn(gen, n, h, D).to(DEV) for _ in range(2))

    def rows(self, f32):
        return (self.k_new, self.v_new) if f32 else (self.k_new.to(self.batch.tdtype), self.v_new.to(self.batch.tdtype))

    def check(self, batch, score0, append, mass=True):
        """The paged batch's outputs against the definition."""
        out, lse, score, q = (f64(x) for x in (batch.out, batch.lse, batch.score, self.q))
        for b, slots in enumerate(self.idx):
            if not len(slots):
                continue
            K, V = (f64(batch.cache_rows(t, b, int(self.resident[b]))) for t in (batch.K, batch.V))
            want, tol = score0[b].copy(), 4 * 2.0 ** -24 * np.abs(score0[b])
            for j in range(self.h * self.G):
                hd = j // self.G
                o, s, p, ot, st, pt = attended(q[b, j][None], K[slots, hd], V[slots, hd], self.D ** -0.5, bf16=self.bf16)
                close(out[b, j][None], o, ot, f"out of sequence {b}, head {j}")
                close(lse[b, j][None], s, st, f"lse of sequence {b}, head {j}")
                want[hd, slots] += p[0]
                tol[hd, slots] += p[0] * pt[0] + 2.0 ** -22 * (1 + want[hd, slots])
            if mass:
                close(score[b], want, tol, f"mass of sequence {b}")


@pytest.mark.parametrize("lists,resident,h,D,dtype,G,page,layout", [
    ([1], 1, 1, 64, "bf16", 0, 16, "head_major"), ([1, 2, 17, 0, 64], [1, 40, 17, 5, 70], 3, 64, "bf16", 0, 16, "slot_major"), ([5, 33, 100], 130, 2, 128, "f32", 0, 32, "head_major"),
    ([427, 300], 468, 20, 64, "bf16", 0, 16, "head_major"), ([673] * 12, 695, 24, 64, "bf16", 0, 64, "head_major"), ([130, 7], [150, 9], 2, 64, "f32", 0, 128, "slot_major"),
    ([2500, 900], [2600, 1000], 2, 128, "bf16", 0, 64, "head_major"), ([5000], 6000, 1, 64, "bf16", 0, 16, "slot_major"), ([3000, 1], [3500, 1], 3, 64, "f32", 0, 8192, "head_major"),
    ([1100] * 3, 1200, 200, 64, "bf16", 0, 16, "head_major"),
    ([1], 1, 1, 64, "bf16", 2, 16, "head_major"), ([1, 2, 17, 0, 64], [1, 40, 17, 5, 70], 3, 64, "bf16", 8, 16, "slot_major"), ([5, 33, 100], 130, 2, 128, "bf16", 16, 32, "head_major"),
    ([300, 1378], 1471, 8, 128, "bf16", 8, 32, "head_major"), ([650] * 50, 700, 8, 64, "bf16", 5, 64, "slot_major"), ([5000, 77], 6000, 1, 128, "bf16", 8, 16, "head_major"),
    ([3000], 3100, 2, 64, "bf16", 3, 64, "head_major"), ([1300] * 40, 1400, 2, 128, "bf16", 16, 16, "head_major")])
@pytest.mark.parametrize("f32_rows,far", [(False, False), (True, False), (True, True)])
def test_single_tokens(lists, resident, h, D, dtype, G, page, layout, f32_rows, far):
    d = Decode(lists, resident, h, D, dtype, G)
    paged = paged_twin(d.batch, page, layout=layout, resident=d.resident, far=far)
    score0 = f64(paged.score)
    k, v = d.rows(f32_rows and d.bf16)
    flags = B.FLAG_APPEND | B.FLAG_ADVANCE | (B.FLAG_NEW_F32 if f32_rows else 0)
    d.batch.attend(d.q, flags, k, v)
    paged.attend(d.q, flags, k, v)
    torch.cuda.synchronize()
    assert same_bits(paged.out, d.batch.out) and same_bits(paged.lse, d.batch.lse)
    if G <= 1:
        assert same_bits(paged.score, d.batch.score)
    same_records(paged, d.batch)
    for b, r in enumerate(d.resident):
        for pool, cache in ((paged.K, d.batch.K), (paged.V, d.batch.V)):
            assert same_bits(paged.cache_rows(pool, b, int(r)).transpose(0, 1), cache[b, :, :int(r)]), b
    d.check(paged, score0, True)


@pytest.mark.parametrize("G,dtype,D", [(0, "bf16", 64), (0, "f32", 128), (4, "bf16", 128)])
def test_single_tokens_whose_rows_are_there(G, dtype, D):
    """Nothing appended, nothing added to the mass, nothing advanced; K and V in one pool."""
    d = Decode([40, 3, 200], [50, 3, 333], 2, D, dtype, G, with_new=False)
    paged = paged_twin(d.batch, 16, resident=d.resident, interleaved=True)
    before = paged.K.clone(), paged.score.clone(), f64(paged.score)
    paged.attend(d.q, B.FLAG_NO_ACCUMULATE)
    torch.cuda.synchronize()
    d.check(paged, before[2], False, mass=False)
    assert same_bits(paged.K, before[0]) and same_bits(paged.score, before[1]) and (paged.read_seqs()["step"] == 4).all()


@pytest.mark.parametrize("G", [0, 4])
@pytest.mark.parametrize("lists,resident", [([30, 40, 50], 60), ([2900, 2950, 2800], 3000)])
@pytest.mark.parametrize("bad", [-1, 1 << 20, (1 << 31) - 1])
def test_single_tokens_on_entries_that_are_no_pages(G, lists, resident, bad):
    d = Decode(lists, resident, 2, 64, "bf16", G, cap=resident + 40)
    paged = paged_twin(d.batch, 16, resident=d.resident, far=bad == -1)
    good = paged_twin(d.batch, 16, resident=d.resident, far=bad == -1)
    k, v = d.rows(False)
    good.attend(d.q, B.FLAG_APPEND, k, v)
    paged.table[1, 0] = bad
    before = paged.K.clone(), paged.score.clone()
    paged.attend(d.q, B.FLAG_APPEND | B.FLAG_ADVANCE, k, v)
    torch.cuda.synchronize()
    r = paged.read_seqs()
    assert list(r["status"]) == [0, B.SEQ_BAD_STATE, 0] and list(r["step"]) == [5, 4, 5]
    assert not paged.out[1].any() and not paged.lse[1].any() and same_bits(paged.score[1], before[1][1])
    for b in (0, 2):
        assert same_bits(paged.out[b], good.out[b]) and same_bits(paged.lse[b], good.lse[b])
    mine = torch.from_numpy(good.table_host[1, :resident // 16 + 1]).long().to(DEV)
    mine = mine[(mine >= 0) & (mine < paged.n_pages)]
    assert same_bits(paged.K[mine], before[0][mine])


def test_single_tokens_listed_beyond_the_resident_ones_stay_in_the_pool():
    """A malformed list reads rows that are there; a count of resident slots that cannot be is refused."""
    d = Decode([30, 40, 50], 60, 2, 64, "bf16", 0, cap=200)
    paged = paged_twin(d.batch, 16, resident=d.resident)
    paged.sel_idx[0, 3], paged.sel_idx[0, 4], paged.sel_idx[0, 5] = 199, -5, 0x7FFFFFF0
    paged.seqs_host["n_res"][1], paged.seqs_host["n_res"][2] = 0, 201
    paged.upload_seqs()
    paged.attend(d.q, 0)
    torch.cuda.synchronize()
    assert list(paged.read_seqs()["status"]) == [0, B.SEQ_BAD_STATE, B.SEQ_BAD_STATE]
    assert torch.isfinite(paged.out.float()).all() and not paged.out[1:].any()


# ---------------------------------------------------------------------------------------------------- eviction
def evicting(n, h, D, W, R, budget, rows, dtype="bf16", prefix=9, seed=1, ties=False, **kw):
    cap = prefix + budget + (R + 1) * W + 4
    p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=64, grid_w=W, win_rows_back=R, win_col_radius=2, dtype=B.F32 if dtype == "f32" else B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=cap, **kw)
    dense = LayerBatch(p, DEV)
    gen = torch.Generator().manual_seed(seed)
    for t in (dense.K, dense.V):
        t.copy_(randn(gen, *t.shape, dtype=dense.tdtype))
    score = torch.rand(n, h, cap, generator=gen)
    dense.score.copy_((score * 3).round() if ties else score)
    rng = np.random.default_rng(seed)
    s = dense.seqs_host
    for b in range(n):
        done = rows + b % 3                                  # completed grid rows
        last = min(R + 1, done) * W
        past = done * W - last
        history = np.sort(rng.permutation(past)[:min(budget, past)])
        pos = np.concatenate([np.arange(prefix), prefix + history, prefix + past + np.arange(last)])
        dense.pos[b, :len(pos)] = torch.from_numpy(pos.astype(np.int32)).to(DEV)
        s[b]["n_res"], s[b]["step"] = len(pos), done * W - (1 if b % 4 == 3 else 0)           # (every fourth has not closed a row)
    s["grid_origin"] = s["n_keep_prefix"] = prefix
    s["budget"] = budget
    dense.upload_seqs()
    return dense


@pytest.mark.parametrize("far", [False, True])
@pytest.mark.parametrize("n,h,D,W,R,budget,rows,dtype,page,layout,ties", [
    (1, 1, 64, 4, 0, 3, 3, "bf16", 16, "head_major", False), (5, 3, 64, 8, 1, 30, 6, "bf16", 16, "slot_major", True), (4, 2, 128, 16, 1, 100, 9, "f32", 32, "head_major", False),
    (6, 24, 64, 32, 1, 512, 22, "bf16", 64, "head_major", False), (3, 14, 128, 24, 2, 600, 30, "bf16", 16, "slot_major", True), (5, 2, 64, 64, 2, 1500, 40, "bf16", 128, "head_major", False),
    (4, 1, 64, 64, 2, 3800, 61, "f32", 16, "head_major", False), (140, 4, 64, 16, 1, 60, 9, "bf16", 16, "head_major", False)])
def test_row_ends(n, h, D, W, R, budget, rows, dtype, page, layout, ties, far):
    dense = evicting(n, h, D, W, R, budget, rows, dtype, ties=ties)
    resident = dense.seqs_host["n_res"].copy()
    paged = paged_twin(dense, page, layout=layout, resident=resident, far=far)
    pos0, score0 = paged.pos.cpu().numpy(), paged.score.cpu().numpy()
    old = [[paged.cache_rows(t, b, int(r)).clone() for t in (paged.K, paged.V)] for b, r in enumerate(resident)]
    dense.compact(B.FLAG_ADVANCE)
    paged.compact(B.FLAG_ADVANCE)
    torch.cuda.synchronize()
    same_records(paged, dense)
    assert same_bits(paged.keep_map, dense.keep_map) and same_bits(paged.pos, dense.pos) and same_bits(paged.score, dense.score)
    after = paged.read_seqs()
    maps, pos1, score1 = paged.keep_map.cpu().numpy(), paged.pos.cpu().numpy(), paged.score.cpu().numpy()
    for b in range(n):
        r, closes = int(resident[b]), b % 4 != 3
        assert after["compacted"][b] == closes
        kept = np.arange(r)
        if closes:                                           # the definition: prefix, last R rows, largest sums (in 32 bits, head by head) of the rest
            done = rows + b % 3
            sums = score0[b, 0, :r].copy()
            for j in range(1, h):
                sums += score0[b, j, :r]
            image = pos0[b, :r] - 9
            fixed = (image < 0) | (image >= (done - min(R, done)) * W)
            best = sorted(np.flatnonzero(~fixed), key=lambda i: (-sums[i], i))[:budget]
            kept = np.sort(np.concatenate([np.flatnonzero(fixed), np.asarray(best, int)]))
            where = np.full(r, -1)
            where[kept] = np.arange(len(kept))
            assert np.array_equal(maps[b, :r], where)
        m = len(kept)
        assert after["n_res"][b] == m and np.array_equal(pos1[b, :m], pos0[b, kept]) and np.array_equal(score1[b, :, :m], score0[b][:, kept])
        at = torch.from_numpy(kept).to(DEV)
        for pool, rows_before in zip((paged.K, paged.V), old[b]):
            assert same_bits(paged.cache_rows(pool, b, m), rows_before[at]), b
    # pages of nobody are as they were
    mine = set(np.concatenate([paged.table_host[b, :-(-int(r) // page)] for b, r in enumerate(resident)]).tolist())
    nobody = [i for i in range(paged.n_pages) if i not in mine]
    assert torch.isnan(paged.K[nobody].float()).all() and torch.isnan(paged.V[nobody].float()).all()


@pytest.mark.parametrize("policy", [B.EVICT_WHEN_FULL, B.EVICT_REUSE_SLOT])
def test_one_by_one_when_full(policy):
    n, h, D, cap, prefix = 3, 2, 64, 70, 5
    p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=30, grid_w=30, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=cap, win_recent_m=8,
                      evict_policy=policy)
    dense = LayerBatch(p, DEV)
    gen = torch.Generator().manual_seed(2)
    for t in (dense.K, dense.V):
        t.copy_(randn(gen, *t.shape, dtype=dense.tdtype))
    dense.score.copy_(torch.rand(n, h, cap, generator=gen))
    dense.pos[:] = torch.arange(cap, dtype=torch.int32, device=DEV)
    s = dense.seqs_host
    s["n_res"], s["step"], s["grid_origin"], s["n_keep_prefix"] = [cap, cap - 1, cap], cap - prefix + 1, prefix, prefix
    dense.upload_seqs()
    paged = paged_twin(dense, 16)
    for t in range(5):                                       # whole steps, the hole taken by the next token under slot reuse
        q, k, v = (randn(gen, n, h, D, dtype=torch.bfloat16).to(DEV) for _ in range(3))
        dense.step(q, k, v)
        paged.step(q, k, v)
        torch.cuda.synchronize()
        same_records(paged, dense)
        assert same_bits(paged.out, dense.out) and same_bits(paged.score, dense.score) and same_bits(paged.pos, dense.pos)
        for b in range(n):
            assert same_bits(paged.cache_rows(paged.K, b, int(paged.seqs_host["n_res"][b])).transpose(0, 1), dense.K[b, :, :int(paged.seqs_host["n_res"][b])])


def test_row_ends_on_entries_that_are_no_pages():
    dense = evicting(5, 3, 64, 8, 1, 30, 6)
    resident = dense.seqs_host["n_res"].copy()
    paged = paged_twin(dense, 16, resident=resident)
    paged.table[0, 1] = paged.n_pages
    paged.table[3, 0] = -1                                   # (closes no row: nothing is looked at)
    before = [t.clone() for t in (paged.K, paged.V, paged.pos, paged.score, paged.keep_map)]
    paged.compact(B.FLAG_ADVANCE)
    torch.cuda.synchronize()
    r = paged.read_seqs()
    assert list(r["status"]) == [B.SEQ_BAD_STATE, 0, 0, 0, 0] and r["n_res"][0] == resident[0] and list(r["compacted"]) == [0, 1, 1, 0, 1]
    mine = torch.from_numpy(paged.table_host[0, :-(-int(resident[0]) // 16)]).long().to(DEV)
    assert same_bits(paged.K[mine], before[0][mine]) and same_bits(paged.V[mine], before[1][mine])
    for now, then in zip((paged.pos, paged.score, paged.keep_map), before[2:]):
        assert same_bits(now[0], then[0])


# ---------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype,G,page,layout", [("bf16", 0, 16, "head_major"), ("f32", 0, 32, "slot_major"), ("bf16", 4, 64, "head_major")])
def test_prompts_and_images_decoded_over_pages(dtype, G, page, layout):
    """Append, attention of the prompt, then steps over several row ends, pages taken as they are needed and given back after evictions: as on dense caches."""
    n, h, D, W, budget, P = 3, 2, 64, 6, 10, [20, 33, 7]
    hq, cap = h * max(G, 1), max(P) + budget + 3 * W
    kw = dict(n_seq=n, n_heads=h, head_dim=D, grid_h=8, grid_w=W, win_rows_back=1, win_col_radius=2, dtype=B.F32 if dtype == "f32" else B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=cap, q_per_kv=G)
    dense = LayerBatch(B.make_params(**kw), DEV)
    paged = PagedBatch(B.make_params(layout=layout, **kw), n_pages=n * -(-cap // page), page_size=page, device=DEV)
    paged.K.fill_(float("nan"))
    paged.V.fill_(float("nan"))
    for batch in (dense, paged):
        s = batch.seqs_host
        s["grid_origin"] = s["n_keep_prefix"] = P
        s["budget"], s["step"] = budget, 0
        batch.upload_seqs()
    for b in range(n):
        paged.reserve(b, P[b])
    paged.upload_table()
    gen = torch.Generator().manual_seed(4)
    T, dt = sum(P), dense.tdtype
    begin = torch.tensor(np.concatenate([[0], np.cumsum(P)]), dtype=torch.int32, device=DEV)
    tokens = B.make_tokens(begin, torch.zeros(n, dtype=torch.int32, device=DEV), T, max(P))
    q, k, v = (randn(gen, T, heads * D, dtype=dt).to(DEV) for heads in (hq, h, h))
    out = [torch.empty(T, hq, D, dtype=dt, device=DEV) for _ in range(4)]
    lse = [torch.empty(T, hq, device=DEV) for _ in range(2)]
    for i, batch in enumerate((dense, paged)):
        batch.append(tokens, None, q, k, v, out[i], flags=B.FLAG_ADVANCE)
        batch.prefill(tokens, out[i], out[2 + i], lse[i], mods=B.make_mods(mask=B.MASK_PREFIX))
    assert same_bits(out[2], out[3]) and same_bits(*lse)
    most = 0
    for t in range(4 * W + 2):
        resident = paged.read_seqs()["n_res"]
        for b in range(n):
            paged.release(b, int(resident[b]))               # what evictions have left empty
            paged.reserve(b, int(resident[b]) + 1)
        paged.upload_table()
        most = max(most, int((paged.table_host >= 0).sum()))
        q, k, v = (randn(gen, n, heads, D, dtype=dt).to(DEV) for heads in (hq, h, h))
        dense.step(q, k, v)
        paged.step(q, k, v)
        torch.cuda.synchronize()
        same_records(paged, dense)
        assert not paged.seqs_host["status"].any()
        # (grouped queries add their mass with atomics on distinct words: the same sums)
        assert same_bits(paged.out, dense.out) and same_bits(paged.lse, dense.lse), t
        close(paged.score, f64(dense.score), 2.0 ** -22 * (1 + f64(dense.score)), "score")
    assert most <= paged.n_pages and len(paged.free_pages) + int((paged.table_host >= 0).sum()) == paged.n_pages


@pytest.mark.parametrize("G", [0, 4])
def test_steps_over_pages_in_a_graph(G):
    """A captured step, replayed between eager ones with tables that change meanwhile, against eager steps on another batch."""
    n, h, D, W, budget, P = 4, 3, 64, 5, 8, 12
    cap = P + budget + 3 * W
    kw = dict(n_seq=n, n_heads=h, head_dim=D, grid_h=9, grid_w=W, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=cap, q_per_kv=G)
    batches = [PagedBatch(B.make_params(**kw), n_pages=4 * n, page_size=16, device=DEV) for _ in range(2)]
    gen = torch.Generator().manual_seed(4)
    K = randn(gen, n, P, h, D, dtype=torch.bfloat16).to(DEV)
    for batch in batches:
        s = batch.seqs_host
        s["grid_origin"] = s["n_keep_prefix"] = s["n_res"] = P
        s["budget"], s["step"] = budget, 1
        batch.upload_seqs()
        batch.pos[:] = torch.arange(cap, dtype=torch.int32, device=DEV)
        for b in range(n):
            batch.reserve(b, cap)
        batch.upload_table()
        for b in range(n):
            batch._put_rows(b, K[b], K[b] * 0.5)
    hq = h * max(G, 1)
    q, k, v = (torch.zeros(n, heads, D, dtype=torch.bfloat16, device=DEV) for heads in (hq, h, h))
    eager, captured = batches
    stream = torch.cuda.Stream()
    saved = [t.clone() for t in (captured.seqs, captured.pos, captured.score, captured.K, captured.V)]
    stream.wait_stream(torch.cuda.current_stream())              # after the copies, which the step must not overtake
    with torch.cuda.stream(stream):
        captured.step(q, k, v)
    torch.cuda.synchronize()
    for t, x in zip((captured.seqs, captured.pos, captured.score, captured.K, captured.V), saved):
        t.copy_(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured.step(q, k, v)
    for t in range(3 * W + 2):
        for x in (q, k, v):
            x.copy_(randn(gen, *x.shape, dtype=torch.bfloat16))
        if t == 4:                                           # another sequence's pages change places
            a = captured.table_host[1, 0]
            free = [i for i in range(captured.n_pages) if i not in captured.table_host]
            if free:
                captured.K[free[0]], captured.V[free[0]] = captured.K[int(a)].clone(), captured.V[int(a)].clone()
                captured.table_host[1, 0] = free[0]
                captured.upload_table()
        eager.step(q, k, v)
        if t % 5 == 3:
            captured.step(q, k, v)
        else:
            graph.replay()
        torch.cuda.synchronize()
        same_records(eager, captured)
        assert same_bits(eager.out, captured.out) and same_bits(eager.lse, captured.lse) and same_bits(eager.pos, captured.pos), t
        close(captured.score, f64(eager.score), 2.0 ** -22 * (1 + f64(eager.score)), "score")


def test_prefixes_shared_by_tables():
    """Two images whose first pages are the same pages: evictions leave them alone."""
    n, h, D, W, budget, P = 2, 2, 64, 8, 20, 32
    cap = P + budget + 3 * W
    kw = dict(n_seq=n, n_heads=h, head_dim=D, grid_h=9, grid_w=W, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=cap)
    own, shares = (PagedBatch(B.make_params(**kw), n_pages=12, page_size=16, device=DEV) for _ in range(2))
    gen = torch.Generator().manual_seed(4)
    rows = randn(gen, P, h, D, dtype=torch.bfloat16).to(DEV)
    for batch in (own, shares):
        s = batch.seqs_host
        s["grid_origin"] = s["n_keep_prefix"] = s["n_res"] = P
        s["budget"], s["step"] = budget, 1
        batch.upload_seqs()
        batch.pos[:] = torch.arange(cap, dtype=torch.int32, device=DEV)
        batch.reserve(0, cap)
        if batch is shares:
            batch.table_host[1, :2] = batch.table_host[0, :2]
        batch.reserve(1, cap)
        batch.upload_table()
        for b in range(n):
            batch._put_rows(b, rows, rows * 2)
    prefix = shares.cache_rows(shares.K, 0, P).clone()
    for t in range(5 * W + 1):
        q, k, v = (randn(gen, n, h, D, dtype=torch.bfloat16).to(DEV) for _ in range(3))
        own.step(q, k, v)
        shares.step(q, k, v)
        torch.cuda.synchronize()
        assert same_bits(own.out, shares.out) and same_bits(own.score, shares.score)
    assert same_bits(shares.cache_rows(shares.K, 0, P), prefix) and not shares.read_seqs()["status"].any()
    assert not np.array_equal(own.table_host[1, :2], own.table_host[0, :2])


def test_rows_beyond_four_gib_of_a_pool():
    """Offsets that pass 32 bits: pages far apart in a pool of more than 8 GiB."""
    n, h, D, page = 2, 2, 128, 64
    n_pages, cap = 300, 200
    stride = 32 * 1024 * 1024 // 2 + 64                      # elements from a page to the next: 32 MiB and a little
    store = [torch.empty(n_pages * stride, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    pools = [t.as_strided((n_pages, h, page, D), (stride, page * D, D, 1)) for t in store]
    d = Decode([100, 150], [150, 190], h, D, "bf16", 0, cap=cap, sel_cap=150)
    p = d.batch.params
    table = torch.tensor([[299, 3, 257, -1], [0, 298, 130, -9]], dtype=torch.int32, device=DEV)
    pages = B.make_pages(*pools, table, page_size=page)
    for b in range(n):
        for slot in range(0, int(d.resident[b]), page):
            m = min(page, int(d.resident[b]) - slot)
            for pool, cache in zip(pools, (d.batch.K, d.batch.V)):
                pool[int(table[b, slot // page]), :, :m] = cache[b, :, slot:slot + m]
    seqs = d.batch.seqs.clone()
    score = d.batch.score.clone()
    k, v = d.rows(False)
    out, lse = torch.zeros_like(d.batch.out), torch.zeros_like(d.batch.lse)
    ws = torch.empty(B.adsa_paged_workspace_bytes(p), dtype=torch.uint8, device=DEV)
    B.adsa_attend_paged(p, pages, d.batch.seqs, d.q, d.batch.sel_idx, d.batch.sel_cnt, out, lse, ws, B.FLAG_APPEND, k, v)
    torch.cuda.synchronize()
    got = out.clone(), lse.clone(), d.batch.score.clone()
    d.batch.seqs.copy_(seqs)
    d.batch.score.copy_(score)
    d.batch.attend(d.q, B.FLAG_APPEND, k, v)
    torch.cuda.synchronize()
    assert same_bits(got[0], d.batch.out) and same_bits(got[1], d.batch.lse) and same_bits(got[2], d.batch.score)
    # ... a chunk over the same pages
    begin, slot0 = torch.tensor([0, 40, 80], dtype=torch.int32, device=DEV), torch.tensor([110, 150], dtype=torch.int32, device=DEV)
    tokens = B.make_tokens(begin, slot0, 80, 40)
    q = randn(torch.Generator().manual_seed(9), 80, h, D, dtype=torch.bfloat16).to(DEV)
    outs, lses = [torch.zeros_like(q) for _ in range(2)], [torch.zeros(80, h, device=DEV) for _ in range(2)]
    d.batch.prefill(tokens, q, outs[0], lses[0], flags=B.FLAG_NO_ACCUMULATE)
    ws = torch.empty(B.adsa_prefill_paged_workspace_bytes(p, pages, tokens), dtype=torch.uint8, device=DEV)
    B.adsa_prefill_paged(p, pages, tokens, None, d.batch.seqs, q, outs[1], lses[1], ws, B.FLAG_NO_ACCUMULATE)
    torch.cuda.synchronize()
    assert same_bits(*outs) and same_bits(*lses)


def test_images_drawn_and_decoded_over_pages_by_the_example():
    """The example's images with drawn tokens, once beside a kept prompt and once with it in caches of pages; fp32 as in its own test: 1e-4 of a logit."""
    spec = importlib.util.spec_from_file_location("shared_prompt", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "shared_prompt.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    args = "--layers 3 --prompts 2 --images 3 --prompt-len 45 --grid 6 --steps 15 --budget 8 --heads 2 --q-per-kv 1 --dtype f32 --vocab 500 --check --page 16 --sample --top-k 20"
    r = m.run(m.parser().parse_args(args.split()))
    assert torch.isfinite(r["logits"]).all() and r["difference"] < 1e-4
    logits, drawn = r["logits"][:-1], r["images"][1:].long()
    rank = (logits > logits.gather(2, drawn[..., None])).sum(2)
    assert int(rank.max()) < 20 and len(drawn.unique()) > 1


def small(n, cap, G, W=5, budget=8, page=16, **kw):
    params = B.make_params(n_seq=n, n_heads=3, head_dim=64, grid_h=9, grid_w=W, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=cap, q_per_kv=G, **kw)
    return PagedBatch(params, n_pages=n * -(-cap // page) + 2, page_size=page, device=DEV)


@pytest.mark.parametrize("G", [0, 4])
def test_sequences_that_share_the_pages_of_a_prompt(G):
    """The pages of a pinned prompt in all sequences' tables, against one copy for each: evictions write behind them only."""
    n, h, D, W, budget, P = 4, 3, 64, 5, 8, 32
    cap = P + budget + 3 * W
    gen = torch.Generator().manual_seed(12)
    K, V = (randn(gen, P, h, D, dtype=torch.bfloat16).to(DEV) for _ in range(2))
    batches = [small(n, cap, G) for _ in range(2)]
    for which, batch in enumerate(batches):
        s = batch.seqs_host
        s["grid_origin"] = s["n_keep_prefix"] = s["n_res"] = P
        s["budget"], s["step"] = budget, 1
        batch.upload_seqs()
        batch.pos[:] = torch.arange(cap, dtype=torch.int32, device=DEV)
        for b in range(n):
            batch.reserve(b, cap)
            if which and b:
                batch.table_host[b, :P // 16] = batch.table_host[0, :P // 16]
        batch.upload_table()
        for b in range(n):
            batch._put_rows(b, K, V)
    hq = h * max(G, 1)
    own, shared = batches
    prompt = shared.cache_rows(shared.K, 0, P).clone(), shared.cache_rows(shared.V, 0, P).clone()
    for t in range(4 * W + 1):
        q, k, v = (randn(gen, n, heads, D, dtype=torch.bfloat16).to(DEV) for heads in (hq, h, h))
        for batch in batches:
            batch.step(q, k, v)
        same_records(own, shared)
        assert same_bits(own.out, shared.out) and same_bits(own.lse, shared.lse), t
    n_res = own.read_seqs()["n_res"]
    assert (n_res < P + 4 * W).all()
    for b in range(n):
        for pools in ((own.K, shared.K), (own.V, shared.V)):
            assert same_bits(*(batch.cache_rows(pool, b, int(n_res[b])) for batch, pool in zip(batches, pools))), b
    assert same_bits(prompt[0], shared.cache_rows(shared.K, 0, P)) and same_bits(prompt[1], shared.cache_rows(shared.V, 0, P))


@pytest.mark.parametrize("G", [0, 4])
def test_prompts_in_a_graph(G):
    """A captured append and prefill, replayed with other rows and tables and with eager ones between, against eager calls on another batch."""
    h, D, lens = 3, 64, [70, 1, 33]
    n, cap, hq, T = len(lens), 96, 3 * max(G, 1), sum(lens)
    begin = torch.tensor([0, 70, 71, 104], dtype=torch.int32, device=DEV)
    tokens = B.make_tokens(begin, torch.zeros(n, dtype=torch.int32, device=DEV), T, max(lens))
    batches = [small(n, cap, G) for _ in range(2)]
    for batch in batches:
        for b in range(n):
            batch.reserve(b, lens[b])
        batch.upload_table()
        batch.seqs_host["step"] = 0
        batch.upload_seqs()
    gen = torch.Generator().manual_seed(21)
    q, k, v = (torch.zeros(T, heads, D, dtype=torch.bfloat16, device=DEV) for heads in (hq, h, h))
    rows = [(torch.zeros(T, hq, D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, hq, D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, hq, device=DEV)) for _ in batches]
    empty = [batch.seqs.clone() for batch in batches]            # (records hold their own batch's addresses)

    def run(i):
        q_out, out, lse = rows[i]
        batches[i].append(tokens, None, q, k, v, q_out, flags=B.FLAG_ADVANCE)
        batches[i].prefill(tokens, q_out, out, lse)

    def reset(i):
        batches[i].seqs.copy_(empty[i])
        batches[i].score.zero_()
        batches[i].K.fill_(float("nan"))
        batches[i].V.fill_(float("nan"))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        run(1)
    for t in range(6):
        for x in (q, k, v):
            x.copy_(randn(gen, *x.shape, dtype=torch.bfloat16))
        if t == 3:
            assert (batches[1].table_host[[0, 2], :3] >= 0).all()
            batches[1].table_host[[0, 2], :3] = batches[1].table_host[[2, 0], :3]        # pages change places (both sequences have three at least)
            batches[1].upload_table()
        for i in range(2):
            reset(i)
        run(0)
        if t % 3 == 1:
            run(1)
        else:
            graph.replay()
        torch.cuda.synchronize()
        same_records(*batches)
        for a, b in zip(*rows):
            assert same_bits(a, b), t
        assert torch.equal(batches[0].score, batches[1].score) and torch.isfinite(rows[0][1].float()).all()
        for b in range(n):
            assert same_bits(batches[0].cache_rows(batches[0].K, b, lens[b]), batches[1].cache_rows(batches[1].K, b, lens[b])), (t, b)


def test_calls_on_two_streams_at_once():
    """Two batches over one pool (other pages of it), each on its own stream, many steps without a wait, against the same one after the other."""
    n, h, D, W, P = 3, 3, 64, 5, 16
    cap, gen = P + 8 + 3 * W, torch.Generator().manual_seed(5)
    rows = [[tuple(randn(gen, n, h, D, dtype=torch.bfloat16).to(DEV) for _ in range(3)) for _ in range(12)] for _ in range(2)]
    K = [randn(gen, n, P, h, D, dtype=torch.bfloat16).to(DEV) for _ in range(2)]
    results = []
    for together in (False, True):
        batches = [small(n, cap, 0) for _ in range(2)]
        pool = [torch.full((2 * batches[0].n_pages, *batches[0].K.shape[1:]), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        for i, batch in enumerate(batches):
            batch.free_pages = list(range(i, 2 * batch.n_pages, 2))
            batch.K, batch.V = pool
            batch.pages = B.make_pages(batch.K, batch.V, batch.table, page_size=16)
            s = batch.seqs_host
            s["grid_origin"] = s["n_keep_prefix"] = s["n_res"] = P
            s["budget"], s["step"] = 8, 1
            batch.upload_seqs()
            batch.pos[:] = torch.arange(cap, dtype=torch.int32, device=DEV)
            for b in range(n):
                batch.reserve(b, cap)
            batch.upload_table()
            for b in range(n):
                batch._put_rows(b, K[i][b], -K[i][b])
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for t in range(12):
            for batch, stream, given in zip(batches, streams, rows):
                batch.step(*given[t], stream=stream)
                if not together:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        results.append([(batch.out.clone(), batch.lse.clone(), batch.score.clone(), batch.read_seqs()["n_res"].copy()) for batch in batches])
    for a, b in zip(*results):
        assert same_bits(a[0], b[0]) and same_bits(a[1], b[1]) and torch.equal(a[2], b[2]) and (a[3] == b[3]).all()


def test_a_batch_without_records_is_inactive():
    """A step writes zeros and no cache; tokens enter whatever a sequence's step is, where it has a page for them."""
    batch = small(2, 64, 0)
    batch.reserve(0, 40)
    batch.upload_table()
    rows = [torch.ones(2, 3, 64, dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    batch.out.fill_(7)
    batch.step(*rows)
    torch.cuda.synchronize()
    assert (batch.out == 0).all() and (batch.K == 0).all() and (batch.read_seqs()["n_res"] == 0).all() and (batch.seqs_host["step"] == -1).all()
    begin = torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    tokens = B.make_tokens(begin, torch.zeros(2, dtype=torch.int32, device=DEV), 2, 1)
    batch.append(tokens, None, *rows, torch.empty_like(rows[0]), flags=B.FLAG_ADVANCE)
    torch.cuda.synchronize()
    assert batch.read_seqs()["n_res"].tolist() == [1, 0] and batch.seqs_host["status"].tolist() == [0, B.SEQ_CACHE_FULL]
    page = int(batch.table_host[0, 0])
    assert (batch.K[page, :, 0] == 1).all() and int((batch.K != 0).sum()) == 3 * 64 and int((batch.V != 0).sum()) == 3 * 64

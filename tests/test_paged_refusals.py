"""What the calls over pages and adsa_sample refuse on the host, before anything is launched, and the host's side of pages.  (No GPU: pointers are numbers
that nobody follows.)"""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2506_18226_amd import binding as B

OK = 0x1000
NULL, SHAPE, DTYPE, ALIGN, CAPACITY, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -6, -8


def params(**kw):
    base = dict(n_seq=4, n_heads=4, head_dim=64, grid_h=8, grid_w=8, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=130, sel_cap=100)
    base.update(kw)
    return B.make_params(**base)


def pages(**kw):
    base = dict(k=OK, v=OK, table=OK, page_stride=4 * 16 * 64, slot_stride=64, head_stride=16 * 64, page_size=16, n_pages=10, table_stride=9)
    base.update(kw)
    return B.AdsaPages(**base)


def tokens(**kw):
    return B.AdsaTokens(**{**dict(n_tokens=20, max_len=9, begin=OK, slot0=OK), **kw})


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def ref(x):
    return None if x is None else C.byref(x)


def append(lib, p=None, g=None, t=None, r=None, **kw):
    a = {**dict(seqs=OK, q=OK, k=OK, v=OK, qo=OK, flags=0), **kw}
    return lib.adsa_append_paged(ref(p or params()), ref(g), ref(t), ref(r), a["seqs"], a["q"], a["k"], a["v"], a["qo"], a["flags"], None)


def prefill(lib, p=None, g=None, t=None, m=None, **kw):
    a = {**dict(seqs=OK, q=OK, out=OK, lse=OK, flags=0, ws=0x10000, bytes=0), **kw}
    return lib.adsa_prefill_paged(ref(p or params()), ref(g), ref(t), ref(m), a["seqs"], a["q"], a["out"], a["lse"], a["flags"], a["ws"], a["bytes"], None)


def attend(lib, p=None, g=None, **kw):
    a = {**dict(seqs=OK, q=OK, kn=OK, vn=OK, idx=OK, cnt=OK, out=OK, lse=OK, flags=0, ws=0x10000, bytes=0), **kw}
    return lib.adsa_attend_paged(ref(p or params()), ref(g), a["seqs"], a["q"], a["kn"], a["vn"], a["idx"], a["cnt"], a["out"], a["lse"], a["flags"], a["ws"], a["bytes"], None)


def compact(lib, p=None, g=None, **kw):
    a = {**dict(seqs=OK, map=OK, flags=0, ws=0x10000, bytes=0), **kw}
    return lib.adsa_compact_paged(ref(p or params()), ref(g), a["seqs"], a["map"], a["flags"], a["ws"], a["bytes"], None)


CALLS = [lambda lib, p, g: append(lib, p, g, tokens()), lambda lib, p, g: prefill(lib, p, g, tokens()), attend, compact]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("what,code", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL), (dict(k=OK + 8), ALIGN), (dict(v=OK + 2), ALIGN), (dict(table=OK + 2), ALIGN),
    (dict(page_size=0), SHAPE), (dict(page_size=8), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=16384), SHAPE), (dict(page_size=-16), SHAPE), (dict(n_pages=0), SHAPE),
    (dict(n_pages=-1), SHAPE), (dict(table_stride=8), SHAPE), (dict(table_stride=65536), SHAPE), (dict(table_stride=-1), SHAPE), (dict(page_stride=0), SHAPE),
    (dict(slot_stride=-64), SHAPE), (dict(head_stride=0), SHAPE), (dict(slot_stride=56), SHAPE), (dict(slot_stride=68), ALIGN), (dict(head_stride=15 * 64), SHAPE),
    (dict(page_stride=3 * 16 * 64), SHAPE), (dict(slot_stride=4 * 64, head_stride=64, page_stride=15 * 4 * 64), SHAPE), (dict(slot_stride=3 * 64, head_stride=64, page_stride=1 << 20), SHAPE),
    (dict(page_stride=1 << 41), SHAPE), (dict(page_stride=(1 << 39) + 8, n_pages=1), UNSUPPORTED), (dict(n_pages=1 << 30, page_stride=1 << 30), UNSUPPORTED),
    (dict(slot_stride=64 + 8, head_stride=16 * 72, page_stride=4 * 16 * 72, n_pages=1 << 30), UNSUPPORTED)])
def test_pools_that_cannot_be(lib, call, what, code):
    assert call(lib, params(), pages(**what)) == code


@pytest.mark.parametrize("call", CALLS)
def test_parameters(lib, call):
    assert call(lib, params(), None) == NULL
    assert call(lib, params(score_mode=B.SCORE_VCOS), pages()) == UNSUPPORTED
    assert call(lib, params(score_mode=B.SCORE_VCOS_FUSED, evict_policy=B.EVICT_REUSE_SLOT, win_recent_m=9), pages()) == UNSUPPORTED
    assert call(lib, params(sel_groups=4), pages()) == UNSUPPORTED
    assert call(lib, params(head_dim=96), pages()) == SHAPE
    assert call(lib, params(cap=B.MAX_CAP + 1), pages()) == CAPACITY
    assert call(lib, params(dtype=7), pages()) == DTYPE
    assert call(lib, params(dtype=B.F32, q_per_kv=2), pages()) == UNSUPPORTED


def test_strides_of_dense_caches_are_not_used(lib):
    p = params()
    p.kv_slot_stride = p.kv_head_stride = 3
    assert lib.adsa_workspace_bytes(C.byref(p)) == 0 and lib.adsa_paged_workspace_bytes(C.byref(p)) == lib.adsa_paged_workspace_bytes(C.byref(params())) > 0
    assert attend(lib, p, pages()) == WORKSPACE and compact(lib, p, pages()) == WORKSPACE


def test_pointers_and_workspaces(lib):
    g, t, n = pages(), tokens(), 1 << 30
    for name in ("seqs", "q", "idx", "cnt", "out", "lse"):
        assert attend(lib, None, g, bytes=n, **{name: None}) == NULL, name
    assert attend(lib, None, g, bytes=n, flags=B.FLAG_APPEND, kn=None) == NULL and attend(lib, None, g, bytes=n, flags=B.FLAG_APPEND, vn=None) == NULL
    assert attend(lib, None, g, bytes=n, q=OK + 8) == ALIGN and attend(lib, None, g, bytes=n, out=OK + 4) == ALIGN
    assert attend(lib, None, g, bytes=n, flags=B.FLAG_APPEND, kn=OK + 8) == ALIGN
    need = lib.adsa_paged_workspace_bytes(C.byref(params()))
    assert attend(lib, None, g, bytes=need - 1) == WORKSPACE and attend(lib, None, g, ws=None, bytes=n) == WORKSPACE and attend(lib, None, g, ws=0x10080, bytes=n) == ALIGN
    for name in ("seqs", "map"):
        assert compact(lib, None, g, bytes=n, **{name: None}) == NULL, name
    assert compact(lib, None, g, bytes=need - 1) == WORKSPACE and compact(lib, None, g, ws=None, bytes=n) == WORKSPACE and compact(lib, None, g, ws=0x10010, bytes=n) == ALIGN
    for name in ("seqs", "q", "out", "lse"):
        assert prefill(lib, None, g, t, bytes=n, **{name: None}) == NULL, name
    need = lib.adsa_prefill_paged_workspace_bytes(C.byref(params()), C.byref(g), C.byref(t))
    assert need > 0 and prefill(lib, None, g, t, bytes=need - 1) == WORKSPACE and prefill(lib, None, g, t, ws=None, bytes=n) == WORKSPACE
    assert prefill(lib, None, g, None, bytes=n) == NULL and prefill(lib, None, g, tokens(max_len=131, n_tokens=200), bytes=n) == SHAPE
    assert prefill(lib, None, g, t, B.AdsaMods(mask=2), bytes=n) == DTYPE and prefill(lib, None, g, t, B.AdsaMods(softcap=-1.0), bytes=n) == SHAPE
    assert prefill(lib, None, g, t, B.AdsaMods(doc=OK, doc_stride=129), bytes=n) == SHAPE
    for name in ("seqs", "k", "v"):
        assert append(lib, None, g, t, **{name: None}) == NULL, name
    assert append(lib, None, g, t, qo=None) == NULL and append(lib, None, g, None) == NULL
    assert append(lib, None, g, tokens(k_stride=4 * 64 - 8)) == SHAPE and append(lib, None, g, t, q=OK + 8) == ALIGN
    assert lib.adsa_prefill_paged_workspace_bytes(C.byref(params()), None, C.byref(t)) == 0
    assert lib.adsa_prefill_paged_workspace_bytes(C.byref(params()), C.byref(pages(page_size=3)), C.byref(t)) == 0
    assert lib.adsa_paged_workspace_bytes(None) == 0 and lib.adsa_paged_workspace_bytes(C.byref(params(score_mode=B.SCORE_VCOS))) == 0


# ---- sampling
def sampling(**kw):
    return B.AdsaSampling(**{**dict(n_rows=3, vocab=100, dtype=B.F32, guided=0, row_stride=0, guidance=1.0, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **kw})


def sample(lib, s=None, **kw):
    a = {**dict(seqs=None, logits=OK, uniform=OK, token=OK, logprob=None), **kw}
    return lib.adsa_sample(ref(s), a["seqs"], a["logits"], a["uniform"], a["token"], a["logprob"], None)


@pytest.mark.parametrize("what,code", [
    (dict(dtype=2), DTYPE), (dict(n_rows=0), SHAPE), (dict(n_rows=(1 << 20) + 1), SHAPE), (dict(vocab=0), SHAPE), (dict(vocab=B.MAX_VOCAB + 1), SHAPE), (dict(guided=2), SHAPE),
    (dict(row_stride=99), SHAPE), (dict(row_stride=-100), SHAPE), (dict(row_stride=1 << 41), SHAPE), (dict(guided=1, guidance=float("inf")), SHAPE),
    (dict(guided=1, guidance=float("nan")), SHAPE), (dict(temperature=-0.5), SHAPE), (dict(temperature=float("nan")), SHAPE), (dict(temperature=float("inf")), SHAPE),
    (dict(top_p=float("nan")), SHAPE), (dict(min_p=float("nan")), SHAPE)])
def test_settings_that_cannot_be(lib, what, code):
    assert sample(lib, sampling(**what)) == code


def test_sampling_pointers(lib):
    assert sample(lib, None) == NULL
    for name in ("logits", "uniform", "token"):
        assert sample(lib, sampling(), **{name: None}) == NULL, name
    assert sample(lib, sampling(), logits=OK + 2) == ALIGN and sample(lib, sampling(dtype=B.BF16), logits=OK + 1) == ALIGN
    for name in ("uniform", "token", "logprob"):
        assert sample(lib, sampling(), **{name: OK + 2}) == ALIGN, name
    for name in ("temperatures", "top_ks", "top_ps", "min_ps"):
        assert sample(lib, sampling(**{name: OK + 1})) == ALIGN, name


def test_struct_sizes_match_the_header():
    """3 addresses, 3 distances, 4 numbers; 4 numbers, a distance, 6 numbers, 4 addresses."""
    assert C.sizeof(B.AdsaPages) == 6 * 8 + 4 * 4 and B.AdsaPages.page_size.offset == 48
    assert C.sizeof(B.AdsaSampling) == 4 * 4 + 8 + 6 * 4 + 4 * 8 and B.AdsaSampling.row_stride.offset == 16 and B.AdsaSampling.temperatures.offset == 48


# ---- the binding's checks
def test_binding_checks_pools_and_tables():
    k = torch.zeros(5, 2, 16, 64, dtype=torch.bfloat16)
    table = torch.zeros(3, 4, dtype=torch.int32)
    g = B.make_pages(k, k.clone(), table, page_size=16)
    assert (g.n_pages, g.page_stride, g.slot_stride, g.head_stride, g.table_stride) == (5, 2 * 16 * 64, 64, 16 * 64, 4)
    g = B.make_pages(k.view(5, 16, 2, 64), k.view(5, 16, 2, 64).clone(), table, page_size=16, layout="slot_major")
    assert (g.slot_stride, g.head_stride) == (128, 64)
    for bad in (lambda: B.make_pages(k, k[:, :, :, :32], table, page_size=16), lambda: B.make_pages(k, k.float(), table, page_size=16),
                lambda: B.make_pages(k, k.clone(), table.long(), page_size=16), lambda: B.make_pages(k, k.clone(), table, page_size=32),
                lambda: B.make_pages(k[0], k[0], table, page_size=16), lambda: B.make_pages(k.transpose(2, 3), k.transpose(2, 3), table, page_size=64)):
        with pytest.raises(ValueError):
            bad()
    g = B.make_pages(k, k.clone(), table, page_size=16)
    with pytest.raises(ValueError):                          # another number of heads
        B.adsa_compact_paged(params(n_seq=3, n_heads=4, cap=64, sel_cap=64), g, OK, OK, None)
    with pytest.raises(ValueError):                          # a table of fewer sequences
        B.adsa_compact_paged(params(n_seq=4, n_heads=2, cap=64, sel_cap=64), g, OK, OK, None)
    with pytest.raises(TypeError):
        B.adsa_attend_paged(params(), tokens(), OK, OK, OK, OK, OK, OK, None)


def test_binding_checks_sampling():
    f = torch.zeros(3, dtype=torch.float32)
    with pytest.raises(ValueError):
        B.make_sampling(4, 10, B.F32, temperature=f)
    with pytest.raises(ValueError):
        B.make_sampling(3, 10, B.F32, top_k=f)
    s = B.make_sampling(3, 10, B.F32, temperature=f, top_k=f.to(torch.int32), guidance=2.0)
    assert s.guided == 1 and s.temperatures == f.data_ptr() and s.top_ps is None
    logits, token = torch.zeros(6, 10), torch.zeros(6, dtype=torch.int32)
    for bad in (dict(logits=logits[:5]), dict(logits=logits.bfloat16()), dict(logits=logits[:, :9]), dict(uniform=f[:2]), dict(token=token[:5]), dict(token=token.long()),
                dict(logprob=f[:2]), dict(seqs=torch.zeros(5 * 96, dtype=torch.uint8)), dict(logits=logits.t().contiguous().t())):
        with pytest.raises(ValueError):
            B.adsa_sample(s, **{**dict(logits=logits, uniform=f, token=token), **bad})
    with pytest.raises(TypeError):
        B.adsa_sample(params(), logits, f, token)
    with pytest.raises(B.AdsaError):
        B.adsa_sample(None, logits, f, token)


def test_pages_are_given_and_taken_back():
    from paper_2506_18226_amd.batch import PagedBatch

    batch = PagedBatch.__new__(PagedBatch)                   # (the host's side alone: no device here)
    batch.params, batch.page_size, batch.n_pages = params(cap=130), 16, 12
    batch.table_host, batch.free_pages = np.full((4, 9), -1, np.int32), list(range(11, -1, -1))
    batch.reserve(0, 17)
    batch.reserve(1, 0)
    batch.reserve(2, 130)
    assert list(batch.table_host[0, :3]) == [0, 1, -1] and (batch.table_host[1] == -1).all() and (batch.table_host[2] >= 0).all() and len(batch.free_pages) == 1
    before = batch.table_host.copy()
    with pytest.raises(MemoryError):
        batch.reserve(0, 100)
    assert np.array_equal(batch.table_host, before) and len(batch.free_pages) == 1
    batch.reserve(0, 10)                                     # (has them)
    assert np.array_equal(batch.table_host, before)
    batch.release(2, 33)
    assert (batch.table_host[2, :3] >= 0).all() and (batch.table_host[2, 3:] == -1).all() and len(batch.free_pages) == 7
    batch.reserve(1, 100)
    taken = batch.table_host[batch.table_host >= 0]
    assert len(set(taken.tolist())) == len(taken) == 12 and not batch.free_pages
    batch.release(1)
    assert (batch.table_host[1] == -1).all() and len(batch.free_pages) == 7
    with pytest.raises(ValueError):
        batch.reserve(0, 131)

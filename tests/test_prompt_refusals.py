"""What the prompt side refuses on the host, before anything is launched.  (No GPU: pointers are numbers that nobody follows.)"""
import ctypes as C

import pytest
import torch

from paper_2506_18226_amd import binding as B

OK = 0x1000
NULL, SHAPE, DTYPE, ALIGN, CAPACITY, WORKSPACE, UNSUPPORTED = -1, -2, -3, -4, -5, -6, -8


def params(**kw):
    base = dict(n_seq=4, n_heads=4, head_dim=64, grid_h=8, grid_w=8, win_rows_back=1, win_col_radius=2, dtype=B.BF16,
                score_mode=B.SCORE_ATTN_MASS, cap=128, sel_cap=100)
    base.update(kw)
    return B.make_params(**base)


def rope(**kw):
    r = B.AdsaRope(OK, 2, 0)
    for name, value in kw.items():
        setattr(r, name, value)
    return r


def tokens(**kw):
    base = dict(n_tokens=20, max_len=9, begin=OK, slot0=OK)
    base.update(kw)
    return B.AdsaTokens(**base)


def shared(**kw):
    base = dict(n_groups=2, max_prompt=64, max_members=3, prompts=OK, members=OK, kv_slot_stride=64, kv_head_stride=64 * 64)
    base.update(kw)
    return B.AdsaShared(**base)


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def ref(x):
    return None if x is None else C.byref(x)


def rotate(lib, p=None, r=None, **kw):
    a = dict(seqs=OK, coords=None, q=OK, k=OK, qs=0, ks=0, qo=OK, ko=OK, flags=0)
    a.update(kw)
    return lib.adsa_rotate(ref(p or params()), ref(r), a["seqs"], a["coords"], a["q"], a["k"], a["qs"], a["ks"], a["qo"], a["ko"], a["flags"], None)


def append(lib, p=None, t=None, r=None, **kw):
    a = dict(seqs=OK, q=OK, k=OK, v=OK, qo=OK, flags=0)
    a.update(kw)
    return lib.adsa_append(ref(p or params()), ref(t), ref(r), a["seqs"], a["q"], a["k"], a["v"], a["qo"], a["flags"], None)


def prefill(lib, p=None, t=None, m=None, **kw):
    a = dict(seqs=OK, q=OK, out=OK, lse=OK, flags=0, ws=OK, bytes=1 << 40)
    a.update(kw)
    return lib.adsa_prefill(ref(p or params()), ref(t), ref(m), a["seqs"], a["q"], a["out"], a["lse"], a["flags"], a["ws"], a["bytes"], None)


def attend(lib, p=None, s=None, m=None, **kw):
    a = dict(seqs=OK, q=OK, kn=OK, vn=OK, idx=OK, cnt=OK, out=OK, lse=OK, flags=B.FLAG_APPEND, ws=OK, bytes=1 << 40)
    a.update(kw)
    return lib.adsa_attend_shared(ref(p or params()), ref(s), ref(m), a["seqs"], a["q"], a["kn"], a["vn"], a["idx"], a["cnt"], a["out"], a["lse"], a["flags"],
                                  a["ws"], a["bytes"], None)


@pytest.mark.parametrize("code,kw", [
    (NULL, dict(r=None)), (NULL, dict(r=rope(freq=None))), (ALIGN, dict(r=rope(freq=OK + 8))), (SHAPE, dict(r=rope(n_axes=0))), (SHAPE, dict(r=rope(n_axes=4))),
    (DTYPE, dict(r=rope(pairing=2))), (UNSUPPORTED, dict(r=rope(), p=params(sel_groups=4))), (SHAPE, dict(r=rope(), p=params(head_dim=96))),
    *[(NULL, dict(r=rope(), **{n: None})) for n in ("seqs", "q", "k", "qo", "ko")], *[(ALIGN, dict(r=rope(), **{n: OK + 8})) for n in ("q", "k", "qo", "ko")],
    (SHAPE, dict(r=rope(), qs=255)), (SHAPE, dict(r=rope(), ks=-256)), (ALIGN, dict(r=rope(), qs=260)), (ALIGN, dict(r=rope(), ks=258, flags=B.FLAG_NEW_F32))])
def test_rotate(lib, code, kw):
    assert rotate(lib, **kw) == code


@pytest.mark.parametrize("code,kw", [
    (NULL, dict(t=None)), (NULL, dict(t=tokens(begin=None))), (NULL, dict(t=tokens(slot0=None))), (SHAPE, dict(t=tokens(n_tokens=0))), (SHAPE, dict(t=tokens(max_len=0))),
    (SHAPE, dict(t=tokens(max_len=129, n_tokens=500))), (SHAPE, dict(t=tokens(max_len=21))), (SHAPE, dict(t=tokens(n_tokens=(1 << 24) + 1))),
    *[(NULL, dict(t=tokens(), **{n: None})) for n in ("seqs", "k", "v", "q", "qo")], *[(ALIGN, dict(t=tokens(), **{n: OK + 4})) for n in ("q", "k", "v", "qo")],
    (SHAPE, dict(t=tokens(v_stride=100))), (ALIGN, dict(t=tokens(k_stride=260))), (NULL, dict(t=tokens(), r=rope(freq=None))), (SHAPE, dict(t=tokens(), r=rope(n_axes=9))),
    (UNSUPPORTED, dict(t=tokens(), p=params(sel_groups=4)))])
def test_append(lib, code, kw):
    assert append(lib, **kw) == code


def test_prefill(lib):
    t = tokens()
    need = B.adsa_prefill_workspace_bytes(params(), t)
    assert need > 0
    for code, kw in [(NULL, dict(t=None)), (SHAPE, dict(t=tokens(max_len=300, n_tokens=300))), *[(NULL, dict(t=t, **{n: None})) for n in ("seqs", "q", "out", "lse")],
                     (ALIGN, dict(t=t, q=OK + 8)), (ALIGN, dict(t=t, out=OK + 2)), (WORKSPACE, dict(t=t, ws=None)), (WORKSPACE, dict(t=t, bytes=need - 1)),
                     (ALIGN, dict(t=t, ws=OK + 16)), (SHAPE, dict(t=t, m=B.AdsaMods(softcap=-1.0))), (SHAPE, dict(t=t, m=B.AdsaMods(softcap=float("nan")))),
                     (SHAPE, dict(t=t, m=B.AdsaMods(softcap=float("inf")))), (DTYPE, dict(t=t, m=B.AdsaMods(mask=2))),
                     (SHAPE, dict(t=t, m=B.AdsaMods(doc=OK, doc_stride=127))), (UNSUPPORTED, dict(t=t, p=params(sel_groups=4)))]:
        assert prefill(lib, **kw) == code, kw
    assert B.adsa_prefill_workspace_bytes(params(sel_groups=4), t) == 0 and B.adsa_prefill_workspace_bytes(params(), tokens(max_len=0)) == 0
    # a launch has less than 2^32 threads
    many = params(n_seq=65535, n_heads=256, cap=4096, sel_cap=4096)
    assert prefill(lib, p=many, t=tokens(n_tokens=1 << 20, max_len=4096)) == UNSUPPORTED
    assert B.adsa_prefill_workspace_bytes(many, tokens(n_tokens=1 << 20, max_len=4096)) == 0


def test_attend_shared(lib):
    s = shared()
    need = B.adsa_shared_workspace_bytes(params(), s)
    assert need > 0
    for code, kw in [(NULL, dict(s=None)), (NULL, dict(s=shared(prompts=None))), (NULL, dict(s=shared(members=None))), (SHAPE, dict(s=shared(n_groups=0))),
                     (SHAPE, dict(s=shared(n_groups=5))), (SHAPE, dict(s=shared(max_members=0))), (SHAPE, dict(s=shared(max_members=5))),
                     (CAPACITY, dict(s=shared(max_prompt=0))), (CAPACITY, dict(s=shared(max_prompt=8193))), (SHAPE, dict(s=shared(kv_slot_stride=0))),
                     (SHAPE, dict(s=shared(kv_head_stride=63 * 64))), (ALIGN, dict(s=shared(kv_slot_stride=68))),
                     *[(NULL, dict(s=s, **{n: None})) for n in ("seqs", "q", "kn", "vn", "idx", "cnt", "out", "lse")],
                     *[(ALIGN, dict(s=s, **{n: OK + 8})) for n in ("q", "kn", "vn", "out")], (WORKSPACE, dict(s=s, ws=None)), (WORKSPACE, dict(s=s, bytes=need - 1)),
                     (ALIGN, dict(s=s, ws=OK + 128)), (SHAPE, dict(s=s, m=B.AdsaMods(softcap=-2.0))), (UNSUPPORTED, dict(s=s, p=params(sel_groups=4))),
                     (UNSUPPORTED, dict(s=s, p=params(score_mode=B.SCORE_VCOS_FUSED, evict_policy=B.EVICT_REUSE_SLOT, win_recent_m=9)))]:
        assert attend(lib, **kw) == code, kw
    assert B.adsa_shared_workspace_bytes(params(), shared(max_members=9)) == 0


def test_struct_mirrors():
    assert C.sizeof(B.AdsaRope) == 8 + 2 * 4 + 4 * 3 * 4 and C.sizeof(B.AdsaTokens) == 2 * 4 + 4 * 8 + 3 * 8
    assert C.sizeof(B.AdsaMods) == 2 * 4 + 2 * 8 + 8 and C.sizeof(B.AdsaShared) == 4 * 4 + 2 * 8 + 2 * 8


def test_python_side_refuses_wrong_tensors():
    f = torch.zeros(2, 32, dtype=torch.float64)
    axes = dict(text=(0, 0), origin=(0, 0), row=(1, 0), col=(0, 1))
    assert B.make_rope(f, pairing="neighbours", **axes).n_axes == 2
    for bad in (f.float(), f[0], f.t(), torch.zeros(4, 32, dtype=torch.float64)):
        with pytest.raises(ValueError):
            B.make_rope(bad, **axes)
    with pytest.raises(ValueError):
        B.make_rope(f, **dict(axes, row=(1,)))
    with pytest.raises(KeyError):
        B.make_rope(f, pairing="thirds", **axes)
    i = torch.zeros(3, dtype=torch.int32)
    for kw in (dict(begin=i.long(), slot0=i), dict(begin=i, slot0=i.float()), dict(begin=i, slot0=i, coords=i.long())):
        with pytest.raises(ValueError):
            B.make_tokens(kw.pop("begin"), kw.pop("slot0"), 2, 1, **kw)
    with pytest.raises(ValueError):
        B.make_mods(slopes=torch.zeros(4, dtype=torch.float64))
    with pytest.raises(ValueError):
        B.make_mods(doc=torch.zeros(4, 4).t().int().t()[:, :2])

"""Tensors of the prompt calls that are shorter than what a call reads, or laid out otherwise, are refused before anything is launched; so are prompts
whose rows are not the sequences' own.  (No GPU: what reaches the library is noted, not run.)"""
import pytest
import torch

from paper_2506_18226_amd import binding as B

AXES = dict(text=(0, 0), origin=(0, 0), row=(1, 0), col=(0, 1))


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def params(**kw):
    base = dict(n_seq=3, n_heads=2, head_dim=64, grid_h=8, grid_w=8, win_rows_back=1, win_col_radius=2, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=40, q_per_kv=2)
    return B.make_params(**dict(base, **kw))


@pytest.fixture
def calls(monkeypatch):
    reached = []
    monkeypatch.setattr(B, "_prompt_call", lambda name, *a: reached.append(name))
    p, x = params(), 1 << 20
    return dict(
        reached=reached,
        rotate=lambda rope, coords=None: B.adsa_rotate(p, rope, x, x, x, x, x, coords),
        append=lambda tokens, rope=None: B.adsa_append(p, tokens, rope, x, x, x, x, x),
        prefill=lambda tokens, mods=None: B.adsa_prefill(p, tokens, mods, x, x, x, x, x),
        shared=lambda shared, mods=None: B.adsa_attend_shared(p, shared, mods, x, x, x, x, x, x, x, x, x))


def rope(width=32, axes=2):
    return B.make_rope(torch.zeros(axes, width, dtype=torch.float64), **{k: v[:axes] for k, v in AXES.items()})


def tokens(**kw):
    a = dict(begin=ints(4), slot0=ints(3), n_tokens=5, max_len=3)
    a.update(kw)
    return B.make_tokens(a.pop("begin"), a.pop("slot0"), a.pop("n_tokens"), a.pop("max_len"), **a)


def shared(groups=2, members=None, records=None, **kw):
    return B.make_shared(params(n_seq=groups, **kw), torch.zeros(96 * (groups if records is None else records), dtype=torch.uint8),
                         ints(groups + 1) if members is None else members, max_members=2)


def test_calls_with_what_they_read_go_through(calls):
    calls["rotate"](rope())
    calls["rotate"](rope(), ints(3, 2))
    calls["rotate"](rope(), 1 << 20)
    for t in (tokens(), tokens(pos0=ints(3), coords=ints(5, 2)), tokens(begin=1 << 20, slot0=1 << 20), B.AdsaTokens(5, 3, 1 << 20, 1 << 20)):
        calls["append"](t, rope())
        calls["append"](t)
        calls["prefill"](t, B.make_mods(slopes=torch.zeros(4), doc=ints(3, 40)))
    calls["shared"](shared(), B.make_mods(slopes=torch.zeros(4)))
    calls["shared"](shared(), B.make_mods(doc=ints(1, 40)))            # (not read)
    calls["rotate"](rope(), (ints(6, 2), 24))                # a tensor and a byte offset, as other pointers
    calls["shared"](shared(q_per_kv=0, cap=77, layout="slot_major"))
    calls["shared"](B.AdsaShared(), B.AdsaMods())
    for name in ("append", "prefill", "shared"):             # (the library says ADSA_ERR_NULL)
        calls[name](None)
    assert len(calls["reached"]) == 23


@pytest.mark.parametrize("call,bad", [
    ("rotate", lambda: (rope(64),)), ("rotate", lambda: (rope(31),)), ("rotate", lambda: (rope(), ints(2, 2))), ("rotate", lambda: (rope(), ints(6))),
    ("rotate", lambda: (rope(), ints(3, 3))), ("rotate", lambda: (rope(axes=1), ints(3, 2))), ("rotate", lambda: (rope(), ints(3, 2).long())),
    ("rotate", lambda: (rope(), ints(2, 3).t())),
    ("append", lambda: (tokens(begin=ints(3)),)), ("append", lambda: (tokens(slot0=ints(2)),)), ("append", lambda: (tokens(pos0=ints(2)),)),
    ("append", lambda: (tokens(coords=ints(5, 3)), rope())), ("append", lambda: (tokens(coords=ints(4, 2)), rope())), ("append", lambda: (tokens(coords=ints(10)), rope())),
    ("append", lambda: (tokens(), rope(16))),
    ("prefill", lambda: (tokens(begin=ints(3)),)), ("prefill", lambda: (tokens(slot0=ints(1)),)), ("prefill", lambda: (tokens(), B.make_mods(slopes=torch.zeros(2)))),
    ("prefill", lambda: (tokens(), B.make_mods(doc=ints(40)))), ("prefill", lambda: (tokens(), B.make_mods(doc=ints(2, 40)))),
    ("shared", lambda: (shared(members=ints(2)),)), ("shared", lambda: (shared(records=1),)), ("shared", lambda: (shared(n_heads=4),)),
    ("shared", lambda: (shared(head_dim=128),)), ("shared", lambda: (shared(dtype=B.F32),)), ("shared", lambda: (shared(), B.make_mods(slopes=torch.zeros(3))))])
def test_others_are_refused(calls, call, bad):
    with pytest.raises(ValueError):
        calls[call](*bad())
    assert not calls["reached"]


def test_records_behind_others():
    """Prompts of a later layer: what lies in front of them counts for nothing."""
    records = torch.zeros(96 * 6, dtype=torch.uint8)
    p = params(n_seq=2)
    assert B.make_shared(p, (records, 96 * 4), ints(3), max_members=2).prompts == records.data_ptr() + 96 * 4
    with pytest.raises(ValueError):
        B.make_shared(p, (records, 96 * 5), ints(3), max_members=2)

"""Workspaces of the prompt calls of a batch: one for each entry point and stream, and none is given up once a call has had it, since a captured
graph may hold its address.  (No GPU: tensors are the host's, and calls do what the library does about a workspace that is too small.)"""
import gc
import weakref

import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch


@pytest.fixture
def batch(monkeypatch):
    monkeypatch.setattr(torch.cuda, "synchronize", lambda device=None: None)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    need = [0]
    seen = []

    def entry(name, params, second, third, flags, stream, workspace, *rest):
        if workspace.numel() < need[0]:
            raise B.AdsaError(B.ERR_WORKSPACE, name)
        seen.append((name, stream, workspace.data_ptr(), weakref.ref(workspace)))

    monkeypatch.setattr(B, "_prompt_call", entry)
    for name in ("adsa_prefill_workspace_bytes", "adsa_shared_workspace_bytes"):
        monkeypatch.setattr(B, name, lambda *a: need[0])
    b = LayerBatch.__new__(LayerBatch)
    b.device, b.params, b.seqs = torch.device("cpu"), B.make_params(n_seq=2, n_heads=1, head_dim=64, grid_h=4, grid_w=4, win_rows_back=1, win_col_radius=1, dtype=B.F32,
                                                                    score_mode=B.SCORE_ATTN_MASS, cap=40), None
    b.sel_idx = b.sel_cnt = b.out = b.lse = b.prompt_workspace = None
    b._prompt_workspaces, b._outgrown = {}, []
    q, mods = torch.zeros(2, 1, 64), None
    tokens = B.make_tokens(torch.tensor([0, 1, 2], dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 2, 1)
    shared = B.AdsaShared()
    b.calls = dict(prefill=lambda stream: b.prefill(tokens, q, q, None, mods, stream=stream), shared=lambda stream: b.attend_shared(shared, q, stream=stream))

    def run(call, bytes_needed, stream=1):
        need[0] = bytes_needed
        b.calls[call](stream)
        return seen[-1][2:]

    b.run = run
    return b


@pytest.mark.parametrize("call", ["prefill", "shared"])
def test_a_workspace_that_a_graph_may_hold_is_kept(batch, call):
    held = [batch.run("shared", 1000)]
    for n in (2000, 2001, 9000, 50000, 300):
        held.append(batch.run(call, n))
    gc.collect()
    for at, ref in held:
        assert ref() is not None and ref().data_ptr() == at
    assert sum(w.numel() for w in batch._outgrown) <= batch.prompt_workspace.numel() + 1000


def test_calls_that_may_run_at_one_time_share_no_workspace(batch):
    places = {(call, stream): batch.run(call, 700, stream)[0] for call in ("prefill", "shared") for stream in (1, 2)}
    assert len(set(places.values())) == 4
    for (call, stream), at in places.items():                # ... and each finds its own again
        assert batch.run(call, 600, stream)[0] == at and batch.prompt_workspace.data_ptr() == at


def test_other_errors_pass_through(batch, monkeypatch):
    batch.run("prefill", 100)

    def refuse(*a):
        raise B.AdsaError(-2, "adsa_prefill")

    monkeypatch.setattr(B, "_prompt_call", refuse)
    kept = batch.prompt_workspace
    with pytest.raises(B.AdsaError) as e:
        batch.calls["prefill"](1)
    assert e.value.code == -2 and batch.prompt_workspace is kept and not batch._outgrown

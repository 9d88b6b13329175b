"""Graphs of prompt calls whose batch has needed larger workspaces since they were captured."""
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch

from test_gpu_shared import Shared

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_graph_outlives_the_growth_of_workspaces():
    s = Shared([3, 2], [60, 20], [40, 7, 33, 1, 90], 2, 64)
    batch, stream = s.batch, torch.cuda.Stream()

    def reset():
        batch.score.copy_(torch.from_numpy(s.score0))
        batch.out.fill_(7.0)
        batch.lse.fill_(7.0)
        torch.cuda.synchronize()

    def attend(shared):
        with torch.cuda.stream(stream):
            batch.attend_shared(shared, s.q, s.kn, s.vn, flags=s.flags)

    attend(s.shared)
    torch.cuda.synchronize()
    want = [t.clone() for t in (batch.out, batch.lse, batch.score)]
    small = batch.prompt_workspace.numel()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        batch.attend_shared(s.shared, s.q, s.kn, s.vn, flags=s.flags)
    # longer prompts' records, which are met in more parts; and a prompt's attention over the same caches
    long = LayerBatch(B.make_params(n_seq=2, n_heads=2, head_dim=64, grid_h=100, grid_w=100, win_rows_back=1, win_col_radius=2, dtype=B.BF16,
                                    score_mode=B.SCORE_ATTN_MASS, cap=2002), DEV)
    attend(B.make_shared(long.params, long.seqs, torch.tensor([0, 3, 5], dtype=torch.int32, device=DEV), max_members=3))
    torch.cuda.synchronize()
    assert batch.prompt_workspace.numel() > small
    int32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    rows = torch.empty(5, 2, 64, dtype=torch.bfloat16, device=DEV)
    batch.prefill(B.make_tokens(int32(0, 1, 2, 3, 4, 5), int32(0, 0, 0, 0, 0), 5, 1), s.q, rows, torch.empty(5, 2, device=DEV), stream=stream)
    torch.cuda.synchronize()
    fresh = [torch.full((small,), 255, dtype=torch.uint8, device=DEV) for _ in range(64)]
    for _ in range(3):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (batch.out, batch.lse, batch.score)))
        assert all((f == 255).all() for f in fresh)
    reset()
    s.run()
    s.check()

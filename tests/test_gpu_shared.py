"""Decode attention of sequences that share prompts, against 64-bit sums on the host and against adsa_attend over caches that hold the
prompt themselves."""
import numpy as np
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch

from prompt_common import attended, close, f64, half_step, randn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


class Shared:
    """Groups of sequences: members (sizes), prompts (slots) and own lists (lengths); the query token's slot is a list's place `new_at`."""

    def __init__(self, members, prompts, lists, h, D, dtype="bf16", G=0, layout="head_major", prompt_layout="head_major", new_f32=False, append=True,
                 new_at=-1, seed=3, q_scale=1.5, prompt_cap=None):
        n, self.h, self.D, self.G = sum(members), h, D, max(G, 1)
        self.members, self.prompts, self.lists = np.concatenate([[0], np.cumsum(members)]), prompts, np.asarray(lists)
        cap = int(self.lists.max()) + 9
        common = dict(n_heads=h, head_dim=D, grid_h=100, grid_w=100, win_rows_back=1, win_col_radius=2, dtype=B.F32 if dtype == "f32" else B.BF16, q_per_kv=G,
                      score_mode=B.SCORE_ATTN_MASS)
        self.batch = LayerBatch(B.make_params(n_seq=n, cap=cap, sel_cap=max(1, int(self.lists.max())), layout=layout, **common), DEV)
        pcap = max(1, max(prompts)) + 2 if prompt_cap is None else prompt_cap
        self.pb = LayerBatch(B.make_params(n_seq=len(prompts), cap=pcap, layout=prompt_layout, **common), DEV)
        gen = torch.Generator().manual_seed(seed)
        dt = self.batch.tdtype
        self.bf16 = dt == torch.bfloat16
        view = lambda t, lay: t if lay == "head_major" else t.transpose(1, 2)
        self.K, self.V = view(self.batch.K, layout), view(self.batch.V, layout)
        self.PK, self.PV = view(self.pb.K, prompt_layout), view(self.pb.V, prompt_layout)
        rng = np.random.default_rng(seed)
        for t in (self.K, self.V):
            t.fill_(NAN)                                     # slots that no list names may hold anything
        for t in (self.PK, self.PV):
            t.copy_(randn(gen, *t.shape, dtype=dt))
            for g, m in enumerate(prompts):
                t[g, :, m:] = NAN
        self.sel, self.pending = [], np.full(n, -1)
        for b, m in enumerate(self.lists):
            s = np.sort(rng.choice(cap, m, replace=False)).astype(np.int64)
            self.sel.append(s)
            self.batch.sel_idx[b, :m] = torch.from_numpy(s).to(torch.int32)
            for t in (self.K, self.V):
                t[b, :, torch.from_numpy(s).to(DEV)] = randn(gen, h, m, D, dtype=dt).to(DEV)
            if append and m:
                self.pending[b] = s[min(new_at, m - 1)] if new_at >= 0 else s[-1]
                for t in (self.K, self.V):
                    t[b, :, self.pending[b]] = NAN           # its row comes with the call
        self.batch.sel_cnt.copy_(torch.from_numpy(self.lists.astype(np.int32)))
        it = torch.float32 if new_f32 else dt
        self.kn, self.vn = randn(gen, n, h, D, dtype=it).to(DEV), randn(gen, n, h, D, dtype=it).to(DEV)
        self.q = randn(gen, n, h * self.G, D, dtype=dt, scale=q_scale).to(DEV)
        s = self.batch.seqs_host
        s["n_res"], s["pending_slot"], s["grid_origin"], s["step"] = cap, self.pending, pcap, 3 * cap
        self.batch.pos[:] = pcap + 3 * torch.arange(cap, dtype=torch.int32, device=DEV)
        self.qpos = pcap + 3 * cap - 1
        self.pb.pos[:] = torch.arange(pcap, dtype=torch.int32, device=DEV)
        self.pb.seqs_host["n_res"] = prompts
        self.batch.upload_seqs()
        self.pb.upload_seqs()
        self.batch.score.uniform_(generator=torch.Generator(device=DEV).manual_seed(seed))
        self.score0 = f64(self.batch.score)
        self.batch.out.fill_(7.0)
        self.batch.lse.fill_(7.0)
        self.flags = (B.FLAG_APPEND if append else 0) | (B.FLAG_NEW_F32 if new_f32 else 0)
        self.shared = B.make_shared(self.pb.params, self.pb.seqs, torch.tensor(self.members, dtype=torch.int32, device=DEV), max_members=max(members))

    def run(self, flags=0, **mods):
        self.batch.attend_shared(self.shared, self.q, self.kn, self.vn, flags=self.flags | flags, mods=B.make_mods(**mods) if mods else None)
        torch.cuda.synchronize()

    def check(self, softcap=0.0, slopes=None, mass=True, dead=(), prompt_from=0):
        K, V, PK, PV, q, out, lse, score = (f64(x) for x in (self.K, self.V, self.PK, self.PV, self.q, self.batch.out, self.batch.lse, self.batch.score))
        kn, vn = f64(self.kn.to(self.batch.tdtype)), f64(self.vn.to(self.batch.tdtype))
        want_score, tol_score = self.score0.copy(), 4 * 2.0 ** -24 * np.abs(self.score0)
        pos = self.batch.pos.cpu().numpy()
        for g, m in enumerate(self.prompts):
            for b in range(self.members[g], self.members[g + 1]):
                if b in dead:
                    assert not out[b].any() and not lse[b].any()
                    continue
                s = self.sel[b]
                if self.pending[b] >= 0:                     # the row is in the cache now
                    assert np.array_equal(K[b, :, self.pending[b]], kn[b]) and np.array_equal(V[b, :, self.pending[b]], vn[b])
                dist = self.qpos - np.concatenate([prompt_from + np.arange(m), pos[b, s]])
                if self.pending[b] >= 0:
                    dist[m + int(np.flatnonzero(s == self.pending[b])[0])] = 0           # its distance to itself
                for j in range(self.h * self.G):
                    hd = j // self.G
                    o, ls, p, ot, st, pt = attended(q[b, j][None], np.concatenate([PK[g, hd, :m], K[b, hd, s]]), np.concatenate([PV[g, hd, :m], V[b, hd, s]]),
                                                    self.D ** -0.5, cap=softcap, slope=0.0 if slopes is None else float(slopes[j]), dist=dist[None], bf16=self.bf16)
                    close(out[b, j][None], o, ot, f"out of sequence {b}, head {j}")
                    close(lse[b, j][None], ls, st, f"lse of sequence {b}, head {j}")
                    want_score[b, hd, s] += p[0, m:]
                    tol_score[b, hd, s] += (p * pt)[0, m:] + 2.0 ** -22 * (1 + want_score[b, hd, s])
        if mass:
            close(score, want_score, tol_score, "score")
        else:
            assert np.array_equal(score, self.score0)


@pytest.mark.parametrize("members,prompts,lists", [
    ([1], [1], [1]), ([2], [0], [5, 1]), ([3, 1, 2], [40, 0, 300], [0, 31, 64, 0, 129, 33]), ([5], [129], [2, 0, 200, 1, 96]), ([33, 1], [65, 500], list(range(34))),
    ([1, 1], [700, 33], [600, 45])])
@pytest.mark.parametrize("h,D,dtype,G,layout,prompt_layout,new_f32", [
    (2, 64, "bf16", 0, "head_major", "head_major", False), (3, 128, "bf16", 0, "slot_major", "head_major", True), (1, 64, "f32", 0, "head_major", "slot_major", False),
    (2, 128, "f32", 0, "slot_major", "slot_major", False), (2, 128, "bf16", 8, "head_major", "slot_major", True), (1, 64, "bf16", 16, "slot_major", "slot_major", False),
    (2, 64, "bf16", 3, "head_major", "head_major", False)])
def test_against_the_definition(members, prompts, lists, h, D, dtype, G, layout, prompt_layout, new_f32):
    s = Shared(members, prompts, lists, h, D, dtype, G, layout, prompt_layout, new_f32)
    s.run(B.FLAG_ADVANCE)
    s.check()
    cap = s.batch.params.cap
    r = s.batch.read_seqs()
    assert (r["step"] == 3 * cap + 1).all() and not r["status"].any()


@pytest.mark.parametrize("h,D,dtype,G", [(2, 64, "bf16", 0), (1, 128, "bf16", 5), (2, 64, "f32", 0), (1, 128, "f32", 0)])
@pytest.mark.parametrize("cap,slope", [(4.0, False), (0.0, True), (15.0, True)])
def test_scores_capped_and_lowered_with_distance(h, D, dtype, G, cap, slope):
    s = Shared([3, 2], [150, 20], [70, 0, 33, 1, 200], h, D, dtype, G, new_at=4, q_scale=4.0)
    mods = dict(softcap=cap, slopes=torch.tensor([2.0 ** -(3 + i) for i in range(h * s.G)], device=DEV) if slope else None)
    s.run(**mods)
    s.check(**mods)


@pytest.mark.parametrize("h,D,dtype,G", [(2, 64, "bf16", 0), (1, 128, "bf16", 5), (1, 64, "bf16", 16), (2, 64, "f32", 0), (1, 128, "f32", 0)])
def test_distances_between_far_positions(h, D, dtype, G):
    """Positions that fp32 does not hold (it counts in steps of 64 there) lie as far apart as near ones."""
    s = Shared([3, 2], [150, 20], [70, 0, 33, 1, 200], h, D, dtype, G, new_at=4)
    far = 1_000_000_000
    s.batch.pos += far
    s.pb.pos += far
    s.batch.seqs_host["grid_origin"] += far
    s.batch.upload_seqs()
    mods = dict(slopes=torch.tensor([2.0 ** -(3 + i) for i in range(h * s.G)], device=DEV))
    s.qpos += far
    s.run(**mods)
    s.check(**mods, prompt_from=far)


@pytest.mark.parametrize("h,D,G", [(2, 64, 0), (1, 128, 0), (1, 128, 5), (2, 64, 2)])
@pytest.mark.parametrize("cap,slope,far", [(4.0, False, 0), (0.0, True, 0), (15.0, True, 0), (0.0, True, 1_000_000_000)])
def test_many_rows_capped_and_lowered_with_distance(h, D, G, cap, slope, far):
    """Groups of more than 32 rows, which meet their prompt 128 at a time."""
    s = Shared([40, 3], [150, 333], [(7 * i) % 65 for i in range(43)], h, D, "bf16", G, q_scale=4.0)
    s.batch.pos += far
    s.pb.pos += far
    s.batch.seqs_host["grid_origin"] += far
    s.batch.upload_seqs()
    s.qpos += far
    mods = dict(softcap=cap, slopes=torch.tensor([2.0 ** -(3 + i) for i in range(h * s.G)], device=DEV) if slope else None)
    s.run(**mods)
    s.check(**mods, prompt_from=far)


def test_scores_of_minus_infinity_gain_nothing():
    s = Shared([2], [0], [5, 40], 2, 64, append=False)
    for t in (s.K, s.q.view(2, 2, 1, 64)):
        t[..., 0] = 1.0
    s.K[..., 0] = -float("inf")
    s.run()
    assert not s.batch.out.any() and (s.batch.lse == -float("inf")).all() and np.array_equal(f64(s.batch.score), s.score0)


def test_without_append_and_without_mass():
    s = Shared([2, 1], [60, 5], [40, 130, 3], 2, 64, append=False)
    s.run(B.FLAG_NO_ACCUMULATE)
    s.check(mass=False)
    assert s.batch.read_seqs()["step"].tolist() == [3 * s.batch.params.cap] * 3


def test_records_that_are_not_attended():
    s = Shared([2, 2, 2], [60, 30, 10], [40, 50, 60, 3, 2, 1], 2, 64)
    r = s.batch.read_seqs()
    r["step"][0], r["status"][3] = -1, B.SEQ_CACHE_FULL
    s.batch.upload_seqs()
    s.pb.seqs_host["n_res"][2] = s.pb.params.cap + 1
    s.pb.upload_seqs()
    s.score0[[0, 3, 4, 5]] = f64(s.batch.score)[[0, 3, 4, 5]]
    s.run(B.FLAG_ADVANCE)
    s.check(dead=(0, 3, 4, 5))
    r = s.batch.read_seqs()
    cap = s.batch.params.cap
    assert r["status"].tolist() == [0, 0, 0, B.SEQ_CACHE_FULL, B.SEQ_BAD_STATE, B.SEQ_BAD_STATE]
    assert r["step"].tolist() == [-1, 3 * cap + 1, 3 * cap + 1, 3 * cap, 3 * cap, 3 * cap]


def test_as_adsa_attend_over_caches_that_hold_the_prompt():
    """Whole steps of both kinds from the same images: the prompt kept once, or in every sequence's cache."""
    n, h, D, P, W, H = 6, 4, 64, 45, 8, 8
    common = dict(n_heads=h, head_dim=D, grid_h=H, grid_w=W, win_rows_back=1, win_col_radius=2, dtype=B.F32, score_mode=B.SCORE_ATTN_MASS)
    rest = 12 + 2 * W
    whole = LayerBatch(B.make_params(n_seq=n, cap=P + rest, **common), DEV)
    own = LayerBatch(B.make_params(n_seq=n, cap=rest, **common), DEV)
    prompt = LayerBatch(B.make_params(n_seq=1, cap=P, **common), DEV)
    gen = torch.Generator().manual_seed(8)
    pk, pv = randn(gen, P, h, D).to(DEV), randn(gen, P, h, D).to(DEV)
    one = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    for batch, copies in ((whole, n), (prompt, 1)):
        batch.seqs_host["grid_origin"] = batch.seqs_host["n_keep_prefix"] = P
        batch.seqs_host["budget"] = 12
        batch.upload_seqs()
        batch.append(B.make_tokens(one(*range(0, copies * P + 1, P)), one(*[0] * copies), copies * P, P), None, None, pk.repeat(copies, 1, 1), pv.repeat(copies, 1, 1), None,
                     flags=B.FLAG_ADVANCE)
    s = own.seqs_host
    s["grid_origin"], s["n_keep_prefix"], s["budget"], s["step"] = P, P, 12, 1
    own.upload_seqs()
    shared = B.make_shared(prompt.params, prompt.seqs, one(0, n), max_members=n)
    for step in range(1, 3 * W + 2):
        q, k, v = (randn(gen, n, h, D).to(DEV) for _ in range(3))
        whole.step(q, k, v)
        own.select(B.FLAG_PLAN_APPEND)
        own.attend_shared(shared, q, k, v, flags=B.FLAG_APPEND)
        own.compact(B.FLAG_ADVANCE)
        a, b = whole.read_seqs(), own.read_seqs()
        assert not a["status"].any() and not b["status"].any() and (a["step"] == b["step"]).all() and (a["n_res"] - P == b["n_res"]).all()
        m = int(b["n_res"][0])
        assert torch.equal(whole.pos[:, P:P + m], own.pos[:, :m]) and torch.equal(whole.K[:, :, P:P + m], own.K[:, :, :m])
        assert (whole.out - own.out).abs().max() < 2e-6 and (whole.lse - own.lse).abs().max() < 1e-5
        assert (whole.score[..., P:P + m] - own.score[..., :m]).abs().max() < 1e-5


def test_a_captured_step_replays():
    """Rotation, selection, shared attention and eviction as one graph, replayed with eager work between the replays."""
    n, h, D, P = 4, 2, 64, 70
    common = dict(n_heads=h, head_dim=D, grid_h=6, grid_w=5, win_rows_back=1, win_col_radius=1, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS)
    gen = torch.Generator().manual_seed(4)
    prompt = LayerBatch(B.make_params(n_seq=2, cap=P, **common), DEV)
    prompt.K.copy_(randn(gen, *prompt.K.shape))
    prompt.V.copy_(randn(gen, *prompt.V.shape))
    prompt.seqs_host["n_res"] = [P, P - 9]
    prompt.upload_seqs()
    freq = torch.rand(2, D // 2, generator=gen, dtype=torch.float64).to(DEV)
    rope = B.make_rope(freq, pairing="neighbours", text=(1, 1), origin=(1, 1), row=(1, 0), col=(0, 1))
    members = torch.tensor([0, 3, 4], dtype=torch.int32, device=DEV)
    shared = B.make_shared(prompt.params, prompt.seqs, members, max_members=3)
    x = [[randn(gen, n, h, D, dtype=torch.bfloat16).to(DEV) for _ in range(3)] for _ in range(12)]

    def make():
        batch = LayerBatch(B.make_params(n_seq=n, cap=20, **common), DEV)
        s = batch.seqs_host
        s["grid_origin"], s["n_keep_prefix"], s["budget"], s["step"] = P, P, 6, 1
        batch.upload_seqs()
        return batch, [t.clone() for t in x[0]], torch.empty(n, h, D, dtype=torch.bfloat16, device=DEV), torch.empty(n, h, D, dtype=torch.bfloat16, device=DEV)

    def step(batch, ins, qo, ko):
        batch.rotate(rope, ins[0], ins[1], qo, ko)
        batch.select(B.FLAG_PLAN_APPEND)
        batch.attend_shared(shared, qo, ko, ins[2], flags=B.FLAG_APPEND)
        batch.compact(B.FLAG_ADVANCE)

    eager, captured = make(), make()
    step(*eager)                                             # (allocates the workspaces; so does the captured side's first step)
    step(*captured)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured)
    for t in range(1, 12):
        for side in (eager, captured):
            for dst, src in zip(side[1], x[t]):
                dst.copy_(src)
        step(*eager)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("out", "lse", "score", "pos", "K", "V"):
            assert torch.equal(getattr(eager[0], name), getattr(captured[0], name)), (t, name)
        a, b = eager[0].read_seqs(), captured[0].read_seqs()
        assert (a["step"] == t + 2).all() and not a["status"].any()
        for f in ("step", "n_res", "compacted", "status"):
            assert (a[f] == b[f]).all()

"""Rotary positions for query tokens and for new tokens on their way into the caches, against 64-bit complex arithmetic on the host."""
import numpy as np
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch

from prompt_common import close, f64, half_step, randn, turned

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
RULES = {"grid": dict(text=(0, 0), origin=(0, 0), row=(1, 0), col=(0, 1)), "thw": dict(text=(1, 1, 1), origin=(1, 1, 1), row=(0, 1, 0), col=(0, 0, 1)),
         "line": dict(text=(3,), origin=(3,), row=(21,), col=(3,))}


def make_rope(D, rule, pairing, gen):
    n = len(RULES[rule]["text"])
    freq = torch.exp(-9.0 * torch.rand(n, D // 2, generator=gen, dtype=torch.float64))
    freq[:, -1] = 0.0                                        # a pair that nothing turns
    dev = freq.to(DEV)
    return freq.numpy(), B.make_rope(dev, pairing=pairing, **RULES[rule])


def coordinates(rule, pos, P, W):
    r = RULES[rule]
    pos, P = np.asarray(pos, np.int64), np.asarray(P, np.int64)
    row, col = (pos - P) // W, (pos - P) % W
    return np.stack([np.where(pos < P, t * pos, o * P + a * row + b * col) for t, o, a, b in zip(r["text"], r["origin"], r["row"], r["col"])], 1)


def make_batch(n, h, D, dtype, cap, G=0, layout="head_major", score_mode=B.SCORE_ATTN_MASS, **kw):
    p = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=9, grid_w=7, win_rows_back=1, win_col_radius=2, dtype=B.F32 if dtype == "f32" else B.BF16,
                      score_mode=score_mode, cap=cap, layout=layout, q_per_kv=G, **kw)
    return LayerBatch(p, DEV)


def rounded(x, dt):
    """Tolerance of the one rounding to the storage type."""
    return half_step(dt) * np.abs(x)


@pytest.mark.parametrize("n,h,G,D,dtype,rule,pairing,in_f32,packed", [
    (1, 1, 0, 64, "bf16", "grid", "neighbours", False, False), (3, 5, 3, 128, "bf16", "thw", "halves", True, True), (70, 4, 0, 64, "f32", "line", "halves", False, True),
    (600, 2, 2, 64, "bf16", "thw", "neighbours", False, False), (1100, 3, 0, 128, "f32", "grid", "neighbours", False, False), (2, 20, 0, 64, "bf16", "grid", "halves", True, False)])
@pytest.mark.parametrize("far", [0, 3_000_000])
def test_query_tokens(n, h, G, D, dtype, rule, pairing, in_f32, packed, far):
    gen = torch.Generator().manual_seed(n + D + far)
    batch = make_batch(n, h, D, dtype, 1, G)
    hq, dt = h * max(G, 1), batch.tdtype
    freq, rope = make_rope(D, rule, pairing, gen)
    it = torch.float32 if in_f32 else dt
    qkv = randn(gen, n, (hq + 2 * h) * D).to(it).to(DEV)
    q, k = (qkv[:, :hq * D], qkv[:, hq * D:(hq + h) * D]) if packed else (qkv[:, :hq * D].contiguous(), qkv[:, hq * D:(hq + h) * D].contiguous())
    s = batch.seqs_host
    P = 10 + far + np.arange(n) % 5
    s["grid_origin"], s["step"] = P, np.arange(n) % 64
    off = np.zeros(n, bool)
    if n > 2:
        s["step"][1], s["status"][2] = -1, B.SEQ_BAD_STATE
        off[1:3] = True
    batch.upload_seqs()
    q_out, k_out = torch.full((n, hq, D), 7.0, dtype=dt, device=DEV), torch.full((n, h, D), 7.0, dtype=dt, device=DEV)
    stride = qkv.shape[1] if packed else 0
    batch.rotate(rope, q, k, q_out, k_out, flags=B.FLAG_NEW_F32 if in_f32 else 0, q_stride=stride, k_stride=stride)
    step = s["step"].astype(np.int64)
    angle = coordinates(rule, P + step - 1, P, 7) @ freq
    for got, x, heads in ((q_out, q, hq), (k_out, k, h)):
        want, tol = turned(f64(x).reshape(n, heads, D), angle, pairing)
        want[off] = 0.0
        close(got, want, tol + rounded(want, dt) if dt != torch.float32 else tol)


def test_given_coordinates_in_place_and_on_a_stream_of_its_own():
    gen = torch.Generator().manual_seed(5)
    n, h, D = 9, 3, 64
    batch = make_batch(n, h, D, "f32", 1)
    batch.seqs_host["step"] = 1
    batch.upload_seqs()
    freq, rope = make_rope(D, "thw", "halves", gen)
    c = torch.randint(-70000, 70000, (n, 3), generator=gen, dtype=torch.int32)
    x = randn(gen, n, h, D)
    q, k = x.to(DEV), x.to(DEV)
    coords = c.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    batch.rotate(rope, q, k, q, k, coords=coords, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    want, tol = turned(f64(x), c.numpy().astype(np.float64) @ freq, "halves")
    close(q, want, tol)
    assert torch.equal(q, k)


@pytest.mark.parametrize("h,G,D,dtype,layout,rule,pairing,in_f32,packed", [
    (3, 0, 64, "bf16", "head_major", "thw", "halves", False, True), (2, 4, 128, "bf16", "slot_major", "grid", "neighbours", True, False),
    (5, 0, 128, "f32", "head_major", "line", "neighbours", False, False), (1, 2, 64, "bf16", "slot_major", "thw", "halves", True, True)])
@pytest.mark.parametrize("n,longest", [(7, 40), (40, 300)])
def test_tokens_enter_the_caches(h, G, D, dtype, layout, rule, pairing, in_f32, packed, n, longest):
    gen = torch.Generator().manual_seed(h + D + longest)
    cap = longest + 21
    batch = make_batch(n, h, D, dtype, cap, G, layout)
    hq, dt = h * max(G, 1), batch.tdtype
    rng = np.random.default_rng(longest)
    lens = rng.integers(0, longest + 1, n)
    lens[:5] = [longest, 0, 1, 2, 17]
    past = rng.integers(0, 21, n)
    past[0] = 0
    P = 11 + longest // 2
    first = np.where(past > 0, rng.integers(0, 5, n), 0)     # position of the first resident token
    lens = np.minimum(lens, P + 63 - past - first)           # a position behind the grid's end is refused
    T = int(lens.sum())
    for t in (batch.K, batch.V):
        t.copy_(randn(gen, *t.shape))
    batch.score.fill_(3.0)
    K0, V0 = f64(batch.K), f64(batch.V)
    for b in range(n):
        batch.pos[b, :past[b]] = torch.arange(first[b], first[b] + past[b], dtype=torch.int32)
    s = batch.seqs_host
    s["n_res"], s["grid_origin"], s["n_keep_prefix"], s["compacted"], s["pending_slot"] = past, P, P, 1, 4
    batch.upload_seqs()
    freq, rope = make_rope(D, rule, pairing, gen)
    it = torch.float32 if in_f32 else dt
    qkv = randn(gen, T, (hq + 2 * h) * D).to(it).to(DEV)
    parts = [qkv[:, :hq * D], qkv[:, hq * D:(hq + h) * D], qkv[:, (hq + h) * D:]]
    if not packed:
        parts = [x.contiguous() for x in parts]
    stride = qkv.shape[1] if packed else 0
    begin = np.concatenate([[0], np.cumsum(lens)])
    tokens = B.make_tokens(torch.tensor(begin, dtype=torch.int32, device=DEV), torch.tensor(past, dtype=torch.int32, device=DEV), T, int(lens.max()),
                           q_stride=stride, k_stride=stride, v_stride=stride)
    q_out = torch.full((T, hq, D), 7.0, dtype=dt, device=DEV)
    flags = B.FLAG_NEW_F32 if in_f32 else 0
    for again in range(2):                                   # the same call may be made again
        batch.append(tokens, rope, *parts, q_out, flags=flags | (B.FLAG_ADVANCE if again else 0))
    pos = np.concatenate([first[b] + past[b] + np.arange(lens[b]) for b in range(n)])
    angle = coordinates(rule, pos, np.full(T, P), 7) @ freq
    q, qt = turned(f64(parts[0]).reshape(T, hq, D), angle, pairing)
    k, kt = turned(f64(parts[1]).reshape(T, h, D), angle, pairing)
    v = f64(parts[2]).reshape(T, h, D)
    one = dt != torch.float32
    close(q_out, q, qt + (rounded(q, dt) if one else 0))
    rows = (lambda x: x) if layout == "head_major" else (lambda x: x.transpose(0, 2, 1, 3))
    K, V, tolK, tolV = rows(K0), rows(V0), np.zeros_like(rows(K0)), np.zeros_like(rows(K0))
    want_pos, want_score = np.zeros((n, cap), np.int64), np.full((n, batch.rows, cap), 3.0)
    for b in range(n):
        a, e, x, y = past[b], past[b] + lens[b], begin[b], begin[b + 1]
        K[b, :, a:e], tolK[b, :, a:e] = k[x:y].transpose(1, 0, 2), (kt + (rounded(k, dt) if one else 0))[x:y].transpose(1, 0, 2)
        V[b, :, a:e], tolV[b, :, a:e] = v[x:y].transpose(1, 0, 2), (rounded(v, dt) if in_f32 else 0 * v)[x:y].transpose(1, 0, 2)
        want_pos[b, :e] = first[b] + np.arange(e)
        want_score[b, :, a:e] = 0.0
    close(rows(f64(batch.K)), K, tolK)
    close(rows(f64(batch.V)), V, tolV)
    assert np.array_equal(batch.pos.cpu().numpy(), want_pos) and np.array_equal(batch.score.cpu().numpy(), want_score)
    r = batch.read_seqs()
    some = lens > 0
    last = first + past + lens - 1
    assert np.array_equal(r["n_res"], past + lens) and not r["status"].any()
    assert np.array_equal(r["step"], np.where(some, np.maximum(0, last + 1 - P) + 1, -1))
    assert np.array_equal(r["compacted"], np.where(some, 0, 1)) and np.array_equal(r["pending_slot"], np.where(some, -1, 4))


def test_records_that_do_not_fit_are_marked_and_left_alone():
    h, D, cap, n = 2, 64, 20, 8
    batch = make_batch(n, h, D, "bf16", cap)
    s = batch.seqs_host
    s["n_res"] = [0, 5, 5, 12, 3, 3, 25, 4]
    s["grid_origin"] = [30, 30, 30, 30, 30, 0, 30, 30]
    s["hole"][4] = 2
    s["status"][7] = B.SEQ_SEL_OVERFLOW
    batch.pos[:] = torch.arange(cap, dtype=torch.int32)
    batch.pos[5, 2] = 62                                     # the next position is behind the 9 x 7 grid
    batch.upload_seqs()
    before = batch.seqs.clone()
    lens = [10, 10, 10, 9, 10, 10, 10, 10]
    slot0 = [0, 5, 6, 12, 3, 3, 2, 4]                        # (2: beyond what is resident; 3: 21 slots)
    T = sum(lens)
    gen = torch.Generator().manual_seed(1)
    q, k, v = (randn(gen, T, h, D, dtype=torch.bfloat16).to(DEV) for _ in range(3))
    q_out = torch.full_like(q, 7.0)
    tokens = B.make_tokens(torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device=DEV), torch.tensor(slot0, dtype=torch.int32, device=DEV), T, 10)
    batch.append(tokens, None, q, k, v, q_out)
    r = batch.read_seqs()
    bad, full = B.SEQ_BAD_STATE, B.SEQ_CACHE_FULL
    assert r["status"].tolist() == [0, 0, bad, full, bad, bad, bad, B.SEQ_SEL_OVERFLOW]
    assert r["n_res"].tolist() == [10, 15, 5, 12, 3, 3, 25, 4]
    at = 0
    for b, m in enumerate(lens):
        fits = b < 2
        assert torch.equal(q_out[at:at + m], q[at:at + m] if fits else torch.zeros_like(q[at:at + m]))
        x = slot0[b]
        assert torch.equal(batch.K[b, :, x:x + m].transpose(0, 1), k[at:at + m]) if fits else not batch.K[b].any()
        if not fits:
            old = before.view(n, 96)[b].clone()
            old[60:64] = batch.seqs.view(n, 96)[b][60:64]
            assert torch.equal(batch.seqs.view(n, 96)[b], old)
        at += m
    # tokens taken back: a smaller slot0; no q wanted; positions given
    lens, T = [3, 0, 0, 0, 0, 0, 0, 0], 3
    tokens = B.make_tokens(torch.tensor([0] + [3] * 8, dtype=torch.int32, device=DEV), torch.tensor([4] * 8, dtype=torch.int32, device=DEV), 3, 3,
                           pos0=torch.tensor([33] * 8, dtype=torch.int32, device=DEV))
    batch.append(tokens, None, None, k, v, None)
    r = batch.read_seqs()
    assert r["n_res"][0] == 7 and r["step"][0] == 6 and r["n_res"][1] == 15
    assert batch.pos[0, :8].tolist() == [0, 1, 2, 3, 33, 34, 35, 7] and torch.equal(batch.V[0, :, 4:7].transpose(0, 1), v[:3])


def test_the_running_v_cosine_state_starts_over():
    batch = make_batch(2, 2, 64, "bf16", 30, score_mode=B.SCORE_VCOS_FUSED, evict_policy=B.EVICT_REUSE_SLOT, win_recent_m=5)
    batch.vcos_u.fill_(2.0)
    batch.seqs_host["grid_origin"] = 30
    batch.upload_seqs()
    k = torch.ones(4, 2, 64, dtype=torch.bfloat16, device=DEV)
    tokens = B.make_tokens(torch.tensor([0, 4, 4], dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV), 4, 4)
    batch.append(tokens, None, None, k, k, None)
    u = batch.vcos_u.cpu()
    assert not u[0, 128:].any() and (u[0, :128] == 2).all() and (u[1] == 2).all()
    assert not batch.score[0, :, :4].any()

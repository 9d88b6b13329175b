"""Operators around a shared prompt, as cases that can be timed and compared: what a decode step of this library needs before and beside
its sparse attention.

  rotate   rotary positions with up to three axes for the query token of every sequence: q and k as the projections leave them, in
           storage type or fp32, packed or not, to rotated rows that the decode attention takes
  append   the same rotation for prompts, on their way into the caches: ragged new tokens behind what is resident, K and V rows, positions
           and counters of every sequence
  prefill  attention of those tokens over the caches: causal, prefix (the prompt sees itself whole) or document masks, scores capped by a
           tanh or lowered with distance, and the attention mass that the decode steps rank by
  shared   decode attention for sequences that share a prompt: each over its own list of resident tokens and over its group's prompt,
           whose rows are kept and read once per group, with the same caps and distances

With `own` false everything is computed in its plain form, by elementary torch operations in 32 bits (angles in 64).  Inputs come from the
seed alone; how long sequences are follows from the case.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"


# --------------------------------------------------------------------------- cases
def _case(name=None, **kw):
    c = dict(kind="rotate", n_seq=1, heads=16, head_dim=64, q_per_kv=1, dtype="bf16", layout="head_major", grid_h=32, grid_w=32)
    kind = kw.get("kind", "rotate")
    if kind in ("rotate", "append"):
        c.update(axes="grid", in_f32=False, packed=False, far=0)
    if kind == "rotate":
        c.update(prefix=120)
    if kind in ("append", "prefill"):
        c.update(new_lo=1, new_hi=1, past=0, prefix=120)
    if kind == "prefill":
        c.update(mask="causal", cap=0.0, slopes=False, doc_len=0, doc_pad=0, mass=False, q_scale=1.0)
    if kind == "shared":
        c.update(groups=1, prefix_lo=120, prefix_hi=120, own_lo=1, own_hi=1, resident=1, cap=0.0, slopes=False, mass=True, in_f32=False, q_scale=1.0)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: ONE image under classifier-free guidance, one layer's q and k of the 36-layer model, rows and columns as axes
        _case("rotate_one_image", kind="rotate", n_seq=2, heads=20, grid_h=24, grid_w=24),
        # serving: 64 sequences of the grouped-query model, fp32 projections q|k|v in one tensor, time, height and width as axes
        _case("rotate_serving", kind="rotate", n_seq=64, heads=8, head_dim=128, q_per_kv=8, axes="thw", in_f32=True, packed=True),
        # text conditions of 64 prompts of 16 to 120 tokens enter the caches of one layer
        _case("append_prompts", kind="append", n_seq=64, heads=24, new_lo=16, new_hi=120, axes="raster"),
        # an image to be continued: half of a 64x64 grid behind 256 prompt tokens, for 4 sequences, from packed projections
        _case("append_image", kind="append", n_seq=4, heads=32, head_dim=128, new_lo=2304, new_hi=2304, grid_h=64, grid_w=64, prefix=256, axes="thw", packed=True),
        # text conditions of a batch: 120 tokens that all see each other
        _case("prefill_text", kind="prefill", n_seq=32, heads=24, new_lo=120, new_hi=120, mask="prefix"),
        # ragged prompts of the grouped-query model, capped scores, in the order of arrival
        _case("prefill_ragged_capped", kind="prefill", n_seq=16, heads=8, head_dim=128, q_per_kv=8, new_lo=16, new_hi=1144, cap=50.0, q_scale=2.8),
        # the largest: 4 sequences of 256 prompt tokens and a whole 64x64 image, causal, with the mass that decode steps rank by
        _case("prefill_image", kind="prefill", n_seq=4, heads=32, head_dim=128, new_lo=4352, new_hi=4352, grid_h=64, grid_w=64, prefix=256, mass=True),
        # a few more tokens behind a long context, scores lowered with distance, [slot][head][D] cache, odd sizes
        _case("prefill_chunk", kind="prefill", n_seq=3, heads=20, new_lo=2, new_hi=7, past=2011, slopes=True, layout="slot_major", grid_h=64, grid_w=64, prefix=37),
        # the fp32 toy model: several short prompts packed into one sequence, padded to 77 tokens each
        _case("prefill_packed_fp32", kind="prefill", n_seq=2, heads=16, dtype="f32", new_lo=385, new_hi=385, mask="prefix", prefix=385, doc_len=77, doc_pad=9),
        # the headline configuration deep in the image: 16 images of one prompt and their 16 unconditional partners, one layer
        _case("shared_guided_batch", kind="shared", n_seq=32, heads=24, groups=2, own_lo=553, own_hi=553, resident=575, q_scale=2.8),
        # long prompts (a reference image and text): 4 prompts with 16 images each, grouped queries
        _case("shared_long_prompts", kind="shared", n_seq=64, heads=8, head_dim=128, q_per_kv=8, groups=4, prefix_lo=2100, prefix_hi=4352, own_lo=200, own_hi=577, resident=640,
              q_scale=2.8),
        # three variations of one image, fp32, capped scores that fall with distance
        _case("shared_few_fp32", kind="shared", n_seq=3, heads=16, dtype="f32", groups=1, prefix_lo=301, prefix_hi=301, own_lo=5, own_hi=97, resident=112, cap=30.0, slopes=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_SHAPES = [(16, 64, 1), (20, 64, 1), (24, 64, 1), (32, 128, 1), (8, 128, 8), (7, 64, 1), (5, 128, 3), (9, 64, 2)]


def draw(rng):
    kind = rng.choice(["rotate", "append", "prefill", "prefill", "shared", "shared"])
    heads, D, G = rng.choice(_SHAPES)
    c = dict(kind=kind, heads=heads, head_dim=D, q_per_kv=G, dtype="bf16" if G > 1 else rng.choice(["bf16", "bf16", "bf16", "f32"]),
             layout=rng.choice(["head_major", "head_major", "slot_major"]), prefix=rng.randint(8, 256), grid_h=64, grid_w=64)
    if kind in ("rotate", "append"):
        c.update(axes=rng.choice(["grid", "thw", "raster"]), in_f32=c["dtype"] == "bf16" and rng.random() < 0.3,
                 packed=heads != 16 and rng.random() < 0.5, far=rng.choice([0, 0, 1000000]))
    if kind == "rotate":
        c["n_seq"] = _log_int(rng, 1, 512)
    if kind == "append":
        hi = _log_int(rng, 4, 4352)
        c.update(n_seq=max(1, min(64, int(rng.uniform(0.2, 1.0) * 9000 / hi))), new_hi=hi, new_lo=rng.randint(1, hi), past=rng.choice([0, 0, rng.randint(1, 900)]))
        if c["past"]:
            c["prefix"] = min(c["prefix"], c["past"])
    if kind == "prefill":
        hi = _log_int(rng, 1, 4352 if c["dtype"] == "bf16" else 2048)
        past = rng.choice([0, 0, _log_int(rng, 8, 2048)])
        pairs = heads * G * D * (hi * float(past) + hi * hi / 2)         # of one sequence: the largest case has 1.6e11 of four
        n = max(1, min(_log_int(rng, 1, 64), int(1.2e11 / pairs)))
        if c["dtype"] == "f32":
            n = max(1, min(n, int(2e10 / pairs)))
        c.update(n_seq=n, new_hi=hi, new_lo=rng.randint(1, hi), past=past, mask=rng.choice(["causal", "causal", "prefix"]),
                 cap=rng.choice([0.0, 0.0, 30.0, 50.0]), slopes=rng.random() < 0.25, mass=rng.random() < 0.3, q_scale=rng.choice([1.0, 2.8]))
        if past:
            c["prefix"] = min(c["prefix"], past)
        if rng.random() < 0.25:
            c["doc_len"] = rng.randint(9, 300)
            c["doc_pad"] = rng.randint(0, c["doc_len"] // 4)
    if kind == "shared":
        groups = _log_int(rng, 1, 8)
        n = groups * _log_int(rng, 1, 96 // groups)
        own_hi = _log_int(rng, 1, 1024)
        pre_hi = _log_int(rng, 1, 4352)
        c.update(groups=groups, n_seq=n, own_hi=own_hi, own_lo=rng.randint(0, own_hi), resident=own_hi + rng.randint(0, 200), prefix_hi=pre_hi,
                 prefix_lo=rng.randint(0, pre_hi), cap=rng.choice([0.0, 0.0, 30.0]), slopes=rng.random() < 0.25, mass=rng.random() < 0.7,
                 in_f32=c["dtype"] == "bf16" and rng.random() < 0.25, q_scale=rng.choice([1.0, 2.8]))
    return _case(**c)


# --------------------------------------------------------------------------- sizes, from the case alone
def _spread(lo, hi, n):
    """n lengths between lo and hi, the longest among them, in no order."""
    if n == 1:
        return [hi]
    return [lo + (hi - lo) * ((i * 7919 + n - 1) % n) // (n - 1) for i in range(n)]


def _eb(c):
    return 4 if c["dtype"] == "f32" else 2


def _storage(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _new(c):
    return _spread(c["new_lo"], c["new_hi"], c["n_seq"])


def _cap_of(c):
    return c["resident"] if c["kind"] == "shared" else c["past"] + c["new_hi"]


def _members(c):
    """First sequence of every group, and the end."""
    return [c["n_seq"] * g // c["groups"] for g in range(c["groups"] + 1)]


def _doc_of(c, n):
    """Document of every slot; -1: padding."""
    slot = np.arange(n)
    return np.where(slot % c["doc_len"] >= c["doc_len"] - c["doc_pad"], -1, slot // c["doc_len"]).astype(np.int32)


def _pairs(c):
    """(query, key) pairs that are attended, over all sequences, per query head."""
    total = 0
    for n in _new(c):
        q = np.arange(c["past"], c["past"] + n)
        end = q + 1
        if c["mask"] == "prefix":
            end = np.where(q < c["prefix"], np.minimum(c["prefix"], c["past"] + n), end)
        if c["doc_len"]:
            doc = _doc_of(c, c["past"] + n)
            alive = np.concatenate([[0], np.cumsum(doc >= 0)])
            begin = q // c["doc_len"] * c["doc_len"]
            end = np.minimum(end, begin + c["doc_len"])
            total += int(np.where(doc[q] >= 0, alive[end] - alive[begin], 0).sum())
        else:
            total += int(end.sum())
    return total


def work(case):
    c = case
    eb, D, h = _eb(c), c["head_dim"], c["heads"]
    hq = h * c["q_per_kv"]
    if c["kind"] in ("rotate", "append"):
        rows = c["n_seq"] if c["kind"] == "rotate" else sum(_new(c))
        ib = 4 if c["in_f32"] else eb
        moved = rows * (hq + h) * D * (ib + eb) + (rows * h * D * (ib + eb) + rows * 4 if c["kind"] == "append" else 0)
        return {"bytes": float(moved), "flops": 3.0 * rows * (hq + h) * D}
    if c["kind"] == "prefill":
        T, keys = sum(_new(c)), sum(c["past"] + n for n in _new(c))
        return {"bytes": float(2 * T * hq * D * eb + 4 * T * hq + 2 * keys * h * D * eb + (4 * keys * h if c["mass"] else 0)), "flops": 4.0 * _pairs(c) * hq * D}
    pre, lists = _spread(c["prefix_lo"], c["prefix_hi"], c["groups"]), _spread(c["own_lo"], c["own_hi"], c["n_seq"])
    m = _members(c)
    attended = sum(lists) + sum(pre[g] * (m[g + 1] - m[g]) for g in range(c["groups"]))
    rows = 2.0 * h * D * eb * (sum(pre) + sum(lists))
    io = c["n_seq"] * (2 * hq * D * eb + 4 * hq + 2 * h * D * (4 if c["in_f32"] else eb)) + 4 * sum(lists) * (1 + (2 * h if c["mass"] else 0))
    return {"bytes": float(rows + io), "flops": 4.0 * attended * hq * D}


# --------------------------------------------------------------------------- inputs
_RULES = {   # coordinate on each axis: of text at position p, text * p; of the image token at (row, column), origin * P + row * r + col * c
    "grid": dict(text=(0, 0), origin=(0, 0), row=(1, 0), col=(0, 1)),
    "thw": dict(text=(1, 1, 1), origin=(1, 1, 1), row=(0, 1, 0), col=(0, 0, 1)),
    "raster": None,
}


def _rule(c):
    return _RULES[c["axes"]] or dict(text=(1,), origin=(1,), row=(c["grid_w"],), col=(1,))


def _pairing(c):
    return "neighbours" if c["axes"] == "grid" else "halves"


def _frequencies(c):
    """[axes][D / 2], radians per unit: what each axis turns each pair of elements by."""
    n = c["head_dim"] // 2
    if c["axes"] == "grid":                                # half of the pairs turn with the row, half with the column
        f = torch.zeros(2, n, dtype=torch.float64)
        one = 10000.0 ** (-torch.arange(n // 2, dtype=torch.float64) / (n // 2))
        f[0, :n // 2], f[1, n // 2:] = one, one
        return f
    base = 10000.0 ** (-torch.arange(n, dtype=torch.float64) / n)
    if c["axes"] == "raster":
        return base[None].clone()
    f = torch.zeros(3, n, dtype=torch.float64)             # a quarter of the pairs for time, the rest for height and width
    a, b = n // 4, n // 4 + (n - n // 4) // 2
    f[0, :a], f[1, a:b], f[2, b:] = base[:a], base[a:b], base[b:]
    return f


def _positions(c):
    """Absolute position and (for rotate) step of every new token, int64 on the host."""
    if c["kind"] == "rotate":
        total = c["grid_h"] * c["grid_w"]
        step = np.array([1 + (i * 7919) % total for i in range(c["n_seq"])])
        return c["prefix"] + c["far"] + step - 1, step
    return np.concatenate([np.arange(c["past"], c["past"] + n) for n in _new(c)]) + (c["far"] if not c["past"] else 0), None


def _coordinates(c, p):
    """int64 [tokens][axes] of positions p."""
    r, P = _rule(c), c["prefix"] + c["far"]
    i = p - P
    row, col = i // c["grid_w"], i % c["grid_w"]
    axes = [np.where(i < 0, t * p, o * P + a * row + b * col) for t, o, a, b in zip(r["text"], r["origin"], r["row"], r["col"])]
    return np.stack(axes, 1)


def _inputs(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 2 + 1)
    dt, h, D, n = _storage(c), c["heads"], c["head_dim"], c["n_seq"]
    hq, cap = h * c["q_per_kv"], _cap_of(c) if c["kind"] != "rotate" else 0

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)

    x = {}
    if c["kind"] in ("rotate", "append"):
        T = n if c["kind"] == "rotate" else sum(_new(c))
        it = torch.float32 if c["in_f32"] else dt
        if c["packed"]:                                    # one projection's output: q, k and v of a token side by side
            x["qkv"] = randn(T, (hq + 2 * h) * D).to(it)
            x["q"], x["k"], x["v"] = x["qkv"][:, :hq * D], x["qkv"][:, hq * D:(hq + h) * D], x["qkv"][:, (hq + h) * D:]
        else:
            x["q"], x["k"], x["v"] = randn(T, hq * D).to(it), randn(T, h * D).to(it), randn(T, h * D).to(it)
        p, _ = _positions(c)
        x["freq"] = _frequencies(c).to(DEV)
        x["coords"] = torch.from_numpy(_coordinates(c, p)).to(DEV)
        if c["kind"] == "append":
            x["K"], x["V"] = randn(n, h, cap, D).to(dt), randn(n, h, cap, D).to(dt)
        return x
    if c["slopes"]:                                        # a geometric sequence over the heads
        x["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device=DEV, dtype=torch.float32) / hq)
    x["K"], x["V"] = randn(n, h, cap, D).to(dt), randn(n, h, cap, D).to(dt)
    if c["kind"] == "prefill":
        x["q"] = (randn(sum(_new(c)), hq, D) * c["q_scale"]).to(dt)
        if c["doc_len"]:
            x["doc"] = torch.from_numpy(_doc_of(c, cap)).to(DEV).repeat(n, 1)
        return x
    # shared: some of the resident tokens are in a sequence's list, the last one is the query token, whose row is still to be stored
    rng = np.random.default_rng([seed & 0x7FFFFFFF, 5])
    lists = _spread(c["own_lo"], c["own_hi"], n)
    idx = np.zeros((n, max(1, c["own_hi"])), np.int32)
    for b, k in enumerate(lists):
        if k:
            idx[b, :k] = np.concatenate([np.sort(rng.permutation(cap - 1)[:k - 1]), [cap - 1]])
    x["idx"], x["cnt"] = torch.from_numpy(idx).to(DEV), torch.tensor(lists, dtype=torch.int32, device=DEV)
    x["q"] = (randn(n, hq, D) * c["q_scale"]).to(dt)
    it = torch.float32 if c["in_f32"] else dt
    x["k_new"], x["v_new"] = randn(n, h, D).to(it), randn(n, h, D).to(it)
    x["PK"], x["PV"] = randn(c["groups"], h, c["prefix_hi"], D).to(dt), randn(c["groups"], h, c["prefix_hi"], D).to(dt)
    x["score"] = torch.rand(n, h, cap, generator=gen, device=DEV)
    return x


def prepare(case, seed):
    c = case
    x = _inputs(c, seed)
    st = {"case": dict(c), "x": x}
    if own:
        _prepare_own(st)
        return st
    n = c["n_seq"]
    if c["kind"] == "append":
        st["K"], st["V"] = x["K"].clone(), x["V"].clone()
        st["pos"] = torch.zeros(n, _cap_of(c), dtype=torch.int32, device=DEV)
        st["pos"][:, :c["past"]] = torch.arange(c["past"], device=DEV, dtype=torch.int32)
        seq = np.repeat(np.arange(n), _new(c))
        slot = np.concatenate([np.arange(c["past"], c["past"] + k) for k in _new(c)])
        st["seq"], st["slot"] = torch.from_numpy(seq).to(DEV), torch.from_numpy(slot).to(DEV)
        st["new_pos"] = torch.from_numpy(_positions(c)[0].astype(np.int32)).to(DEV)
        st["resident"] = torch.tensor([c["past"] + k for k in _new(c)], dtype=torch.int32, device=DEV)
    if c["kind"] == "shared":
        st["K"], st["V"], st["score"] = x["K"].clone(), x["V"].clone(), x["score"].clone()
        width = x["idx"].shape[1]
        st["off"] = torch.arange(width, device=DEV)[None] >= x["cnt"][:, None]             # places behind the end of a list
        st["has"] = torch.tensor([b for b, k in enumerate(_spread(c["own_lo"], c["own_hi"], n)) if k], dtype=torch.long, device=DEV)
    return st


# --------------------------------------------------------------------------- the framework's operators
def _prepare_own(st):
    from paper_2506_18226_amd import binding as B
    from paper_2506_18226_amd.batch import LayerBatch

    c, x = st["case"], st["x"]
    st["B"] = B
    h, D, n = c["heads"], c["head_dim"], c["n_seq"]
    hq = h * c["q_per_kv"]
    cap = _cap_of(c) if c["kind"] != "rotate" else 1

    def layer(n_seq, cap, sel_cap, mass):
        return LayerBatch(B.make_params(
            n_seq=n_seq, n_heads=h, head_dim=D, grid_h=c["grid_h"], grid_w=c["grid_w"], win_rows_back=1, win_col_radius=4,
            dtype=B.F32 if c["dtype"] == "f32" else B.BF16, score_mode=B.SCORE_ATTN_MASS if mass else B.SCORE_EXT_LARGEST, cap=cap, sel_cap=sel_cap,
            layout=c["layout"], q_per_kv=c["q_per_kv"]), DEV)

    batch = st["batch"] = layer(n, cap, max(1, c["own_hi"]) if c["kind"] == "shared" else cap, c.get("mass", False))
    rows = (lambda t: t) if c["layout"] == "head_major" else (lambda t: t.transpose(1, 2))
    s = batch.seqs_host
    st["K"], st["V"] = rows(batch.K), rows(batch.V)
    if c["kind"] in ("rotate", "append"):
        st["rope"] = B.make_rope(x["freq"], pairing=_pairing(c), **_rule(c))
        st["flags"] = B.FLAG_NEW_F32 if c["in_f32"] and c["dtype"] == "bf16" else 0
    if c["kind"] == "rotate":
        s["grid_origin"], s["step"] = c["prefix"] + c["far"], _positions(c)[1]
        st["out"] = torch.empty(n, hq, D, dtype=batch.tdtype, device=DEV), torch.empty(n, h, D, dtype=batch.tdtype, device=DEV)
    if c["kind"] in ("append", "prefill"):
        new = _new(c)
        begin = torch.tensor([0] + np.cumsum(new).tolist(), dtype=torch.int32, device=DEV)
        slot0 = torch.full((n,), c["past"], dtype=torch.int32, device=DEV)
        s["n_keep_prefix"] = s["grid_origin"] = c["prefix"] + c.get("far", 0)
        st["K"].copy_(x["K"])
        st["V"].copy_(x["V"])
    if c["kind"] == "append":
        s["n_res"] = c["past"]
        batch.pos[:, :c["past"]] = torch.arange(c["past"], device=DEV, dtype=torch.int32)
        stride = x["q"].stride(0) if c["packed"] else 0
        st["coords"] = x["coords"].to(torch.int32) if c["far"] and not c["past"] else None       # positions that do not follow from the slots
        st["tokens"] = B.make_tokens(begin, slot0, sum(new), max(new), coords=st["coords"], q_stride=stride, k_stride=stride, v_stride=stride)
        st["q_out"] = torch.empty(sum(new), hq, D, dtype=batch.tdtype, device=DEV)
    if c["kind"] == "prefill":
        s["n_res"] = [c["past"] + k for k in new]
        batch.pos[:] = torch.arange(cap, device=DEV, dtype=torch.int32)
        st["tokens"] = B.make_tokens(begin, slot0, sum(new), max(new))
        st["mods"] = B.make_mods(softcap=c["cap"], mask=B.MASK_PREFIX if c["mask"] == "prefix" else B.MASK_CAUSAL, slopes=x.get("slopes"), doc=x.get("doc"))
        st["out"] = torch.empty(sum(new), hq, D, dtype=batch.tdtype, device=DEV)
        st["lse"] = torch.empty(sum(new), hq, dtype=torch.float32, device=DEV)
    if c["kind"] == "shared":
        st["K"].copy_(x["K"])
        st["V"].copy_(x["V"])
        batch.pos[:] = torch.arange(cap, device=DEV, dtype=torch.int32) + c["prefix_hi"]
        s["n_res"], s["grid_origin"], s["n_keep_prefix"], s["step"] = cap, c["prefix_hi"], c["prefix_hi"], cap
        s["pending_slot"] = [cap - 1 if k else -1 for k in _spread(c["own_lo"], c["own_hi"], n)]
        batch.sel_idx.copy_(x["idx"])
        batch.sel_cnt.copy_(x["cnt"])
        prompts = st["prompts"] = layer(c["groups"], c["prefix_hi"], c["prefix_hi"], False)
        rows(prompts.K).copy_(x["PK"])
        rows(prompts.V).copy_(x["PV"])
        prompts.pos[:] = torch.arange(c["prefix_hi"], device=DEV, dtype=torch.int32)
        prompts.seqs_host["n_res"] = _spread(c["prefix_lo"], c["prefix_hi"], c["groups"])
        prompts.upload_seqs()
        m = _members(c)
        st["members"] = torch.tensor(m, dtype=torch.int32, device=DEV)
        st["shared"] = B.make_shared(prompts.params, prompts.seqs, st["members"], max_members=max(b - a for a, b in zip(m, m[1:])))
        st["mods"] = B.make_mods(softcap=c["cap"], slopes=x.get("slopes"))
        st["flags"] = B.FLAG_APPEND | (B.FLAG_NEW_F32 if c["in_f32"] else 0)
    batch.upload_seqs()


def _run_own(st):
    c, x, B, batch = st["case"], st["x"], st["B"], st["batch"]
    if c["kind"] == "rotate":
        stride = x["q"].stride(0) if c["packed"] else 0
        batch.rotate(st["rope"], x["q"], x["k"], *st["out"], flags=st["flags"], q_stride=stride, k_stride=stride)
        return st["out"]
    if c["kind"] == "append":
        batch.append(st["tokens"], st["rope"], x["q"], x["k"], x["v"], st["q_out"], flags=st["flags"])
        res = batch.seqs.view(torch.int32).view(c["n_seq"], -1)[:, 8]
        pos = batch.pos if st["coords"] is None else None
        return {"q": st["q_out"], "K": st["K"], "V": st["V"], "resident": res, "pos": pos}
    if c["kind"] == "prefill":
        if c["mass"]:
            batch.score.zero_()                            # (a prompt starts without mass, whichever pass this is)
        batch.prefill(st["tokens"], x["q"], st["out"], st["lse"], mods=st["mods"])
        return {"out": st["out"], "lse": st["lse"], "mass": batch.score if c["mass"] else None}
    if c["mass"]:
        batch.score.copy_(x["score"])                      # (every pass adds to the same scores)
    batch.attend_shared(st["shared"], x["q"], x["k_new"], x["v_new"], flags=st["flags"], mods=st["mods"])
    return {"out": batch.out, "lse": batch.lse, "K": st["K"], "V": st["V"], "score": batch.score if c["mass"] else None}


# --------------------------------------------------------------------------- plain forms
def _turn(x, angle, pairing):
    """Rows x [T][heads][D], as fp32, with every pair of elements turned by angle [T][D / 2] (fp64)."""
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = x.float()
    if pairing == "halves":
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)


def _weights(c, z):
    """(exp(z - max), their sum, log of the sum of exp(z)) over the last axis; a row without a finite score gives zeros and -inf."""
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = (z - m).exp()
    l = e.sum(-1, keepdim=True)
    return e, l, (m + l.log()).squeeze(-1)


def run(st):
    if own:
        return _run_own(st)
    c, x = st["case"], st["x"]
    h, D, n, G = c["heads"], c["head_dim"], c["n_seq"], c["q_per_kv"]
    hq, dt = h * G, _storage(c)
    if c["kind"] in ("rotate", "append"):
        angle = x["coords"].double() @ x["freq"]
        q = _turn(x["q"].unflatten(1, (hq, D)), angle, _pairing(c)).to(dt)
        k = _turn(x["k"].unflatten(1, (h, D)), angle, _pairing(c)).to(dt)
        if c["kind"] == "rotate":
            return q, k
        st["K"][st["seq"], :, st["slot"]] = k
        st["V"][st["seq"], :, st["slot"]] = x["v"].unflatten(1, (h, D)).to(dt)
        st["pos"][st["seq"], st["slot"]] = st["new_pos"]
        return {"q": q, "K": st["K"], "V": st["V"], "resident": st["resident"], "pos": st["pos"] if not c["far"] or c["past"] else None}
    scale = 1.0 / math.sqrt(D)
    if c["kind"] == "prefill":
        T, at = x["q"].shape[0], 0
        out, lse = torch.empty(T, hq, D, dtype=dt, device=DEV), torch.empty(T, hq, device=DEV)
        mass = torch.zeros(n, h, _cap_of(c), device=DEV) if c["mass"] else None
        for b, k in enumerate(_new(c)):
            keys = c["past"] + k
            K, V = x["K"][b, :, :keys].float(), x["V"][b, :, :keys].float()
            q = x["q"][at:at + k].float().view(k, h, G, D).permute(1, 2, 0, 3).reshape(h, G * k, D)
            z = (torch.matmul(q, K.transpose(1, 2).contiguous()) * scale).view(h, G, k, keys)
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
            qs, ks = torch.arange(c["past"], keys, device=DEV)[:, None], torch.arange(keys, device=DEV)[None]
            if c["slopes"]:
                z = z - x["slopes"].view(h, G, 1, 1) * (qs - ks).abs()
            seen = ks <= qs
            if c["mask"] == "prefix":
                seen = seen | ((qs < c["prefix"]) & (ks < c["prefix"]))
            if c["doc_len"]:
                doc = x["doc"][b, :keys]
                seen = seen & (doc[c["past"]:, None] == doc[None]) & (doc[None] >= 0)
            e, l, lg = _weights(c, z.masked_fill(~seen, -math.inf))
            del z
            w = e / torch.where(l == 0, torch.ones_like(l), l)
            del e
            out[at:at + k] = torch.matmul(w.view(h, G * k, keys), V).view(h, G, k, D).permute(2, 0, 1, 3).reshape(k, hq, D).to(dt)
            lse[at:at + k] = lg.permute(2, 0, 1).reshape(k, hq)
            if mass is not None:
                mass[b, :, :keys] = w.sum((1, 2))
            at += k
        return {"out": out, "lse": lse, "mass": mass}
    # shared
    st["K"][st["has"], :, -1], st["V"][st["has"], :, -1] = x["k_new"][st["has"]].to(dt), x["v_new"][st["has"]].to(dt)
    idx = x["idx"].long()
    width, pre = idx.shape[1], c["prefix_hi"]
    at = idx[:, None, :, None].expand(n, h, width, D)
    K, V = st["K"].gather(2, at).float(), st["V"].gather(2, at).float()
    q = x["q"].float().view(n, h, G, D)
    z = torch.empty(n, h, G, pre + width, device=DEV)
    m, lens = _members(c), _spread(c["prefix_lo"], pre, c["groups"])
    for g in range(c["groups"]):
        a, b = m[g], m[g + 1]
        rows = q[a:b].transpose(0, 1).reshape(h, (b - a) * G, D)
        z[a:b, ..., :pre] = torch.matmul(rows, x["PK"][g].float().transpose(1, 2).contiguous()).view(h, b - a, G, pre).transpose(0, 1)
    z[..., pre:] = torch.matmul(q, K.transpose(2, 3).contiguous())
    z *= scale
    if c["cap"]:
        z = c["cap"] * torch.tanh(z / c["cap"])
    if c["slopes"]:
        there = pre + _cap_of(c) - 1                       # the query token's position
        dist = torch.cat([(there - torch.arange(pre, device=DEV)).expand(n, pre), there - (pre + idx)], 1)
        z = z - x["slopes"].view(1, h, G, 1) * dist[:, None, None]
    for g in range(c["groups"]):
        z[m[g]:m[g + 1], ..., lens[g]:pre] = -math.inf
    z[..., pre:].masked_fill_(st["off"][:, None, None], -math.inf)
    e, l, lse = _weights(c, z)
    w = e / torch.where(l == 0, torch.ones_like(l), l)
    out = torch.matmul(w[..., pre:], V)
    for g in range(c["groups"]):
        a, b = m[g], m[g + 1]
        rows = w[a:b, ..., :pre].transpose(0, 1).reshape(h, (b - a) * G, pre)
        out[a:b] += torch.matmul(rows, x["PV"][g].float()).view(h, b - a, G, D).transpose(0, 1)
    score = None
    if c["mass"]:
        gain = w[..., pre:].sum(2).masked_fill(st["off"][:, None], 0.0)
        st["score"].copy_(x["score"])
        score = st["score"].scatter_add_(2, idx[:, None].expand(n, h, width), gain)
    return {"out": out.view(n, hq, D).to(dt), "lse": lse.view(n, hq), "K": st["K"], "V": st["V"], "score": score}


# --------------------------------------------------------------------------- from the definitions, in 64 bits
def _turned(x, coords, freq, pairing):
    """Each pair of elements as a complex number, times exp(i * angle)."""
    n = x.shape[-1] // 2
    x = x.double()
    z = torch.complex(x[..., :n], x[..., n:]) if pairing == "halves" else torch.view_as_complex(x.unflatten(-1, (n, 2)).contiguous())
    angle = (coords.double()[:, :, None] * freq[None]).sum(1)
    z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.cat([z.real, z.imag], -1) if pairing == "halves" else torch.view_as_real(z).flatten(-2)


def _attended(c, z, V):
    """Softmax of scores z [..., keys] times V [keys][D]: (output, lse, probabilities)."""
    lse = torch.logsumexp(z, -1)
    p = torch.exp(z - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[..., None])
    return p @ V, lse, p


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    h, D, n, G = c["heads"], c["head_dim"], c["n_seq"], c["q_per_kv"]
    hq, dt = h * G, _storage(c)
    if c["kind"] in ("rotate", "append"):
        q = _turned(x["q"].unflatten(1, (hq, D)), x["coords"], x["freq"], _pairing(c))
        k = _turned(x["k"].unflatten(1, (h, D)), x["coords"], x["freq"], _pairing(c))
        if c["kind"] == "rotate":
            return q, k
        K, V = x["K"].double(), x["V"].double()
        v, at = x["v"].unflatten(1, (h, D)), 0
        pos = torch.zeros(n, _cap_of(c), dtype=torch.int32, device=DEV)
        for b, new in enumerate(_new(c)):
            a, e = c["past"], c["past"] + new
            K[b, :, a:e], V[b, :, a:e] = k[at:at + new].transpose(0, 1), v[at:at + new].transpose(0, 1).double()
            pos[b, :e] = torch.arange(e, device=DEV)
            at += new
        res = torch.tensor([c["past"] + new for new in _new(c)], dtype=torch.int32, device=DEV)
        return {"q": q, "K": K, "V": V, "resident": res, "pos": pos if not c["far"] or c["past"] else None}

    def bent(z, head, dist):
        z = z / math.sqrt(D)
        if c["cap"]:
            z = c["cap"] * torch.tanh(z / c["cap"])
        return z - x["slopes"][head].double() * dist.abs() if c["slopes"] else z

    if c["kind"] == "prefill":
        out, lse = torch.empty(x["q"].shape[0], hq, D, dtype=torch.float64, device=DEV), torch.empty(x["q"].shape[0], hq, dtype=torch.float64, device=DEV)
        mass = torch.zeros(n, h, _cap_of(c), dtype=torch.float64, device=DEV) if c["mass"] else None
        at = 0
        for b, new in enumerate(_new(c)):
            keys = c["past"] + new
            dist = (torch.arange(c["past"], keys, device=DEV)[:, None] - torch.arange(keys, device=DEV)[None]).double()
            hidden = dist < 0
            if c["mask"] == "prefix":
                there = torch.arange(keys, device=DEV) < c["prefix"]
                hidden &= ~(there[c["past"]:, None] & there[None])
            if c["doc_len"]:
                doc = x["doc"][b, :keys]
                hidden |= doc[c["past"]:, None] != doc[None]
                hidden |= (doc < 0)[None]
            for j in range(hq):
                z = bent(x["q"][at:at + new, j].double() @ x["K"][b, j // G, :keys].double().t(), j, dist)
                z[hidden] = -math.inf
                o, s, p = _attended(c, z, x["V"][b, j // G, :keys].double())
                out[at:at + new, j], lse[at:at + new, j] = o, s
                if mass is not None:
                    mass[b, j // G, :keys] += p.sum(0)
            at += new
        return {"out": out, "lse": lse, "mass": mass}
    pre, lists, m = _spread(c["prefix_lo"], c["prefix_hi"], c["groups"]), _spread(c["own_lo"], c["own_hi"], n), _members(c)
    out, lse = torch.zeros(n, hq, D, dtype=torch.float64, device=DEV), torch.zeros(n, hq, dtype=torch.float64, device=DEV)
    K, V, score = x["K"].double(), x["V"].double(), x["score"].double()
    for g in range(c["groups"]):
        for b in range(m[g], m[g + 1]):
            slots = x["idx"][b, :lists[b]].long()
            if lists[b]:                                   # (the row as the cache stores it)
                K[b, :, -1], V[b, :, -1] = x["k_new"][b].to(dt).double(), x["v_new"][b].to(dt).double()
            keys = torch.cat([x["PK"][g, :, :pre[g]].double(), K[b][:, slots]], 1)
            vals = torch.cat([x["PV"][g, :, :pre[g]].double(), V[b][:, slots]], 1)
            z = (x["q"][b].double().view(h, G, D) @ keys.transpose(1, 2)).reshape(hq, -1)
            dist = c["prefix_hi"] + _cap_of(c) - 1 - torch.cat([torch.arange(pre[g], device=DEV), c["prefix_hi"] + slots]).double()
            z = bent(z, torch.arange(hq, device=DEV)[:, None], dist[None]) if c["slopes"] else bent(z, None, dist)
            if not z.shape[1]:
                lse[b] = -math.inf
                continue
            o, s, p = _attended(c, z.view(h, G, -1), vals)
            out[b], lse[b] = o.reshape(hq, D), s.reshape(hq)
            score[b][:, slots] += p[..., pre[g]:].sum(1)
    return {"out": out, "lse": lse, "K": K, "V": V, "score": score if c["mass"] else None}

"""A decode step over caches that are kept in pages, and the next token, as cases that can be timed and compared.

  append   tokens enter the pages of their sequences: q and k turned by rotary positions, K and V rows to the pages that a table names
  prefill  attention of a chunk of new tokens behind what is resident in the pages, any number of tokens from one on: causal, or a prefix
           that sees itself whole; scores capped by a tanh or lowered with distance; the attention mass that evictions rank by
  attend   the form for single tokens: one query token over a list of its sequence's slots, its own row stored on the way, mass added
  compact  the eviction at the end of a grid row: prefix, the last rows and the largest accumulated mass stay, rows close up in their pages
  sample   the next token from logits and given random numbers: temperature, top-k, top-p and min-p, of guided pairs or single rows

With `own` false everything is computed in its plain form, by elementary torch operations in 32 bits (angles and what tokens are drawn
by in 64).  Inputs come from the seed alone; how long sequences are follows from the case.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"


# --------------------------------------------------------------------------- cases
def _case(name=None, **kw):
    c = dict(kind=kw["kind"])
    if c["kind"] == "sample":
        c.update(rows=1, vocab=16384, dtype="bf16", guided=False, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, per_row=False)
    else:
        c.update(n_seq=1, heads=16, head_dim=64, q_per_kv=1, dtype="bf16", page=64, layout="head_major", grid_h=32, grid_w=32, prefix=120)
    if c["kind"] in ("append", "prefill"):
        c.update(new_lo=1, new_hi=1, past_lo=0, past_hi=0)
    if c["kind"] == "append":
        c.update(axes="grid", in_f32=False)
    if c["kind"] == "prefill":
        c.update(mask="causal", cap=0.0, slopes=False, mass=False, q_scale=1.0)
    if c["kind"] == "attend":
        c.update(own_lo=1, own_hi=1, resident=1, mass=True, in_f32=False, q_scale=1.0)
    if c["kind"] == "compact":
        c.update(rows_back=1, budget=16, row=8)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one image to be edited enters its cache and its unconditional partner's: a few rows of a 24x24 grid behind the text
        _case("append_rows", kind="append", n_seq=2, heads=20, new_lo=72, new_hi=72, past_lo=120, past_hi=120, page=16, grid_h=24, grid_w=24),
        # half of a 64x64 grid behind 256 prompt tokens, 4 sequences, time, height and width as axes, fp32 projections
        _case("append_image", kind="append", n_seq=4, heads=32, head_dim=128, new_lo=2304, new_hi=2304, grid_h=64, grid_w=64, prefix=256, axes="thw", in_f32=True),
        # a few more tokens behind a long context, scores lowered with distance, small pages that hold all heads of a slot, odd sizes
        _case("prefill_few", kind="prefill", n_seq=3, heads=20, new_lo=2, new_hi=7, past_lo=1500, past_hi=2011, page=16, slopes=True, layout="slot_major", grid_h=64, grid_w=64, prefix=37),
        # serving: chunks of prompts of different lengths, grouped queries, capped scores
        _case("prefill_chunks", kind="prefill", n_seq=16, heads=8, head_dim=128, q_per_kv=8, new_lo=100, new_hi=256, past_lo=0, past_hi=1100, cap=50.0, q_scale=2.8),
        # the largest: the second half of a 64x64 image of 4 sequences, behind the first and 256 prompt tokens, with the mass that evictions rank by
        _case("prefill_image", kind="prefill", n_seq=4, heads=32, head_dim=128, new_lo=2048, new_hi=2048, past_lo=2304, past_hi=2304, mass=True, grid_h=64, grid_w=64, prefix=256),
        # the smallest decode call: one guided image, one layer of the 36-layer model
        _case("attend_one_image", kind="attend", n_seq=2, heads=20, own_lo=427, own_hi=427, resident=468, page=16, grid_h=24, grid_w=24, q_scale=2.8),
        # the headline configuration deep in the image, one layer
        _case("attend_batch", kind="attend", n_seq=32, heads=24, own_lo=673, own_hi=673, resident=695, q_scale=2.8),
        # grouped queries over long ragged lists, fp32 rows of the query token
        _case("attend_grouped", kind="attend", n_seq=32, heads=8, head_dim=128, q_per_kv=8, own_lo=300, own_hi=1378, resident=1471, page=32, in_f32=True, q_scale=2.8),
        # a grid row ends: the headline configuration
        _case("compact_batch", kind="compact", n_seq=32, heads=24, budget=512, row=24),
        # ... and a few sequences of a 64x64 grid, small pages
        _case("compact_long", kind="compact", n_seq=4, heads=32, head_dim=128, page=16, grid_h=64, grid_w=64, prefix=256, rows_back=2, budget=1024, row=40),
        # the next token of one guided image
        _case("sample_one_image", kind="sample", rows=1, guided=True, top_k=2000, top_p=0.95),
        # the next tokens of a serving batch, each row with settings of its own
        _case("sample_serving", kind="sample", rows=256, vocab=65536, dtype="f32", per_row=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_SHAPES = [(16, 64, 1), (20, 64, 1), (24, 64, 1), (32, 128, 1), (8, 128, 8), (7, 64, 1), (5, 128, 3), (9, 64, 2)]


def draw(rng):
    kind = rng.choice(["append", "prefill", "prefill", "attend", "attend", "compact", "sample", "sample"])
    if kind == "sample":
        vocab = _log_int(rng, 500, 131072)
        return _case(kind=kind, vocab=vocab, rows=min(_log_int(rng, 1, 512), (1 << 24) // vocab), dtype=rng.choice(["bf16", "f32"]), guided=rng.random() < 0.5,
                     temperature=rng.choice([0.0, 0.7, 1.0, 1.3]), top_k=rng.choice([0, 1, 50, 2000]), top_p=rng.choice([1.0, 0.95, 0.8, 0.3]),
                     min_p=rng.choice([0.0, 0.0, 0.02]), per_row=rng.random() < 0.3)
    heads, D, G = rng.choice(_SHAPES)
    c = dict(kind=kind, heads=heads, head_dim=D, q_per_kv=G, dtype="bf16" if G > 1 else rng.choice(["bf16", "bf16", "bf16", "f32"]),
             layout=rng.choice(["head_major", "head_major", "slot_major"]), prefix=rng.randint(8, 256), grid_h=64, grid_w=64, page=rng.choice([16, 32, 64, 128]))
    if kind in ("append", "prefill"):
        hi = _log_int(rng, 1, 2304 if kind == "append" or c["dtype"] == "bf16" else 1024)
        past = rng.choice([0, _log_int(rng, 8, 2048), _log_int(rng, 8, 2048)])
        if kind == "append":
            n = max(1, min(_log_int(rng, 1, 64), int(9000 / hi), int(20000 / (hi + past))))
            c.update(axes=rng.choice(["grid", "thw"]), in_f32=c["dtype"] == "bf16" and rng.random() < 0.4)
        else:
            pairs = heads * G * D * (hi * float(past) + hi * hi / 2)
            n = max(1, min(_log_int(rng, 1, 64), int(1.0e11 / pairs)))
            if c["dtype"] == "f32":
                n = max(1, min(n, int(2e10 / pairs)))
            c.update(mask=rng.choice(["causal", "causal", "prefix"]), cap=rng.choice([0.0, 0.0, 50.0]), slopes=rng.random() < 0.25, mass=rng.random() < 0.4,
                     q_scale=rng.choice([1.0, 2.8]))
        c.update(n_seq=n, new_hi=hi, new_lo=rng.randint(1, hi), past_hi=past, past_lo=rng.randint(0, past))
        c["prefix"] = max(1, min(c["prefix"], hi + past))
    if kind == "attend":
        n, own_hi = _log_int(rng, 1, 128), _log_int(rng, 1, 1400)
        n = max(1, min(n, int(1.0e9 / (own_hi * heads * D * 8))))
        c.update(n_seq=n, own_hi=own_hi, own_lo=rng.randint(1, own_hi), resident=own_hi + rng.randint(0, 200), mass=rng.random() < 0.7,
                 in_f32=c["dtype"] == "bf16" and rng.random() < 0.3, q_scale=rng.choice([1.0, 2.8]))
    if kind == "compact":
        W, R = rng.choice([16, 24, 32, 64]), rng.randint(0, 2)
        budget = _log_int(rng, 4, 1024)
        row = min(64, (budget + W - 1) // W + R + 1 + rng.randint(0, 20))
        n = max(1, min(_log_int(rng, 1, 64), int(6.0e8 / ((c["prefix"] + budget + 3 * W) * heads * D * 8))))
        c.update(n_seq=n, grid_w=W, grid_h=64, rows_back=R, budget=budget, row=row, q_per_kv=1)
    return _case(**c)


# --------------------------------------------------------------------------- sizes, from the case alone
def _spread(lo, hi, n, turn=0):
    """n lengths between lo and hi, the longest among them, in no order."""
    if n == 1:
        return [hi]
    return [lo + (hi - lo) * (((i + turn) * 7919 + n - 1) % n) // (n - 1) for i in range(n)]


def _eb(c):
    return 4 if c["dtype"] == "f32" else 2


def _storage(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _new(c):
    return _spread(c["new_lo"], c["new_hi"], c["n_seq"])


def _past(c):
    return _spread(c["past_lo"], c["past_hi"], c["n_seq"], 1)


def _resident(c):
    """Slots of every sequence that hold something once the call is done (compact: before it)."""
    if c["kind"] in ("append", "prefill"):
        return [a + b for a, b in zip(_past(c), _new(c))]
    if c["kind"] == "attend":
        return [c["resident"]] * c["n_seq"]
    rows = min(c["rows_back"] + 1, c["row"])
    history = min(c["budget"], (c["row"] - rows) * c["grid_w"])
    return [c["prefix"] + history + rows * c["grid_w"]] * c["n_seq"]


def _kept(c):
    rest = _resident(c)[0] - c["prefix"] - min(c["rows_back"], c["row"]) * c["grid_w"]
    return _resident(c)[0] - max(0, rest - c["budget"])


def _pages(c):
    return [-(-n // c["page"]) for n in _resident(c)]


def _pairs(c):
    """(query, key) pairs that are attended, over all sequences, per query head."""
    total = 0
    for past, new in zip(_past(c), _new(c)):
        q = np.arange(past, past + new)
        end = q + 1
        if c["mask"] == "prefix":
            end = np.where(q < c["prefix"], np.maximum(end, min(c["prefix"], past + new)), end)
        total += int(end.sum())
    return total


def work(case):
    c = case
    if c["kind"] == "sample":
        logits = c["rows"] * (2 if c["guided"] else 1) * c["vocab"]
        return {"bytes": float(logits * _eb(c) + 12 * c["rows"]), "flops": 4.0 * logits}
    eb, D, h = _eb(c), c["head_dim"], c["heads"]
    hq, table = h * c["q_per_kv"], 4 * sum(_pages(c))
    if c["kind"] == "append":
        T, ib = sum(_new(c)), 4 if c["in_f32"] else eb
        return {"bytes": float(T * ((hq + 2 * h) * D * (ib + eb) + 4) + table), "flops": 3.0 * T * (hq + h) * D}
    if c["kind"] == "prefill":
        T, keys = sum(_new(c)), sum(_resident(c))
        return {"bytes": float(2 * T * hq * D * eb + 4 * T * hq + 2 * keys * h * D * eb + (4 * keys * h if c["mass"] else 0) + table), "flops": 4.0 * _pairs(c) * hq * D}
    if c["kind"] == "attend":
        lists = sum(_spread(c["own_lo"], c["own_hi"], c["n_seq"]))
        io = c["n_seq"] * (2 * hq * D * eb + 4 * hq + 2 * h * D * (4 if c["in_f32"] else eb)) + 4 * lists * (1 + (2 * h if c["mass"] else 0))
        return {"bytes": float(2 * lists * h * D * eb + io + table), "flops": 4.0 * lists * hq * D}
    n, kept = _resident(c)[0], _kept(c)
    rest = n - c["prefix"] - min(c["rows_back"], c["row"]) * c["grid_w"]
    moved = max(0, kept - c["prefix"] - rest // (n - kept + 1)) if kept < n else 0            # behind the first that goes, of any order of scores
    return {"bytes": float(c["n_seq"] * (moved * (4 * h * D * eb + 4 * h + 4) + n * (4 * h + 8)) + table), "flops": float(c["n_seq"] * n * h)}


# --------------------------------------------------------------------------- inputs
_RULES = {   # coordinate on each axis: of text at position p, text * p; of the image token at (row, column), origin * P + row * r + col * c
    "grid": dict(text=(0, 0), origin=(0, 0), row=(1, 0), col=(0, 1)),
    "thw": dict(text=(1, 1, 1), origin=(1, 1, 1), row=(0, 1, 0), col=(0, 0, 1)),
}


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
    f = torch.zeros(3, n, dtype=torch.float64)             # a quarter of the pairs for time, the rest for height and width
    a, b = n // 4, n // 4 + (n - n // 4) // 2
    f[0, :a], f[1, a:b], f[2, b:] = base[:a], base[a:b], base[b:]
    return f


def _coordinates(c):
    """int64 [tokens][axes] of the new tokens."""
    p, r, P = np.concatenate([np.arange(a, a + n) for a, n in zip(_past(c), _new(c))]), _RULES[c["axes"]], c["prefix"]
    row, col = (p - P) // c["grid_w"], (p - P) % c["grid_w"]
    axes = [np.where(p < P, t * p, o * P + a * row + b * col) for t, o, a, b in zip(r["text"], r["origin"], r["row"], r["col"])]
    return np.stack(axes, 1)


def _inputs(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 2 + 1)
    rng = np.random.default_rng([seed & 0x7FFFFFFF, 6])

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)

    x = {}
    if c["kind"] == "sample":
        rows, V = c["rows"], c["vocab"]
        x["logits"] = (randn(rows * (2 if c["guided"] else 1), V) * 2.0).to(_storage(c))
        if c["guided"]:                                    # the condition changes some of what the model says without it
            x["logits"][:rows] = (x["logits"][rows:].float() + 0.5 * x["logits"][:rows].float()).to(_storage(c))
        x["uniform"] = torch.rand(rows, generator=gen, device=DEV)
        one = dict(temperature=c["temperature"], top_k=c["top_k"], top_p=c["top_p"], min_p=c["min_p"])
        if c["per_row"]:
            some = dict(temperature=rng.choice([0.0, 0.6, 0.9, 1.0, 1.2], rows), top_k=rng.choice([0, 0, 20, 100, 1000], rows), top_p=rng.choice([1.0, 0.95, 0.9, 0.7], rows),
                        min_p=rng.choice([0.0, 0.0, 0.05], rows))
        else:
            some = {k: np.full(rows, v) for k, v in one.items()}
        x["settings"] = {k: torch.from_numpy(v.astype(np.int32 if k == "top_k" else np.float32)).to(DEV) for k, v in some.items()}
        return x
    dt, h, D, n, P = _storage(c), c["heads"], c["head_dim"], c["n_seq"], c["page"]
    hq, pages, res = h * c["q_per_kv"], _pages(c), _resident(c)
    cap = max(res)
    # every sequence's pages lie anywhere in the pool; some pages are nobody's
    total = sum(pages) + 3
    order = rng.permutation(total)
    table = np.full((n, max(pages)), -1, np.int32)
    at = 0
    for b, k in enumerate(pages):
        table[b, :k] = order[at:at + k]
        at += k
    x["table"] = torch.from_numpy(table).to(DEV)
    shape = (total, h, P, D) if c["layout"] == "head_major" else (total, P, h, D)
    x["K"], x["V"] = randn(*shape).to(dt), randn(*shape).to(dt)
    if c["kind"] == "append":
        T, it = sum(_new(c)), torch.float32 if c["in_f32"] else dt
        x["q"], x["k"], x["v"] = randn(T, hq * D).to(it), randn(T, h * D).to(it), randn(T, h * D).to(it)
        x["freq"] = _frequencies(c).to(DEV)
        x["coords"] = torch.from_numpy(_coordinates(c)).to(DEV)
    if c["kind"] == "prefill":
        x["q"] = (randn(sum(_new(c)), hq, D) * c["q_scale"]).to(dt)
        if c["slopes"]:                                    # a geometric sequence over the heads
            x["slopes"] = 2.0 ** (-8.0 * torch.arange(1, hq + 1, device=DEV, dtype=torch.float32) / hq)
    if c["kind"] == "attend":                              # some of the resident tokens are in a sequence's list, the last one is the query token
        lists = _spread(c["own_lo"], c["own_hi"], n)
        idx = np.zeros((n, c["own_hi"]), np.int32)
        for b, k in enumerate(lists):
            idx[b, :k] = np.concatenate([np.sort(rng.permutation(cap - 1)[:k - 1]), [cap - 1]])
        x["idx"], x["cnt"] = torch.from_numpy(idx).to(DEV), torch.tensor(lists, dtype=torch.int32, device=DEV)
        x["q"] = (randn(n, hq, D) * c["q_scale"]).to(dt)
        it = torch.float32 if c["in_f32"] else dt
        x["k_new"], x["v_new"] = randn(n, h, D).to(it), randn(n, h, D).to(it)
    if c["kind"] == "compact":                             # prefix, what earlier row ends kept, and the last rows whole
        rows, W = min(c["rows_back"] + 1, c["row"]), c["grid_w"]
        past = (c["row"] - rows) * W
        pos = np.empty((n, cap), np.int32)
        for b in range(n):
            history = np.sort(rng.permutation(past)[:min(c["budget"], past)])
            pos[b] = np.concatenate([np.arange(c["prefix"]), c["prefix"] + history, c["prefix"] + past + np.arange(rows * W)])
        x["pos"] = torch.from_numpy(pos).to(DEV)
    if c["kind"] in ("attend", "compact"):
        x["score"] = torch.rand(n, h, cap, generator=gen, device=DEV)
    return x


def _slots(c, x):
    """Page and place in it of every slot of every sequence, [n_seq][slots]."""
    n = max(_resident(c))
    slot = torch.arange(n, device=DEV)
    return x["table"].long()[:, slot // c["page"]].clamp(min=0), (slot % c["page"]).expand(c["n_seq"], n)


def _rows_of(c, pool, page, place):
    """Rows [..., heads, D] of the pool."""
    return pool[page, :, place] if c["layout"] == "head_major" else pool[page, place]


def prepare(case, seed):
    c = case
    x = _inputs(c, seed)
    st = {"case": dict(c), "x": x}
    if own:
        _prepare_own(st)
        return st
    if c["kind"] == "sample":
        return st
    st["K"], st["V"] = x["K"].clone(), x["V"].clone()
    st["page"], st["place"] = _slots(c, x)
    n, cap = c["n_seq"], max(_resident(c))
    if c["kind"] == "append":
        st["pos"] = torch.zeros(n, cap, dtype=torch.int32, device=DEV)
        for b, past in enumerate(_past(c)):
            st["pos"][b, :past] = torch.arange(past, device=DEV, dtype=torch.int32)
        seq = np.repeat(np.arange(n), _new(c))
        slot = np.concatenate([np.arange(a, a + k) for a, k in zip(_past(c), _new(c))])
        st["seq"], st["slot"] = torch.from_numpy(seq).to(DEV), torch.from_numpy(slot).to(DEV)
        st["resident"] = torch.tensor(_resident(c), dtype=torch.int32, device=DEV)
    if c["kind"] == "attend":
        st["score"] = x["score"].clone()
        st["off"] = torch.arange(x["idx"].shape[1], device=DEV)[None] >= x["cnt"][:, None]              # places behind the end of a list
    return st


# --------------------------------------------------------------------------- the framework's operators
def _prepare_own(st):
    from paper_2506_18226_amd import binding as B
    from paper_2506_18226_amd import batch as batches

    c, x = st["case"], st["x"]
    st["B"] = B
    if c["kind"] == "sample":
        per_row = x["settings"] if c["per_row"] else {k: c[k] for k in x["settings"]}
        st["sampler"] = batches.Sampler(c["rows"], c["vocab"], B.F32 if c["dtype"] == "f32" else B.BF16, guidance=3.0 if c["guided"] else None, device=DEV, **per_row)
        return
    h, D, n, G = c["heads"], c["head_dim"], c["n_seq"], c["q_per_kv"]
    hq, cap, res = h * G, max(_resident(c)), _resident(c)
    mass = c["kind"] == "compact" or c.get("mass", False)
    params = B.make_params(n_seq=n, n_heads=h, head_dim=D, grid_h=c["grid_h"], grid_w=c["grid_w"], win_rows_back=c.get("rows_back", 1), win_col_radius=4,
                           dtype=B.F32 if c["dtype"] == "f32" else B.BF16, score_mode=B.SCORE_ATTN_MASS if mass else B.SCORE_EXT_LARGEST, cap=cap,
                           sel_cap=c["own_hi"] if c["kind"] == "attend" else cap, layout=c["layout"], q_per_kv=G)
    batch = st["batch"] = batches.PagedBatch(params, n_pages=x["K"].shape[0], page_size=c["page"], device=DEV)
    batch.K.copy_(x["K"])
    batch.V.copy_(x["V"])
    batch.table.copy_(x["table"])
    s = batch.seqs_host
    s["n_keep_prefix"] = s["grid_origin"] = c["prefix"]
    if c["kind"] in ("append", "prefill"):
        new = _new(c)
        begin = torch.tensor([0] + np.cumsum(new).tolist(), dtype=torch.int32, device=DEV)
        slot0 = torch.tensor(_past(c), dtype=torch.int32, device=DEV)
        st["tokens"] = B.make_tokens(begin, slot0, sum(new), max(new))
        s["n_res"] = _past(c) if c["kind"] == "append" else res
        st["out"] = torch.empty(sum(new), hq, D, dtype=batch.tdtype, device=DEV)
    if c["kind"] == "append":
        for b, past in enumerate(_past(c)):
            batch.pos[b, :past] = torch.arange(past, device=DEV, dtype=torch.int32)
        st["rope"] = B.make_rope(x["freq"], pairing=_pairing(c), **_RULES[c["axes"]])
        st["flags"] = B.FLAG_NEW_F32 if c["in_f32"] else 0
    if c["kind"] == "prefill":
        batch.pos[:] = torch.arange(cap, device=DEV, dtype=torch.int32)
        st["mods"] = B.make_mods(softcap=c["cap"], mask=B.MASK_PREFIX if c["mask"] == "prefix" else B.MASK_CAUSAL, slopes=x.get("slopes"))
        st["lse"] = torch.empty(sum(new), hq, dtype=torch.float32, device=DEV)
    if c["kind"] == "attend":
        batch.pos[:] = torch.arange(cap, device=DEV, dtype=torch.int32)
        s["n_res"], s["step"], s["pending_slot"] = cap, 1, cap - 1
        batch.sel_idx.copy_(x["idx"])
        batch.sel_cnt.copy_(x["cnt"])
        st["flags"] = B.FLAG_APPEND | (B.FLAG_NEW_F32 if c["in_f32"] else 0)
    if c["kind"] == "compact":
        s["n_res"], s["step"], s["budget"] = cap, c["row"] * c["grid_w"], c["budget"]
    batch.upload_seqs()
    if c["kind"] == "compact":
        st["seqs"] = batch.seqs.clone()


def _run_own(st):
    c, x, B = st["case"], st["x"], st["B"]
    if c["kind"] == "sample":
        st["sampler"].sample(x["logits"], x["uniform"])
        return {"token": st["sampler"].token[:c["rows"]], "logprob": st["sampler"].logprob}
    batch = st["batch"]
    if c["kind"] == "append":
        batch.append(st["tokens"], st["rope"], x["q"], x["k"], x["v"], st["out"], flags=st["flags"])
        return {"q": st["out"], "K": batch.K, "V": batch.V, "resident": batch.seqs.view(torch.int32).view(c["n_seq"], -1)[:, 8], "pos": batch.pos}
    if c["kind"] == "prefill":
        if c["mass"]:
            batch.score.zero_()                            # (a prompt starts without mass, whichever pass this is)
        batch.prefill(st["tokens"], x["q"], st["out"], st["lse"], mods=st["mods"])
        return {"out": st["out"], "lse": st["lse"], "mass": batch.score if c["mass"] else None}
    if c["kind"] == "attend":
        if c["mass"]:
            batch.score.copy_(x["score"])                  # (every pass adds to the same scores)
        batch.attend(x["q"], st["flags"], x["k_new"], x["v_new"])
        return {"out": batch.out, "lse": batch.lse, "K": batch.K, "V": batch.V, "score": batch.score if c["mass"] else None}
    batch.score.copy_(x["score"])                          # (every pass ends the same row of the same records)
    batch.pos.copy_(x["pos"])
    batch.seqs.copy_(st["seqs"])
    batch.compact()
    return {"map": batch.keep_map, "resident": batch.seqs.view(torch.int32).view(c["n_seq"], -1)[:, 8], "pos": batch.pos, "score": batch.score, "K": batch.K, "V": batch.V}


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


def _weights(z):
    """(exp(z - max), their sum, log of the sum of exp(z)) over the last axis; every row has a finite score."""
    m = z.amax(-1, keepdim=True)
    e = (z - m).exp()
    l = e.sum(-1, keepdim=True)
    return e, l, (m + l.log()).squeeze(-1)


def _put(c, pool, page, place, rows):
    if c["layout"] == "head_major":
        pool[page, :, place] = rows
    else:
        pool[page, place] = rows


def _run_sample(c, x):
    n, s = c["rows"], x["settings"]
    z = x["logits"].float()
    if c["guided"]:                                        # rounded to 32 bits once
        a, b = z[:n].double(), z[n:].double()
        z = (b + 3.0 * (a - b)).float()
    T = s["temperature"].double()[:, None]
    greedy = T == 0
    d = (z.double() - z.double().amax(1, keepdim=True)) / torch.where(greedy, torch.ones_like(T), T)
    w = d.exp()
    order = torch.sort(z, dim=1, descending=True, stable=True)[1]                # ties: the lowest index first
    ws = w.gather(1, order)
    place = torch.arange(c["vocab"], device=DEV)[None]
    k = s["top_k"][:, None]
    keep = (place < k) | (k <= 0)
    ws = ws * keep
    sums = ws.cumsum(1)
    p = s["top_p"].double()[:, None]
    keep &= (sums - ws < p * sums[:, -1:]) | (p >= 1)
    keep &= ws >= s["min_p"].double()[:, None]
    keep = torch.where(greedy, place == 0, keep)
    w = w * torch.zeros_like(keep).scatter(1, order, keep)
    sums = w.cumsum(1)
    total = sums[:, -1:]
    token = (sums > x["uniform"].double()[:, None] * total).long().argmax(1)     # (the first that passes)
    logprob = d.gather(1, token[:, None]) - total.log()
    return {"token": token.to(torch.int32), "logprob": logprob[:, 0].float()}


def run(st):
    if own:
        return _run_own(st)
    c, x = st["case"], st["x"]
    if c["kind"] == "sample":
        return _run_sample(c, x)
    h, D, n, G = c["heads"], c["head_dim"], c["n_seq"], c["q_per_kv"]
    hq, dt, scale = h * G, _storage(c), 1.0 / math.sqrt(c["head_dim"])
    if c["kind"] == "append":
        angle = x["coords"].double() @ x["freq"]
        q = _turn(x["q"].unflatten(1, (hq, D)), angle, _pairing(c)).to(dt)
        k = _turn(x["k"].unflatten(1, (h, D)), angle, _pairing(c)).to(dt)
        page, place = st["page"][st["seq"], st["slot"]], st["place"][st["seq"], st["slot"]]
        _put(c, st["K"], page, place, k)
        _put(c, st["V"], page, place, x["v"].unflatten(1, (h, D)).to(dt))
        st["pos"][st["seq"], st["slot"]] = st["slot"].to(torch.int32)
        return {"q": q, "K": st["K"], "V": st["V"], "resident": st["resident"], "pos": st["pos"]}
    if c["kind"] == "prefill":
        T, at = x["q"].shape[0], 0
        out, lse = torch.empty(T, hq, D, dtype=dt, device=DEV), torch.empty(T, hq, device=DEV)
        mass = torch.zeros(n, h, max(_resident(c)), device=DEV) if c["mass"] else None
        for b, (past, k) in enumerate(zip(_past(c), _new(c))):
            keys = past + k
            K, V = (_rows_of(c, st[name], st["page"][b, :keys], st["place"][b, :keys]).float().transpose(0, 1).contiguous() for name in "KV")
            q = x["q"][at:at + k].float().view(k, h, G, D).permute(1, 2, 0, 3).reshape(h, G * k, D)
            z = (torch.matmul(q, K.transpose(1, 2).contiguous()) * scale).view(h, G, k, keys)
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
            qs, ks = torch.arange(past, keys, device=DEV)[:, None], torch.arange(keys, device=DEV)[None]
            if c["slopes"]:
                z = z - x["slopes"].view(h, G, 1, 1) * (qs - ks).abs()
            seen = ks <= qs
            if c["mask"] == "prefix":
                seen = seen | ((qs < c["prefix"]) & (ks < c["prefix"]))
            e, l, lg = _weights(z.masked_fill(~seen, -math.inf))
            del z
            w = e / l
            del e
            out[at:at + k] = torch.matmul(w.view(h, G * k, keys), V).view(h, G, k, D).permute(2, 0, 1, 3).reshape(k, hq, D).to(dt)
            lse[at:at + k] = lg.permute(2, 0, 1).reshape(k, hq)
            if mass is not None:
                mass[b, :, :keys] = w.sum((1, 2))
            at += k
        return {"out": out, "lse": lse, "mass": mass}
    seq = torch.arange(n, device=DEV)[:, None]
    if c["kind"] == "attend":
        _put(c, st["K"], st["page"][:, -1], st["place"][:, -1], x["k_new"].to(dt))
        _put(c, st["V"], st["page"][:, -1], st["place"][:, -1], x["v_new"].to(dt))
        idx = x["idx"].long()
        K, V = (_rows_of(c, st[name], st["page"][seq, idx], st["place"][seq, idx]).float().transpose(1, 2).contiguous() for name in "KV")     # [n][h][entries][D]
        z = torch.matmul(x["q"].float().view(n, h, G, D), K.transpose(2, 3).contiguous()) * scale
        e, l, lse = _weights(z.masked_fill(st["off"][:, None, None], -math.inf))
        w = e / l
        out, score = torch.matmul(w, V), None
        if c["mass"]:
            st["score"].copy_(x["score"])
            score = st["score"].scatter_add_(2, idx[:, None].expand(n, h, idx.shape[1]), w.sum(2))       # (places behind the end of a list add 0)
        return {"out": out.view(n, hq, D).to(dt), "lse": lse.view(n, hq), "K": st["K"], "V": st["V"], "score": score}
    # compact: what the prefix and the last rows hold stays, of the rest the `budget` largest sums of scores (over heads, one after the other)
    cap, pos, score = x["pos"].shape[1], x["pos"], x["score"]
    rank = score[:, 0].clone()
    for j in range(1, h):
        rank += score[:, j]
    image = pos - c["prefix"]
    fixed = (pos < c["prefix"]) | (image >= (c["row"] - min(c["rows_back"], c["row"])) * c["grid_w"])
    order = torch.sort(rank.masked_fill(fixed, -math.inf), dim=1, descending=True, stable=True)[1]
    best = torch.zeros_like(fixed).scatter(1, order[:, :c["budget"]], True)
    keep = fixed | best
    new = keep.to(torch.int32).cumsum(1, dtype=torch.int32)
    where = torch.where(keep, new - 1, -torch.ones_like(new))
    src = torch.sort(where.masked_fill(~keep, cap), dim=1, stable=True)[1][:, :_kept(c)]                 # kept slots in order
    K, V = (_rows_of(c, st[name], st["page"][seq, src], st["place"][seq, src]) for name in "KV")
    _put(c, st["K"], st["page"][:, :_kept(c)], st["place"][:, :_kept(c)], K)
    _put(c, st["V"], st["page"][:, :_kept(c)], st["place"][:, :_kept(c)], V)
    pos_out, score_out = pos.clone(), score.clone()
    pos_out[:, :_kept(c)] = pos.gather(1, src)
    score_out[:, :, :_kept(c)] = score.gather(2, src[:, None].expand(n, h, _kept(c)))
    return {"map": where, "resident": new[:, -1], "pos": pos_out, "score": score_out, "K": st["K"], "V": st["V"]}


# --------------------------------------------------------------------------- from the definitions, in 64 bits
def _turned(x, coords, freq, pairing):
    """Each pair of elements as a complex number, times exp(i * angle)."""
    n = x.shape[-1] // 2
    x = x.double()
    z = torch.complex(x[..., :n], x[..., n:]) if pairing == "halves" else torch.view_as_complex(x.unflatten(-1, (n, 2)).contiguous())
    angle = (coords.double()[:, :, None] * freq[None]).sum(1)
    z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.cat([z.real, z.imag], -1) if pairing == "halves" else torch.view_as_real(z).flatten(-2)


def _attended(z, V):
    """Softmax of scores z [..., keys] times V [keys][D]: (output, lse, probabilities)."""
    lse = torch.logsumexp(z, -1)
    p = torch.exp(z - lse[..., None])
    return p @ V, lse, p


def _cached(c, pool, table, n):
    """Rows [heads][n][D] of one sequence, page by page, in 64 bits."""
    at = 1 if c["layout"] == "head_major" else 0
    rows = torch.cat([pool[int(k)] for k in table[:-(-n // c["page"])]], at)
    return (rows if at else rows.transpose(0, 1))[:, :n].double()


def _exact_sample(c, x):
    n, rows = c["rows"], {"token": [], "logprob": []}
    s = {k: v.double().cpu() for k, v in x["settings"].items()}
    for r in range(n):
        z = x["logits"][r].double()
        if c["guided"]:
            free = x["logits"][n + r].double()
            z = (free + 3.0 * (z - free)).float().double()
        T, k, p, m = (float(s[name][r]) for name in ("temperature", "top_k", "top_p", "min_p"))
        if T == 0:
            rows["token"].append(torch.nonzero(z == z.max())[0, 0])
            rows["logprob"].append(torch.zeros((), dtype=torch.float64, device=DEV))
            continue
        order = torch.argsort(-z, stable=True)
        if k > 0:
            order = order[:int(k)]
        prob = torch.softmax(z[order] / T, 0)
        count = int((prob >= m * prob[0]).sum())
        if p < 1:                                          # as few as reach p
            count = min(count, int((torch.cumsum(prob, 0) < p).sum()) + 1)
        chosen = torch.sort(order[:count])[0]
        final = torch.log_softmax(z[chosen] / T, 0)
        at = int((torch.cumsum(final.exp(), 0) <= x["uniform"][r].double()).sum())
        at = min(at, len(chosen) - 1)
        rows["token"].append(chosen[at])
        rows["logprob"].append(final[at])
    return {"token": torch.stack(rows["token"]).to(torch.int32), "logprob": torch.stack(rows["logprob"])}


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    if c["kind"] == "sample":
        return _exact_sample(c, x)
    h, D, n, G = c["heads"], c["head_dim"], c["n_seq"], c["q_per_kv"]
    hq, dt, P = h * G, _storage(c), c["page"]
    table = x["table"].cpu().numpy()
    if c["kind"] == "append":
        q = _turned(x["q"].unflatten(1, (hq, D)), x["coords"], x["freq"], _pairing(c))
        k = _turned(x["k"].unflatten(1, (h, D)), x["coords"], x["freq"], _pairing(c))
        v = x["v"].unflatten(1, (h, D)).double()
        K, V, at = x["K"].double(), x["V"].double(), 0
        views = [t if c["layout"] == "slot_major" else t.transpose(1, 2) for t in (K, V)]                # [pages][slots][heads][D]
        pos = torch.zeros(n, max(_resident(c)), dtype=torch.int32, device=DEV)
        for b, (past, new) in enumerate(zip(_past(c), _new(c))):
            for page in range(past // P, -(-(past + new) // P)):
                lo, hi = max(past, page * P), min(past + new, (page + 1) * P)
                for view, rows in zip(views, (k, v)):
                    view[int(table[b, page]), lo - page * P:hi - page * P] = rows[at + lo - past:at + hi - past]
            pos[b, :past + new] = torch.arange(past + new, device=DEV)
            at += new
        return {"q": q, "K": K, "V": V, "resident": torch.tensor(_resident(c), dtype=torch.int32, device=DEV), "pos": pos}
    if c["kind"] == "prefill":
        out, lse = torch.empty(x["q"].shape[0], hq, D, dtype=torch.float64, device=DEV), torch.empty(x["q"].shape[0], hq, dtype=torch.float64, device=DEV)
        mass = torch.zeros(n, h, max(_resident(c)), dtype=torch.float64, device=DEV) if c["mass"] else None
        at = 0
        for b, (past, new) in enumerate(zip(_past(c), _new(c))):
            keys = past + new
            K, V = _cached(c, x["K"], table[b], keys), _cached(c, x["V"], table[b], keys)
            dist = (torch.arange(past, keys, device=DEV)[:, None] - torch.arange(keys, device=DEV)[None]).double()
            hidden = dist < 0
            if c["mask"] == "prefix":
                there = torch.arange(keys, device=DEV) < c["prefix"]
                hidden &= ~(there[past:, None] & there[None])
            for j in range(hq):
                z = x["q"][at:at + new, j].double() @ K[j // G].t() / math.sqrt(D)
                if c["cap"]:
                    z = c["cap"] * torch.tanh(z / c["cap"])
                if c["slopes"]:
                    z -= x["slopes"][j].double() * dist.abs()
                z[hidden] = -math.inf
                o, s, p = _attended(z, V[j // G])
                out[at:at + new, j], lse[at:at + new, j] = o, s
                if mass is not None:
                    mass[b, j // G, :keys] += p.sum(0)
            at += new
        return {"out": out, "lse": lse, "mass": mass}
    K, V, score = x["K"].double(), x["V"].double(), x["score"].double()
    if c["kind"] == "attend":
        out, lse = torch.empty(n, hq, D, dtype=torch.float64, device=DEV), torch.empty(n, hq, dtype=torch.float64, device=DEV)
        last = c["resident"] - 1
        for b, count in enumerate(_spread(c["own_lo"], c["own_hi"], n)):
            page, place = int(table[b, last // P]), last % P
            for pool, row in ((K, x["k_new"][b]), (V, x["v_new"][b])):
                view = pool[page] if c["layout"] == "slot_major" else pool[page].transpose(0, 1)
                view[place] = row.to(dt).double()          # (the row as the cache stores it)
            slots = x["idx"][b, :count].long()
            keys, vals = _cached(c, K, table[b], last + 1)[:, slots], _cached(c, V, table[b], last + 1)[:, slots]
            o, s, p = _attended(x["q"][b].double().view(h, G, D) @ keys.transpose(1, 2) / math.sqrt(D), vals)
            out[b], lse[b] = o.reshape(hq, D), s.reshape(hq)
            score[b][:, slots] += p.sum(1)
        return {"out": out, "lse": lse, "K": K, "V": V, "score": score if c["mass"] else None}
    # compact: slot by slot, on the host; ranks as the definition has them, sums in 32 bits in the order of the heads
    pos, sums = x["pos"].cpu().numpy(), x["score"].cpu().numpy()
    rank = sums[:, 0].copy()
    for j in range(1, h):
        rank += sums[:, j]
    first_row = (c["row"] - min(c["rows_back"], c["row"])) * c["grid_w"]
    where, pos_out = np.full(pos.shape, -1, np.int32), pos.copy()
    old_k, old_v, old_score = K.clone(), V.clone(), score.clone()
    for b in range(n):
        rest = [i for i in range(pos.shape[1]) if c["prefix"] <= pos[b, i] < c["prefix"] + first_row]
        best = set(sorted(rest, key=lambda i: (-rank[b, i], i))[:c["budget"]])
        kept = [i for i in range(pos.shape[1]) if i in best or not c["prefix"] <= pos[b, i] < c["prefix"] + first_row]
        where[b, kept] = np.arange(len(kept))
        pos_out[b, :len(kept)] = pos[b, kept]
        score[b, :, :len(kept)] = old_score[b][:, torch.tensor(kept, device=DEV)]
        src, dst = torch.tensor(kept, device=DEV), torch.arange(len(kept), device=DEV)
        t = x["table"][b].long()
        for new, old in ((K, old_k), (V, old_v)):
            if c["layout"] == "slot_major":
                new[t[dst // P], dst % P] = old[t[src // P], src % P]
            else:
                new[t[dst // P], :, dst % P] = old[t[src // P], :, src % P]
    return {"map": torch.from_numpy(where).to(DEV), "resident": torch.full((n,), _kept(c), dtype=torch.int32, device=DEV), "pos": torch.from_numpy(pos_out).to(DEV), "score": score,
            "K": K, "V": V}

"""Several images to each prompt, with the prompts kept once: a small decoder with random weights, one HIP layer batch per layer.

    python examples/shared_prompt.py                       # 4 prompts, 8 images each, bf16
    python examples/shared_prompt.py --dtype f32 --check   # ... and the same images with the prompt in every image's own cache

A step of the loop is what a serving program does around its matrix products:

    prompts:  adsa_append  (rotary positions on the way into the caches)  ->  adsa_prefill (the prompt sees itself whole)
    images:   adsa_rotate  ->  adsa_select  ->  adsa_attend_shared (own list and the group's prompt)  ->  adsa_compact

Rows and columns are the rotary axes of image tokens, text counts along both.  With --check the images are decoded a second time by
adsa_step over caches that hold the prompt themselves, and the logits of the two runs are compared.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2506_18226_amd import binding as B  # noqa: E402
from paper_2506_18226_amd.batch import LayerBatch  # noqa: E402

DEV = "cuda:0"


def int32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Decoder:
    """Embedding, layers of attention and a gated product, logits by the embedding; bf16 or fp32."""

    def __init__(self, layers, heads, q_per_kv, head_dim, vocab, dtype, seed):
        self.h, self.hq, self.D, self.dtype = heads, heads * q_per_kv, head_dim, dtype
        d = self.hq * head_dim
        gen = torch.Generator(device=DEV).manual_seed(seed)

        def w(*shape):
            return (torch.randn(*shape, generator=gen, device=DEV) * shape[0] ** -0.5).to(dtype)

        self.emb = torch.randn(vocab, d, generator=gen, device=DEV).to(dtype)
        self.layers = [dict(qkv=w(d, (self.hq + 2 * heads) * head_dim), out=w(d, d), up=w(d, 2 * d), down=w(d, d)) for _ in range(layers)]
        # half of a row's pairs turn with the image row, half with the column
        n = head_dim // 2
        freq = torch.zeros(2, n, dtype=torch.float64, device=DEV)
        freq[0, :n // 2] = freq[1, n // 2:] = 10000.0 ** (-torch.arange(n // 2, dtype=torch.float64, device=DEV) / (n // 2))
        self.rope = B.make_rope(freq, pairing="neighbours", text=(1, 1), origin=(1, 1), row=(1, 0), col=(0, 1))

    @staticmethod
    def norm(x):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def split(self, x, layer):
        """q, k and v of every token, side by side in one product's rows."""
        qkv = self.norm(x) @ layer["qkv"]
        a, b = self.hq * self.D, (self.hq + self.h) * self.D
        return qkv[:, :a], qkv[:, a:b], qkv[:, b:]

    def rest(self, x, layer, attended):
        x = x + attended.reshape(x.shape) @ layer["out"]
        gate, up = (self.norm(x) @ layer["up"]).chunk(2, -1)
        return x + (torch.nn.functional.silu(gate) * up) @ layer["down"]

    def prompts(self, batches, lens, prompts):
        """The prompts' tokens (packed one behind the other) enter the layers' caches; every token sees its whole prompt."""
        x, T = self.emb[prompts], int(sum(lens))
        begin = torch.cumsum(torch.tensor([0] + list(lens)), 0).to(torch.int32).to(DEV)
        stride = (self.hq + 2 * self.h) * self.D
        tokens = B.make_tokens(begin, torch.zeros(len(lens), dtype=torch.int32, device=DEV), T, max(lens), q_stride=stride, k_stride=stride, v_stride=stride)
        q_rot, out = (torch.empty(T, self.hq, self.D, dtype=self.dtype, device=DEV) for _ in range(2))
        lse, whole = torch.empty(T, self.hq, device=DEV), B.make_mods(mask=B.MASK_PREFIX)
        for layer, batch in zip(self.layers, batches):
            q, k, v = self.split(x, layer)
            batch.append(tokens, self.rope, q, k, v, q_rot, flags=B.FLAG_ADVANCE)
            batch.prefill(tokens, q_rot, out, lse, mods=whole)
            x = self.rest(x, layer, out)

    def step(self, batches, tokens, attend):
        """Logits behind one image token per sequence; attend(number of the layer, q, k, v)."""
        x = self.emb[tokens]
        for i, (layer, batch) in enumerate(zip(self.layers, batches)):
            q, k, v = self.split(x, layer)
            n, stride = len(tokens), q.stride(0)
            qr, kr = (torch.empty(n, heads, self.D, dtype=self.dtype, device=DEV) for heads in (self.hq, self.h))
            batch.rotate(self.rope, q, k, qr, kr, q_stride=stride, k_stride=stride)
            attend(i, qr, kr, v.contiguous())
            x = self.rest(x, layer, batch.out)
        return self.norm(x).float() @ self.emb.float().t()


def run(args):
    dtype = torch.float32 if args.dtype == "f32" else torch.bfloat16
    model = Decoder(args.layers, args.heads, args.q_per_kv, args.head_dim, args.vocab, dtype, args.seed)
    groups, each, W = args.prompts, args.images, args.grid
    n = groups * each
    lens = [args.prompt_len - 3 * g for g in range(groups)]                  # ragged
    gen = torch.Generator().manual_seed(args.seed)
    prompts = [torch.randint(args.vocab, (k,), generator=gen) for k in lens]
    images = torch.randint(args.vocab, (args.steps, n), generator=gen).to(DEV)
    common = dict(n_heads=args.heads, head_dim=args.head_dim, grid_h=W, grid_w=W, win_rows_back=1, win_col_radius=2, q_per_kv=args.q_per_kv,
                  dtype=B.F32 if args.dtype == "f32" else B.BF16, score_mode=B.SCORE_ATTN_MASS)
    own_cap = args.budget + 3 * W

    def caches(n_seq, cap, prefix, step):
        out = []
        for _ in model.layers:
            batch = LayerBatch(B.make_params(n_seq=n_seq, cap=cap, **common), DEV)
            s = batch.seqs_host
            s["grid_origin"] = s["n_keep_prefix"] = prefix
            s["budget"], s["step"] = args.budget, step
            batch.upload_seqs()
            out.append(batch)
        return out

    of_image = [k for k in lens for _ in range(each)]
    # ---- prompts kept once
    kept = caches(groups, max(lens), lens, 0)
    model.prompts(kept, lens, torch.cat(prompts).to(DEV))
    own = caches(n, own_cap, of_image, 1)
    members = int32(*range(0, n + 1, each))
    shared = [B.make_shared(p.params, p.seqs, members, max_members=each) for p in kept]

    def attend_shared(i, q, k, v):
        own[i].select(B.FLAG_PLAN_APPEND)
        own[i].attend_shared(shared[i], q, k, v, flags=B.FLAG_APPEND)
        own[i].compact(B.FLAG_ADVANCE)

    logits, ms = [], 0.0
    for t in range(args.steps):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        out = model.step(own, images[t], attend_shared)
        torch.cuda.synchronize()
        ms += (time.perf_counter() - t0) * 1e3 if t else 0.0                 # (the first step allocates workspaces)
        logits.append(out.cpu())
    for batch in own + kept:
        assert not batch.read_seqs()["status"].any()
    rows = 2 * args.layers * args.heads * args.head_dim * (4 if args.dtype == "f32" else 2)
    result = dict(logits=torch.stack(logits), ms_per_step=ms / max(1, args.steps - 1), cache_mib=rows * (sum(lens) + n * own_cap) / 2 ** 20,
                  cache_mib_whole=rows * (sum(of_image) + n * own_cap) / 2 ** 20)
    print(f"{groups} prompts of up to {max(lens)} tokens, {each} images each, {args.layers} layers: {result['ms_per_step']:.3f} ms a step; "
          f"caches {result['cache_mib']:.1f} MiB, with the prompt in each {result['cache_mib_whole']:.1f}", flush=True)
    if args.check:
        # ---- the prompt in every image's own cache
        whole = caches(n, own_cap + max(lens), of_image, 0)
        model.prompts(whole, of_image, torch.cat([p for p in prompts for _ in range(each)]).to(DEV))
        ref = [model.step(whole, images[t], lambda i, q, k, v: whole[i].step(q, k, v)).cpu() for t in range(args.steps)]
        result["difference"] = float((torch.stack(ref) - result["logits"]).abs().max() / result["logits"].abs().max())
        print(f"largest difference of logits from caches that hold the prompt: {result['difference']:.2e} of the largest logit", flush=True)
    return result


def parser():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("layers", 4), ("heads", 4), ("q_per_kv", 2), ("head_dim", 64), ("vocab", 1024), ("prompts", 4), ("images", 8), ("prompt_len", 120),
                        ("grid", 16), ("steps", 40), ("budget", 24), ("seed", 0)):
        p.add_argument("--" + name.replace("_", "-"), type=int, default=value)
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    p.add_argument("--check", action="store_true")
    return p


if __name__ == "__main__":
    run(parser().parse_args())

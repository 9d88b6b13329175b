"""Prompt calls of a ModelBatch, a layer at a time, give what a LayerBatch of that layer gives, bit by bit."""
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch, ModelBatch

from prompt_common import randn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def int32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_layers_of_a_model_as_batches_of_their_own():
    """Prompts enter, see themselves, and are shared by images that select, attend and evict."""
    layers, groups, each, h, G, D, W, budget = 3, 2, 3, 2, 2, 64, 6, 8
    n, lens = groups * each, [45, 41]
    common = dict(n_heads=h, head_dim=D, grid_h=W, grid_w=W, win_rows_back=1, win_col_radius=2, q_per_kv=G, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS)
    prompt_params, own_params = B.make_params(n_seq=groups, cap=max(lens), **common), B.make_params(n_seq=n, cap=budget + 3 * W, **common)
    gen = torch.Generator().manual_seed(2)
    rope = B.make_rope(torch.rand(2, D // 2, generator=gen, dtype=torch.float64).to(DEV), text=(1, 1), origin=(1, 1), row=(1, 0), col=(0, 1))
    T = sum(lens)
    tokens = B.make_tokens(int32(0, lens[0], T), int32(0, 0), T, max(lens))
    members, whole = int32(0, each, n), B.make_mods(mask=B.MASK_PREFIX)
    bf16 = lambda *s: randn(gen, *s, dtype=torch.bfloat16).to(DEV)
    prompt_in = [[bf16(T, x, D) for x in (h * G, h, h)] for _ in range(layers)]
    steps = [[[bf16(n, x, D) for x in (h * G, h, h)] for _ in range(layers)] for _ in range(2 * W)]

    def fill(seqs, prefixes, step):
        seqs["grid_origin"] = seqs["n_keep_prefix"] = prefixes
        seqs["budget"], seqs["step"] = budget, step

    def buffers(rows):
        return torch.empty(rows, h * G, D, dtype=torch.bfloat16, device=DEV), torch.empty(rows, h, D, dtype=torch.bfloat16, device=DEV), torch.empty(rows, h * G, device=DEV)

    of_image = [x for x in lens for _ in range(each)]
    model_prompts, model = ModelBatch(prompt_params, layers, DEV), ModelBatch(own_params, layers, DEV)
    for layer in range(layers):
        fill(model_prompts.seqs_host[layer * groups:(layer + 1) * groups], lens, 0)
        fill(model.seqs_host[layer * n:(layer + 1) * n], of_image, 1)
    single = []
    for layer in range(layers):
        p, o = LayerBatch(prompt_params, DEV), LayerBatch(own_params, DEV)
        fill(p.seqs_host, lens, 0)
        fill(o.seqs_host, of_image, 1)
        single.append((p, o))
    for batch in (model_prompts, model, *(x for pair in single for x in pair)):
        batch.upload_seqs()
    shared, model_shared = [], []
    for layer, (p, o) in enumerate(single):
        q, k, v = prompt_in[layer]
        (qa, _, la), (qb, _, lb) = buffers(T), buffers(T)
        oa, ob = torch.empty_like(qa), torch.empty_like(qb)
        p.append(tokens, rope, q, k, v, qa, flags=B.FLAG_ADVANCE)
        p.prefill(tokens, qa, oa, la, mods=whole)
        model_prompts.append_layer(layer, tokens, rope, q, k, v, qb, flags=B.FLAG_ADVANCE)
        model_prompts.prefill_layer(layer, tokens, qb, ob, lb, mods=whole)
        assert torch.equal(qa, qb) and torch.equal(oa, ob) and torch.equal(la, lb)
        shared.append(B.make_shared(prompt_params, p.seqs, members, max_members=each))
        model_shared.append(B.make_shared(prompt_params, model_prompts.records(layer), members, max_members=each))
    for at, step in enumerate(steps):
        model.select_all(B.FLAG_PLAN_APPEND)
        for layer, (p, o) in enumerate(single):
            q, k, v = step[layer]
            (qa, ka, _), (qb, kb, _) = buffers(n), buffers(n)
            o.rotate(rope, q, k, qa, ka)
            o.select(B.FLAG_PLAN_APPEND)
            o.attend_shared(shared[layer], qa, ka, v, flags=B.FLAG_APPEND)
            o.compact(B.FLAG_ADVANCE)
            model.rotate_layer(layer, rope, q, k, qb, kb)
            model.attend_shared_layer(layer, model_shared[layer], qb, kb, v, flags=B.FLAG_APPEND)
            assert torch.equal(qa, qb) and torch.equal(ka, kb)
            rows = slice(layer * n, (layer + 1) * n)
            assert torch.equal(o.out, model.out[rows]) and torch.equal(o.lse, model.lse[rows]), (at, layer)
        model.compact_all(B.FLAG_ADVANCE)
    for layer, (p, o) in enumerate(single):
        rows = slice(layer * n, (layer + 1) * n)
        for name in ("K", "V", "pos", "score"):
            assert torch.equal(getattr(o, name), getattr(model, name)[rows]), name
    assert not model.read_seqs()["status"].any() and not model_prompts.read_seqs()["status"].any()


def test_layers_that_are_not_there_are_refused():
    model = ModelBatch(B.make_params(n_seq=1, n_heads=1, head_dim=64, grid_h=4, grid_w=4, win_rows_back=1, win_col_radius=1, dtype=B.F32, score_mode=B.SCORE_ATTN_MASS, cap=40),
                       2, DEV)
    x = torch.zeros(1, 1, 64, device=DEV)
    for layer in (-1, 2):
        for call in (lambda: model.rotate_layer(layer, None, x, x, x, x), lambda: model.append_layer(layer, None, None, x, x, x, x),
                     lambda: model.prefill_layer(layer, None, x, x, x), lambda: model.attend_shared_layer(layer, None, x), lambda: model.records(layer)):
            with pytest.raises(B.AdsaError) as e:
                call()
            assert e.value.code == -1

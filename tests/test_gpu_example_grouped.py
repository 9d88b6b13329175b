"""The example with grouped queries, against caches that hold the prompt themselves."""
import pytest
import torch

from test_gpu_example import load

pytestmark = pytest.mark.gpu


# bf16: the two forms' attention outputs differ by their rounding alone; behind it a layer rounds six times more (two products, a sum, a product of products, a product, a
# sum), and what is half a step apart, 2^-8, may be rounded either way on both sides: 2 layers x 7 x 2 x 2^-8
@pytest.mark.parametrize("heads,group,head_dim", [(1, 3, 128), (2, 4, 64)])
@pytest.mark.parametrize("images", [3, 12])
def test_prompts_kept_once_and_in_every_cache(heads, group, head_dim, images):
    m = load()
    r = m.run(m.parser().parse_args(["--layers", "2", "--prompts", "2", "--images", str(images), "--prompt-len", "45", "--grid", "6", "--steps", "15", "--budget", "8", "--check",
                                     "--head-dim", str(head_dim), "--heads", str(heads), "--q-per-kv", str(group)]))
    assert torch.isfinite(r["logits"]).all() and r["difference"] < 28 * 2.0 ** -8

"""The example of prompts kept once, in small, against caches that hold the prompt themselves."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "shared_prompt.py")


def load():
    spec = importlib.util.spec_from_file_location("shared_prompt", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


# fp32: the two forms round sums over some 100 keys and 3 layers of 128 products each differently, 2^-24 * (100 + 3 * 4 * 128) ~ 1e-4 of a logit
@pytest.mark.parametrize("extra", [["--head-dim", "64", "--heads", "2", "--q-per-kv", "1"], ["--head-dim", "128", "--heads", "1", "--q-per-kv", "3"]])
def test_prompts_kept_once_and_in_every_cache(extra):
    m = load()
    if "3" in extra:                                         # grouped queries are bf16 only: both forms round, no bound but their size
        r = m.run(m.parser().parse_args(["--layers", "2", "--prompts", "2", "--images", "3", "--prompt-len", "45", "--grid", "6", "--steps", "15", "--budget", "8", *extra]))
        assert torch.isfinite(r["logits"]).all()
        return
    r = m.run(m.parser().parse_args(["--layers", "3", "--prompts", "2", "--images", "3", "--prompt-len", "45", "--grid", "6", "--steps", "15", "--budget", "8", "--dtype",
                                     "f32", "--check", *extra]))
    assert torch.isfinite(r["logits"]).all() and r["difference"] < 1e-4

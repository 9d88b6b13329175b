"""Caps whose fp32 constants (their reciprocal times the softmax scale, their multiple by log2 e) are no normal numbers are refused."""
import pytest

from paper_2506_18226_amd import binding as B

from test_prompt_refusals import attend, lib, params, prefill, shared, tokens  # noqa: F401  (lib is a fixture)

SHAPE, WORKSPACE = -2, -6


@pytest.mark.parametrize("softcap,scale,code", [(3e38, 0.0, SHAPE), (2.4e38, 0.0, SHAPE), (1e38, 0.0, SHAPE), (1e-45, 0.0, SHAPE), (1e-39, 1.0, SHAPE), (1e30, 1e-20, SHAPE),
                                                (1e30, 0.0, WORKSPACE), (1e37, 0.0, WORKSPACE), (1e-30, 0.0, WORKSPACE), (50.0, 0.0, WORKSPACE), (0.0, 0.0, WORKSPACE)])
def test_caps(lib, softcap, scale, code):  # noqa: F811
    p, m = params(softmax_scale=scale), B.AdsaMods(softcap=softcap)
    assert prefill(lib, p=p, t=tokens(), m=m, ws=None) == code
    assert attend(lib, p=p, s=shared(), m=m, ws=None) == code

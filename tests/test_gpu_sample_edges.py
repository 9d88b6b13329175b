"""adsa_sample where its numbers end: masked logits of guided pairs, the largest vocabulary, the largest temperatures.  Bounds as in test_gpu_sample."""
import numpy as np
import pytest
import torch

from test_gpu_sample import DEV, INF, NAN, draw, reference, some

pytestmark = pytest.mark.gpu


def check_rows(z, u, got, **settings):
    """z: the logits as the definition has them, fp32 values on the host."""
    token, logprob = got
    T = min(float(np.float32(settings.get("temperature", 1.0))), 1e300)          # (an infinite one: weights of 1, and -infinity / 1e300 stays what it is)
    for r in range(len(z)):
        right, logs = reference(z[r], u[r].item(), T, settings.get("top_k", 0), settings.get("top_p", 1.0), settings.get("min_p", 0.0))
        assert token[r] in right, (r, token[r], right)
        assert any(logprob[r] == x or abs(logprob[r] - x) <= 2.0 ** -24 * abs(x) + len(z[r]) * 2.0 ** -44 + 2.0 ** -46 for x in logs[token[r]]), (r, logprob[r], logs[token[r]])


# ---------------------------------------------------------------------------------------------------- guided pairs
def mixed(c, f, g):
    """The definition: a token that either row masks is masked; guidance 1 is the conditional row alone."""
    if g == 1.0:
        return c
    with np.errstate(invalid="ignore", over="ignore"):
        z = (f.astype(np.float64) + np.float64(np.float32(g)) * (c.astype(np.float64) - f.astype(np.float64))).astype(np.float32)
    return np.where((c == -np.inf) | (f == -np.inf), np.float32(-np.inf), z)


@pytest.mark.parametrize("V", [40, 5003, 70001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("g", [-1.0, 0.0, 0.5, 1.0, 3.0])
@pytest.mark.parametrize("settings", [dict(temperature=0.0), dict(top_k=9), dict(top_p=0.8), dict()])
def test_tokens_that_a_row_of_a_pair_masks(V, dtype, g, settings):
    n = 7
    logits, _ = some(2 * n, V, dtype, V + 3)
    u = torch.tensor([0.0, 0.2, 0.4, 0.6, 0.8, 0.95, 0.5], device=DEV)
    c, f = logits[:n], logits[n:]
    c[0, ::3] = -INF                                         # in the conditional row only
    f[1, ::3] = -INF                                         # in the unconditional row only
    c[2, ::2], f[2, ::2] = -INF, -INF                        # in both
    c[3, :V // 2], f[3, V // 3:] = -INF, -INF                # in one or the other: with most guidances none is left
    c[4, 5:], f[4, 7:] = -INF, -INF
    f[5] = -INF                                              # the whole unconditional row
    c[6, 3], c[6, 4], f[6, 8], f[6, 9] = INF, NAN, INF, NAN
    z = mixed(c.float().cpu().numpy(), f.float().cpu().numpy(), g)
    token, logprob = draw(logits, u, g, **settings)
    assert np.array_equal(token[:n], token[n:])
    check_rows(z, u, (token, logprob), **settings)


# ---------------------------------------------------------------------------------------------------- the largest numbers
@pytest.mark.parametrize("V", [50, 3000, 20000, 70001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1e30, 2e36, 5e37, 1.5e38, 3.4e38, INF])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=40), dict(top_k=3000, top_p=0.7), dict(top_p=0.5), dict(min_p=0.3)])
def test_logits_and_temperatures_as_large_as_there_are(V, dtype, T, settings):
    """What is below the largest by less than 31 temperatures has a weight, also where the distance, or 31 temperatures, pass the largest number."""
    gen = torch.Generator().manual_seed(V)
    logits = ((torch.rand(6, V, generator=gen) * 2 - 1) * 3.38e38).to(dtype)
    logits[1, ::2] = -INF
    logits[2] *= 0.3
    logits[3, 0], logits[3, 1:] = 3.38e38, -3.38e38
    logits[4, :V // 2] = INF
    assert torch.isfinite(logits[0]).all()
    u = torch.tensor([0.1, 0.3, 0.5, 0.7, 0.9, 0.99], device=DEV)
    got = draw(logits.to(DEV), u, temperature=torch.full((6,), T, device=DEV), **settings)
    check_rows(logits.float().numpy(), u, got, **dict(settings, temperature=T))


# ---------------------------------------------------------------------------------------------------- the largest vocabulary
LAST = torch.tensor([0.0, 0.37, 0.99999994], device=DEV if torch.cuda.is_available() else "cpu")


@pytest.mark.parametrize("V", [262144, 262143])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("settings", [dict(), dict(temperature=0.0), dict(top_k=1000), dict(top_k=1024, top_p=0.9), dict(top_k=5000), dict(top_k=200000, top_p=0.8, min_p=0.001), dict(top_p=0.9),
                                      dict(top_p=0.01), dict(top_k=262142), dict(min_p=0.5)])
def test_the_largest_vocabulary(V, dtype, settings):
    """Few candidates and many, and the draw at its ends."""
    logits, _ = some(3, V, dtype, V)
    logits[:, -1] = logits.max()                             # the last index is a candidate, and the last of them
    token, logprob = draw(logits, LAST, **settings)
    check_rows(logits.float().cpu().numpy(), LAST, (token, logprob), **settings)
    if settings.get("temperature", 1.0) > 0:
        assert token[2] == V - 1


@pytest.mark.parametrize("V", [262144, 262143])
@pytest.mark.parametrize("levels", [1, 2, 7])
@pytest.mark.parametrize("settings", [dict(top_k=262142), dict(top_k=37), dict(top_p=0.6), dict(top_k=100000, top_p=0.99), dict()])
def test_ties_in_the_largest_vocabulary(V, levels, settings):
    gen = torch.Generator().manual_seed(levels)
    logits = torch.randint(0, levels, (3, V), generator=gen).float().to(DEV) * 0.5
    check_rows(logits.cpu().numpy(), LAST, draw(logits, LAST, **settings), **settings)


@pytest.mark.parametrize("V", [70001, 262143, 262144])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=50), dict(top_k=6000, top_p=0.9), dict(top_p=0.9), dict(temperature=0.0)])
def test_guided_pairs_of_large_vocabularies(V, dtype, settings):
    """Rows of which most is read again in every pass, both of a pair."""
    logits, _ = some(6, V, dtype, V + 1)
    c, f = (x.float().cpu().numpy() for x in logits.chunk(2))
    token, logprob = draw(logits, LAST, 2.5, **settings)
    assert np.array_equal(token[:3], token[3:])
    check_rows(mixed(c, f, 2.5), LAST, (token, logprob), **settings)

"""adsa_sample against its definition in 64 bits: limits alone and together, ties, odd sizes and rows, guided pairs, settings by row, what is not a number.

Bounds.  A weight is off by 2^-45 of the largest one's (it is a whole number of 2^-44 of it) and, relative to itself, by its polynomial's (ln(2) / 512)^5 / 120 =
2^-54.5 and by two roundings of 1 / T, each 2^-53 of the exponent, which is 31.2 at most: 2^-47; the reference's own quotient is rounded once, 2^-48 the same way.
Together less than 2^-46, so sums over V logits are off by V 2^-45 + 2^-46 of themselves: where a limit or the random number falls closer to a border than twice
that, either side is right (`off`).  logprob is rounded to 32 bits once, and off by the sum's error besides."""
import numpy as np
import pytest
import torch

from paper_2506_18226_amd import binding as B
from paper_2506_18226_amd.batch import LayerBatch, Sampler

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


def reference(z, u, T=1.0, k=0, p=1.0, m=0.0):
    """(tokens that are right, the first of them as the definition has it; logprobs that are right, by token) of one row of logits z (fp32 values)."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    V, top = len(z), z.max()
    if top == -np.inf:
        return [-1], {-1: [-np.inf]}
    if not T > 0:
        t = int(np.argmax(z))
        return [t], {t: [0.0]}
    with np.errstate(invalid="ignore", over="ignore"):
        d = np.where(z == top, 0.0, (z - top) / np.float64(T))
    w = np.exp(d)
    off = V * 2.0 ** -44 + 2.0 ** -45 * w.sum()              # twice a sum's error
    order = np.argsort(-z, kind="stable")
    if 0 < k < V:
        order = order[:k]
    ends = [len(order)]
    if p < 1:
        ws = w[order]
        sums = np.cumsum(ws)
        share = max(float(np.float32(p)), 0.0) * sums[-1]
        ends = [min(int((sums < x).sum()) + 1, len(order)) for x in (share, share - 2 * off, share + 2 * off)]
        if p <= 0:
            ends = [1]
    right, logs = [], {}
    for end in ends:
        chosen = np.sort(order[:end])
        chosen = chosen[w[chosen] >= min(float(np.float32(m)), 1.0)] if m > 0 else chosen
        sums = np.cumsum(w[chosen])
        at = (min(float(u), 1 - 2.0 ** -24) if u >= 0 else 0.0) * sums[-1]
        for x in (at, at - off, at + off):
            t = int(chosen[min(int((sums <= max(x, 0.0)).sum()), len(chosen) - 1)])
            right.append(t)
            logs.setdefault(t, []).append(d[t] - np.log(sums[-1]))
    return list(dict.fromkeys(right)), logs


def draw(logits, u, guidance=None, row_stride=0, seqs=None, stream=None, out=None, **settings):
    rows, V = logits.shape
    n = rows // (1 if guidance is None else 2)
    kind = B.F32 if logits.dtype == torch.float32 else B.BF16
    s = Sampler(n, V, kind, guidance=guidance, row_stride=row_stride, device=DEV, **settings)
    s.token.fill_(-77)
    s.logprob.fill_(-77.0)
    s.sample(logits, u, seqs, stream)
    torch.cuda.synchronize()
    return s.token.cpu().numpy(), s.logprob.cpu().numpy()


def guided(logits, g):
    c, f = logits.float().chunk(2)
    c, f = c.double(), f.double()
    return (f + g * (c - f)).float()


def check(logits, u, guidance=None, ambiguous=0.02, **settings):
    token, logprob = draw(logits, u, guidance, **settings)
    z = (logits.float() if guidance is None else guided(logits.cpu(), float(np.float32(guidance)))).cpu().numpy()
    n, several = len(z), 0
    row = lambda name, r, default: settings[name][r].item() if torch.is_tensor(settings.get(name)) else settings.get(name, default)
    for r in range(n):
        T = float(np.float32(row("temperature", r, 1.0)))
        right, logs = reference(z[r], u[r].item(), T, row("top_k", r, 0), row("top_p", r, 1.0), row("min_p", r, 0.0))
        several += len(right) > 1
        assert token[r] in right, (r, token[r], right)
        wants = logs[token[r]]
        assert any(logprob[r] == x or abs(logprob[r] - x) <= 2.0 ** -24 * abs(x) + len(z[r]) * 2.0 ** -44 + 2.0 ** -46 for x in wants), (r, logprob[r], wants)
    if guidance is not None:
        assert np.array_equal(token[:n], token[n:])
    assert several <= max(1, ambiguous * n)
    return token, logprob


def some(rows, V, dtype=torch.float32, seed=0, scale=2.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, V, generator=gen) * scale).to(dtype).to(DEV), torch.rand(rows, generator=gen).to(DEV)


SIZES = [1, 2, 3, 5, 64, 255, 256, 257, 1000, 1024, 1025, 4096, 4099, 16384, 16387, 32768, 50001, 65536, 70001, 131072]


@pytest.mark.parametrize("V", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("settings", [dict(), dict(temperature=0.0), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.05), dict(temperature=0.7, top_k=100, top_p=0.8, min_p=0.01),
                                      dict(temperature=1.5, top_k=2000, top_p=0.97)])
def test_sizes_and_limits(V, dtype, settings):
    logits, u = some(5, V, dtype, V)
    check(logits, u, **settings)


@pytest.mark.parametrize("V", [7, 1024, 16384, 20001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("g", [1.0, 0.0, 3.0, 7.5, -1.0])
def test_guided_pairs(V, dtype, g):
    logits, u = some(8, V, dtype, V + 1)
    check(logits, u[:4], g, top_k=50)
    check(logits, u[:4], g, top_p=0.9, temperature=0.8)
    check(logits, u[:4], g, temperature=0.0)


@pytest.mark.parametrize("k", [1, 2, 10, 999, 1000, 1001, 5000, -3])
@pytest.mark.parametrize("p", [1.0, 0.5, 0.001, 0.0, -1.0, 1e-30, 0.9999999, 2.0])
def test_limits_at_their_ends(k, p):
    logits, u = some(6, 1000, torch.float32, 4)
    check(logits, u, top_k=k, top_p=p)


@pytest.mark.parametrize("V", [300, 4000, 16384, 100000])
@pytest.mark.parametrize("levels", [1, 2, 7])
@pytest.mark.parametrize("settings", [dict(top_k=37), dict(top_p=0.4), dict(top_k=3000, top_p=0.6), dict(top_k=299, min_p=0.3), dict()])
def test_ties_go_to_the_lowest_index(V, levels, settings):
    """Few different values: a limit falls among many equal logits, and what is in is decided by index."""
    gen = torch.Generator().manual_seed(V + levels)
    logits = torch.randint(0, levels, (6, V), generator=gen).float().to(DEV) * 0.5
    u = torch.tensor([0.0, 0.1, 0.5, 0.9, 0.999, 0.99999994], device=DEV)
    check(logits, u, ambiguous=1.0, **settings)


@pytest.mark.parametrize("V", [4000, 16384, 20001, 70000, 200000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.01, 0.5, 60.0])
@pytest.mark.parametrize("settings", [dict(top_p=0.999, min_p=0.6), dict(top_p=0.3, min_p=0.97), dict(top_k=2500, top_p=0.999, min_p=0.6), dict(top_k=2048, top_p=0.5), dict(top_k=2049, min_p=0.5),
                                      dict(top_p=0.02), dict(min_p=0.9)])
def test_few_and_many_candidates(V, dtype, scale, settings):
    """Flat rows, of which a limit leaves thousands, and steep ones; what min_p asks above and below where top_p ends."""
    logits, u = some(4, V, dtype, V + 5, scale)
    check(logits, u, ambiguous=1.0, **settings)


@pytest.mark.parametrize("V", [300, 16384, 70000])
@pytest.mark.parametrize("T", [0.01, 1.0, 50.0])
@pytest.mark.parametrize("settings", [dict(top_p=0.9), dict(top_k=2), dict(top_p=0.5, min_p=0.1), dict(top_k=50, top_p=0.9), dict()])
def test_rows_of_which_a_mask_leaves_one_or_a_few(V, T, settings):
    gen = torch.Generator().manual_seed(V)
    logits = torch.full((6, V), -INF)
    for r, left in enumerate((1, 2, 3, 1, 600 if V > 600 else 200, 2)):
        at = torch.randperm(V, generator=gen)[:left]
        logits[r, at] = torch.randn(left, generator=gen) if r < 3 else torch.tensor(INF if r == 5 else -3.0)
    u = torch.tensor([0.3, 0.6, 0.95, 0.0, 0.5, 0.7])
    check(logits.to(DEV), u.to(DEV), temperature=T, ambiguous=1.0, **settings)


def test_signed_zeros_are_equal():
    z = torch.zeros(4, 50, device=DEV)
    z[:, ::2] = -0.0
    token, _ = draw(z, torch.tensor([0.0, 0.3, 0.6, 0.99], device=DEV), top_k=3)
    assert list(token) == [0, 0, 1, 2]
    assert list(draw(z, torch.rand(4, device=DEV), temperature=0.0)[0]) == [0] * 4


def test_the_largest_of_several():
    z = torch.randn(7, 9000, device=DEV)
    for r, at in enumerate([0, 1, 4095, 4096, 5000, 8998, 8999]):
        z[r, at:] = torch.where(torch.rand(9000 - at, device=DEV) < 0.01, torch.full((), 50.0, device=DEV), z[r, at:])
        z[r, at] = 50.0
    token, logprob = draw(z, torch.rand(7, device=DEV), temperature=0.0)
    assert list(token) == [0, 1, 4095, 4096, 5000, 8998, 8999] and not logprob.any()


@pytest.mark.parametrize("V", [40, 5000, 70000])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=9), dict(top_p=0.7), dict(top_k=4000, top_p=0.5), dict(temperature=0.0), dict(min_p=0.2)])
def test_masked_infinite_and_not_numbers(V, settings):
    logits, u = some(9, V, torch.float32, 8)
    logits[0] = -INF
    logits[1] = NAN
    logits[2, 3:] = -INF                                     # three left
    logits[3, : V - 1] = torch.finfo(torch.float32).min     # one left, masked by the lowest value
    logits[4, ::2] = NAN
    logits[5, [5, 9, 30]] = INF                              # only these
    logits[6, 1:] = -INF
    logits[7] = torch.finfo(torch.float32).min               # all alike
    logits[8, ::3] = -1e30
    check(logits, u, ambiguous=1.0, **settings)


@pytest.mark.parametrize("T", [1e-42, 1e-30, 1e-3, 0.05, 30.0, 1e10, 3e38])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=40), dict(top_p=0.5)])
def test_temperatures(T, settings):
    logits, u = some(6, 3000, torch.float32, 3)
    check(logits, u, ambiguous=1.0, temperature=T, **settings)


def test_random_numbers_at_their_ends():
    logits, _ = some(7, 2000, torch.float32, 3)
    u = torch.tensor([0.0, -1.0, NAN, 1.0, 5.0, 0.99999994, INF], device=DEV)
    token, _ = draw(logits, u, top_k=20)
    for r in range(7):
        best = np.sort(np.argsort(-logits[r].cpu().numpy(), kind="stable")[:20])
        assert token[r] == best[0 if r < 3 else -1], r


@pytest.mark.parametrize("V", [500, 16384])
def test_settings_by_row(V):
    rows = 60
    logits, u = some(rows, V, torch.bfloat16, 5)
    rng = np.random.default_rng(2)
    T = torch.tensor(rng.choice([0.0, 0.5, 1.0, 1.5], rows), dtype=torch.float32)
    k = torch.tensor(rng.choice([0, 1, 20, 400, V, -5], rows), dtype=torch.int32)
    p = torch.tensor(rng.choice([1.0, 0.9, 0.3, 0.0, 1.5], rows), dtype=torch.float32)
    m = torch.tensor(rng.choice([0.0, 0.01, 0.5, 2.0], rows), dtype=torch.float32)
    check(logits, u, temperature=T.to(DEV), top_k=k.to(DEV), top_p=p.to(DEV), min_p=m.to(DEV))
    # what cannot be, on the device
    T[:3], p[3:5], m[5:7] = torch.tensor([-1.0, NAN, -INF]), NAN, NAN
    token, _ = draw(logits, u, temperature=T.to(DEV), top_k=0, top_p=p.to(DEV), min_p=m.to(DEV))
    z = logits.float().cpu().numpy()
    for r in range(3):
        assert token[r] == np.argmax(z[r])
    for r in range(3, 7):
        right, _ = reference(z[r], u[r].item(), float(T[r]), 0, 1.0 if r < 5 else float(p[r]), 0.0 if r >= 5 else float(m[r]))
        assert token[r] in right


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,stride,offset", [(1000, 1001, 1), (1000, 1003, 3), (4096, 5000, 2), (20000, 20002, 0), (70000, 70004, 1)])
def test_rows_of_a_wider_tensor(dtype, V, stride, offset):
    wide, u = some(6, stride, dtype, 9)
    logits = wide.reshape(-1)[offset:]
    logits = logits.as_strided((5, V), (stride, 1))
    a = draw(logits, u[:5], row_stride=stride, top_p=0.9)
    b = draw(logits.contiguous(), u[:5], top_p=0.9)
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_sequences_that_are_not_active_get_no_token():
    p = B.make_params(n_seq=8, n_heads=1, head_dim=64, grid_h=4, grid_w=4, win_rows_back=1, win_col_radius=1, dtype=B.BF16, score_mode=B.SCORE_ATTN_MASS, cap=16)
    batch = LayerBatch(p, DEV)
    batch.seqs_host["step"] = [1, -1, 2, 3, 1, 1, 2, 3]
    batch.seqs_host["status"] = [0, 0, B.SEQ_CACHE_FULL, 0, 0, 0, 0, B.SEQ_BAD_STATE]
    batch.upload_seqs()
    logits, u = some(8, 700, torch.float32, 1)
    every = draw(logits, u)[0]
    token, logprob = draw(logits, u, seqs=batch.seqs)
    off = [1, 2, 7]
    assert all(token[r] == -1 and logprob[r] == 0 for r in off) and all(token[r] == every[r] for r in range(8) if r not in off)
    pairs = draw(logits, u[:4], 2.0)[0]
    token, _ = draw(logits, u[:4], 2.0, seqs=batch.seqs)     # a pair goes by its conditional row
    assert list(token) == [pairs[0], -1, -1, pairs[3]] * 2


def test_shares_of_many_draws():
    """The random numbers of a grid: every candidate gets its share of them, to one either way."""
    gen = torch.Generator().manual_seed(1)
    row = torch.randn(300, generator=gen) * 2
    n = 20000
    logits = row.expand(n, 300).contiguous().to(DEV)
    u = ((torch.arange(n) + 0.5) / n).to(torch.float32).to(DEV)
    token, logprob = draw(logits, u, top_k=25)
    z = row.double().numpy()
    best = np.argsort(-z, kind="stable")[:25]
    w = np.zeros(300)
    w[best] = np.exp(z[best])
    w /= w.sum()
    count = np.bincount(token, minlength=300)
    assert (np.abs(count - n * w) <= 1 + n * 2.0 ** -23).all() and (np.diff(token) >= 0).all()


def test_streams_and_graphs():
    logits, u = some(6, 16384, torch.bfloat16, 2)
    kw = dict(top_k=300, top_p=0.9)
    want = draw(logits, u, **kw)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = draw(logits, u, stream=other, **kw)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    s = Sampler(6, 16384, B.BF16, device=DEV, **kw)
    x, v = torch.zeros_like(logits), torch.zeros_like(u)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.sample(x, v)
    for seed in range(4):
        a, b = some(6, 16384, torch.bfloat16, 20 + seed)
        want = draw(a, b, **kw)
        x.copy_(a)
        v.copy_(b)
        s.token.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(s.token.cpu().numpy(), want[0]) and np.array_equal(s.logprob.cpu().numpy(), want[1])

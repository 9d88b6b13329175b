"""Plain implementations, in 64 bits on the host, of what the prompt side computes, with the error that the kernels' roundings allow.

Bounds.  u = 2^-24 (half a step of fp32).  A score q.k over D products and its scaling is off by at most (D + 4) u sum|q_i k_i| * scale; the cap
passes errors on undiminished at most and adds 4 u * 2 cap of its own (tanh as 1 - 2 / (e + 1): three roundings of numbers below 2), the
distance 2 u * slope * distance.  With scores off by d, a probability is off by the factor 1 +- (2 d + 32 u): the scores' own errors in numerator and sum,
the hardware's exp2 and log2, sums and weights.  A bf16 cache has probabilities rounded by 2^-9 (half a step is 2^-8 of the value, and rounds a sum's
terms either way: 2^-8 is taken whole) and the result rounded by 2^-8 of itself."""
import numpy as np
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def randn(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype)


def f64(x):
    return x.detach().cpu().double().numpy()


def turned(x, angle, pairing):
    """Rows x [T][heads][D] turned by angle [T][D/2], and the bound of fp32 arithmetic: sine and cosine within 4 u, two products and a sum."""
    n = x.shape[-1] // 2
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = (x[..., :n], x[..., n:]) if pairing == "halves" else (x[..., 0::2], x[..., 1::2])
    ya, yb, size = a * c - b * s, b * c + a * s, 8 * U * (np.abs(a) + np.abs(b))
    if pairing == "halves":
        return np.concatenate([ya, yb], -1), np.concatenate([size, size], -1)
    return np.stack([ya, yb], -1).reshape(x.shape), np.stack([size, size], -1).reshape(x.shape)


def attended(q, k, v, scale, *, seen=None, cap=0.0, slope=0.0, dist=None, bf16=False):
    """One query head: q [n][D], keys k, v [m][D], seen [n][m].  Returns out, lse, p, and bounds of out, lse and (relative) of p."""
    n, m = q.shape[0], k.shape[0]
    if m == 0:
        return np.zeros((n, v.shape[1])), np.full(n, -np.inf), np.zeros((n, 0)), np.zeros((n, v.shape[1])), np.zeros(n), np.zeros((n, 0))
    seen = np.ones((n, m), bool) if seen is None else seen
    with np.errstate(invalid="ignore", over="ignore"):
        z = q @ k.T * scale
        d = (q.shape[1] + 4) * U * (np.abs(q) @ np.abs(k).T) * scale
        if cap:
            z, d = cap * np.tanh(z / cap), d + 8 * U * cap
        if slope:
            z, d = z - slope * np.abs(dist), d + 4 * U * slope * np.abs(dist)
    z, d = np.where(seen, z, -np.inf), np.where(seen, d, 0.0)
    top = z.max(1, keepdims=True)
    e = np.exp(z - np.where(np.isinf(top), 0.0, top))
    l = e.sum(1, keepdims=True)
    p = np.divide(e, l, out=np.zeros_like(e), where=l > 0)
    with np.errstate(divide="ignore"):
        lse = np.where(l[:, 0] > 0, np.where(np.isinf(top[:, 0]), 0.0, top[:, 0]) + np.log(l[:, 0]), -np.inf)
    worst = d.max(1)
    rel = 2 * worst + 32 * U
    vv = np.where(seen.any(0)[:, None], v, 0.0)              # (a value that nobody sees may be anything)
    out = p @ vv
    size = p @ np.abs(vv)
    tol = (rel[:, None] + (2.0 ** -8 if bf16 else 0.0)) * size + (2.0 ** -8 if bf16 else U) * np.abs(out) + 1e-30
    return out, lse, p, tol, worst + 32 * U * (1 + np.abs(np.where(np.isinf(lse), 0.0, lse))), np.broadcast_to(rel[:, None], p.shape)


def close(got, want, tol, what=""):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    err = np.abs(got[~inf] - want[~inf])
    tol = np.broadcast_to(tol, want.shape)[~inf]
    assert not np.isnan(err).any(), (what, "NaN")
    assert (err <= tol).all(), (what, float(err.max()), float((err / np.maximum(tol, 1e-300)).max()))

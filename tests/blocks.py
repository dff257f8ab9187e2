"""The feed-forward operators over row groups in 64 bits, from their definitions, and how far the library's results
may be from them.

Error bounds are per element and follow the library's documented roundings: every stored bf16 value is off by at
most BF = 2^-8 of itself (half a step), a product of depth n summed in fp32 by n * 2 * 2^-24 of the sum of its
terms' magnitudes (twice the usual bound: the order of a matrix instruction's additions is its own), and the
activation by a few fp32 roundings, of which the exponential's argument is the largest."""
import math

import numpy as np

BF = 2.0 ** -8
F32 = 2.0 ** -24
ATOL = 1e-30  # what a flushed exponential can lose


def running_offsets(off, T, G):
    """Offsets as the library reads them: the running maximum of the offsets clamped to [0, T]."""
    if off is None:
        return np.array([0, T])
    return np.maximum.accumulate(np.clip(np.asarray(off, np.int64), 0, T))


def act(v, name):
    """(activation, derivative, fp32 error of each) of a float64 array."""
    if name == "silu":
        z, dz = v, np.ones_like(v)
    else:
        c = 2.0 * math.sqrt(2.0 / math.pi)
        z, dz = c * (v + 0.044715 * v ** 3), c * (1.0 + 3 * 0.044715 * v ** 2)
    with np.errstate(over="ignore"):
        s = 1.0 / (1.0 + np.exp(-z))
    t = s * (1.0 - s)
    a, da = v * s, s + v * t * dz
    # relative errors: of s (6 |z| + 8) roundings, of t the same and those of 1 - s (s rounded: 2^-24 of 1)
    rel = (6 * np.abs(z) + 8) * F32
    return a, da, rel * np.abs(a), (rel + 8 * F32) * (np.abs(s) + np.abs(v * t * dz)) + np.abs(v * dz * s) * 4 * F32


def forward(x, off, w1, w3, w2, name, rows):
    """y, gate, up and their bounds; NaN in rows of no group (bounds 0)."""
    T, H = x.shape
    G, _, F = w1.shape
    y, gate, up = np.full((T, H), np.nan), np.full((T, F), np.nan), np.full((T, F), np.nan)
    by, bg, bu = np.zeros((T, H)), np.zeros((T, F)), np.zeros((T, F))
    o = running_offsets(off, T, G)
    for g in range(G):
        r = slice(o[g], o[g + 1])
        if o[g + 1] <= o[g]:
            continue
        X = x[r]
        gate[r], up[r] = X @ w1[g], X @ w3[g]
        eg, eu = 2 * H * F32 * (np.abs(X) @ np.abs(w1[g])), 2 * H * F32 * (np.abs(X) @ np.abs(w3[g]))
        a, da, ea, _ = act(gate[r], name)
        h = a * up[r]
        # activations have slopes of at most 1.13
        eh = BF * np.abs(h) + (ea + 1.13 * eg) * (np.abs(up[r]) + eu) + np.abs(a) * eu + 4 * F32 * np.abs(h)
        y[r] = h @ w2[g]
        by[r] = BF * np.abs(y[r]) + (eh + 2 * F * F32 * np.abs(h)) @ np.abs(w2[g]) * (1 + BF) + ATOL
        bg[r], bu[r] = BF * np.abs(gate[r]) + eg * (1 + BF) + ATOL, BF * np.abs(up[r]) + eu * (1 + BF) + ATOL
    return (y, gate, up), (by, bg, bu)


def backward(dy, x, off, w1, w3, w2, gate, up, name):
    """dx (NaN in rows of no group), dw1, dw3, dw2 and their bounds."""
    T, H = x.shape
    G, _, F = w1.shape
    out = [np.full((T, H), np.nan), np.zeros((G, H, F)), np.zeros((G, H, F)), np.zeros((G, F, H))]
    bound = [np.zeros_like(v) for v in out]
    o = running_offsets(off, T, G)
    for g in range(G):
        r = slice(o[g], o[g + 1])
        n = o[g + 1] - o[g]
        if n <= 0:
            continue
        D, X, U = dy[r], x[r], up[r]
        a, da, ea, eda = act(gate[r], name)
        dh = D @ w2[g].T
        edh = 2 * H * F32 * (np.abs(D) @ np.abs(w2[g].T))
        h, dg, du = a * U, dh * U * da, dh * a
        eh = BF * np.abs(h) + ea * np.abs(U) + 4 * F32 * np.abs(h)
        edg = BF * np.abs(dg) + (1 + BF) * (edh * np.abs(U * da) + (np.abs(dh) + edh) * np.abs(U) * eda) + 4 * F32 * np.abs(dg)
        edu = BF * np.abs(du) + (1 + BF) * (edh * np.abs(a) + (np.abs(dh) + edh) * ea) + 4 * F32 * np.abs(du)
        out[0][r] = dg @ w1[g].T + du @ w3[g].T
        out[1][g], out[2][g], out[3][g] = X.T @ dg, X.T @ du, h.T @ D
        k = 4 * F * F32
        bound[0][r] = (edg + k * np.abs(dg)) @ np.abs(w1[g].T) + (edu + k * np.abs(du)) @ np.abs(w3[g].T)
        k = 2 * n * F32
        bound[1][g], bound[2][g] = np.abs(X.T) @ (edg + k * np.abs(dg)), np.abs(X.T) @ (edu + k * np.abs(du))
        bound[3][g] = (eh + k * np.abs(h)).T @ np.abs(D)
    return out, [b * (1 + BF) + BF * np.abs(np.nan_to_num(v)) + ATOL for v, b in zip(out, bound)]


def quantize_rows(x):
    """x fp32 -> (q int8, scale fp32): the definition in IEEE fp32 divisions."""
    x = np.asarray(x, np.float32)
    amax = np.max(np.abs(x), axis=-1)
    ok = np.isfinite(amax)
    scale = np.where(ok, amax / np.float32(127), np.float32("nan")).astype(np.float32)
    with np.errstate(all="ignore"):
        q = np.rint(x / scale[..., None])
    q = np.where((scale > 0)[..., None], np.clip(q, -127, 127), 0)
    return q.astype(np.int8), scale


def gemm_i8(xq, sx, off, wq, sw, name):
    """y and its bound; NaN in rows of no group (bound 0)."""
    T, K = xq.shape
    G, N, _ = wq.shape
    out = N if name == "none" else N // 2
    y, by = np.full((T, out), np.nan), np.zeros((T, out))
    o = running_offsets(off, T, G)
    for g in range(G):
        r = slice(o[g], o[g + 1])
        if o[g + 1] <= o[g]:
            continue
        # (float64 products of whole numbers below 2^53 are exact)
        v = (xq[r].astype(np.float64) @ wq[g].astype(np.float64).T) * sx[r, None].astype(np.float64) * sw[g].astype(np.float64)
        ev = 3 * F32 * np.abs(v)
        if name == "none":
            y[r], by[r] = v, BF * np.abs(v) + (1 + BF) * ev + ATOL
        else:
            a, _, ea, _ = act(v[:, :out], name)
            u = v[:, out:]
            y[r] = a * u
            by[r] = BF * np.abs(y[r]) + (1 + BF) * ((ea + 1.13 * ev[:, :out]) * np.abs(u) * (1 + 4 * F32) + np.abs(a) * ev[:, out:]) \
                + 4 * F32 * np.abs(y[r]) + ATOL
    return y, by


def check(name, got, ref, bound):
    """got float64; where ref is NaN nothing is said."""
    some = ~np.isnan(ref)
    assert not np.isnan(got[some]).any(), f"{name}: NaN"
    far = np.abs(got[some] - ref[some]) - bound[some]
    assert far.size == 0 or far.max() <= 0, f"{name}: {int((far > 0).sum())} of {far.size} beyond the bound, by up to {far.max():.3g}"


def norms(name, got, ref, whole=4e-3, line=6.5e-3):
    """2-norms of got - ref against those of ref: of the whole matrix, and of every row, column and 32 x 64 block of it.

    A stored value is rounded by up to 2^-8 of itself, evenly: 2^-8 / sqrt(3) = 2.3e-3 of a norm at most.  Results are
    rounded once and the rounded factors of their sums once, independently: sqrt(2) times that, 3.2e-3.  A line can
    be the multiple of one rounded factor: 2^-8 of it and 2.3e-3.  fp32 sums add less than 1e-4 of the mean line.  A
    part p of a sum's depth that is lost is sqrt(p) of the norm: 3e-2 for 32 of 32768.
    The factors' roundings are 2^-8 / sqrt(3) of the root of the terms' squares, which a line's own norm is on average
    but may fall below: of n values with a spread of chi^2 over n, n = 32 by a factor of 0.55 once in 20000, and 2.3e-3 /
    0.55 and 2.3e-3 together are still 4.8e-3; one value alone may cancel to nothing.  So lines of fewer than 32 values
    are left to the bounds of single values."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    if got.ndim == 3:
        for g, r in zip(got, ref):
            norms(name, g, r, whole, line)
        return
    some = ~np.isnan(ref).any(1)
    got, ref = got[some], ref[some]
    if not ref.size:
        return
    e, r = (got - ref) ** 2, ref ** 2
    assert e.sum() <= whole ** 2 * r.sum(), f"{name}: off by {math.sqrt(e.sum() / r.sum()):.2e} of its norm"
    i, j = np.arange(0, ref.shape[0], 32), np.arange(0, ref.shape[1], 64)
    blocks = [np.add.reduceat(np.add.reduceat(v, i, 0), j, 1) for v in (e, r)]
    size = np.minimum(32, ref.shape[0] - i)[:, None] * np.minimum(64, ref.shape[1] - j)
    for what, a, b, n in (("row", e.sum(1), r.sum(1), ref.shape[1]), ("column", e.sum(0), r.sum(0), ref.shape[0]),
                          ("block", *blocks, size)):
        if np.max(n) < 32:
            continue
        a = np.where(np.asarray(n) < 32, 0.0, a)
        far = np.sqrt(a) - line * np.sqrt(b) - 1e-4 * math.sqrt(b.mean())
        assert far.max() <= 0, f"{name}: {what} {np.unravel_index(far.argmax(), far.shape)} is off by " \
            f"{math.sqrt(a.flat[far.argmax()] / max(b.flat[far.argmax()], 1e-300)):.2e} of its norm"

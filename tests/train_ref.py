"""The norm, the gate, the routing's losses and the optimizer's step in 64 bits, from their definitions, and how far
the library's results may be from them.

Bounds are per element.  F32 = 2^-24 is half a step of fp32 (a rounding), BF = 2^-8 half a step of bf16.  Sums of
positive terms are off by their number of additions in a chain, other sums by that many times the sum of the terms'
magnitudes."""
import numpy as np

from tests.blocks import BF, F32

TINY = 2.0 ** -133  # half a step of a subnormal bf16


def bf16(v):
    """fp32 values rounded to bf16, to the nearest, halves to even."""
    u = np.asarray(v, np.float32).view(np.uint32)
    r = (u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)
    return np.where(np.isnan(v), np.float32(np.nan), r.view(np.float32))


def offsets(off, S, T):
    """Offsets as the library reads them."""
    return np.array([0, T]) if off is None else np.maximum.accumulate(np.clip(np.asarray(off, np.int64), 0, T))


# ---- norm: a thread adds at most 64 squares, then 8 folds and 4 wavefronts: 80 roundings of a positive sum -------------
CHAIN = 80


def norm(x, residual, w, eps):
    """(s, rstd, y, scale) from bf16 values in float32, s as it is kept."""
    s = x if residual is None else bf16(x.astype(np.float32) + residual.astype(np.float32))
    v = s.astype(np.float64)
    r = 1.0 / np.sqrt((v * v).mean(1) + eps)
    y = v * w.astype(np.float64) * r[:, None]
    return s, r, y, np.abs(y).max(1) / 127.0


RSTD = (CHAIN / 2 + 4) * F32   # relative: half of the sum's, and division, addition, root and reciprocal
Y = RSTD + 2 * F32             # before the rounding to bf16
SCALE = Y + 2 * F32


def norm_grad(dy, dsum, s, w, r):
    """dx, its bound, dweight, its bound, from float64 arrays."""
    H = s.shape[1]
    n, g = s * r[:, None], dy * w
    t = g * n
    c, size = t.mean(1, keepdims=True), np.abs(t).mean(1, keepdims=True)
    dx = r[:, None] * (g - n * c)
    err = np.abs(r[:, None]) * (4 * F32 * (np.abs(g) + np.abs(n * c)) + np.abs(n) * (CHAIN + 6) * F32 * size)
    if dsum is not None:
        err = err + 2 * F32 * (np.abs(dsum) + np.abs(dx))
        dx = dx + dsum
    dw, many = dy * n, s.shape[0] + 16
    return dx, err + BF * (np.abs(dx) + err) + TINY, dw.sum(0), many * F32 * np.abs(dw).sum(0) + 1e-37


# ---- gate: products of bf16 values are exact in fp32, a sum of depth n is off by 2 n roundings of the magnitudes' --------
def gate_logits(x, wg, bias):
    l = x @ wg + bias
    return l, 2 * x.shape[1] * F32 * (np.abs(x) @ np.abs(wg)) + 2 * F32 * (np.abs(l) + np.abs(bias))


def gate_grad(dl32, x, wg):
    """dx, dwg, dbias and their bounds from fp32 dlogits, which the products take in bf16."""
    d = bf16(dl32).astype(np.float64)
    dx, dwg, db = d @ wg.T, x.T @ d, dl32.astype(np.float64).sum(0)
    T, E = d.shape
    ex = 2 * E * F32 * (np.abs(d) @ np.abs(wg).T)
    ew = 2 * T * F32 * (np.abs(x).T @ np.abs(d))
    return (dx, ex + BF * (np.abs(dx) + ex) + TINY), (dwg, ew + BF * (np.abs(dwg) + ew) + TINY), \
        (db, 2 * T * F32 * np.abs(dl32.astype(np.float64)).sum(0) + 1e-37)


# ---- losses ---------------------------------------------------------------------------------------------------------
def softmax(l):
    """p and lse of float64 logits; rows of -inf alone have p = 0."""
    with np.errstate(invalid="ignore", divide="ignore"):
        top = l.max(1, keepdims=True)
        top = np.where(np.isneginf(top), 0.0, top)
        e = np.exp(l - top)
        total = e.sum(1, keepdims=True)
        return np.where(total > 0, e / total, np.where(np.isnan(total), np.nan, 0.0)), (np.log(total) + top)[:, 0]


# lse: exp(x) by 2^(x log2 e) is off by 2 |x| + 2 roundings of itself (the difference's, the product's and the
# hardware's), e^-x x weighs at most 8 for 512 logits, 16 additions; the logarithm and its sum
def lse_bound(lse):
    return (2 * 8 + 2 + 16 + 16) * F32 + 4 * F32 * np.abs(lse)


def loss(l, idx, off, E, k):
    """counts, lse, (balance, z), relative bound of balance and bound of z."""
    p, lse = softmax(l)
    S = len(off) - 1
    counts = np.zeros((S, E), np.int64)
    parts, N = [], off[-1] - off[0]
    for s in range(S):
        a, b = off[s], off[s + 1]
        if b == a:
            continue
        chosen = idx[a:b].ravel()
        counts[s] = np.bincount(chosen[(chosen >= 0) & (chosen < E)], minlength=E)
        parts.append(E / (k * (b - a) ** 2) * (counts[s] * p[a:b].sum(0)).sum())
    some = lse[off[0]:off[-1]]
    some = np.where(np.isneginf(some), 0.0, some)
    z = (some ** 2).mean() if N else 0.0
    zb = (2 * np.abs(some) * lse_bound(some)).mean() + (N + 8) * F32 * z if N else 0.0
    return counts, lse, (np.mean(parts) if parts else 0.0, z), (N + 300) * F32, zb + 1e-37


def loss_grad(l, idx, w, off, counts, lse, dloss, dw, E, k):
    """dlogits and its bound, on the rows of the sequences; lse, w and dw as they are given."""
    T = len(l)
    d, err = np.zeros((T, E)), np.zeros((T, E))
    live, N = sum(b > a for a, b in zip(off, off[1:])), off[-1] - off[0]
    for s, (a, b) in enumerate(zip(off, off[1:])):
        if b == a:
            continue
        dead = np.isneginf(lse[a:b])[:, None]
        with np.errstate(invalid="ignore"):
            arg = l[a:b] - lse[a:b, None]
            p = np.where(dead, 0.0, np.exp(arg))
            far = np.where(p > 0, 2 * np.abs(arg) + 4, 0.0) * F32
            zl = np.where(dead, 0.0, dloss[1] * 2.0 / N * lse[a:b, None])
        c = dloss[0] * E / (k * (b - a) ** 2 * live) * counts[s].astype(np.float64)
        dot = (c * p).sum(1, keepdims=True)
        edot = (np.abs(c) * p * (far + 26 * F32)).sum(1, keepdims=True)
        v = p * (c - dot + zl)
        d[a:b] = v
        err[a:b] = p * far * np.abs(c - dot + zl) + p * (8 * F32 * np.abs(c) + edot + 4 * F32 * np.abs(dot) + 8 * F32 * np.abs(zl)) \
            + 4 * F32 * np.abs(v)
    if dw is not None:
        t = w * (dw - (w * dw).sum(1, keepdims=True))
        et = (k + 6) * F32 * np.abs(w) * (np.abs(dw) + np.abs(w * dw).sum(1, keepdims=True))
        for row in range(off[0], off[-1]):
            for j in range(k):
                if 0 <= idx[row, j] < E:
                    d[row, idx[row, j]] += t[row, j]
                    err[row, idx[row, j]] += et[row, j] + 2 * F32 * np.abs(t[row, j])
        err[off[0]:off[-1]] += 2 * F32 * np.abs(d[off[0]:off[-1]])
    return d, err + 1e-37


# ---- AdamW ------------------------------------------------------------------------------------------------------------
M32 = 0xFFFFFFFF


def mixed(h):
    h = ((h ^ (h >> 16)) * 0x761BCE4B) & M32
    h = ((h ^ (h >> 15)) * 0xA0D73955) & M32
    return h ^ (h >> 16)


def random_bits(seed, step, place, n, first=0):
    """(16 bits for m, 16 for v, 16 for the weight) of values first .. first + n of a tensor."""
    key = mixed((mixed((seed + step * 0xD22CD251) & M32) + place * 0xA5375919) & M32)
    out = np.empty((3, n), np.uint64)
    i = np.arange(first, first + n, dtype=np.uint64)
    m = np.uint64(M32)
    h = (np.uint64(key) + (i & m) * np.uint64(0x946BAFCD) + (i >> np.uint64(32)) * np.uint64(0x8952E2D3)) & m
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x761BCE4B)) & m
    h = ((h ^ (h >> np.uint64(15))) * np.uint64(0xA0D73955)) & m
    h = h ^ (h >> np.uint64(16))
    out[0], out[1], out[2] = h & np.uint64(0xFFFF), h >> np.uint64(16), ((h * np.uint64(0x761BCE4B)) & m) >> np.uint64(16)
    return out


def block_max(v):
    n = len(v)
    full = np.zeros(-(-n // 256) * 256)
    full[:n] = np.abs(v)
    return full.reshape(-1, 256).max(1)


def rounded_at_random(v, scale, u, bits, least, most, above_zero):
    """Values of a format with `bits` bits of mantissa times their block's scale: (value, step) with v's sign."""
    s = np.repeat(scale, 256)[:len(v)]
    x = np.where(s > 0, np.abs(v) / np.where(s > 0, s, 1.0), 0.0)
    e = np.maximum(np.frexp(x)[1] - 1, least)
    unit = np.ldexp(1.0, e - bits)
    steps = np.floor(x / unit + u.astype(np.float64) / 65536.0)
    if above_zero:
        steps = np.where((np.abs(v) > 0) & (s > 0), np.maximum(steps, 1.0), steps)
    return np.copysign(np.minimum(steps * unit, most), v), unit


def adamw(w, g, m, v, cfg, decay):
    """The new (w, m, v) in float64 and their bounds before any rounding to fewer bits; cfg: a dict."""
    b1, b2 = float(cfg["beta1"]), float(cfg["beta2"])
    t = float(cfg["step"])
    c1, c2 = -np.expm1(t * np.log(b1)) if b1 else 1.0, -np.expm1(t * np.log(b2)) if b2 else 1.0
    g = g * float(cfg["grad_scale"])
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    em = 5 * F32 * (np.abs(b1 * m) + np.abs((1 - b1) * g)) + 2.0 ** -148
    ev = 7 * F32 * (np.abs(b2 * v) + (1 - b2) * g * g) + 2.0 ** -148
    root = np.sqrt(v1 / c2)
    den = root + float(cfg["eps"])
    u = m1 / c1 / den
    # the corrections (8 roundings each), the root and its argument's error (never more than the root itself), quotients
    eroot = np.minimum(ev / c2, root * root + ev / c2) / np.maximum(root, np.sqrt(ev / c2)) + 8 * F32 * root
    eu = em / c1 / den + np.abs(u) * (16 * F32 + eroot / den)
    w1 = w - float(cfg["lr"]) * (decay * w + u)
    ew = 4 * F32 * np.abs(w) + float(cfg["lr"]) * (eu + 8 * F32 * np.abs(u) + 8 * F32 * decay * np.abs(w)) + F32 * np.abs(w1)
    return (w1, ew + 1e-40), (m1, em), (v1, ev)

"""CPU oracle for the layers of a decoder block: masked attention, rotary positions, the gated layer, dropout.

TEST INFRASTRUCTURE ONLY: plain float64 statements of what the CUDA library computes, sharing no code with it, and beside each result a
bound of its error, formed from the roundings that the library's formats cannot avoid:

    U = 2^-8   half a step of bf16,     E = 2^-24   half a step of fp32

Bounds are sums of absolute values: every rounding is taken at its worst and none cancels.
"""
from __future__ import annotations

import numpy as np

U, E = 2.0 ** -8, 2.0 ** -24


# ------------------------------------------------------------------------------------------ attention
def visible(M, begin, causal, prefix):
    """[M x M]: row i sees key j."""
    see = np.zeros((M, M), dtype=bool)
    for q in range(len(begin) - 1):
        b, e = (min(max(int(v), 0), M) for v in begin[q:q + 2])
        for i in range(b, e):
            last = e
            if causal:
                last = min(e, max(i + 1, b + max(int(prefix[q]), 0) if prefix is not None else 0))
            see[i, b:last] = True
    return see


def _softmax_rows(z, see):
    z = np.where(see, z, -np.inf)
    m = z.max(axis=-1, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    p = np.exp(z - m)
    total = p.sum(axis=-1, keepdims=True)
    return p / np.where(total == 0, 1.0, total)


def attention(x, heads, kv, dim, see, scale=None, cap=0.0, slopes=None, dy=None):
    """(y, y_err) or with dy (y, y_err, dx, dx_err).  x: [M x (heads + 2 kv) dim].

    Scores: `dim` fp32 products and sums and the scale, E (dim + 4) sum |q k| scale.  The cap's tanh is off by 2^-20 of itself (at most
    sixteen fp32 roundings: of the argument and its square, of a numerator and a denominator, of one reciprocal for four and the products
    that part it), which is 2^-20 of the score, whatever the cap.  The distance's product is off by E.  All of it enters a weight p through
    exp (2^-21 more), in the numerator and in the normalising sum.
    P is rounded to bf16 before P v and P^T dO, dS before dS K and dS^T Q.  D is formed from the stored (bf16) y."""
    M = x.shape[0]
    g = heads // kv
    scale = 1.0 / np.sqrt(dim) if not scale else scale
    blocks = x.reshape(M, heads + 2 * kv, dim)
    y, y_err = np.zeros((M, heads, dim)), np.zeros((M, heads, dim))
    dx, dx_err = np.zeros_like(blocks), np.zeros_like(blocks)
    away = np.abs(np.arange(M)[:, None] - np.arange(M)[None])
    for h in range(heads):
        q, k, v = blocks[:, h], blocks[:, heads + h // g], blocks[:, heads + kv + h // g]
        raw = q @ k.T * scale
        delta = E * (dim + 4) * (np.abs(q) @ np.abs(k).T) * scale
        slope = np.ones_like(raw)
        z = raw
        if cap:
            t = np.tanh(raw / cap)
            z, slope = cap * t, 1 - t * t
            delta = delta + np.abs(z) * 2.0 ** -20
        if slopes is not None:
            z = z - slopes[h] * away
            delta = delta + 2 * E * np.abs(slopes[h]) * away
        delta = delta + 2 * E * np.abs(z)                                # the sum with the maximum (or the log-sum-exp)
        p = _softmax_rows(z, see)
        worst = np.where(see, delta, 0.0).max(axis=1, keepdims=True)
        rel = delta + worst + 2.0 ** -20                                 # of every p
        ay = p @ np.abs(v)
        y[:, h] = p @ v
        y_err[:, h] = (p * (U + rel)) @ np.abs(v) + U * np.abs(y[:, h]) + E * M * ay
        if dy is None:
            continue
        do = dy.reshape(M, heads, dim)[:, h]
        dp = do @ v.T
        D = (do * y[:, h]).sum(axis=1, keepdims=True)
        ds = p * (dp - D) * slope
        inner = E * (dim + 4) * (np.abs(do) @ np.abs(v).T) + (np.abs(do) * (y_err[:, h] + U * np.abs(y[:, h]))).sum(axis=1, keepdims=True)
        slope_err = (1 - slope) * 2.0 ** -19 + 2 * E if cap else 0.0     # 2 t times t's error; errors of both factors of a product meet
        ds_err = U * np.abs(ds) + p * (np.abs(slope) + slope_err) * inner + np.abs(ds) * rel + p * np.abs(dp - D) * slope_err
        add = lambda at, val, err: (np.add(dx[:, at], val, out=dx[:, at]), np.add(dx_err[:, at], err, out=dx_err[:, at]))  # noqa: E731
        add(h, scale * ds @ k, scale * (ds_err + E * M * np.abs(ds)) @ np.abs(k))
        add(heads + h // g, scale * ds.T @ q, scale * (ds_err + E * M * np.abs(ds)).T @ np.abs(q))
        add(heads + kv + h // g, p.T @ do, (p * (U + rel + E * M)).T @ np.abs(do))
    y, y_err = y.reshape(M, -1), y_err.reshape(M, -1)
    if dy is None:
        return y, y_err
    dx, dx_err = dx.reshape(M, -1), dx_err.reshape(M, -1)
    return y, y_err, dx, dx_err + U * np.abs(dx)


# ------------------------------------------------------------------------------------------ rotary
def rotary(x, heads, kv, dim, sections, positions, theta, adjacent=False, own_spectrum=False, back=False):
    """y, and the size of what each element is made of (|x| + |y| of its pair).  positions: [axes][M]."""
    M = x.shape[0]
    out = np.array(x, dtype=np.float64).reshape(M, -1, dim)
    size = np.zeros_like(out)
    n, k = sum(sections), 0
    src = out.copy()
    for a, count in enumerate(sections):
        for j in range(count):
            e = j / count if own_spectrum else k / n
            angle = np.asarray(positions[a], dtype=np.float64) * np.float64(theta) ** -e * (-1 if back else 1)
            c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
            i0, i1 = (2 * k, 2 * k + 1) if adjacent else (k, n + k)
            u, w = src[:, :heads + kv, i0], src[:, :heads + kv, i1]
            out[:, :heads + kv, i0], out[:, :heads + kv, i1] = u * c - w * s, w * c + u * s
            size[:, :heads + kv, i0] = size[:, :heads + kv, i1] = np.abs(u) + np.abs(w)
            k += 1
    return out.reshape(M, -1), size.reshape(M, -1)


# ------------------------------------------------------------------------------------------ gated
def act(z, kind):
    """Value, slope and a bound of the second derivative.  1 = GELU (tanh form), 2 = ReLU, 3 = SiLU."""
    if kind == 3:
        g = 1 / (1 + np.exp(-z))
        return z * g, g * (1 + z * (1 - g)), 0.5
    if kind == 2:
        return np.maximum(z, 0), (z > 0).astype(np.float64), 0.0
    c0, c1 = np.sqrt(2 / np.pi), 0.044715
    t = np.tanh(c0 * (z + c1 * z ** 3))
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c0 * (1 + 3 * c1 * z * z), 1.2


def gated(x, W, b, kind, dy, u, uz=None, dy_err=0.0):
    """Results and bounds of a gated layer by itself: y, dx, dW, db.  u: half a step of the storage type; uz: of the type that Z is kept in
    (bf16 stacks: fp16, 2^-11); dy_err: bound of the error that dy comes with."""
    uz = (2.0 ** -11 if u == U else u) if uz is None else uz
    M, K = x.shape
    h = W.shape[1] // 2
    z = x @ W + b
    zerr = E * (K + 3) * (np.abs(x) @ np.abs(W) + np.abs(b))
    zg, zu = z[:, :h], z[:, h:]
    f, s, curve = act(zg, kind)
    near = 2.0 ** -19                                    # the activations' own error, relative to |z| + 1
    ferr = 1.2 * zerr[:, :h] + near * (np.abs(zg) + 1)
    y = f * zu
    out = {"y": (y, ferr * np.abs(zu) + np.abs(f) * zerr[:, h:] + (u + 2 * E) * np.abs(y))}
    zerr = zerr + uz * np.abs(z) + (2.0 ** -25 if uz == 2.0 ** -11 else 0.0)     # as Z is kept (fp16: steps of 2^-24 near 0)
    serr = curve * zerr[:, :h] + near * (np.abs(zg) + 1)
    if kind == 2:
        serr = serr + (np.abs(zg) <= zerr[:, :h])
    ferr = 1.2 * zerr[:, :h] + near * (np.abs(zg) + 1)
    dg, du = dy * zu * s, dy * f
    dz = np.concatenate([dg, du], axis=1)
    derr = np.concatenate([np.abs(dy) * (np.abs(zu) * serr + np.abs(s) * zerr[:, h:]), np.abs(dy) * ferr], axis=1)
    derr = derr + (u + 3 * E) * np.abs(dz) + np.concatenate([dy_err * np.abs(zu * s), dy_err * np.abs(f)], axis=1)
    dx = dz @ W.T
    out["dx"] = (dx, (derr + E * (2 * h + 2) * np.abs(dz)) @ np.abs(W).T + u * np.abs(dx))
    out["dW"] = (x.T @ dz, np.abs(x).T @ (derr + E * (M + 2) * np.abs(dz)))
    out["db"] = (dz.sum(axis=0), (derr + E * (M + 2) * np.abs(dz)).sum(axis=0))
    return out


# ------------------------------------------------------------------------------------------ dropout
def philox(counter, key):
    """Philox 4x32 with ten rounds (Salmon et al. 2011) on Python integers."""
    c0, c1, c2, c3 = counter
    k0, k1 = key
    low = 0xFFFFFFFF
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32) ^ c1 ^ k0, b & low, (a >> 32) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def kept(first, count, p, seed, step, layer):
    """Elements first .. first + count - 1 (first a multiple of 4) that stay."""
    low = 0xFFFFFFFF
    limit = round(p * 2 ** 32)
    words = []
    for block in range(first // 4, (first + count + 3) // 4):
        words += philox((block & low, block >> 32, step & low, layer), (seed & low, (seed >> 32) & low))
    return np.array(words[:count], dtype=np.uint64) >= limit

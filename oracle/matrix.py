"""fp64 numpy forms of the matrix operators: Newton-Schulz orthogonalisation, the optimiser step built on it, and
microscaled 4-bit quantisation with its packed layout.  Shares no code with the CUDA path."""
import math

import numpy as np

COEF = (3.4445, -4.7750, 2.0315)


def newton_schulz(g, steps=5, coef=COEF, eps=1e-7):
    """The singular values pushed through sigma <- a sigma + b sigma^3 + c sigma^5, written with matrix products."""
    x = np.asarray(g, dtype=np.float64)
    a, b, c = coef
    x = x / (np.sqrt(np.sum(x * x)) + eps)
    eye = np.eye(min(x.shape))
    for _ in range(steps):
        if x.shape[0] <= x.shape[1]:
            s = x @ x.T
            x = (a * eye + b * s + c * (s @ s)) @ x
        else:
            s = x.T @ x
            x = x @ (a * eye + b * s + c * (s @ s))
    return x


def muon(w, m, g, lr, beta, nesterov, weight_decay, scale, **kw):
    """(w, m) after one step."""
    w, m, g = (np.asarray(t, dtype=np.float64) for t in (w, m, g))
    m = beta * m + (1 - beta) * g
    u = beta * m + (1 - beta) * g if nesterov else m
    return (1 - lr * weight_decay) * w - lr * scale * newton_schulz(u, **kw), m


E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mx_quantize(x):
    """(codes [rows, blocks, 32], exponents [rows, blocks]) of x; the exponent of a block that holds an infinity or
    NaN is None (128)."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // 32)
    p = np.zeros((rows, nb * 32))
    p[:, :cols] = x
    p = p.reshape(rows, nb, 32)
    codes = np.zeros(p.shape, dtype=np.uint8)
    exps = np.zeros((rows, nb), dtype=np.int64)
    for r in range(rows):
        for k in range(nb):
            top = np.max(np.abs(p[r, k]))
            if not np.isfinite(top):
                exps[r, k] = 128
                continue
            e = -127 if top == 0 else min(127, max(-127, math.frexp(top)[1] - 3))
            exps[r, k] = e
            y = np.abs(p[r, k]) * 2.0 ** -e
            d = np.abs(y[:, None] - E2M1[None, :])
            best = np.argmin(d, axis=1)                       # the lower of two equally near ones
            tie = (best < 7) & (d[np.arange(32), best] == d[np.arange(32), np.minimum(best + 1, 7)])
            best = np.where(tie & (best % 2 == 1), best + 1, best)
            codes[r, k] = best + 8 * np.signbit(p[r, k])
    return codes, exps


def mx_values(codes, exps, cols):
    v = np.where(codes & 8, -1.0, 1.0) * E2M1[codes & 7] * 2.0 ** np.minimum(exps, 127)[..., None]
    v[exps == 128] = np.nan
    return v.reshape(codes.shape[0], -1)[:, :cols]


def mx_pack(codes, exps):
    """The library's bytes: (codes, scales)."""
    rows, nb, _ = codes.shape
    c = codes.reshape(rows, -1)
    packed = (c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8)
    tiles = -(-nb // 8)
    scales = np.zeros((-(-rows // 128)) * tiles * 1024, dtype=np.uint8)
    for r in range(rows):
        for k in range(nb):
            at = ((r // 128) * tiles + k // 8) * 1024 + (k % 8 // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + k % 4
            scales[at] = exps[r, k] + 127
    return packed.reshape(-1), scales

"""float64 reference of the serving operators: rows and channels in 8-bit
integers, the expert FFN on them, and elementwise bounds for the layer of a few
tokens.  Test infrastructure only; written from the definitions, plain and slow."""
from __future__ import annotations

import numpy as np

from .moe_oracle import round_bf16


def quant_rows(x):
    """(integers, fp32 scale) of the rows of x (bf16 values): scale = max|x| / 127, the
    integers 127 x / max|x| rounded to nearest, ties to even.  A row of zeros has scale 0;
    a row with an infinity or NaN has a NaN scale and zero integers."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore"):
        top = np.max(np.abs(x), axis=-1)
    fine = np.isfinite(top)
    safe = np.where(fine & (top > 0), top, 1.0)
    q = np.rint(127.0 * np.where(fine[..., None], x, 0.0) / safe[..., None])
    scale = np.where(fine, np.where(fine, top, 0.0) / 127.0, np.nan).astype(np.float32)
    return q, scale


def quant_weights(W):
    """(integers [E, N, Kd], scale [E, N]) of W [E, Kd, N] per output channel."""
    return quant_rows(np.swapaxes(np.asarray(W, np.float64), -1, -2))


def product_i8(q, sx, Wq, sw):
    """sx[r] sw[n] sum_k q[r, k] Wq[n, k], the sum exact."""
    return (q @ Wq.T) * sx.astype(np.float64)[:, None] * sw.astype(np.float64)


def ffn_i8(x, W1q, s1, W2q, s2):
    """One expert: (h, y) with h = bf16(max(u, 0)^2) and its rows quantised."""
    q, sx = quant_rows(x)
    h = round_bf16(np.maximum(product_i8(q, sx, W1q, s1), 0.0) ** 2)
    hq, sh = quant_rows(h)
    return h, product_i8(hq, sh, W2q, s2)


def ffn_bound(x, W1, W2):
    """(y, b): one bf16 expert on rows x, and how far y may be off where sums of n
    terms are taken in fp32 in any order (each off by at most n 2^-24 times the sum of
    the terms' magnitudes) and h is rounded to bf16 (half a step, 2^-8)."""
    x, W1, W2 = (np.asarray(a, np.float64) for a in (x, W1, W2))
    D, F = W1.shape
    u = np.maximum(x @ W1, 0.0)
    du = D * 2.0 ** -24 * (np.abs(x) @ np.abs(W1))
    h = u * u
    dh = 2 * u * du + du * du + (2.0 ** -8 + 2.0 ** -23) * (u + du) ** 2
    y = h @ W2
    return y, dh @ np.abs(W2) + F * 2.0 ** -24 * ((h + dh) @ np.abs(W2))

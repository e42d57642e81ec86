"""The operators after a macro-step's attention in plain fp64 numpy (TEST INFRASTRUCTURE ONLY: the
tests and `__graft_entry__.smoke()` use it; the product path never imports this package).

8-bit rows: e4m3 codes and, for each 128 elements, a scale byte s standing for 2^(s - 127).  The scale
of a block whose largest magnitude is m 2^E (0.5 <= m < 1) is 2^(E - 8), E - 8 clamped to [-124, 119],
and 1 for a block of zeros.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
FINE = 2.0 ** 31


def scale_bytes(k: int) -> int:
    """Scale bytes of a row of k elements."""
    return 4 * ((k + 4 * BLOCK - 1) // (4 * BLOCK))


def code_values() -> np.ndarray:
    """Values of the 256 e4m3 codes: sign, 4 exponent bits of bias 7, 3 mantissa bits; the two codes
    with every other bit set are NaN."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m / 8 * 2.0 ** -6, (1 + m / 8) * 2.0 ** (e - 7))
    v[(c & 127) == 127] = np.nan
    return np.where(c >> 7, -v, v)


def block_exponent(top: np.ndarray) -> np.ndarray:
    """Exponent of the scale of blocks whose largest magnitudes are `top`."""
    return np.where(top > 0, np.clip(np.frexp(top)[1] - 8, -124, 119), 0)


def step_of(q: np.ndarray) -> np.ndarray:
    """Distance of neighbouring e4m3 values at q (below 2^-6 all 2^-9 apart)."""
    return 2.0 ** np.maximum(np.frexp(np.abs(q))[1] - 4, -9)


def encode_rows(x: np.ndarray):
    """fp64 rows [T][K] -> (values the codes stand for, scaled back; exponents [T][blocks])."""
    t, k = x.shape
    nb = -(-k // BLOCK)
    p = np.zeros((t, nb * BLOCK))
    p[:, :k] = x
    p = p.reshape(t, nb, BLOCK)
    e = block_exponent(np.abs(p).max(axis=2))
    q = p * 2.0 ** -e[:, :, None].astype(np.float64)
    s = step_of(q)
    v = np.rint(q / s) * s * 2.0 ** e[:, :, None].astype(np.float64)
    return v.reshape(t, -1)[:, :k], e


def decode_rows(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """fp64 values of 8-bit rows (uint8 codes [T][K], scale bytes [T][scale_bytes(K)])."""
    k = codes.shape[1]
    p = np.repeat(2.0 ** (scales.astype(np.float64) - 127), BLOCK, axis=1)[:, :k]
    return code_values()[codes] * p


def decode_weight(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """fp64 values of an 8-bit weight (one scale for each 128 x 128 block)."""
    return decode_rows(codes, np.repeat(scales, BLOCK, axis=0)[:codes.shape[0]])


def add_norm(x, residual, weight, eps):
    """(h, y): h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight."""
    h = x if residual is None else x + residual
    return h, h / np.sqrt((h * h).mean(axis=1, keepdims=True) + eps) * weight


def silu(g):
    """g / (1 + exp(-g)), without overflow."""
    return g * np.exp(np.minimum(g, 0)) / (1 + np.exp(-np.abs(g)))


def gated(x, w_gate, w_up):
    """(G, U, silu(G) U) of the gated block's first half."""
    g, u = x @ w_gate.T, x @ w_up.T
    return g, u, silu(g) * u


def kept_weights(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Weights of one row's kept tokens (0 elsewhere), in units of the likeliest token's / 2^31."""
    l = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    top = l.max()
    if top == -np.inf:
        return np.zeros(len(l))
    if not temperature > 0:
        w = np.zeros(len(l))
        w[int(np.argmax(l))] = FINE
        return w
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.where(l == top, 0.0, (l - top) / temperature)
    w = np.floor(FINE * np.exp(x))
    order = np.lexsort((np.arange(len(l)), -l))
    if 0 < top_k < len(l):
        order = order[:top_k]
    if top_p < 1:
        run = np.cumsum(w[order])
        before = run - w[order]
        order = order[(before < top_p * run[-1]) | (np.arange(len(order)) == 0)]
    order = order[w[order] >= min(min_p, 1.0) * FINE]
    kept = np.zeros(len(l))
    kept[order] = w[order]
    return kept


def sample(logits, u, **settings):
    """(token, probability) of one row."""
    kept = kept_weights(logits, **settings)
    run = np.cumsum(kept)
    if run[-1] == 0:
        return -1, 0.0
    aim = min(np.floor(u * run[-1]), run[-1] - 1)
    token = int(np.searchsorted(run, aim, "right"))
    return token, kept[token] / run[-1]

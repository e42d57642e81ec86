"""Set-up and tolerances shared by the tests of the operators after the attention."""
import numpy as np

from oracle import ops
from paper_2505_20438_gb300 import ham


def bf16(x, rng=None):
    """fp array -> (CUDA bf16 tensor, its fp64 values)."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16()
    return t.cuda(), t.double().numpy()


def rows(rng, t, k, spread=True):
    """Rows as a residual stream has them: N(0, 1), one channel in 64 eight times as large; with
    `spread` the rows' sizes run over 2^-12 .. 2^12."""
    x = rng.standard_normal((t, k))
    x[:, 5::64] *= 8
    if spread:
        x *= 2.0 ** rng.integers(-12, 13, (t, 1))
    return x


def random_codes(rng, t, k, weight=False):
    """Finite e4m3 codes and scale bytes (2^-14 .. 2^2) of t rows (weight: of a weight)."""
    c = rng.integers(0, 256, (t, k)).astype(np.uint8)
    c[(c & 127) == 127] = 0
    n = -(-t // 128) if weight else t
    return c, rng.integers(113, 130, (n, ops.scale_bytes(k))).astype(np.uint8)


def dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def empty_rows(t, k):
    """Output codes and scales, filled with a pattern that no encoder writes (NaN codes, scale 255)."""
    import torch
    return (torch.full((t, k), 0x7f, dtype=torch.uint8, device="cuda"),
            torch.full((t, ops.scale_bytes(k)), 255, dtype=torch.uint8, device="cuda"))


def check_bf16(got, want, slack):
    """got (a bf16 or fp32 tensor) is a value within `slack` of `want`; a bf16 one its rounding: it lies
    between the roundings of want - slack and want + slack."""
    import torch
    g = got.double().cpu().numpy()
    lo, hi = want - slack, want + slack
    if got.dtype == torch.bfloat16:
        lo, hi = (_round_bf16(v) for v in (lo, hi))
    bad = ~((g >= lo) & (g <= hi))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), g[bad][:4], want[bad][:4])


def _round_bf16(x):
    """fp64 -> the nearest bf16 value, ties to even (8 significant bits; no overflow here)."""
    step = 2.0 ** (np.maximum(np.frexp(x)[1], -125) - 8)
    return np.rint(x / step) * step


def check_codes(codes, scales, want, slack):
    """8-bit rows of values that lie within `slack` of `want`: each block's scale is that of a largest
    magnitude within the slack, each code is a nearest e4m3 value for some value within the slack, and
    the padding is scale 1."""
    c, s = codes.cpu().numpy(), scales.cpu().numpy().astype(np.int64)
    t, k = want.shape
    nb = -(-k // 128)
    assert (s[:, nb:] == 127).all()
    assert np.isfinite(ops.code_values()[c]).all()
    slack = np.broadcast_to(slack, want.shape)
    for b in range(nb):
        w, d = want[:, 128 * b:128 * (b + 1)], slack[:, 128 * b:128 * (b + 1)]
        lo = ops.block_exponent(np.max(np.maximum(np.abs(w) - d, 0), axis=1))
        hi = ops.block_exponent(np.max(np.abs(w) + d, axis=1))
        e = s[:, b] - 127
        zero = (np.max(np.abs(w) - d, axis=1) <= 0) & (e == 0)
        assert (((e >= lo) & (e <= hi)) | zero).all(), (b, e, lo, hi)
        p = 2.0 ** e[:, None].astype(np.float64)
        q, dq = w / p, d / p
        v = ops.code_values()[c[:, 128 * b:128 * (b + 1)]]
        near = ops.step_of(np.abs(q) + dq) / 2 + dq
        bad = np.abs(v - q) > near * (1 + 1e-12)
        assert not bad.any(), (b, int(bad.sum()), v[bad][:4], q[bad][:4])


def product_slack(x, w):
    """Bound of a product's error before its rounding.  A tensor-core product adds 32 exact terms at a
    time to a running fp32 sum, each addition off by at most one unit of 2^-23 of the magnitudes that
    meet in it (truncation included), which sum|x w| bounds: k / 32 additions and two spare."""
    return (x.shape[1] / 32 + 2) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T)


def gated_slack(x, wg, wu, g, u):
    """The same carried through silu(G) U (|silu'| <= 1.1), and 2^-20 of the value for the fp32
    exponential, division and products (some ten roundings of 2^-24, doubled)."""
    dg, du = product_slack(x, wg), product_slack(x, wu)
    silu = np.abs(ops.silu(g))
    return 1.1 * dg * (np.abs(u) + du) + silu * du + 2.0 ** -20 * silu * np.abs(u)


def norm_slack(y):
    """fp32 sum of squares in a tree (each thread at most 32 terms in a row, then 10 levels), the
    reciprocal root (2 units), three products: below 64 roundings of 2^-24 of the value."""
    return 2.0 ** -18 * np.abs(y)


def alloc_weight(n, k, w, up=None):
    return ham.ham_fp8_weight_alloc(n, k, dev(w[0]), dev(w[1]), *((dev(up[0]), dev(up[1])) if up else ()))

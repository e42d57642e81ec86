"""Gated results that leave fp32's range, and NaN among finite ones: the block's scale is the header's, with rows by index and
rows sorted first."""
import numpy as np
import pytest

from oracle import ops
from paper_2505_20438_gb300 import ham
from tests.ops_helpers import alloc_weight, dev, empty_rows
from tests.test_gpu_experts import alloc, grouping

pytestmark = pytest.mark.gpu

# (by index; sorted first; the sizes of test_rows_sorted_first)
SIZES = [([5, 0, 40], 384, 128), ([257, 0, 300], 4096, 1024)]


def _weights(rng, experts, n, k, exponent):
    """Weights of one column: codes [experts][n][k], zeros from the second column on, and scales 2^exponent[tile]."""
    c = np.zeros((experts, n, k), np.uint8)
    c[:, :, 0] = rng.integers(0, 256, (experts, n))
    c[:, :, 0][(c[:, :, 0] & 127) == 127] = 0
    s = np.full((experts, -(-n // 128), ops.scale_bytes(k)), 127, np.uint8)
    s[:, :, 0] = 127 + np.resize(exponent, s.shape[1])
    return c, s


def _rows(rng, rows, k):
    """Rows of one column, 1 and 1/2 in turn."""
    x = np.zeros((rows, k), np.uint8)
    x[:, 0] = np.where(np.arange(rows) % 2, 0x30, 0x38)
    return x, np.full((rows, ops.scale_bytes(k)), 127, np.uint8)


def _want(x, w, up):
    """The codes' values and the scale bytes of slots x with weights w and up (codes, scales): every product is exact, of eight
    significant bits at most, and its gate far from zero or zero (silu(g) is max(g, 0)); beyond 2^128 it is infinite."""
    g, u = (x @ ops.decode_weight(*v).T for v in (w, up))
    h = np.maximum(g, 0) * u
    h[np.abs(h) >= 2.0 ** 128] = np.inf * np.sign(h[np.abs(h) >= 2.0 ** 128])
    t, n = h.shape
    p = np.zeros((t, -(-n // 128) * 128))
    p[:, :n] = h
    p = p.reshape(t, p.shape[1] // 128, 128)
    top = np.abs(p).max(axis=2)
    e = np.where(np.isinf(top), 119, ops.block_exponent(np.where(np.isinf(top), 0, top)))
    q = np.clip(p * 2.0 ** -e[:, :, None].astype(float), -1e30, 1e30)
    step = ops.step_of(q)
    v = np.clip(np.rint(q / step) * step, -448, 448).reshape(t, p.shape[1] * 128)[:, :n]
    return v, e + 127


def _call(counts, n, k, w, up, x):
    rows = len(x[0])
    offsets, order = grouping(np.random.default_rng(1), counts, 1, rows)
    h = alloc(n, k, w, up)
    codes, scales = empty_rows(rows, n)
    ham.ham_fp8_experts_gated(h, *map(dev, x), dev(offsets), dev(order), 1, codes, scales)
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE
    return offsets, order, codes.cpu().numpy(), scales.cpu().numpy()


@pytest.mark.parametrize("counts,n,k", SIZES, ids=["by index", "sorted"])
def test_an_infinite_result_has_the_largest_scale(counts, n, k):
    """Tiles with many products past 2^128, with a few, with none."""
    rng = np.random.default_rng(n)
    exponent = np.array([57, 55, 50])
    w, up = (_weights(rng, len(counts), n, k, exponent) for _ in range(2))
    x = _rows(rng, sum(counts), k)
    offsets, order, codes, scales = _call(counts, n, k, w, up, x)
    x64 = ops.decode_rows(*x)[order]
    seen = set()
    for e in range(len(counts)):
        i = slice(offsets[e], offsets[e + 1])
        v, s = _want(x64[i], (w[0][e], w[1][e]), (up[0][e], up[1][e]))
        assert (scales[i, :s.shape[1]] == s).all()
        assert (ops.code_values()[codes[i]] == v).all()
        seen |= set(s.reshape(-1) == 246)
    assert seen == {False, True}


@pytest.mark.parametrize("rows", [5, 300])
def test_as_the_dense_half_has_it(rows):
    """The same weights and rows through ham_fp8_gated: the same bits."""
    import torch
    rng = np.random.default_rng(rows)
    n, k = 384, 128
    w, up = (_weights(rng, 1, n, k, np.array([57, 55, 50])) for _ in range(2))
    x = _rows(rng, rows, k)
    dense = alloc_weight(n, k, (w[0][0], w[1][0]), (up[0][0], up[1][0]))
    c, s = empty_rows(rows, n)
    ham.ham_fp8_gated(dense, *map(dev, x), c, s)
    codes, scales = empty_rows(rows, n)
    order = dev(np.arange(rows, dtype=np.int32))
    ham.ham_fp8_experts_gated(alloc(n, k, w, up), *map(dev, x), dev(np.int32([0, rows])), order, 1, codes, scales)
    assert torch.equal(c, codes) and torch.equal(s, scales)


@pytest.mark.parametrize("counts,n,k", SIZES, ids=["by index", "sorted"])
def test_nan_counts_for_nothing_in_a_scale(counts, n, k):
    """A weight's NaN makes its feature NaN and leaves the others and their scales as they are; a row's NaN makes the whole row
    NaN, with scale 1."""
    rng = np.random.default_rng(n + 1)
    w, up = (_weights(rng, len(counts), n, k, np.array([3, 0, -5])) for _ in range(2))
    w[0][:, 7, 0] = 0                              # the feature that is NaN below
    x = _rows(rng, sum(counts), k)
    offsets, order, codes, scales = _call(counts, n, k, w, up, x)
    w[0][:, 7, 1] = 0x7f
    x[0][4, 3] = 0xff
    _, _, got, got_scales = _call(counts, n, k, w, up, x)
    row = order == 4
    assert row.sum() == 1
    blocks = -(-n // 128)
    assert ((got[row] & 127) == 127).all() and (got_scales[row] == 127).all()
    assert ((got[~row, 7] & 127) == 127).all()
    got[:, 7], got[row], got_scales[row] = codes[:, 7], codes[row], scales[row]
    assert (got == codes).all() and (got_scales == scales).all() and (scales[:, blocks:] == 127).all()

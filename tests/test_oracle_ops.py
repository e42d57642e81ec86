"""Pins of the fp64 oracle of the operators after the attention (oracle/ops.py) to things other than
itself: torch's e4m3 conversion, hand-worked rows, brute-force definitions."""
import math

import numpy as np
import pytest

from oracle import ops


def test_code_values_are_torchs():
    import torch
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(ops.code_values(), codes.astype(np.float64))


def test_encoding_rounds_as_torch_does():
    import torch
    x = np.random.default_rng(0).standard_normal((5, 300)).astype(np.float32) * \
        np.float32(2.0) ** np.arange(-40, 60, 20, dtype=np.float32)[:, None]
    v, e = ops.encode_rows(x.astype(np.float64))
    for b in range(3):
        s = slice(128 * b, 128 * (b + 1))
        p = (2.0 ** -e[:, b:b + 1].astype(np.float64)).astype(np.float32)
        t = torch.from_numpy(x[:, s] * p).to(torch.float8_e4m3fn).double().numpy()
        np.testing.assert_array_equal(v[:, s] / 2.0 ** e[:, b:b + 1].astype(np.float64), t)


def test_scale_of_a_block_by_hand():
    #  1.0 = 0.5 2^1: E = 1, scale 2^-7, the code's value 128
    np.testing.assert_array_equal(ops.block_exponent(np.array([1.0, 0.75, 255.0, 256.0, 0.0])), [-7, -8, 0, 1, 0])
    np.testing.assert_array_equal(ops.block_exponent(np.array([2.0 ** -130, 2.0 ** 127])), [-124, 119])
    assert [ops.scale_bytes(k) for k in (16, 128, 512, 528, 4096)] == [4, 4, 4, 8, 32]


def test_norm_and_gate_by_hand():
    h, y = ops.add_norm(np.array([[3.0, 4.0]]), np.array([[0.0, 0.0]]), np.array([1.0, 2.0]), 0.0)
    np.testing.assert_allclose(y, [[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]], rtol=1e-15)
    g, u, v = ops.gated(np.array([[1.0, 2.0]]), np.array([[1.0, 0.0]]), np.array([[0.0, 1.0]]))
    assert (g, u) == (1.0, 2.0)
    np.testing.assert_allclose(v, 2 / (1 + math.exp(-1)), rtol=1e-15)


@pytest.mark.parametrize("k,p,m,kept", [
    # weights 0.25, 1, 0.5, 0.5 of the largest: order 1, 2, 3, 0, sum 2.25
    (0, 1.0, 0.0, [0, 1, 2, 3]),
    (2, 1.0, 0.0, [1, 2]),           # the largest, then the first of the two equal ones
    (0, 0.5, 0.0, [1, 2]),           # 1.125: the largest alone does not reach it
    (0, 0.7, 0.0, [1, 2, 3]),        # 1.575
    (3, 0.7, 0.0, [1, 2]),           # of the three: 1.4
    (0, 0.0, 0.0, [1]),
    (3, 1.0, 0.6, [1]),
    (0, 1.0, 0.4, [1, 2, 3]),
    (0, 1.0, 7.0, [1]),              # the likeliest stays
])
def test_cuts_by_hand(k, p, m, kept):
    l = np.log(np.array([1.0, 4.0, 2.0, 2.0]))
    l[3] = l[2]
    w = ops.kept_weights(l, top_k=k, top_p=p, min_p=m)
    assert list(np.flatnonzero(w)) == kept
    np.testing.assert_allclose(w[kept] / 2.0 ** 31, np.array([0.25, 1, 0.5, 0.5])[kept], rtol=1e-8)


def test_sample_walks_the_running_sum():
    l = np.log(np.array([1.0, 4.0, 2.0, 1.0]))
    got = [ops.sample(l, u)[0] for u in (0.0, 0.1249, 0.1251, 0.62, 0.63, 0.874, 0.876, 0.99999)]
    assert got == [0, 0, 1, 1, 2, 2, 3, 3]
    assert ops.sample(l, 0.3, temperature=0.0) == (1, 1.0)
    assert ops.sample(np.full(4, -np.inf), 0.3) == (-1, 0.0)
    assert ops.sample(np.array([np.nan, -np.inf, 3.0]), 0.9)[0] == 2

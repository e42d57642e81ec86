"""ham_fp8_linear and ham_fp8_gated against the fp64 oracle: the streaming kernel (few rows) and the
pair kernel (many), ragged sizes, scales over their range."""
import numpy as np
import pytest

from oracle import ops
from ops_helpers import (alloc_weight, check_bf16, check_codes, dev, empty_rows, gated_slack, product_slack,
                         random_codes)
from paper_2505_20438_gb300 import ham

pytestmark = pytest.mark.gpu


def _linear(t, k, n, f32, seed=0):
    import torch
    rng = np.random.default_rng(seed + 7 * t + 11 * k + 13 * n)
    x, w = random_codes(rng, t, k), random_codes(rng, n, k, weight=True)
    handle = alloc_weight(n, k, w)
    y = torch.full((t, n), float("nan"), dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    ham.ham_fp8_linear(handle, dev(x[0]), dev(x[1]), y)
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(handle) == 0
    x64, w64 = ops.decode_rows(*x), ops.decode_weight(*w)
    check_bf16(y, x64 @ w64.T, product_slack(x64, w64))


# one K block and a part of one, few and many blocks (splits over a cluster), scale words ending
# anywhere; rows and features off every tile
@pytest.mark.parametrize("t,k,n", [
    (1, 16, 1), (1, 128, 128), (1, 4096, 256), (2, 144, 130), (3, 512, 127), (8, 528, 384), (16, 640, 1000),
    (17, 2064, 257), (33, 1536, 200), (64, 1024, 640), (100, 272, 129), (128, 1664, 300), (129, 400, 140),
    (300, 896, 513), (5, 16400, 136),
])
@pytest.mark.parametrize("f32", [False, True])
def test_linear_streams_match_oracle(t, k, n, f32):
    _linear(t, k, n, f32)


@pytest.mark.parametrize("t,k,n", [
    (2560, 128, 2048), (2561, 144, 2049), (2300, 528, 2500), (2304, 1024, 2304), (1281, 640, 4003),
    (5000, 256, 4096),
])
@pytest.mark.parametrize("f32", [False, True])
def test_linear_pairs_match_oracle(t, k, n, f32):
    _linear(t, k, n, f32)


def _gated(t, k, f):
    import torch
    rng = np.random.default_rng(3 * t + 5 * k + 7 * f)
    x, g, u = random_codes(rng, t, k), random_codes(rng, f, k, weight=True), random_codes(rng, f, k, weight=True)
    # scales about 2^-10, so that G is of the order of one and both sides of the SiLU are met
    size = int(np.log2(np.sqrt(k) * 100.0 ** 2)) // 2
    for s in (x[1], g[1], u[1]):
        s[:] = 127 - size + (s & 3)
    handle = alloc_weight(f, k, g, u)
    codes, scales = empty_rows(t, f)
    ham.ham_fp8_gated(handle, dev(x[0]), dev(x[1]), codes, scales)
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(handle) == 0
    x64, g64, u64 = ops.decode_rows(*x), ops.decode_weight(*g), ops.decode_weight(*u)
    G, U, h = ops.gated(x64, g64, u64)
    assert 0.05 < np.mean(G < -1) < 0.95
    check_codes(codes, scales, h, gated_slack(x64, g64, u64, G, U))


@pytest.mark.parametrize("t,k,f", [(1, 16, 16), (1, 512, 128), (2, 144, 144), (8, 2048, 400), (20, 1040, 528),
                                   (64, 528, 256), (128, 640, 272), (200, 400, 640)])
def test_gated_streams_match_oracle(t, k, f):
    _gated(t, k, f)


@pytest.mark.parametrize("t,k,f", [(2560, 128, 1024), (2561, 144, 1040), (1300, 1152, 2064), (4500, 528, 528)])
def test_gated_pairs_match_oracle(t, k, f):
    _gated(t, k, f)


@pytest.mark.parametrize("n", [2496, 2504, 2500, 2502, 2503])
@pytest.mark.parametrize("f32", [False, True])
def test_linear_pairs_write_at_every_alignment(n, f32):
    """Rows that begin at multiples of 32 down to 2 bytes, an output that begins at one of 16 alone, and what lies
    around it left as it is."""
    import torch
    t, k = 300, 272
    rng = np.random.default_rng(n)
    x, w = random_codes(rng, t, k), random_codes(rng, n, k, weight=True)
    x64, w64 = ops.decode_rows(*x), ops.decode_weight(*w)
    handle = alloc_weight(n, k, w)
    dtype = torch.float32 if f32 else torch.bfloat16
    for first in (0, 4 if f32 else 8):
        room = torch.full((first + t * n + 64,), 7.0, dtype=dtype, device="cuda")
        y = room[first:first + t * n].view(t, n)
        ham.ham_fp8_linear(handle, dev(x[0]), dev(x[1]), y)
        check_bf16(y, x64 @ w64.T, product_slack(x64, w64))
        assert (room[:first] == 7).all() and (room[first + t * n:] == 7).all()


def test_scales_over_their_range():
    """Each operand's scales from 2^-124 to 2^119 (their products within fp32)."""
    import torch
    t, k, n = 4, 256, 128
    rng = np.random.default_rng(0)
    x, w = random_codes(rng, t, k), random_codes(rng, n, k, weight=True)
    for sx, sw in ((127 - 124, 127 + 119), (127 + 119, 127 - 124), (127 - 60, 127 - 50), (127 + 50, 127 + 50)):
        x[1][:], w[1][:] = sx, sw
        y = torch.empty(t, n, dtype=torch.float32, device="cuda")
        ham.ham_fp8_linear(alloc_weight(n, k, w), dev(x[0]), dev(x[1]), y)
        x64, w64 = ops.decode_rows(*x), ops.decode_weight(*w)
        check_bf16(y, x64 @ w64.T, product_slack(x64, w64))


def test_padding_of_the_scales_is_not_read_as_numbers():
    """Scale bytes past the last block may hold anything (255 is NaN), and rows past the call's are
    not touched."""
    import torch
    rng = np.random.default_rng(1)
    for t in (3, 2561):
        k, n = 640, 2304
        x, w = random_codes(rng, t, k), random_codes(rng, n, k, weight=True)
        x[1][:, 5:], w[1][:, 5:] = 255, 255
        y = torch.full((t + 2, n), 7.0, dtype=torch.bfloat16, device="cuda")
        ham.ham_fp8_linear(alloc_weight(n, k, w), dev(x[0]), dev(x[1]), y[:t])
        x64, w64 = ops.decode_rows(*x), ops.decode_weight(*w)
        check_bf16(y[:t], x64 @ w64.T, product_slack(x64, w64))
        assert (y[t:] == 7).all()


def test_same_answer_on_every_call_and_row_position():
    """Sums run in one order: calls repeat bit for bit, and a row's result does not depend on the
    rows beside it within one call's kernel."""
    import torch
    rng = np.random.default_rng(2)
    k, n = 4096, 512
    x, w = random_codes(rng, 16, k), random_codes(rng, n, k, weight=True)
    handle = alloc_weight(n, k, w)
    ys = []
    for _ in range(3):
        y = torch.empty(16, n, dtype=torch.float32, device="cuda")
        ham.ham_fp8_linear(handle, dev(x[0]), dev(x[1]), y)
        ys.append(y)
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])
    y1 = torch.empty(1, n, dtype=torch.float32, device="cuda")
    ham.ham_fp8_linear(handle, dev(x[0][9:10]), dev(x[1][9:10]), y1)
    assert torch.equal(y1[0], ys[0][9])


def test_products_in_a_graph_and_back_to_back():
    """The chain encode -> linear -> norm -> gated -> linear, captured and replayed, equals the calls
    made one by one."""
    import torch
    rng = np.random.default_rng(4)
    t, h, f = 24, 1024, 2048
    wo, w2 = alloc_weight(h, h, random_codes(rng, h, h, True)), alloc_weight(h, f, random_codes(rng, h, f, True))
    w13 = alloc_weight(f, h, random_codes(rng, f, h, True), random_codes(rng, f, h, True))
    nw = torch.ones(h, dtype=torch.bfloat16, device="cuda") * 2.0 ** -6
    x = torch.randn(t, h, device="cuda").bfloat16()
    c1, s1 = empty_rows(t, h)
    c2, s2 = empty_rows(t, h)
    c3, s3 = empty_rows(t, f)
    y1, total, y2 = (torch.empty_like(x) for _ in range(3))

    def chain():
        ham.ham_fp8_encode(x, c1, s1)
        ham.ham_fp8_linear(wo, c1, s1, y1)
        ham.ham_add_norm(y1, nw, 1e-5, residual=x, sum_out=total, codes=c2, scales=s2)
        ham.ham_fp8_gated(w13, c2, s2, c3, s3)
        ham.ham_fp8_linear(w2, c3, s3, y2)

    chain()
    torch.cuda.synchronize()
    want = [v.clone() for v in (c1, s1, y1, total, c2, s2, c3, s3, y2)]
    assert torch.isfinite(y2.float()).all()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for _ in range(4):
            chain()
    for v in (y1, total, y2):
        v.fill_(float("nan"))
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, (c1, s1, y1, total, c2, s2, c3, s3, y2)):
        assert torch.equal(a, b)


def test_no_rows_and_refusals():
    import torch
    rng = np.random.default_rng(5)
    k, n = 256, 160
    w = random_codes(rng, n, k, True)
    plain, gated = alloc_weight(n, k, w), alloc_weight(n, k, w, w)
    x, s = empty_rows(2, k)
    y = torch.empty(2, n, dtype=torch.bfloat16, device="cuda")
    ham.ham_fp8_linear(plain, x[:0], s[:0], y[:0])
    with pytest.raises(ham.HamError, match="gated"):
        ham.ham_fp8_linear(gated, x, s, y)
    with pytest.raises(ham.HamError, match="gated"):
        ham.ham_fp8_gated(plain, x, s, *empty_rows(2, n))
    with pytest.raises(ValueError, match="x_codes must have shape"):
        ham.ham_fp8_linear(plain, x[:, :128].contiguous(), s, y)
    with pytest.raises(ValueError, match="contiguous"):
        ham.ham_fp8_linear(plain, torch.empty(k, 2, dtype=torch.uint8, device="cuda").t(), s, y)
    buf = torch.zeros(4 * k * n, dtype=torch.uint8, device="cuda")
    with pytest.raises(ham.HamError, match="overlap"):
        ham.ham_fp8_linear(plain, buf[:2 * k].view(2, k), s, buf[k:k + 4 * n].view(torch.bfloat16).view(2, n))
    for bad in (dict(n=0), dict(k=24), dict(k=0)):
        a = dict(n=n, k=k)
        a.update(bad)
        with pytest.raises((ham.HamError, ValueError)):
            ham.ham_fp8_weight_alloc(a["n"], a["k"], dev(w[0]), dev(w[1]))

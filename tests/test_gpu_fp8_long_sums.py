"""Long sums of the 8-bit products: parts of K of their own, added in fp32, so that the error does not grow
with K as one accumulator's does; every form of the pair kernel, with accumulators used again."""
import numpy as np
import pytest

from oracle import ops
from ops_helpers import alloc_weight, check_bf16, check_codes, dev, empty_rows, random_codes
from paper_2505_20438_gb300 import ham

pytestmark = pytest.mark.gpu


def slack(x, w):
    """A part of at most 4096 terms adds 32 of them at a time, off by at most a unit of 2^-23 of the magnitudes
    that meet in it, which sum|x w| bounds; then at most K / 2048 parts are added, half a unit each; two spare."""
    k = x.shape[1]
    return (min(k, 4096) / 32 + k / 4096 + 2) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T)


def _pair_tiles(rows, features, gated):
    """Tiles of 256 rows a pair of CTAs computes at least, of a product that the pair kernel takes."""
    import torch
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    tiles = -(-rows // 256) * (-(-features // 128) if gated else -(-features // 256))
    assert rows > 128 and tiles * 8 >= sms
    return -(-tiles // (sms // 2))


def _linear(t, k, n, f32):
    import torch
    rng = np.random.default_rng(t + 3 * k + 5 * n)
    x, w = random_codes(rng, t, k), random_codes(rng, n, k, weight=True)
    handle = alloc_weight(n, k, w)
    y = torch.full((t, n), float("nan"), dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    ham.ham_fp8_linear(handle, dev(x[0]), dev(x[1]), y)
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(handle) == 0
    x64, w64 = ops.decode_rows(*x), ops.decode_weight(*w)
    check_bf16(y, x64 @ w64.T, slack(x64, w64))


def _gated(t, k, f):
    import torch
    rng = np.random.default_rng(3 * t + 7 * k + 5 * f)
    x, g, u = random_codes(rng, t, k), random_codes(rng, f, k, weight=True), random_codes(rng, f, k, weight=True)
    size = int(np.log2(np.sqrt(k) * 100.0 ** 2)) // 2    # G of the order of one
    for s in (x[1], g[1], u[1]):
        s[:] = 127 - size + (s & 3)
    codes, scales = empty_rows(t, f)
    handle = alloc_weight(f, k, g, u)
    ham.ham_fp8_gated(handle, dev(x[0]), dev(x[1]), codes, scales)
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(handle) == 0
    x64, g64, u64 = ops.decode_rows(*x), ops.decode_weight(*g), ops.decode_weight(*u)
    G, U, h = ops.gated(x64, g64, u64)
    dg, du = slack(x64, g64), slack(x64, u64)
    silu = np.abs(ops.silu(G))
    check_codes(codes, scales, h, 1.1 * dg * (np.abs(U) + du) + silu * du + 2.0 ** -20 * silu * np.abs(U))


# one part of K and a block more, parts that end inside a scale word, odd numbers of blocks, many parts; row and
# column tiles in odd numbers, rows and features off every tile
@pytest.mark.parametrize("t,k,n", [(2304, 2048, 2304), (1281, 2064, 1000), (1300, 4096, 1030), (700, 6160, 2500),
                                   (513, 16400, 1800), (1100, 16384, 1281)])
@pytest.mark.parametrize("f32", [False, True])
def test_pairs_over_many_blocks(t, k, n, f32):
    _pair_tiles(t, n, False)
    _linear(t, k, n, f32)


@pytest.mark.parametrize("t,k,f", [(2561, 144, 2064), (1300, 2064, 528), (1100, 16400, 528)])
def test_gated_pairs_over_many_blocks(t, k, f):
    _pair_tiles(t, f, True)
    _gated(t, k, f)


@pytest.mark.parametrize("k", [144, 2304])
@pytest.mark.parametrize("kind", ["plain", "gated"])
def test_three_tiles_and_more_a_pair(kind, k):
    t, n = (5900, 2320) if kind == "plain" else (4600, 1100 // 16 * 16)
    assert _pair_tiles(t, n, kind == "gated") >= 3
    if kind == "plain":
        _linear(t, k, n, False)
    else:
        _gated(t, k, n)


# few rows: several accumulators a CTA, several splits, and so long that a CTA takes fewer rows
@pytest.mark.parametrize("t,k,n", [(8, 16400, 136), (128, 36880, 130), (100, 131072, 136), (5, 262144, 128), (16, 6160, 20000)])
def test_streams_over_many_blocks(t, k, n):
    _linear(t, k, n, True)


@pytest.mark.parametrize("t,k,f", [(8, 16400, 144), (128, 40960, 144), (16, 6160, 20000), (128, 6160, 256)])
def test_gated_streams_over_many_blocks(t, k, f):
    _gated(t, k, f)


def _decoded(codes, scales, down):
    import torch
    p = ((scales.to(torch.int64) + 896) << 52).view(torch.float64)     # 2^(s - 127)
    return codes.view(torch.float8_e4m3fn).double() * \
        p.repeat_interleave(128, 1)[:, :codes.shape[1]].repeat_interleave(down, 0)[:codes.shape[0]]


@pytest.mark.parametrize("t,k,n", [(2304, 4096, 2304), (2304, 16384, 2304), (8, 4096, 40064), (8, 16384, 40064),
                                   (64, 16384, 20480), (64, 16384, 256), (128, 65536, 1024)])
def test_error_does_not_grow_with_the_length(t, k, n):
    """Of sums of random terms, the error's norm stays below four units of fp32's last place of the sums' norm
    at every length (cut off at each addition in one accumulator, it passes that from some 8192 terms on)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(k + n)
    x = torch.randn((t, k), generator=g, device="cuda").bfloat16()
    xc, xs = empty_rows(t, k)
    ham.ham_fp8_encode(x, xc, xs)
    w = torch.randn((n, k), generator=g, device="cuda").mul_(k ** -0.5).bfloat16()
    wc, ws = empty_rows(n, k)
    ws = ws[:-(-n // 128)].contiguous()
    ham.ham_fp8_encode_weight(w, wc, ws)
    del x, w
    y = torch.empty((t, n), device="cuda")
    ham.ham_fp8_linear(ham.ham_fp8_weight_alloc(n, k, wc, ws), xc, xs, y)
    x64 = _decoded(xc, xs, 1)
    off = size = 0.0
    for r in range(0, n, 4096):
        want = x64 @ _decoded(wc[r:r + 4096], ws[r // 128:-(-min(n, r + 4096) // 128)], 128).T
        off += (y[:, r:r + 4096].double() - want).square().sum().item()
        size += want.square().sum().item()
    assert (off / size) ** 0.5 <= 4 * 2.0 ** -23, (off / size) ** 0.5

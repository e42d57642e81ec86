"""ham_add_norm, ham_fp8_encode and ham_fp8_encode_weight against the fp64 oracle."""
import numpy as np
import pytest

from oracle import ops
from ops_helpers import bf16, check_bf16, check_codes, dev, empty_rows, norm_slack, rows
from paper_2505_20438_gb300 import ham

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.mark.parametrize("t,h", [(1, 16), (3, 128), (2, 144), (5, 1040), (7, 4096), (9, 5136), (2, 8208),
                                 (1, 16384), (2, 32768), (400, 2048)])
@pytest.mark.parametrize("residual", [False, True])
def test_add_norm_matches_oracle(t, h, residual):
    import torch
    rng = np.random.default_rng(t * 100003 + h)
    x, x64 = bf16(rows(rng, t, h))
    r, r64 = bf16(rows(rng, t, h)) if residual else (None, None)
    w, w64 = bf16(1 + 0.2 * rng.standard_normal(h))
    total = torch.full_like(x, float("nan"))
    out = torch.full_like(x, float("nan"))
    codes, scales = empty_rows(t, h)
    ham.ham_add_norm(x, w, EPS, residual=r, sum_out=total, out=out, codes=codes, scales=scales)
    torch.cuda.synchronize()
    h64, y = ops.add_norm(x64, r64, w64, EPS)
    check_bf16(total, h64, 2.0 ** -24 * np.abs(h64))
    check_bf16(out, y, norm_slack(y))
    check_codes(codes, scales, y, norm_slack(y))
    # each output alone gives the same bits
    out2 = torch.empty_like(out)
    ham.ham_add_norm(x, w, EPS, residual=r, out=out2)
    codes2, scales2 = empty_rows(t, h)
    ham.ham_add_norm(x, w, EPS, residual=r, codes=codes2, scales=scales2)
    assert torch.equal(out, out2) and torch.equal(codes, codes2) and torch.equal(scales, scales2)


def test_add_norm_in_place():
    """The residual stream updated where it stands, the norm where the addend stood."""
    import torch
    rng = np.random.default_rng(3)
    x, _ = bf16(rows(rng, 33, 2064))
    r, _ = bf16(rows(rng, 33, 2064))
    w, _ = bf16(np.ones(2064))
    total, out = torch.empty_like(x), torch.empty_like(x)
    ham.ham_add_norm(x, w, EPS, residual=r, sum_out=total, out=out)
    ham.ham_add_norm(x, w, EPS, residual=r, sum_out=r, out=x)
    assert torch.equal(r, total) and torch.equal(x, out)


def test_add_norm_rows_of_zeros_and_of_what_is_not_a_number():
    """A row of zeros gives zeros at scale 1; infinities and NaN stay in their own row, and a NaN
    element gives NaN codes there."""
    import torch
    x = np.ones((4, 256))
    x[1] = 0
    x[2, 3] = np.inf
    x[3, 5] = np.nan
    xt, _ = bf16(x)
    w, _ = bf16(np.ones(256))
    out = torch.empty_like(xt)
    codes, scales = empty_rows(4, 256)
    ham.ham_add_norm(xt, w, EPS, out=out, codes=codes, scales=scales)
    o = out.float().cpu().numpy()
    assert np.isfinite(o[:2]).all() and (o[1] == 0).all()
    assert (codes[1] == 0).all() and (scales[1] == 127).all()
    assert np.isnan(o[2, 3]) and (o[2, :3] == 0).all() and np.isnan(o[3]).all()
    assert (codes[3] & 127 == 127).all()


def test_no_rows_launch_nothing():
    import torch
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    x = torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    codes, scales = empty_rows(0, 64)
    ham.ham_add_norm(x, w, EPS, out=x)
    ham.ham_fp8_encode(x, codes, scales)


@pytest.mark.parametrize("t,k", [(1, 16), (2, 128), (3, 400), (1, 512), (5, 528), (17, 4096), (300, 1808), (1, 65552)])
def test_encode_is_exact(t, k):
    """Bit for bit the oracle's encoding, over sizes from below the smallest scale to the largest."""
    import torch
    rng = np.random.default_rng(k + t)
    x = rng.standard_normal((t, k)) * 2.0 ** rng.integers(-30, 30, (t, k))
    x[rng.random((t, k)) < 0.1] = 0
    if t > 2:
        x[1] = 0
        x[2] *= 2.0 ** -110
    xt, x64 = bf16(x)
    codes, scales = empty_rows(t, k)
    ham.ham_fp8_encode(xt, codes, scales)
    want, e = ops.encode_rows(x64)
    nb = e.shape[1]
    s = scales.cpu().numpy()
    np.testing.assert_array_equal(s[:, :nb].astype(np.int64) - 127, e)
    assert (s[:, nb:] == 127).all()
    np.testing.assert_array_equal(ops.decode_rows(codes.cpu().numpy(), s), want)


def test_encode_at_the_ends_of_the_range():
    import torch
    x = torch.zeros(3, 256, dtype=torch.bfloat16, device="cuda")
    x[0, 0], x[0, 1], x[0, 2] = float("inf"), -float("inf"), float("nan")
    x[1, 0] = 3.3e38
    x[2, 0] = 1e-40                              # below the normal range: 0.0021 of 2^-124
    codes, scales = empty_rows(3, 256)
    ham.ham_fp8_encode(x, codes, scales)
    c = ops.code_values()[codes.cpu().numpy()]
    assert scales[0, 0] == 119 + 127 and c[0, 0] == 448 and c[0, 1] == -448 and np.isnan(c[0, 2])
    assert scales[1, 0] == 119 + 127 and 448 >= c[1, 0] > 200
    assert scales[2, 0] == 127 - 124 and c[2, 0] == 2.0 ** -9


@pytest.mark.parametrize("n,k", [(1, 16), (128, 128), (129, 144), (300, 1040), (257, 2048)])
def test_encode_weight_is_exact(n, k):
    import torch
    rng = np.random.default_rng(n + k)
    wt, w64 = bf16(rng.standard_normal((n, k)) * 2.0 ** rng.integers(-8, 8, (n, 1)))
    codes = torch.full((n, k), 0x7f, dtype=torch.uint8, device="cuda")
    scales = torch.full((-(-n // 128), ops.scale_bytes(k)), 255, dtype=torch.uint8, device="cuda")
    ham.ham_fp8_encode_weight(wt, codes, scales)
    s = scales.cpu().numpy()
    nb = -(-k // 128)
    assert (s[:, nb:] == 127).all()
    v = ops.code_values()[codes.cpu().numpy()]
    for i in range(-(-n // 128)):
        for b in range(nb):
            blk = w64[128 * i:128 * (i + 1), 128 * b:128 * (b + 1)]
            e = int(ops.block_exponent(np.abs(blk).max()))
            assert int(s[i, b]) - 127 == e
            q = blk / 2.0 ** e
            step = ops.step_of(q)
            np.testing.assert_array_equal(v[128 * i:128 * (i + 1), 128 * b:128 * (b + 1)], np.rint(q / step) * step)


def test_calls_run_on_the_current_stream():
    """A tensor made on a side stream is normed there, and again by an explicit stream."""
    import torch
    side = torch.cuda.Stream()
    w, w64 = bf16(np.ones(1024))
    base, b64 = bf16(rows(np.random.default_rng(0), 2000, 1024))
    torch.cuda.synchronize()
    want = ops.add_norm(4 * b64, None, w64, EPS)[1]
    with torch.cuda.stream(side):
        x = base * 4
        out = torch.empty_like(x)
        ham.ham_add_norm(x, w, EPS, out=out)
        twice = torch.empty_like(x)
        ham.ham_add_norm(out, w, EPS, out=twice, stream=side)
    side.synchronize()
    check_bf16(out, want, norm_slack(want))
    assert torch.isfinite(twice.float()).all()


@pytest.mark.parametrize("change,message", [
    (dict(hidden=24), "multiple of 16"), (dict(hidden=32784), "multiple of 16"), (dict(eps=-1.0), "eps"),
    (dict(out=False), "required"), (dict(codes=True), "come together"), (dict(overlap=True), "overlap"),
])
def test_add_norm_refuses(change, message):
    import torch
    h = change.get("hidden", 256)
    buf = torch.zeros(4 * h + 4096, dtype=torch.bfloat16, device="cuda")
    x, w = buf[:2 * h].view(2, h), torch.ones(h, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(2, h, dtype=torch.bfloat16, device="cuda")
    kw = dict(out=out)
    if change.get("out") is False:
        kw = {}
    if change.get("codes"):
        kw["codes"] = torch.empty(2, h, dtype=torch.uint8, device="cuda")
    if change.get("overlap"):
        kw["out"] = buf[h:3 * h].view(2, h)
    with pytest.raises(ham.HamError, match=message) as e:
        ham.ham_add_norm(x, w, change.get("eps", EPS), **kw)
    assert e.value.status == ham.HAM_EINVAL

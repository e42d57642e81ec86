"""ham_add_norm over the whole range of bf16: rows whose squares leave fp32's range are normed like any other."""
import numpy as np
import pytest

from oracle import ops
from ops_helpers import bf16, check_bf16, check_codes, empty_rows, norm_slack
from paper_2505_20438_gb300 import ham

pytestmark = pytest.mark.gpu

SIZES = [-133, -126, -100, -75, -62, -51, -50, -49, 0, 49, 58, 62, 63, 64, 100, 126]


@pytest.mark.parametrize("h", [16, 1040, 4096, 8208, 32768])
@pytest.mark.parametrize("residual", [False, True])
def test_rows_of_every_size(h, residual):
    """Rows of about 2^size, with no eps (the smallest lie below the normal numbers) and beside one row of
    another size."""
    import torch
    rng = np.random.default_rng(h)
    t = len(SIZES)
    scale = 2.0 ** np.array(SIZES, np.float64)[:, None]
    draw = lambda: np.clip(rng.standard_normal((t, h)), -1.9, 1.9) * scale / (2 if residual else 1)
    x, x64 = bf16(draw())
    r, r64 = bf16(draw()) if residual else (None, None)
    w, w64 = bf16(1 + 0.2 * rng.standard_normal(h))
    out, total = torch.empty_like(x), torch.empty_like(x)
    codes, scales = empty_rows(t, h)
    ham.ham_add_norm(x, w, 0.0, residual=r, sum_out=total, out=out, codes=codes, scales=scales)
    h64, y = ops.add_norm(x64, r64, w64, 0.0)
    assert np.abs(y).max() > 1 and (np.sqrt((h64 * h64).mean(axis=1)) > 0).all()
    check_bf16(out, y, norm_slack(y))
    check_codes(codes, scales, y, norm_slack(y))
    check_bf16(total, h64, 2.0 ** -24 * np.abs(h64))


def test_eps_beside_rows_of_every_size():
    import torch
    rng = np.random.default_rng(1)
    t, h = len(SIZES), 2064
    x, x64 = bf16(np.clip(rng.standard_normal((t, h)), -1.9, 1.9) * 2.0 ** np.array(SIZES, np.float64)[:, None])
    w, w64 = bf16(np.ones(h))
    for eps in (1e-5, 1e-12, 2.0 ** -110, 2.0 ** -140):
        out = torch.empty_like(x)
        ham.ham_add_norm(x, w, eps, out=out)
        _, y = ops.add_norm(x64, None, w64, float(np.float32(eps)))
        check_bf16(out, y, norm_slack(y) + 2.0 ** -149)

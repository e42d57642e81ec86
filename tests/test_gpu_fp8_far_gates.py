"""Gates far below zero in ham_fp8_gated, where exp(-g) leaves fp32: the values are the formula's, however small, as the
experts' products have them."""
import numpy as np
import pytest

from oracle import ops
from paper_2505_20438_gb300 import ham
from tests.ops_helpers import alloc_weight, check_codes, dev, empty_rows, product_slack
from tests.test_gpu_experts import _exact_codes

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 40, 300, 3000])
def test_gates_far_from_zero(rows):
    """Gates down to -105 (where exp(g) leaves fp32's normal numbers and then fp32) and up to 300, a block each."""
    rng = np.random.default_rng(12)
    n, k = 128 * 6, 128
    far = np.repeat([-85.0, -88.0, -95.0, -105.0, 60.0, 300.0], 128)
    wg, wu = np.zeros((1, n, k)), rng.standard_normal((1, n, k)) * 64
    wg[0, :, 0] = far / 4
    (gc, gs), (uc, us) = _exact_codes(wg), _exact_codes(wu)
    xc = rng.integers(0, 40, (rows, k)).astype(np.uint8)
    xc[:, 0] = 0x48                          # 4
    xs = np.full((rows, ops.scale_bytes(k)), 127, np.uint8)
    h = alloc_weight(n, k, (gc[0], gs[0]), (uc[0], us[0]))
    codes, scales = empty_rows(rows, n)
    ham.ham_fp8_gated(h, dev(xc), dev(xs), codes, scales)
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE
    x, wg, wu = ops.decode_rows(xc, xs), ops.decode_weight(gc[0], gs[0]), ops.decode_weight(uc[0], us[0])
    g, u, want = ops.gated(x, wg, wu)
    assert (np.abs(g - far) <= np.abs(far) / 16).all()
    # (A gate is one product, exact; the rest as in gated_slack.  2^-149: the exponential's last place, where it is not a
    # normal number, once for itself and once for its product with the gate.)
    silu = np.abs(ops.silu(g))
    check_codes(codes, scales, want, silu * product_slack(x, wu) + 2.0 ** -20 * silu * np.abs(u) + 2.0 ** -148 * np.abs(g * u))

"""How exact the routing's weights are where they leave fp32's normal numbers: far logits of a softmax that is not
renormalised, and small scales."""
import numpy as np
import pytest

from oracle import experts as ox
from paper_2505_20438_gb300 import ham
from tests.test_gpu_route import _logits, _outputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1.0, 2.5, -3.0, 2.0 ** 60, 2.0 ** -20, 1e-30, 1e-38, 2.0 ** -149, 0.0])
@pytest.mark.parametrize("sigmoid,renorm", [(False, False), (False, True), (True, False), (True, True)])
def test_weights_near_the_end_of_the_range(scale, sigmoid, renorm):
    """2^-18 of themselves; |scale| 2^-140 for a score below the normal numbers (its exponential, its quotient: a few units of
    2^-149, times the scale), 2^-149 for a product that is (half a unit)."""
    experts, k = 16, 16
    l = np.stack([-np.arange(experts) * s for s in (0.5, 5.0, 6.0, 6.9, 7.3, 9.0)] * 4)
    t, ref = _logits(l)
    got = _outputs(len(l), k, experts)
    ham.ham_route(t, *got, score=ham.HAM_SCORE_SIGMOID if sigmoid else ham.HAM_SCORE_SOFTMAX, renorm=renorm, scale=scale)
    expert, weight = got[0].cpu().numpy(), got[1].double().cpu().numpy()
    s = float(np.float32(scale))
    for i, row in enumerate(ref):
        e, w = ox.choose(row, k, sigmoid=sigmoid, renorm=renorm, scale=s)
        assert expert[i].tolist() == e.tolist()
        assert (np.abs(weight[i] - w) <= 2.0 ** -18 * np.abs(w) + abs(s) * 2.0 ** -140 + 2.0 ** -149).all(), (weight[i], w)

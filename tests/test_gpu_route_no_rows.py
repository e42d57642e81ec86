"""An empty batch routes to no slots: buffers that a program keeps hold no grouping of the call before."""
import numpy as np
import pytest

from paper_2505_20438_gb300 import ham
from tests.ops_helpers import dev, random_codes
from tests.test_gpu_experts import alloc, weights
from tests.test_gpu_route import _logits, _outputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("experts", [1, 60, 512])
@pytest.mark.parametrize("captured", [False, True])
def test_no_rows_leave_no_slots(experts, captured):
    import torch
    rng = np.random.default_rng(experts)
    n, k = 128, 128
    t, _ = _logits(rng.standard_normal((5, experts)))
    got = _outputs(5, 1, experts)
    none, empty = t[:0], (got[0][:0], got[1][:0], got[2], got[3][:0], got[4][:0])
    h = alloc(n, k, weights(rng, experts, n, k))
    x = [dev(v) for v in random_codes(rng, 5, k)]
    y = torch.full((5, n), -7.0, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                ham.ham_route(none, *empty)
                ham.ham_fp8_experts_linear(h, *x, got[2], y)
        ham.ham_route(t, *got)
        before = got[2].clone()
        if captured:
            graph.replay()
        else:
            ham.ham_route(none, *empty)
            ham.ham_fp8_experts_linear(h, *x, got[2], y)
    torch.cuda.synchronize()
    assert before[-1] == 5 and (got[2] == 0).all()
    assert (y == -7).all()                           # (the fixed buffers' rows belong to no expert)
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE

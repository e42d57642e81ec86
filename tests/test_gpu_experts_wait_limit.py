"""A wait of the experts' products that runs out is reported through the weights' error word, and the weights keep
working afterwards: the waits are made to run out on a healthy GPU by shortening their limit to a nanosecond
(ham_fp8_weight_set_wait_limit_ns), as in test_gpu_fp8_wait_limit.py."""
import numpy as np
import pytest

from paper_2505_20438_gb300 import ham
from tests.ops_helpers import dev, empty_rows, random_codes
from tests.test_gpu_experts import alloc, grouping, weights

pytestmark = pytest.mark.gpu


# rows by index and rows that are sorted first; tiles of one half and of two; one tile a pair of CTAs and several
@pytest.mark.parametrize("counts,n,k", [([40, 0, 7], 384, 4096), ([300, 200], 512, 8208), ([1] * 200, 256, 2304),
                                        ([500, 3, 90, 225] * 12, 512, 2064)], ids=["few", "sorted", "many", "mixed"])
@pytest.mark.parametrize("gated", [False, True])
def test_a_wait_runs_out_and_the_weights_recover(counts, n, k, gated):
    import torch
    rng = np.random.default_rng(len(counts) + k)
    slots = int(np.sum(counts))
    w = weights(rng, len(counts), n, k)
    x = [dev(a) for a in random_codes(rng, slots, k)]
    offsets, order = grouping(rng, counts, 1, slots)
    h = alloc(n, k, w, w if gated else None)
    offsets, order = dev(offsets), dev(order)

    def call():
        if gated:
            out = empty_rows(slots, n)
            ham.ham_fp8_experts_gated(h, *x, offsets, order, 1, *out)
            return out
        y = torch.empty(slots, n, device="cuda")
        ham.ham_fp8_experts_linear(h, *x, offsets, y)
        return (y,)

    want = call()
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE
    ham.ham_fp8_weight_set_wait_limit_ns(h, 1)
    for _ in range(3):
        call()
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_TIMEOUT
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE     # read and cleared
    ham.ham_fp8_weight_set_wait_limit_ns(h, 0)
    for _ in range(2):
        for a, b in zip(want, call()):
            assert torch.equal(a, b)
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE

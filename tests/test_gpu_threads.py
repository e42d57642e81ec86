"""Calls from a thread that has made no CUDA call before: it has no context yet, and the calls give it one."""
import threading

import numpy as np
import pytest

from paper_2505_20438_gb300 import ham
from tests.ops_helpers import alloc_weight, dev, empty_rows, random_codes
from tests.test_gpu_experts import alloc, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["linear", "gated", "experts_linear", "experts_gated", "route", "combine"])
def test_first_call_of_a_thread(call):
    import torch
    rng = np.random.default_rng(1)
    n, k, rows = 128, 256, 6
    x = [dev(v) for v in random_codes(rng, rows, k)]
    w = weights(rng, 2, n, k)
    offsets, order = dev(np.int32([0, 2, rows])), dev(np.arange(rows, dtype=np.int32))
    logits = torch.randn((rows, 8), device="cuda")
    ints = [torch.empty(s, dtype=torch.int32, device="cuda") for s in ((rows, 2), (9,), (2 * rows,), (rows, 2))]
    share = torch.rand((rows, 2), device="cuda")
    place = dev(np.arange(2 * rows, dtype=np.int32).reshape(rows, 2))
    results = torch.randn((2 * rows, n), device="cuda")

    def outputs():
        if call in ("gated", "experts_gated"):
            return empty_rows(rows, n)
        if call == "route":
            return (*[torch.zeros_like(i) for i in ints], torch.zeros_like(share))
        if call == "combine":
            return (torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda"),)
        return (torch.zeros((rows, n), device="cuda"),)

    one = [(w[0][0], w[1][0])] * 2
    h = {"linear": lambda: alloc_weight(n, k, one[0]), "gated": lambda: alloc_weight(n, k, *one),
         "experts_linear": lambda: alloc(n, k, w), "experts_gated": lambda: alloc(n, k, w, w)}.get(call, lambda: None)()
    run = {"linear": lambda o: ham.ham_fp8_linear(h, *x, *o), "gated": lambda o: ham.ham_fp8_gated(h, *x, *o),
           "experts_linear": lambda o: ham.ham_fp8_experts_linear(h, *x, offsets, *o),
           "experts_gated": lambda o: ham.ham_fp8_experts_gated(h, *x, offsets, order, 1, *o),
           "route": lambda o: ham.ham_route(logits, o[0], o[4], o[1], o[2], o[3]),
           "combine": lambda o: ham.ham_experts_combine(results, share, place, *o)}[call]
    want, got, failed = outputs(), outputs(), []
    run(want)
    torch.cuda.synchronize()

    def work():
        try:
            run(got)
        except Exception as e:      # (raised in the test, not in the thread)
            failed.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    assert all(torch.equal(a, b) for a, b in zip(got, want))

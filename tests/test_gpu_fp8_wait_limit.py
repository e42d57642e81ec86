"""A wait of the 8-bit products that runs out is reported through the weight's error word, and the weight
keeps working afterwards.

The waits are made to run out on a healthy GPU by shortening their limit to a nanosecond
(ham_fp8_weight_set_wait_limit_ns): every CTA has more blocks of K than stages or scale words, and finds one
that is not free again by the first poll, so it gives up, with copies and products on their way.  The kernel
waits for those, frees its tensor memory and ends.  No fault, trap or endless loop is involved.
"""
import numpy as np
import pytest

from ops_helpers import alloc_weight, dev, empty_rows, random_codes
from paper_2505_20438_gb300 import ham

pytestmark = pytest.mark.gpu


# the stream kernel's CTAs alone and in clusters that share K; the pair kernel with one part of K and with several
@pytest.mark.parametrize("t,k,n", [(8, 4096, 40000), (8, 16400, 136), (200, 2064, 300), (5900, 1280, 4096),
                                   (2304, 16400, 2304), (2304, 8208, 4000)])
@pytest.mark.parametrize("gated", [False, True])
def test_a_wait_runs_out_and_the_weight_recovers(t, k, n, gated):
    import torch
    n = n // 2 // 16 * 16 if gated else n
    rng = np.random.default_rng(t + k + n)
    x = [dev(a) for a in random_codes(rng, t, k)]
    w = alloc_weight(n, k, *(random_codes(rng, n, k, True) for _ in range(1 + gated)))

    def call():
        if gated:
            out = empty_rows(t, n)
            ham.ham_fp8_gated(w, *x, *out)
            return out
        y = torch.empty(t, n, device="cuda")
        ham.ham_fp8_linear(w, *x, y)
        return (y,)

    want = call()
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(w) == ham.HAM_DEVERR_NONE
    ham.ham_fp8_weight_set_wait_limit_ns(w, 1)
    for _ in range(3):
        call()
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(w) == ham.HAM_DEVERR_TIMEOUT
    assert ham.ham_fp8_weight_status(w) == ham.HAM_DEVERR_NONE     # read and cleared
    ham.ham_fp8_weight_set_wait_limit_ns(w, 0)
    for _ in range(2):
        for a, b in zip(want, call()):
            assert torch.equal(a, b)
    assert ham.ham_fp8_weight_status(w) == ham.HAM_DEVERR_NONE


def test_wait_limit_above_the_default_is_rejected():
    w = alloc_weight(128, 128, random_codes(np.random.default_rng(0), 128, 128, True))
    with pytest.raises(ham.HamError, match="above the default") as e:
        ham.ham_fp8_weight_set_wait_limit_ns(w, 3_000_000_000)
    assert e.value.status == ham.HAM_EINVAL


def test_the_call_before_does_not_count():
    """A product's CTAs may start while the call before still runs (a sampling lets them at its beginning, and its
    256 CTAs leave room on some SMs): its waits begin when that call has ended."""
    import torch
    rng = np.random.default_rng(1)
    x = [dev(a) for a in random_codes(rng, 8, 4096)]
    w = alloc_weight(512, 4096, random_codes(rng, 512, 4096, True))
    y = torch.empty(8, 512, device="cuda")
    logits = torch.randn((256, 128256), device="cuda")
    u, p = torch.rand(256, device="cuda"), torch.full((256,), 0.9, device="cuda")
    tokens = torch.empty(256, dtype=torch.int32, device="cuda")

    def calls():
        ham.ham_sample(logits, u, tokens, top_p=p)      # some 90 us
        ham.ham_fp8_linear(w, *x, y)                    # some 6
    calls()
    torch.cuda.synchronize()
    want = y.clone()
    ham.ham_fp8_weight_set_wait_limit_ns(w, 40_000)
    torch.cuda._sleep(2_000_000)
    for _ in range(10):
        calls()
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(w) == ham.HAM_DEVERR_NONE
    assert torch.equal(y, want)

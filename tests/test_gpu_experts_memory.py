"""The memory of the rows that are sorted first: the results are those of rows by index, a call without memory falls back to
them, and what the library kept goes back with the last weights that take it."""
import gc

import numpy as np
import pytest

from paper_2505_20438_gb300 import ham
from tests.ops_helpers import dev, empty_rows, random_codes
from tests.test_gpu_experts import alloc, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,k", [(4096, 1024), (4112, 1040)])
@pytest.mark.parametrize("counts", [[5, 0, 9], [30, 0, 70], [1, 1, 1]], ids=str)
def test_sorted_rows_give_the_same_bits(n, k, counts):
    """A batch so small that its rows are read by index, and the same among buffers so long that they are sorted."""
    import torch
    rng = np.random.default_rng(sum(counts))
    total, many = sum(counts), 600
    h = alloc(n, k, weights(rng, 3, n, k), weights(rng, 3, n, k))
    x = [dev(v) for v in random_codes(rng, many, k)]
    offsets = dev(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32))
    order = np.full(many, -1, np.int32)
    order[:total] = rng.permutation(total)
    few, long = empty_rows(total, n), empty_rows(many, n)
    ham.ham_fp8_experts_gated(h, x[0][:total], x[1][:total], offsets, dev(order[:total]), 1, *few)
    ham.ham_fp8_experts_gated(h, *x, offsets, dev(order), 1, *long)
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE
    assert torch.equal(few[0], long[0][:total]) and torch.equal(few[1], long[1][:total])
    assert (long[0][total:] == 0x7f).all() and (long[1][total:] == 255).all()


def test_without_memory_the_rows_are_read_by_index():
    """Buffers whose sorted rows would need more than the device has."""
    import torch
    rng = np.random.default_rng(3)
    n, k, top_k, total = 144, 1 << 16, 32, 40
    rows = int(torch.cuda.mem_get_info()[1] * 1.1) // (k * top_k) + 1
    assert rows * top_k <= 1 << 26
    h = alloc(n, k, weights(rng, 2, n, k), weights(rng, 2, n, k))
    xc, xs = random_codes(rng, 2, k)
    x = (torch.empty((rows, k), dtype=torch.uint8, device="cuda"), torch.empty((rows, xs.shape[1]), dtype=torch.uint8, device="cuda"))
    x[0][:2], x[1][:2] = dev(xc), dev(xs)
    offsets = dev(np.int32([0, 15, total]))
    pairs = rng.permutation(2 * top_k)[:total].astype(np.int32)
    order = torch.full((rows * top_k,), -1, dtype=torch.int32, device="cuda")
    order[:total] = dev(pairs)
    long, few = empty_rows(rows * top_k, n), empty_rows(2 * top_k, n)
    ham.ham_fp8_experts_gated(h, *x, offsets, order, top_k, *long)
    ham.ham_fp8_experts_gated(h, dev(xc), dev(xs), offsets, order[:2 * top_k].contiguous(), top_k, *few)
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE
    assert torch.equal(few[0][:total], long[0][:total]) and torch.equal(few[1][:total], long[1][:total])
    assert (long[0][total:] == 0x7f).all()


def test_the_last_weights_give_the_memory_back():
    import torch
    rng = np.random.default_rng(4)
    n, k, top_k, rows = 16, 1 << 14, 8, 2048
    w = weights(rng, 2, n, k)
    x = [dev(v) for v in random_codes(rng, rows, k)]
    offsets, order = dev(np.int32([0, 3, 7])), dev(np.arange(rows * top_k, dtype=np.int32))
    out = empty_rows(rows * top_k, n)
    h = alloc(n, k, w, w)
    ham.ham_fp8_experts_gated(h, *x, offsets, order, top_k, *out)   # (what a first call loads stays)
    h.close()
    gc.collect()
    torch.cuda.synchronize()
    start = torch.cuda.mem_get_info()[0]
    for _ in range(2):
        first, second = alloc(n, k, w, w), alloc(n, k, w, w)
        for h in (first, second):
            ham.ham_fp8_experts_gated(h, *x, offsets, order, top_k, *out)
        torch.cuda.synchronize()
        sorted_rows = rows * top_k * k
        assert torch.cuda.mem_get_info()[0] < start - sorted_rows     # (the rows were sorted, and their memory kept)
        first.close()
        ham.ham_fp8_experts_gated(second, *x, offsets, order, top_k, *out)
        assert ham.ham_fp8_weight_status(second) == ham.HAM_DEVERR_NONE
        second.close()
        assert torch.cuda.mem_get_info()[0] > start - sorted_rows // 4

"""How exact the experts' sums are: parts of K of their own, added in fp32, so that the tensor cores' cutting off of each
addition does not carry them further from the exact sums than an fp32 product in the usual order is."""
import pytest

from paper_2505_20438_gb300 import ham
from tests.ops_helpers import empty_rows
from tests.test_gpu_fp8_long_sums import _decoded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [128, 1024, 1408, 1424, 2048, 2064, 3328, 4096, 4112, 8192, 16384])
def test_sums_are_as_exact_as_fp32(k):
    """Of random terms the error's norm stays below three quarters of a unit of fp32's last place of the sums' norm (the
    bias that up to 1408 terms leave in one accumulator; 2048 leave a whole unit), or, where sums are so long that an fp32
    product passes that, below five quarters of such a product's."""
    import torch
    t, n, experts = 384, 1024, 2
    g = torch.Generator(device="cuda").manual_seed(k)
    xc, xs = empty_rows(t, k)
    ham.ham_fp8_encode(torch.randn((t, k), generator=g, device="cuda").bfloat16(), xc, xs)
    wc = torch.empty((experts, n, k), dtype=torch.uint8, device="cuda")
    ws = torch.empty((experts, n // 128, ham.fp8_scale_bytes(k)), dtype=torch.uint8, device="cuda")
    for e in range(experts):
        ham.ham_fp8_encode_weight((torch.randn((n, k), generator=g, device="cuda") * k ** -0.5).bfloat16(), wc[e], ws[e])
    y = torch.empty((t, n), device="cuda")
    half = t // 2
    offsets = torch.tensor([0, half, t], dtype=torch.int32, device="cuda")
    ham.ham_fp8_experts_linear(ham.ham_fp8_experts_alloc(experts, n, k, wc, ws), xc, xs, offsets, y)
    off = plain = size = 0.0
    for e in range(experts):
        i = slice(e * half, (e + 1) * half)
        x, w = _decoded(xc[i], xs[i], 1), _decoded(wc[e], ws[e], 128)
        want = x @ w.T
        off += (y[i].double() - want).square().sum().item()
        plain += ((x.float() @ w.float().T).double() - want).square().sum().item()
        size += want.square().sum().item()
    error, usual = (off / size) ** 0.5, (plain / size) ** 0.5
    print(k, error, usual)
    assert error <= max(0.75 * 2.0 ** -23, 1.25 * usual), (error, usual)

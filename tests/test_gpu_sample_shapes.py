"""ham_sample at the shapes where the number of CTAs a row changes: the same tokens as the definition's."""
import numpy as np
import pytest

from test_gpu_sample import SETTINGS, _logits, check_exact

pytestmark = pytest.mark.gpu


# 152 SMs: eight, four, two and one CTA a row, a CTA an SM and two, each side of a change; vocabularies at the most
# logits of a CTA
@pytest.mark.parametrize("b,v", [(19, 32000), (20, 32000), (38, 32000), (39, 32000), (76, 32000), (77, 32000), (152, 40000),
                                 (153, 40000), (20, 128256), (38, 170001), (39, 170001), (5, 1025), (5, 2049), (9, 8193)])
@pytest.mark.parametrize("f32", [True, False])
def test_each_number_of_ctas(b, v, f32):
    rng = np.random.default_rng(b * 31 + v)
    pick = np.arange(b) % len(SETTINGS)
    t, k, p, m = (np.array([SETTINGS[i][j] for i in pick]) for j in range(4))
    check_exact(_logits(rng, b, v, 2.0, f32), rng.random(b).astype(np.float32), t.astype(np.float32),
                np.minimum(k, 2 ** 30).astype(np.int32), p.astype(np.float32), m.astype(np.float32))


@pytest.mark.parametrize("b,v", [(76, 150001), (76, 131072), (60, 140000), (38, 262144), (152, 65536), (150, 65537)])
def test_one_bin_holds_a_whole_row(b, v):
    """All but one of a row's tokens weigh the same, a weight whose lower 16 bits are nearly all set: the sums of
    such weights over a CTA's tokens, as a histogram's bin adds them up, pass 2^32 from 2^16 tokens on."""
    import torch
    d = torch.arange(1, 4096, dtype=torch.float32).div(4096).bfloat16().unique().float().cuda()
    low = (torch.exp(-d) * 2.0 ** 31).to(torch.int64) & 0xffff
    worst = d[low.argmax()].item()
    assert low.max() > 0xf000
    l = torch.full((b, v), -worst, device="cuda")
    l[torch.arange(b), torch.arange(b) * 7 % v] = 0.0
    u = np.linspace(0, 0.9999, b).astype(np.float32)
    for s in ((1.0, 0, 0.9, 0.0), (1.0, 0, 0.37, 0.0), (1.0, v - 5, 0.8, 0.0), (1.0, 0, 1.0, 0.0)):
        check_exact(l.bfloat16(), u, *s)

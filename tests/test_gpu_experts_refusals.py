"""What the experts' products refuse on the host of a call that is right but for one pointer: buffers that overlap, and
alignments."""
import numpy as np
import pytest

from paper_2505_20438_gb300 import ham
from tests.ops_helpers import dev
from tests.test_gpu_experts import alloc, weights

pytestmark = pytest.mark.gpu
E, N, K, S = 2, 128, 256, 4
# Each buffer has 4 KiB of one allocation to itself, so that a pointer that is moved stays within it.
PLACE = dict(x_codes=1, x_scales=2, offsets=3, order=4, codes=5, scales=6, out=7)
BYTES = dict(x_codes=S * K, x_scales=S * 4, offsets=4 * (E + 1), order=4 * S, codes=S * N, scales=S * 4, out=4 * S * N)


@pytest.fixture(scope="module")
def setup():
    import torch
    rng = np.random.default_rng(1)
    w = weights(rng, E, N, K)
    memory = torch.zeros(9 * 4096, dtype=torch.uint8, device="cuda")   # (offsets of zeros: no slots)
    assert memory.data_ptr() % 16 == 0
    return alloc(N, K, w), alloc(N, K, w, w), memory


def _at(memory, moved):
    p = {name: memory.data_ptr() + 4096 * i for name, i in PLACE.items()}
    for name, (other, by) in moved.items():
        p[name] = (p[other] if other else p[name]) + by
    return p


def _linear(setup, f32=True, **moved):
    p = _at(setup[2], moved)
    return ham.lib().ham_fp8_experts_linear(setup[0], p["x_codes"], p["x_scales"], S, p["offsets"], p["out"],
                                            ham.HAM_DTYPE_F32 if f32 else ham.HAM_DTYPE_BF16, ham._stream_ptr(None))


def _gated(setup, **moved):
    p = _at(setup[2], moved)
    return ham.lib().ham_fp8_experts_gated(setup[1], p["x_codes"], p["x_scales"], S, p["offsets"], p["order"], 1, p["codes"],
                                           p["scales"], ham._stream_ptr(None))


def _refused(rc, words):
    assert rc == ham.HAM_EINVAL and words in ham.ham_last_error(), (rc, ham.ham_last_error())


def _last(name, align):
    """The last aligned place within a buffer."""
    return (BYTES[name] - 1) // align * align


@pytest.mark.parametrize("other", ["x_codes", "x_scales", "offsets"])
@pytest.mark.parametrize("f32", [True, False])
def test_linear_refuses_an_output_over_an_input(setup, other, f32):
    bytes_out = BYTES["out"] if f32 else BYTES["out"] // 2
    _refused(_linear(setup, f32, out=(other, 0)), "out overlaps an input")
    _refused(_linear(setup, f32, out=(other, _last(other, 16))), "out overlaps an input")
    align = 16 if other == "x_codes" else 4
    _refused(_linear(setup, f32, **{other: ("out", bytes_out - align)}), "out overlaps an input")
    # one after another is no overlap
    assert _linear(setup, f32, **{other: ("out", bytes_out)}) == ham.HAM_OK
    assert _linear(setup, f32, out=(other, -(-BYTES[other] // 16) * 16)) == ham.HAM_OK


@pytest.mark.parametrize("out", ["codes", "scales"])
@pytest.mark.parametrize("other", ["x_codes", "x_scales", "offsets", "order"])
def test_gated_refuses_an_output_over_an_input(setup, out, other):
    align = 16 if out == "codes" else 4
    _refused(_gated(setup, **{out: (other, 0)}), "an output overlaps an input")
    _refused(_gated(setup, **{out: (other, _last(other, align))}), "an output overlaps an input")
    _refused(_gated(setup, **{other: (out, BYTES[out] - (16 if other == "x_codes" else 4))}), "an output overlaps an input")
    assert _gated(setup, **{out: (other, -(-BYTES[other] // 16) * 16)}) == ham.HAM_OK


def test_gated_refuses_outputs_over_each_other(setup):
    for by in (0, BYTES["codes"] - 4):
        _refused(_gated(setup, scales=("codes", by)), "two outputs overlap")
    _refused(_gated(setup, codes=("scales", 0)), "two outputs overlap")
    assert _gated(setup, scales=("codes", BYTES["codes"])) == ham.HAM_OK


@pytest.mark.parametrize("name,by,words", [("x_codes", 8, "16-byte"), ("out", 8, "16-byte"), ("x_scales", 2, "4-byte"),
                                           ("offsets", 2, "4-byte")])
def test_linear_refuses_alignments(setup, name, by, words):
    _refused(_linear(setup, **{name: (None, by)}), words)


@pytest.mark.parametrize("name,by,words", [("x_codes", 8, "16-byte"), ("codes", 4, "16-byte"), ("x_scales", 1, "4-byte"),
                                           ("offsets", 2, "4-byte"), ("order", 2, "4-byte"), ("scales", 2, "4-byte")])
def test_gated_refuses_alignments(setup, name, by, words):
    _refused(_gated(setup, **{name: (None, by)}), words)


def test_a_weight_of_one_block_serves_no_experts(setup):
    from tests.ops_helpers import alloc_weight
    w = weights(np.random.default_rng(2), 1, N, K)
    one = alloc_weight(N, K, (w[0][0], w[1][0]))
    p = _at(setup[2], {})
    rc = ham.lib().ham_fp8_experts_linear(one, p["x_codes"], p["x_scales"], S, p["offsets"], p["out"], ham.HAM_DTYPE_F32,
                                          ham._stream_ptr(None))
    _refused(rc, "plain weights")

"""More of what the calls after the attention refuse on the host, without a GPU."""
import pytest

from paper_2505_20438_gb300 import build as build_mod
from paper_2505_20438_gb300 import ham


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return ham.lib()


def test_wait_limit_wants_a_handle(lib):
    assert lib.ham_fp8_weight_set_wait_limit_ns(None, 1000) == ham.HAM_EINVAL
    assert "handle" in ham.ham_last_error()


P = 1 << 20         # an aligned address; every call with it is refused before anything is launched


@pytest.mark.parametrize("a,words", [
    (dict(tokens=P + 4 * 99), "input"), (dict(tokens=P + 2 * 4 * 100 - 4), "input"), (dict(probs=P + 64), "input"),
    (dict(tokens=2 * P + 4), "input"), (dict(probs=2 * P), "input"), (dict(temperature=5 * P - 4), "input"),
    (dict(top_k=5 * P), "input"), (dict(top_p=6 * P + 4), "input"), (dict(min_p=6 * P - 4), "input"),
    (dict(probs=5 * P + 4), "two outputs"), (dict(probs=5 * P), "two outputs"),
])
def test_sample_refuses_outputs_that_overlap(lib, a, words):
    v = dict(logits=P, dtype=ham.HAM_DTYPE_F32, rows=2, vocab=100, u=2 * P, temperature=None, top_k=None, top_p=None,
             min_p=None, tokens=5 * P, probs=6 * P)
    v.update(a)
    rc = lib.ham_sample(*[v[n] for n in ("logits", "dtype", "rows", "vocab", "u", "temperature", "top_k", "top_p",
                                         "min_p", "tokens", "probs")], None)
    assert rc == ham.HAM_EINVAL and words in ham.ham_last_error() and "overlap" in ham.ham_last_error()

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

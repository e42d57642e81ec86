"""What ham_route refuses of an empty batch on the host, without a GPU."""
import pytest

from paper_2505_20438_gb300 import ham
from tests.test_experts_abi_cpu import P, _refused, _route, lib  # noqa: F401

NONE = dict(rows=0, logits=None, expert=None, weight=None, order=None, place=None)


@pytest.mark.parametrize("a,words", [
    (dict(bias=None, offsets=5 * P + 2), "aligned"), (dict(offsets=2 * P + 4 * 63), "overlaps an input"),
    (dict(offsets=2 * P - 4 * 64), "overlaps an input"),
])
def test_an_empty_batch_keeps_the_offsets_rules(lib, a, words):  # noqa: F811
    _refused(_route(lib, **NONE, **a), words)


def test_an_empty_batch_may_leave_them_out(lib):  # noqa: F811
    assert _route(lib, **NONE, offsets=None) == ham.HAM_OK

"""The experts' calls without a GPU: what the library refuses on the host, and the binding's checks."""
import ctypes

import pytest

from paper_2505_20438_gb300 import build as build_mod
from paper_2505_20438_gb300 import ham


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return ham.lib()


P = 1 << 20         # an aligned address; every call with it is refused before anything is launched
BF16, F32 = ham.HAM_DTYPE_BF16, ham.HAM_DTYPE_F32


def _refused(rc, words, status=ham.HAM_EINVAL):
    assert rc == status and words in ham.ham_last_error(), ham.ham_last_error()


def _route(lib, **a):
    v = dict(logits=P, dtype=F32, bias=2 * P, rows=4, experts=64, top_k=8, score=0, groups=1, top_groups=1, renorm=1,
             scale=1.0, expert=3 * P, weight=4 * P, offsets=5 * P, order=6 * P, place=7 * P)
    v.update(a)
    return lib.ham_route(*v.values(), None)


@pytest.mark.parametrize("a,words", [
    (dict(dtype=2), "logits_dtype"), (dict(score=2), "score"), (dict(rows=-1), "rows"), (dict(rows=(1 << 24) + 1), "rows"),
    (dict(experts=0), "experts"), (dict(experts=513), "experts"), (dict(groups=0), "groups"), (dict(groups=3), "groups"),
    (dict(groups=64), "groups"), (dict(groups=8, top_groups=9), "top_groups"), (dict(top_groups=0), "top_groups"),
    (dict(top_k=0), "top_k"), (dict(top_k=33), "top_k"), (dict(experts=4, top_k=5), "top_k"),
    (dict(groups=8, top_groups=1, top_k=9), "top_k"), (dict(scale=float("nan")), "scale"),
    (dict(scale=float("inf")), "scale"), (dict(logits=None), "required"), (dict(expert=None), "required"),
    (dict(weight=None), "required"), (dict(offsets=None), "required"), (dict(order=None), "required"),
    (dict(place=None), "required"), (dict(logits=P + 2), "aligned"), (dict(bias=2 * P + 2), "aligned"),
    (dict(order=6 * P + 1), "aligned"), (dict(dtype=BF16, logits=P + 1), "aligned"),
    (dict(expert=P + 4 * 255), "input"), (dict(offsets=2 * P - 4 * 64), "input"), (dict(place=6 * P + 4 * 31), "two outputs"),
    (dict(weight=3 * P), "two outputs"), (dict(offsets=6 * P - 4 * 64), "two outputs"),
])
def test_route_refuses(lib, a, words):
    _refused(_route(lib, **a), words)


def test_no_rows_need_no_buffers(lib):
    none = dict(logits=None, bias=None, expert=None, weight=None, offsets=None, order=None, place=None)
    assert _route(lib, rows=0, **none) == ham.HAM_OK
    assert lib.ham_experts_combine(None, BF16, None, None, None, 0, 8, 128, None, None) == ham.HAM_OK


@pytest.mark.parametrize("experts,n,k,up,words", [
    (0, 128, 128, None, "experts 0"), (513, 128, 128, None, "experts 513"), (4, 0, 128, None, "n 0"),
    (4, 128, 24, None, "k 24"), (4, 100, 128, P, "gated"), (4, 1 << 23, 128, None, "n 8388608"),
])
def test_alloc_refuses(lib, experts, n, k, up, words):
    out = ctypes.c_void_p(7)
    _refused(lib.ham_fp8_experts_alloc(experts, n, k, P, P, up, up, ctypes.byref(out)), words)
    assert out.value is None


def test_alloc_refuses_pointers_and_sizes(lib):
    out = ctypes.c_void_p(7)
    alloc = lib.ham_fp8_experts_alloc
    _refused(alloc(4, 128, 128, P, P, None, None, None), "out")
    _refused(alloc(4, 128, 128, None, P, None, None, ctypes.byref(out)), "required")
    _refused(alloc(4, 128, 128, P, None, None, None, ctypes.byref(out)), "required")
    _refused(alloc(4, 128, 128, P, P, P, None, ctypes.byref(out)), "come together")
    _refused(alloc(4, 128, 128, P + 8, P, None, None, ctypes.byref(out)), "aligned")
    _refused(alloc(512, 1 << 22, 1 << 20, P, P, None, None, ctypes.byref(out)), "too large", ham.HAM_EUNSUPPORTED)
    assert out.value is None


def test_calls_want_a_handle(lib):
    _refused(lib.ham_fp8_experts_gated(None, P, P, 1, P, P, 1, P, P, None), "handle")
    _refused(lib.ham_fp8_experts_linear(None, P, P, 1, P, P, 0, None), "handle")


@pytest.mark.parametrize("a,words", [
    (dict(dtype=3), "y_dtype"), (dict(rows=-1), "rows"), (dict(top_k=0), "top_k"), (dict(top_k=33), "top_k"),
    (dict(n=0), "n 0"), (dict(n=(1 << 20) + 1), "n 1048577"), (dict(y=None), "required"), (dict(weight=None), "required"),
    (dict(place=None), "required"), (dict(out=None), "required"), (dict(y=P + 8), "aligned"), (dict(add=2 * P + 2), "aligned"),
    (dict(out=9 * P + 8), "aligned"), (dict(weight=3 * P + 1), "aligned"), (dict(out=P + 16 * 64), "overlaps"),
    (dict(out=3 * P), "overlaps"), (dict(out=4 * P), "overlaps"), (dict(out=2 * P + 16), "overlaps"),
])
def test_combine_refuses(lib, a, words):
    v = dict(y=P, dtype=BF16, weight=3 * P, place=4 * P, add=2 * P, rows=4, top_k=2, n=256, out=9 * P)
    v.update(a)
    _refused(lib.ham_experts_combine(*v.values(), None), words)


def test_binding_rejects_host_tensors():
    import types

    import torch
    f, b, i = torch.zeros(2, 4), torch.zeros(2, 256, dtype=torch.uint8), torch.zeros(2, 4, dtype=torch.int32)
    w = types.SimpleNamespace(n=128, k=256, experts=4)
    for call, name in ((lambda: ham.ham_route(f, i, f, i, i, i), "logits"),
                       (lambda: ham.ham_fp8_experts_alloc(2, 4, 256, b, b), "codes"),
                       (lambda: ham.ham_fp8_experts_gated(w, b, b, i, i, 2, b, b), "x_codes"),
                       (lambda: ham.ham_fp8_experts_linear(w, b, b, i, f), "x_codes"),
                       (lambda: ham.ham_experts_combine(f, f, i, f), "y")):
        with pytest.raises(ValueError, match=f"^{name} must be a CUDA tensor"):
            call()

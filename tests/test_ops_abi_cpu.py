"""The calls after the attention without a GPU: what the library refuses on the host, and the binding's
checks of its tensors."""
import ctypes

import pytest

from paper_2505_20438_gb300 import build as build_mod
from paper_2505_20438_gb300 import ham


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return ham.lib()


P = 4096            # an aligned address; every call with it is refused before anything is launched


def _refused(rc, status, *words):
    assert rc == status, ham.ham_last_error()
    for w in words:
        assert w in ham.ham_last_error()


@pytest.mark.parametrize("a,words", [
    (dict(rows=-1), ["rows"]), (dict(hidden=8), ["hidden"]), (dict(hidden=40), ["hidden"]),
    (dict(hidden=65536), ["hidden"]), (dict(eps=-1.0), ["eps"]), (dict(eps=float("nan")), ["eps"]),
    (dict(x=None), ["x and weight"]), (dict(weight=None), ["x and weight"]), (dict(x=P + 8), ["aligned"]),
    (dict(scales=2), ["aligned"]), (dict(codes=None), ["come together"]),
    (dict(out=None, codes=None, scales=None), ["required"]), (dict(codes=P), ["overlap"]),
    (dict(out=P + 16), ["overlap"]), (dict(sum_out=64 * P, out=64 * P), ["two outputs overlap"]),
])
def test_add_norm_refuses(lib, a, words):
    v = dict(x=P, residual=None, weight=2 * P, eps=1e-5, rows=4, hidden=256, sum_out=None, out=32 * P, codes=64 * P,
             scales=128 * P)
    v.update(a)
    args = [v[n] for n in ("x", "residual", "weight", "eps", "rows", "hidden", "sum_out", "out", "codes", "scales")]
    _refused(lib.ham_add_norm(*args, None), ham.HAM_EINVAL, *words)


def test_no_rows_need_no_buffers(lib):
    assert lib.ham_add_norm(None, None, None, 1e-5, 0, 256, None, None, None, None, None) == ham.HAM_OK
    assert lib.ham_fp8_encode(None, 0, 256, None, None, None) == ham.HAM_OK
    assert lib.ham_sample(None, 1, 0, 100, None, None, None, None, None, None, None, None) == ham.HAM_OK


def test_encoders_refuse(lib):
    _refused(lib.ham_fp8_encode(P, 2, 100, 2 * P, 3 * P, None), ham.HAM_EINVAL, "k 100")
    _refused(lib.ham_fp8_encode(P, 2, 128, None, 3 * P, None), ham.HAM_EINVAL, "required")
    _refused(lib.ham_fp8_encode(P, 64, 128, P + 64, 9 * P, None), ham.HAM_EINVAL, "overlap")
    _refused(lib.ham_fp8_encode(P, 64, 128, 9 * P + 1, 20 * P, None), ham.HAM_EINVAL, "aligned")
    _refused(lib.ham_fp8_encode_weight(P, 0, 128, 9 * P, 20 * P, None), ham.HAM_EINVAL, "n 0")
    _refused(lib.ham_fp8_encode_weight(None, 4, 128, 9 * P, 20 * P, None), ham.HAM_EINVAL, "required")


@pytest.mark.parametrize("n,k,up,words", [
    (0, 128, None, "n 0"), (128, 0, None, "k 0"), (128, 24, None, "k 24"), (1 << 23, 128, None, "n 8388608"),
    (100, 128, P, "gated"),
])
def test_weight_alloc_refuses(lib, n, k, up, words):
    out = ctypes.c_void_p(7)
    _refused(lib.ham_fp8_weight_alloc(n, k, P, P, up, up, ctypes.byref(out)), ham.HAM_EINVAL, words)
    assert out.value is None


def test_weight_calls_refuse_nothing_given(lib):
    out = ctypes.c_void_p(7)
    _refused(lib.ham_fp8_weight_alloc(128, 128, None, P, None, None, ctypes.byref(out)), ham.HAM_EINVAL, "required")
    _refused(lib.ham_fp8_weight_alloc(128, 128, P, P, P, None, ctypes.byref(out)), ham.HAM_EINVAL, "come together")
    _refused(lib.ham_fp8_weight_alloc(128, 128, P + 4, P, None, None, ctypes.byref(out)), ham.HAM_EINVAL, "aligned")
    _refused(lib.ham_fp8_weight_alloc(128, 128, P, P, None, None, None), ham.HAM_EINVAL, "out")
    _refused(lib.ham_fp8_linear(None, P, P, 1, P, 0, None), ham.HAM_EINVAL, "handle")
    _refused(lib.ham_fp8_gated(None, P, P, 1, P, P, None), ham.HAM_EINVAL, "handle")
    _refused(lib.ham_fp8_weight_status(None, None, None), ham.HAM_EINVAL, "handle")
    assert lib.ham_fp8_weight_free(None) == ham.HAM_OK


@pytest.mark.parametrize("a,status,words", [
    (dict(dtype=7), ham.HAM_EINVAL, "logits_dtype"), (dict(rows=-1), ham.HAM_EINVAL, "rows"),
    (dict(rows=70000), ham.HAM_EINVAL, "rows"), (dict(vocab=0), ham.HAM_EINVAL, "vocab"),
    (dict(vocab=(1 << 18) + 1), ham.HAM_EUNSUPPORTED, "vocab"), (dict(logits=None), ham.HAM_EINVAL, "required"),
    (dict(u=None), ham.HAM_EINVAL, "required"), (dict(tokens=None), ham.HAM_EINVAL, "required"),
    (dict(logits=P + 2), ham.HAM_EINVAL, "aligned"), (dict(top_k=P + 2), ham.HAM_EINVAL, "aligned"),
])
def test_sample_refuses(lib, a, status, words):
    v = dict(logits=P, dtype=1, rows=2, vocab=100, u=P, temperature=None, top_k=None, top_p=None, min_p=None, tokens=P,
             probs=None)
    v.update(a)
    _refused(lib.ham_sample(*[v[n] for n in ("logits", "dtype", "rows", "vocab", "u", "temperature", "top_k", "top_p",
                                             "min_p", "tokens", "probs")], None), status, words)


def test_binding_rejects_host_tensors():
    import types

    import torch
    x, b = torch.zeros(2, 256, dtype=torch.bfloat16), torch.zeros(2, 256, dtype=torch.uint8)
    w = types.SimpleNamespace(n=128, k=256)
    s = torch.zeros(2, 4, dtype=torch.uint8)
    for call, name in ((lambda: ham.ham_add_norm(x, x[0], 1e-5, out=x), "x"), (lambda: ham.ham_fp8_encode(x, b, s), "x"),
                       (lambda: ham.ham_fp8_encode_weight(x, b, s), "w"),
                       (lambda: ham.ham_fp8_weight_alloc(2, 256, b, s), "codes"),
                       (lambda: ham.ham_fp8_linear(w, b, s, x), "x_codes"),
                       (lambda: ham.ham_fp8_gated(w, b, s, b, s), "x_codes"),
                       (lambda: ham.ham_sample(x, x, x), "logits")):
        with pytest.raises(ValueError, match=f"^{name} must be a CUDA tensor"):
            call()


def test_scale_bytes():
    assert [ham.fp8_scale_bytes(k) for k in (16, 128, 512, 513, 4096)] == [4, 4, 4, 8, 32]

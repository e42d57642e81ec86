"""The example's macro-step (examples/macro_step.py): every call of it against the fp64 oracle, from the
buffers that the step left, and the step replayed from a graph."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import ops
from ops_helpers import check_bf16, check_codes, gated_slack, norm_slack, product_slack
from paper_2505_20438_gb300 import ham

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "macro_step.py")
    spec = importlib.util.spec_from_file_location("macro_step", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _f64(t):
    return t.double().cpu().numpy()


def _rows(pair):
    return ops.decode_rows(pair[0].cpu().numpy(), pair[1].cpu().numpy())


def _weight(pair):
    return ops.decode_weight(pair[0].cpu().numpy(), pair[1].cpu().numpy())


def test_each_call_of_a_step_matches_the_oracle():
    """The last layer's calls and the head, each from the inputs that the step gave it."""
    import torch
    ex = _example()
    m = ex.Model(seed=3)
    b, c = m.cfg.batch, m.cfg
    u = torch.rand(b, device="cuda")
    settings = dict(temperature=torch.full((b,), 0.9, device="cuda"), top_p=torch.full((b,), 0.9, device="cuda"))
    seen = {}
    add_norm = ham.ham_add_norm

    def spy(x, *a, **k):      # the residual stream is updated in place: keep the inputs of each norm
        seen.setdefault("norm", []).append((x.clone(), None if k.get("residual") is None else k["residual"].clone()))
        add_norm(x, *a, **k)

    ham.ham_add_norm = spy
    try:
        for _ in range(3):
            seen.clear()
            m.step(u, **settings)
    finally:
        ham.ham_add_norm = add_norm
    torch.cuda.synchronize()
    m.check()
    w = m.w[-1]
    # the final norm, from the feed-forward's branch and the residual before it
    x, r = seen["norm"][-1]
    h, y = ops.add_norm(_f64(x), _f64(r), _f64(m.norm), c.eps)
    check_codes(*m.normed8, y, norm_slack(y))
    # the second projection of the feed-forward block gave that branch
    inner, down = _rows(m.inner8), _weight(w["down"])
    check_bf16(x, inner @ down.T, product_slack(inner, down))
    # the norm before the block, and the block's first half
    x2, r2 = seen["norm"][-2]
    h2, y2 = ops.add_norm(_f64(x2), _f64(r2), _f64(w["norm2"]), c.eps)
    check_bf16(r, h2, 2.0 ** -24 * np.abs(h2))           # (the stream that the final norm read)
    codes, scales = torch.empty_like(m.normed8[0]), torch.empty_like(m.normed8[1])
    ham.ham_add_norm(x2, w["norm2"], c.eps, residual=r2, codes=codes, scales=scales)
    check_codes(codes, scales, y2, norm_slack(y2))
    n8, gate, up = _rows((codes, scales)), _weight(w["gate"]), _weight(w["up"])
    G, U, want = ops.gated(n8, gate, up)
    check_codes(*m.inner8, want, gated_slack(n8, gate, up, G, U))
    # the output projection of the attention's rows
    a64, e = ops.encode_rows(_f64(m.attn.view(b, -1)))
    np.testing.assert_array_equal(_rows(m.attn8), a64)
    o = _weight(w["o"])
    check_bf16(x2, a64 @ o.T, product_slack(a64, o))
    # the head and the tokens
    f8, head = _rows(m.normed8), _weight(m.head_w)
    check_bf16(m.logits, f8 @ head.T, product_slack(f8, head))
    for i in range(b):
        token, prob = ops.sample(_f64(m.logits[i]), float(u[i]), temperature=np.float32(0.9), top_p=np.float32(0.9))
        kept = ops.kept_weights(_f64(m.logits[i]), temperature=np.float32(0.9), top_p=np.float32(0.9))
        run = np.cumsum(kept)
        t = int(m.tokens[i])
        # (the weights' fp32 exponentials: 2.6e-6 of the sum, a unit a token)
        slack = 2 * (2.6e-6 * run[-1] + c.vocab)
        assert kept[t] > 0 and run[t] - kept[t] - slack <= float(u[i]) * run[-1] <= run[t] + slack
    assert list(ham.ham_slot_lengths(m.kv)[0]) == [3] * b


def test_a_replayed_step_gives_the_same_tokens():
    import torch
    ex = _example()
    b = ex.Config.batch
    u = torch.rand((5, b), device="cuda")
    runs = []
    for captured in (False, True):
        m = ex.Model(seed=1)
        now = torch.zeros(b, device="cuda")
        if captured:
            m.step(now)
            ham.ham_kv_reset(m.kv)
            m.tokens.zero_()
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                m.step(now)
        got = []
        for i in range(5):
            now.copy_(u[i])
            g.replay() if captured else m.step(now)
            got.append((m.tokens.clone(), m.probs.clone(), m.logits.clone()))
        m.check()
        runs.append(got)
    for (t0, p0, l0), (t1, p1, l1) in zip(*runs):
        assert torch.equal(t0, t1) and torch.equal(p0, p1) and torch.equal(l0, l1)

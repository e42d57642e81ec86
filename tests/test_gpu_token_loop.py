"""Macro-steps one after the other: the tokens that ham_sample writes are the ones that the next
ham_embed_tokens embeds, with nothing between the two calls and the work queued ahead of the GPU."""
import importlib.util
import os

import numpy as np
import pytest

from paper_2505_20438_gb300 import ham

pytestmark = pytest.mark.gpu


def _embedder(hidden, heads, batch, vocab, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()

    table = normal(vocab, hidden)
    e = ham.ham_embedder_alloc(hidden, heads, batch, 4, *(normal(hidden, hidden, scale=hidden ** -0.5) for _ in range(4)),
                               normal(4, hidden))
    ham.ham_embedder_set_vocab(e, table)
    return e, table


# a row a cluster and a row a CTA (two rows of CTAs an SM and more)
@pytest.mark.parametrize("batch,vocab", [(6, 32003), (240, 20011)])
def test_the_tokens_just_chosen_are_embedded(batch, vocab):
    import torch
    H, rounds = 256, 16
    e, table = _embedder(H, 8, batch, vocab, 7)
    g = torch.Generator(device="cuda").manual_seed(8)
    logits = [torch.randn((batch, vocab), generator=g, device="cuda") * 3 for _ in range(rounds)]
    u = torch.rand((rounds, batch), generator=g, device="cuda")
    k = torch.full((batch,), 40, dtype=torch.int32, device="cuda")
    tokens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    lone = torch.arange(batch + 1, dtype=torch.int32, device="cuda")
    pairs = torch.arange(0, batch + 1, 2, dtype=torch.int32, device="cuda")
    alone = torch.zeros((rounds, batch, H), dtype=torch.bfloat16, device="cuda")     # a token a sequence: its row
    fused = torch.zeros((rounds, batch // 2, H), dtype=torch.bfloat16, device="cuda")  # two

    def loop(after_each=lambda i: None):
        for i in range(rounds):
            ham.ham_sample(logits[i], u[i], tokens, top_k=k)
            after_each(i)
            ham.ham_embed_tokens(e, tokens, pairs, fused[i])
            after_each(i)
            ham.ham_sample(logits[rounds - 1 - i], u[i], tokens, top_k=k)
            after_each(i)
            ham.ham_embed_tokens(e, tokens, lone, alone[i])
            after_each(i)

    chosen = []

    def wait(i):
        torch.cuda.synchronize()
        chosen.append(tokens.clone())

    loop(wait)
    want = alone.clone(), fused.clone()
    for i in range(rounds):     # the tokens were other ones in every round, and their rows came out
        assert torch.equal(want[0][i], table[chosen[4 * i + 3].long()])
        assert i == 0 or not torch.equal(chosen[4 * i + 3], chosen[4 * i - 1])
    assert ham.ham_embedder_status(e) == ham.HAM_DEVERR_NONE

    def check():
        torch.cuda.synchronize()
        assert torch.equal(alone, want[0]) and torch.equal(fused, want[1])
        for t in (alone, fused):
            t.zero_()
        tokens.zero_()
        torch.cuda.synchronize()

    for t in (alone, fused):
        t.zero_()
    tokens.zero_()
    for _ in range(3):
        torch.cuda._sleep(2_000_000)        # (a millisecond: the loop is queued before its first call runs)
        loop()
        check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop()
    for _ in range(3):
        graph.replay()
        check()
    assert ham.ham_embedder_status(e) == ham.HAM_DEVERR_NONE


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "macro_step.py")
    spec = importlib.util.spec_from_file_location("macro_step", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_whole_steps_back_to_back(monkeypatch):
    """Macro-steps of the example with nothing between them, one by one and several in one graph, give the
    bits of the same steps with a synchronisation after every call."""
    import torch
    ex = _example()
    steps, b = 6, ex.Config.batch
    u = torch.rand((steps, b), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))

    def results(m):
        torch.cuda.synchronize()
        m.check()
        assert list(ham.ham_slot_lengths(m.kv)[0]) == [steps] * b
        return [t.clone() for t in (m.tokens, m.probs, m.logits, m.attn, m.inner8[0], m.branch)]

    def fresh():
        m = ex.Model(seed=4)
        m.tokens.copy_(torch.arange(b, dtype=torch.int32))
        torch.cuda.synchronize()
        return m

    m = fresh()
    with monkeypatch.context() as patch:
        for name in [n for n in dir(ham) if n.startswith("ham_") and callable(getattr(ham, n))]:
            def waits(*a, _call=getattr(ham, name), **kw):
                r = _call(*a, **kw)
                torch.cuda.synchronize()
                return r
            patch.setattr(ham, name, waits)
        for i in range(steps):
            m.step(u[i])
        want = results(m)
    for captured in (False, True, False, True):
        m = fresh()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                for i in range(steps):
                    m.step(u[i])
            graph.replay()
        else:
            torch.cuda._sleep(2_000_000)
            for i in range(steps):
                m.step(u[i])
        for a, w in zip(results(m), want):
            assert np.array_equal(a.view(torch.uint8).cpu().numpy(), w.view(torch.uint8).cpu().numpy())

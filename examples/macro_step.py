"""Macro-steps of a small decoder, from the tokens of the last one to the tokens of the next, with
every operation in the library's kernels: the compositional embedder, the layers (norm, layer front,
attention over the paged cache, output projection, gated feed-forward block) with 8-bit weights, the
head and the choice of each sequence's token.

    python examples/macro_step.py [steps]

The weights are random: the point is how the calls fit together.  A macro-step is captured in a CUDA
graph once and replayed, as a serving loop does.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2505_20438_gb300 import ham  # noqa: E402


class Config:
    layers, batch, hidden, n_q_heads, n_kv_heads, head_dim = 2, 6, 1024, 8, 2, 128
    ffn, vocab, page_slots, max_slots, eps = 2048, 5003, 16, 64, 1e-5


def encoded(w):
    """An 8-bit weight's codes and scales from bf16 [n][k]."""
    n, k = w.shape
    codes = torch.empty((n, k), dtype=torch.uint8, device="cuda")
    scales = torch.empty((-(-n // 128), ham.fp8_scale_bytes(k)), dtype=torch.uint8, device="cuda")
    ham.ham_fp8_encode_weight(w, codes, scales)
    return codes, scales


class Model:
    def __init__(self, cfg=Config, seed=0):
        self.cfg, c = cfg, cfg
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, scale=1.0):
            return (torch.randn(shape, generator=g, device="cuda") * scale).bfloat16()

        H, d, q = c.hidden, c.head_dim, c.n_q_heads * c.head_dim
        self.w = []        # the bf16 weights and 8-bit codes, for whoever wants to check a result
        self.layers = []
        for _ in range(c.layers):
            w = dict(norm1=1 + normal(H, scale=0.1), norm2=1 + normal(H, scale=0.1),
                     qkv=normal(q + 2 * c.n_kv_heads * d, H, scale=H ** -0.5),
                     o=encoded(normal(H, q, scale=q ** -0.5)), gate=encoded(normal(c.ffn, H, scale=H ** -0.5)),
                     up=encoded(normal(c.ffn, H, scale=H ** -0.5)), down=encoded(normal(H, c.ffn, scale=c.ffn ** -0.5)))
            self.w.append(w)
            self.layers.append(dict(
                norm1=w["norm1"], norm2=w["norm2"], qkv=w["qkv"],
                o=ham.ham_fp8_weight_alloc(H, q, *w["o"]),
                gate_up=ham.ham_fp8_weight_alloc(c.ffn, H, *w["gate"], *w["up"]),
                down=ham.ham_fp8_weight_alloc(H, c.ffn, *w["down"])))
        self.norm, self.head_w = 1 + normal(H, scale=0.1), encoded(normal(c.vocab, H, scale=2 * H ** -0.5))
        self.head = ham.ham_fp8_weight_alloc(c.vocab, H, *self.head_w)
        self.table = normal(c.vocab, H)
        self.embedder = ham.ham_embedder_alloc(H, c.n_q_heads, c.batch, 4,
                                               *(normal(H, H, scale=H ** -0.5) for _ in range(4)), normal(4, H))
        ham.ham_embedder_set_vocab(self.embedder, self.table)
        self.kv = ham.ham_kv_alloc(c.layers, c.batch, c.n_q_heads, c.n_kv_heads, d, c.page_slots, c.max_slots, page_seed=1)

        def rows(k):
            return (torch.empty((c.batch, k), dtype=torch.uint8, device="cuda"),
                    torch.empty((c.batch, ham.fp8_scale_bytes(k)), dtype=torch.uint8, device="cuda"))

        def state():
            return torch.empty((c.batch, H), dtype=torch.bfloat16, device="cuda")

        self.hidden, self.normed, self.branch = state(), state(), state()
        self.q_rot = torch.empty((c.batch, c.n_q_heads, d), dtype=torch.bfloat16, device="cuda")
        self.attn = torch.empty_like(self.q_rot)
        self.attn8, self.normed8, self.inner8 = rows(q), rows(H), rows(c.ffn)
        self.logits = torch.empty((c.batch, c.vocab), device="cuda")
        self.ntok = torch.ones(c.batch, dtype=torch.int32, device="cuda")
        self.offsets = torch.arange(c.batch + 1, dtype=torch.int32, device="cuda")
        self.tokens = torch.zeros(c.batch, dtype=torch.int32, device="cuda")
        self.probs = torch.empty(c.batch, device="cuda")

    def step(self, u, temperature=None, top_k=None, top_p=None, min_p=None):
        """One macro-step of every sequence from self.tokens (one token a sequence here), u [B] its
        random numbers: leaves the next tokens in self.tokens and their probabilities in self.probs."""
        c, x, y = self.cfg, self.hidden, self.branch
        ham.ham_embed_tokens(self.embedder, self.tokens, self.offsets, x)
        first = True
        for layer, w in enumerate(self.layers):
            # the residual stream stays in x; a layer's branch comes back in y and is added by the next norm
            if first:
                ham.ham_add_norm(x, w["norm1"], c.eps, out=self.normed)
            else:
                ham.ham_add_norm(y, w["norm1"], c.eps, residual=x, sum_out=x, out=self.normed)
            ham.ham_qkv_append(self.kv, layer, self.normed, w["qkv"], self.ntok, self.q_rot)
            ham.ham_decode_attn(self.kv, layer, self.q_rot, self.attn)
            ham.ham_fp8_encode(self.attn.view(c.batch, -1), *self.attn8)
            ham.ham_fp8_linear(w["o"], *self.attn8, y)
            ham.ham_add_norm(y, w["norm2"], c.eps, residual=x, sum_out=x, codes=self.normed8[0], scales=self.normed8[1])
            ham.ham_fp8_gated(w["gate_up"], *self.normed8, *self.inner8)
            ham.ham_fp8_linear(w["down"], *self.inner8, y)
            first = False
        ham.ham_add_norm(y, self.norm, c.eps, residual=x, codes=self.normed8[0], scales=self.normed8[1])
        ham.ham_fp8_linear(self.head, *self.normed8, self.logits)
        ham.ham_sample(self.logits, u, self.tokens, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p,
                       probs=self.probs)

    def check(self):
        """Raise if a kernel recorded an error (a full sequence, for one)."""
        bad = [ham.ham_kv_status(self.kv), ham.ham_embedder_status(self.embedder), ham.ham_fp8_weight_status(self.head)]
        bad += [ham.ham_fp8_weight_status(w[n]) for w in self.layers for n in ("o", "gate_up", "down")]
        if any(bad):
            raise RuntimeError(f"device error words {bad}")


def main(steps=16):
    m = Model()
    b = m.cfg.batch
    u = torch.rand((steps, b), device="cuda")
    now = torch.empty(b, device="cuda")
    settings = dict(temperature=torch.full((b,), 0.8, device="cuda"), top_p=torch.full((b,), 0.95, device="cuda"),
                    top_k=torch.full((b,), 200, dtype=torch.int32, device="cuda"))
    now.copy_(u[0])
    m.step(now, **settings)             # (the first calls set the kernels up: not in a capture)
    ham.ham_kv_reset(m.kv)
    m.tokens.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.step(now, **settings)
    for i in range(steps):
        now.copy_(u[i])
        graph.replay()
        print(i, m.tokens.tolist(), [round(p, 3) for p in m.probs.tolist()])
    m.check()
    slots, _ = ham.ham_slot_lengths(m.kv)
    print("slots held:", slots.tolist())


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 16)

"""The experts' block as a decoder runs it: norm, the router's logits, the choice, both products, the weighted sum, the
next norm; captured in a graph and replayed on other rows, with other experts and other counts."""
import numpy as np
import pytest

from oracle import experts as ox
from oracle import ops
from paper_2505_20438_gb300 import ham
from tests.ops_helpers import dev

pytestmark = pytest.mark.gpu


def _encoded(x):
    """bf16 rows of one weight -> codes, scales on the GPU and their values."""
    import torch
    n, k = x.shape
    codes = torch.empty((n, k), dtype=torch.uint8, device="cuda")
    scales = torch.empty((-(-n // 128), ham.fp8_scale_bytes(k)), dtype=torch.uint8, device="cuda")
    ham.ham_fp8_encode_weight(torch.from_numpy(np.float32(x)).bfloat16().cuda(), codes, scales)
    return codes, scales, ops.decode_weight(codes.cpu().numpy(), scales.cpu().numpy())


class Block:
    def __init__(self, rng, hidden, experts, f):
        import torch
        self.hidden, self.experts, self.f = hidden, experts, f

        def several(n, k):
            each = [_encoded(rng.standard_normal((n, k)) * k ** -0.5) for _ in range(experts)]
            return torch.stack([e[0] for e in each]), torch.stack([e[1] for e in each]), [e[2] for e in each]

        self.router = _encoded(2 * rng.standard_normal((experts, hidden)) * hidden ** -0.5)
        self.gate, self.up, self.down = several(f, hidden), several(f, hidden), several(hidden, f)
        self.h_router = ham.ham_fp8_weight_alloc(experts, hidden, *self.router[:2])
        self.h_gated = ham.ham_fp8_experts_alloc(experts, f, hidden, *self.gate[:2], *self.up[:2])
        self.h_down = ham.ham_fp8_experts_alloc(experts, hidden, f, *self.down[:2])
        self.norm = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")

    def buffers(self, t, k):
        import torch

        def rows(n, w):
            return (torch.empty((n, w), dtype=torch.uint8, device="cuda"),
                    torch.empty((n, ham.fp8_scale_bytes(w)), dtype=torch.uint8, device="cuda"))

        def ints(*shape):
            return torch.empty(shape, dtype=torch.int32, device="cuda")

        self.x8, self.h8 = rows(t, self.hidden), rows(t * k, self.f)
        self.logits = torch.empty((t, self.experts), device="cuda")
        self.expert, self.weight, self.place = ints(t, k), torch.empty((t, k), device="cuda"), ints(t, k)
        self.offsets, self.order = ints(self.experts + 1), ints(t * k)
        self.y = torch.empty((t * k, self.hidden), dtype=torch.bfloat16, device="cuda")
        self.out, self.next = (torch.empty((t, self.hidden), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def run(self, x, k, **settings):
        ham.ham_add_norm(x, self.norm, 1e-5, codes=self.x8[0], scales=self.x8[1])
        ham.ham_fp8_linear(self.h_router, *self.x8, self.logits)
        ham.ham_route(self.logits, self.expert, self.weight, self.offsets, self.order, self.place, **settings)
        ham.ham_fp8_experts_gated(self.h_gated, *self.x8, self.offsets, self.order, k, *self.h8)
        ham.ham_fp8_experts_linear(self.h_down, *self.h8, self.offsets, self.y)
        ham.ham_experts_combine(self.y, self.weight, self.place, self.out, add=x)
        ham.ham_add_norm(self.out, self.norm, 1e-5, out=self.next)

    def check(self, x, k, settings):
        """The block's sum from its own 8-bit rows and logits.  The inner rows' 8-bit codes are off by 2^-4 of a
        value at most, of random sign, and y by 2^-8: over f terms the sum's error is below 2^-5 of its norm."""
        rows = ops.decode_rows(*(v.cpu().numpy() for v in self.x8))
        settings = dict(settings)
        settings["sigmoid"] = settings.pop("score", 0) == ham.HAM_SCORE_SIGMOID
        if settings.get("bias") is not None:
            settings["bias"] = settings["bias"].double().cpu().numpy()
        want = ox.block(rows, self.logits.double().cpu().numpy(), self.gate[2], self.up[2], self.down[2], top_k=k, **settings)
        got = self.out.double().cpu().numpy() - x.double().cpu().numpy()
        err = np.linalg.norm(got - want, axis=1) / np.linalg.norm(want, axis=1)
        assert err.max() < 2.0 ** -4, err.max()   # (2^-5, and x + sum rounded to bf16)
        h = self.out.double().cpu().numpy()
        n = h / np.sqrt((h * h).mean(axis=1, keepdims=True) + 1e-5)
        assert np.abs(self.next.double().cpu().numpy() - n).max() <= 2.0 ** -8 * np.abs(n).max()
        assert ham.ham_fp8_weight_status(self.h_gated) == ham.ham_fp8_weight_status(self.h_down) == 0


@pytest.mark.parametrize("t,k,settings", [
    (1, 2, {}), (6, 4, dict(score=ham.HAM_SCORE_SIGMOID, groups=4, top_groups=2, scale=2.0)),
    (70, 3, dict(renorm=False)), (400, 2, {})])
def test_block(t, k, settings):
    import torch
    rng = np.random.default_rng(t)
    b = Block(rng, 512, 16, 384)
    b.buffers(t, k)
    x = torch.randn((t, 512), device="cuda").bfloat16() * 0.25
    b.run(x, k, **settings)
    b.check(x, k, settings)


@pytest.mark.parametrize("t,k,width", [(40, 2, 256), (400, 3, 1024)])    # rows by index; sorted first
def test_block_captured(t, k, width):
    """Every replay routes its own rows; nothing depends on the counts of the capture."""
    import torch
    rng = np.random.default_rng(1)
    b = Block(rng, width, 8, width)
    b.buffers(t, k)
    bias = dev(np.float32(0.1 * rng.standard_normal(8)))
    settings = dict(score=ham.HAM_SCORE_SIGMOID, bias=bias)
    x = torch.randn((t, width), device="cuda").bfloat16() * 0.25
    b.run(x, k, **settings)                 # (the first calls set the kernels up: not in a capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.run(x, k, **settings)
    for i in range(4):
        x.copy_(torch.randn((t, width), device="cuda") * 0.25)
        if i == 2:
            bias.copy_(dev(np.float32([9, 9, 0, 0, 0, 0, 0, 0])))   # two experts take every row
        graph.replay()
        torch.cuda.synchronize()
        b.check(x, k, settings)


def test_a_padded_batch():
    """Rows of -inf logits take no expert: their sum is what was added, and nothing is computed for them."""
    import torch
    rng = np.random.default_rng(2)
    b = Block(rng, 256, 8, 128)
    t, k = 24, 2
    b.buffers(t, k)
    x = torch.randn((t, 256), device="cuda").bfloat16()
    b.run(x, k)
    live, order = b.out.clone(), b.logits.clone()
    order[16:] = float("-inf")
    b.y.fill_(float("nan"))
    b.h8[0].fill_(0x7f)
    ham.ham_route(order, b.expert, b.weight, b.offsets, b.order, b.place)
    ham.ham_fp8_experts_gated(b.h_gated, *b.x8, b.offsets, b.order, k, *b.h8)
    ham.ham_fp8_experts_linear(b.h_down, *b.h8, b.offsets, b.y)
    ham.ham_experts_combine(b.y, b.weight, b.place, b.out, add=x)
    assert int(b.offsets[-1]) == 32
    assert torch.equal(b.out[:16], live[:16]) and torch.equal(b.out[16:], x[16:])
    assert torch.isnan(b.y[32:].float()).all()


def test_two_graphs_and_a_stream_at_once():
    """Two captured blocks of many rows and calls on a third stream share the weights: each has memory of its own for the
    sorted rows."""
    import torch
    rng = np.random.default_rng(3)
    t, k = 700, 2
    b = Block(rng, 1024, 8, 1024)
    b.buffers(t, k)
    x = [torch.randn((t, 1024), device="cuda").bfloat16() for _ in range(3)]
    b.run(x[0], k)
    rows = []
    for v in x:
        ham.ham_add_norm(v, b.norm, 1e-5, codes=b.x8[0], scales=b.x8[1])
        rows.append([a.clone() for a in b.x8])
    outs = [[torch.zeros_like(a) for a in b.h8] for _ in x]

    def call(i, stream=None):
        ham.ham_fp8_experts_gated(b.h_gated, *rows[i], b.offsets, b.order, k, *outs[i], stream=stream)

    want = []
    for i in range(3):
        call(i)
        want.append([a.clone() for a in outs[i]])
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in range(3)]
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            for _ in range(3):
                call(i)
    for o in outs:
        for a in o:
            a.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        call(2, streams[2])
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(a, c) for a, c in zip(o, w))
    assert ham.ham_fp8_weight_status(b.h_gated) == ham.HAM_DEVERR_NONE

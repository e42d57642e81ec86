"""The experts' products on the GPU against the fp64 oracle, slot by slot."""
import numpy as np
import pytest

from oracle import experts as ox
from oracle import ops
from paper_2505_20438_gb300 import ham
from tests.ops_helpers import check_bf16, check_codes, dev, empty_rows, gated_slack, product_slack, random_codes

pytestmark = pytest.mark.gpu


def weights(rng, experts, n, k):
    """Codes [experts][n][k], scales, and their values."""
    c, s = random_codes(rng, experts * n, k)
    c = c.reshape(experts, n, k)
    s = rng.integers(113, 130, (experts, -(-n // 128), ops.scale_bytes(k))).astype(np.uint8)
    return c, s, Values(c, s)


class Values:
    """The experts' weights in fp64, one at a time."""

    def __init__(self, codes, scales):
        self.codes, self.scales = codes, scales

    def __getitem__(self, e):
        return ops.decode_weight(self.codes[e], self.scales[e])


def alloc(n, k, w, up=None):
    return ham.ham_fp8_experts_alloc(len(w[0]), n, k, dev(w[0]), dev(w[1]), *((dev(up[0]), dev(up[1])) if up else ()))


def grouping(rng, counts, top_k, rows, missing=0):
    """offsets, order for experts with `counts` slots: each slot a random pair of its own."""
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    assert offsets[-1] + missing <= rows * top_k
    order = np.full(rows * top_k, -1, np.int32)
    order[:offsets[-1]] = rng.permutation(rows * top_k)[:offsets[-1]]
    return offsets, order


def run_gated(rng, counts, n, k, top_k=2, rows=None, stream=None):
    import torch
    total = int(np.sum(counts))
    rows = rows or max(1, -(-total // top_k))
    w, up = weights(rng, len(counts), n, k), weights(rng, len(counts), n, k)
    xc, xs = random_codes(rng, rows, k)
    offsets, order = grouping(rng, counts, top_k, rows)
    h = alloc(n, k, w, up)
    codes, scales = empty_rows(rows * top_k, n)
    args = [dev(v) for v in (xc, xs, offsets, order)]
    torch.cuda.synchronize()
    ham.ham_fp8_experts_gated(h, *args, top_k, codes, scales, stream=stream)
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE
    x = ops.decode_rows(xc, xs)
    for e in range(len(counts)):
        a, b = offsets[e], offsets[e + 1]
        if a < b:
            mine = x[order[a:b] // top_k]
            wg, wu = w[2][e], up[2][e]
            g, u, want = ops.gated(mine, wg, wu)
            check_codes(codes[a:b], scales[a:b], want, gated_slack(mine, wg, wu, g, u))
    # rows behind the last slot are left as they were
    assert (codes[total:] == 0x7f).all() and (scales[total:] == 255).all()
    return h, args, codes, scales


def run_linear(rng, counts, n, k, out="bf16", slots=None, stream=None):
    import torch
    total = int(np.sum(counts))
    slots = slots or max(total, 1)
    w = weights(rng, len(counts), n, k)
    xc, xs = random_codes(rng, slots, k)
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    h = alloc(n, k, w)
    y = torch.full((slots, n), -7.0, dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    args = [dev(v) for v in (xc, xs, offsets)]
    torch.cuda.synchronize()
    ham.ham_fp8_experts_linear(h, *args, y, stream=stream)
    torch.cuda.synchronize()
    assert ham.ham_fp8_weight_status(h) == ham.HAM_DEVERR_NONE
    x = ops.decode_rows(xc, xs)
    for e in range(len(counts)):
        a, b = offsets[e], offsets[e + 1]
        if a < b:
            we = w[2][e]
            check_bf16(y[a:b], x[a:b] @ we.T, product_slack(x[a:b], we))
    assert (y[total:] == -7).all()
    return h, args, y


COUNTS = [[1], [0, 0, 1, 0], [3, 0, 1, 2], [16, 17, 15], [31, 33, 32, 0, 1], [64, 65, 0, 63], [127, 0, 129], [128, 1, 255],
          [257, 0, 0, 300], [513, 2]]


@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("n,k", [(128, 128), (256, 512)])
def test_counts_of_rows(counts, n, k):
    rng = np.random.default_rng(len(counts) + n)
    run_gated(rng, counts, n, k)
    run_linear(rng, counts, n, k)


@pytest.mark.parametrize("counts", [[128, 1, 255], [257, 0, 0, 300], [513, 2], [130, 200, 97]], ids=str)
@pytest.mark.parametrize("n,k", [(4096, 1024), (4112, 1040)])
def test_rows_sorted_first(counts, n, k):
    """Products so large that their rows are copied into slot order before."""
    run_gated(np.random.default_rng(len(counts) + n), counts, n, k, top_k=3)


@pytest.mark.parametrize("n,k", [(16, 16), (128, 48), (144, 128), (272, 144), (528, 2064), (112, 640), (384, 1040)])
@pytest.mark.parametrize("counts", [[2, 0, 5], [40, 7], [130, 200]], ids=str)
def test_gated_sizes(n, k, counts):
    run_gated(np.random.default_rng(n + k), counts, n, k, top_k=3)


@pytest.mark.parametrize("n,k", [(1, 16), (7, 48), (100, 128), (129, 144), (130, 256), (255, 640), (1000, 528), (257, 2064), (260, 1040)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[2, 0, 5], [40, 7], [130, 200]], ids=str)
def test_linear_sizes(n, k, out, counts):
    run_linear(np.random.default_rng(n + k), counts, n, k, out)


@pytest.mark.parametrize("k", [2048, 2176, 4096, 6160])
def test_long_sums(k):
    """K in several parts, with few rows and with many."""
    rng = np.random.default_rng(k)
    for counts in ([3, 0, 20], [200, 90]):
        run_gated(rng, counts, 128, k)
        run_linear(rng, counts, 256, k, "f32")


@pytest.mark.parametrize("counts", ["ones", "mixed", "large"])
def test_tiles_one_after_another(counts):
    """Several tiles a pair of CTAs, K in several parts: tiles of one and of two halves in every order."""
    rng = np.random.default_rng(len(counts))
    c = {"ones": np.ones(100, int), "mixed": rng.choice([0, 1, 40, 130, 200], 90), "large": rng.choice([3, 128, 256], 80)}[counts]
    run_gated(rng, c, 256, 2304, top_k=4)
    run_linear(rng, c, 400, 2304)


def test_no_slots_and_rows_behind_the_last():
    rng = np.random.default_rng(2)
    run_gated(rng, [0, 0, 0], 128, 256, rows=5)
    run_linear(rng, [0, 0], 128, 256, slots=9)
    run_gated(rng, [3, 4], 128, 256, rows=40)
    run_linear(rng, [5, 0, 200], 128, 256, slots=300)


@pytest.mark.parametrize("counts,n,k", [([5, 9], 128, 256), ([90, 150], 3200, 2048)])
def test_offsets_may_begin_anywhere(counts, n, k):
    """The experts of one part of the slots: the others' rows are neither looked at nor written."""
    import torch
    rng = np.random.default_rng(4)
    slots, first = sum(counts) + 20, 11
    w, up = weights(rng, 2, n, k), weights(rng, 2, n, k)
    hg, hl = alloc(n, k, w, up), alloc(n, k, w)
    xc, xs = (dev(v) for v in random_codes(rng, slots, k))
    offsets = np.int32([0, counts[0], sum(counts)]) + first
    order = rng.permutation(slots).astype(np.int32)
    order[:first], order[sum(counts) + first:] = 1 << 30, -5
    codes, scales = empty_rows(slots, n)
    y = torch.full((slots, n), -7.0, device="cuda")
    ham.ham_fp8_experts_gated(hg, xc, xs, dev(offsets), dev(order), 1, codes, scales)
    ham.ham_fp8_experts_linear(hl, xc, xs, dev(offsets), y)
    assert ham.ham_fp8_weight_status(hg) == ham.ham_fp8_weight_status(hl) == ham.HAM_DEVERR_NONE
    inside = np.zeros(slots, bool)
    inside[first:first + sum(counts)] = True
    assert (y[~inside] == -7).all() and (codes[~inside] == 0x7f).all() and (scales[~inside] == 255).all()
    x = ops.decode_rows(xc.cpu().numpy(), xs.cpu().numpy())
    for e in range(2):
        a, b = offsets[e], offsets[e + 1]
        check_bf16(y[a:b], x[a:b] @ w[2][e].T, product_slack(x[a:b], w[2][e]))
        mine = x[order[a:b]]
        g, u, want = ops.gated(mine, w[2][e], up[2][e])
        check_codes(codes[a:b], scales[a:b], want, gated_slack(mine, w[2][e], up[2][e], g, u))


def test_many_experts():
    rng = np.random.default_rng(3)
    counts = rng.integers(0, 4, 512)
    run_gated(rng, counts, 64, 128, top_k=8)
    run_linear(rng, counts, 130, 128)


def test_a_slot_does_not_depend_on_the_others():
    """The same bits for a slot alone and among hundreds."""
    import torch
    rng = np.random.default_rng(5)
    n, k = 384, 2304
    w, up = weights(rng, 3, n, k), weights(rng, 3, n, k)
    hg, hl = alloc(n, k, w, up), alloc(n, k, w)
    xc, xs = (dev(v) for v in random_codes(rng, 300, k))
    codes, scales = empty_rows(300, n)
    y = torch.empty((300, n), device="cuda")
    offsets = dev(np.int32([0, 10, 10, 300]))
    ham.ham_fp8_experts_gated(hg, xc, xs, offsets, dev(np.arange(300, dtype=np.int32)), 1, codes, scales)
    ham.ham_fp8_experts_linear(hl, xc, xs, offsets, y)
    for slot, e in ((0, 0), (9, 0), (10, 2), (177, 2), (299, 2)):
        one = [0, 0, 0, 0]
        one[e + 1:] = [1] * (3 - e)
        c, s = empty_rows(1, n)
        z = torch.empty((1, n), device="cuda")
        ham.ham_fp8_experts_gated(hg, xc[slot:slot + 1], xs[slot:slot + 1], dev(np.int32(one)), dev(np.int32([0])), 1, c, s)
        ham.ham_fp8_experts_linear(hl, xc[slot:slot + 1], xs[slot:slot + 1], dev(np.int32(one)), z)
        assert torch.equal(c[0], codes[slot]) and torch.equal(s[0], scales[slot]) and torch.equal(z[0], y[slot])


def test_the_same_row_for_several_slots():
    """A row that many slots take, of one expert too."""
    import torch
    rng = np.random.default_rng(6)
    n, k = 128, 256
    w, up = weights(rng, 2, n, k), weights(rng, 2, n, k)
    h = alloc(n, k, w, up)
    xc, xs = random_codes(rng, 4, k)
    order = np.int32([5, 5, 4, 5, 0, 5, 7, 6])
    codes, scales = empty_rows(8, n)
    ham.ham_fp8_experts_gated(h, dev(xc), dev(xs), dev(np.int32([0, 5, 8])), dev(order), 2, codes, scales)
    mine = ops.decode_rows(xc, xs)[order // 2]
    for e, (a, b) in enumerate(((0, 5), (5, 8))):
        g, u, want = ops.gated(mine[a:b], w[2][e], up[2][e])
        check_codes(codes[a:b], scales[a:b], want, gated_slack(mine[a:b], w[2][e], up[2][e], g, u))
    assert torch.equal(codes[0], codes[1]) and torch.equal(codes[1], codes[3])


def test_nan_stays_in_its_row():
    import torch
    rng = np.random.default_rng(7)
    w = weights(rng, 2, 256, 256)
    h = alloc(256, 256, w)
    xc, xs = random_codes(rng, 40, 256)
    clean = torch.empty((40, 256), device="cuda")
    offsets = dev(np.int32([0, 20, 40]))
    ham.ham_fp8_experts_linear(h, dev(xc), dev(xs), offsets, clean)
    xc[7, 100] = 0x7f
    y = torch.empty_like(clean)
    ham.ham_fp8_experts_linear(h, dev(xc), dev(xs), offsets, y)
    assert torch.isnan(y[7]).all()
    y[7] = clean[7]
    assert torch.equal(y, clean)


def test_gates_far_from_zero():
    """Gates down to -105 (where exp(g) leaves fp32's normal numbers and then fp32) and up to 300, a block each: the
    values are the formula's, however small."""
    rng = np.random.default_rng(12)
    n, k, rows = 128 * 6, 128, 40
    far = np.repeat([-85.0, -88.0, -95.0, -105.0, 60.0, 300.0], 128)
    wg, wu = np.zeros((1, n, k)), rng.standard_normal((1, n, k)) * 64
    wg[0, :, 0] = far / 4
    (gc, gs), (uc, us) = _exact_codes(wg), _exact_codes(wu)
    xc = rng.integers(0, 40, (rows, k)).astype(np.uint8)
    xc[:, 0] = 0x48                          # 4
    xs = np.full((rows, ops.scale_bytes(k)), 127, np.uint8)
    h = alloc(n, k, (gc, gs), (uc, us))
    codes, scales = empty_rows(rows, n)
    ham.ham_fp8_experts_gated(h, dev(xc), dev(xs), dev(np.int32([0, rows])), dev(np.arange(rows, dtype=np.int32)), 1, codes, scales)
    x, wg, wu = ops.decode_rows(xc, xs), ops.decode_weight(gc[0], gs[0]), ops.decode_weight(uc[0], us[0])
    g, u, want = ops.gated(x, wg, wu)
    assert (np.abs(g - far) <= np.abs(far) / 16).all()
    # (A gate is one product, exact; the rest as in gated_slack.  2^-149: the exponential's last place, where it is not a
    # normal number.)
    silu = np.abs(ops.silu(g))
    check_codes(codes, scales, want, silu * product_slack(x, wu) + 2.0 ** -20 * silu * np.abs(u) + 2.0 ** -149 * np.abs(g * u))


def _exact_codes(w):
    """e4m3 codes and block scales nearest to weights [experts][n][k] (n, k multiples of 128)."""
    e, n, k = w.shape
    b = w.reshape(e, n // 128, 128, k // 128, 128)
    x = ops.block_exponent(np.abs(b).max(axis=(2, 4)))
    q = (b * 2.0 ** -x[:, :, None, :, None].astype(float)).reshape(e, n, k)
    values = ops.code_values()
    order = np.argsort(np.where(np.isnan(values), np.inf, values))[:254]
    at = np.clip(np.searchsorted(values[order], q), 1, 253)
    near = np.where(q - values[order][at - 1] < values[order][at] - q, at - 1, at)
    s = np.full((e, n // 128, ops.scale_bytes(k)), 127, np.uint8)
    s[:, :, :k // 128] = x + 127
    return order[near].astype(np.uint8), s


def test_bad_offsets_and_order_are_reported():
    """Offsets that are no grouping compute nothing, an order entry out of range counts as entry 0; both are reported."""
    import torch
    rng = np.random.default_rng(8)
    n, k = 128, 128
    w, up = weights(rng, 3, n, k), weights(rng, 3, n, k)
    hg, hl = alloc(n, k, w, up), alloc(n, k, w)
    xc, xs = (dev(v) for v in random_codes(rng, 16, k))
    y = torch.empty((16, n), device="cuda")
    for bad in ([0, 4, 3, 16], [0, 4, 8, 17], [-1, 4, 8, 16], [0, 4, 1 << 30, 16]):
        y.fill_(-7)
        ham.ham_fp8_experts_linear(hl, xc, xs, dev(np.int32(bad)), y)
        assert ham.ham_fp8_weight_status(hl) == ham.HAM_DEVERR_ROUTE
        assert (y == -7).all()
    codes, scales = empty_rows(16, n)
    order = np.arange(16, dtype=np.int32)
    order[5], order[9] = -1, 16
    ham.ham_fp8_experts_gated(hg, xc, xs, dev(np.int32([0, 4, 8, 16])), dev(order), 1, codes, scales)
    assert ham.ham_fp8_weight_status(hg) == ham.HAM_DEVERR_ROUTE
    assert ham.ham_fp8_weight_status(hg) == ham.HAM_DEVERR_NONE
    fixed = np.where((order < 0) | (order > 15), 0, order)
    want = empty_rows(16, n)
    ham.ham_fp8_experts_gated(hg, xc, xs, dev(np.int32([0, 4, 8, 16])), dev(fixed), 1, *want)
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    assert ham.ham_fp8_weight_status(hl) == ham.HAM_DEVERR_NONE


def test_handles_serve_their_own_calls():
    import torch
    rng = np.random.default_rng(10)
    w = weights(rng, 2, 128, 128)
    h, g = alloc(128, 128, w), alloc(128, 128, w, w)
    one = ham.ham_fp8_weight_alloc(128, 128, dev(w[0][0]), dev(w[1][0]))
    xc, xs = (dev(v) for v in random_codes(rng, 4, 128))
    y, (c, s), off, order = torch.empty((4, 128), device="cuda"), empty_rows(4, 128), dev(np.int32([0, 1, 4])), dev(np.arange(4, dtype=np.int32))
    for call in (lambda: ham.ham_fp8_linear(h, xc, xs, y), lambda: ham.ham_fp8_gated(g, xc, xs, c, s),
                 lambda: ham.ham_fp8_experts_linear(g, xc, xs, off, y),
                 lambda: ham.ham_fp8_experts_gated(h, xc, xs, off, order, 1, c, s),
                 lambda: ham.lib().ham_fp8_experts_linear(one, xc.data_ptr(), xs.data_ptr(), 4, off.data_ptr(), y.data_ptr(), 1, None) and ham._check(1)):
        with pytest.raises(ham.HamError, match="HAM_EINVAL"):
            call()
    for args in ((y, off), (xc, off)):       # an output over an input
        with pytest.raises((ham.HamError, ValueError)):
            ham.ham_fp8_experts_linear(h, xc, xs, args[1], xc.view(torch.bfloat16).view(4, -1) if args[0] is xc else y[:3])
    with pytest.raises(ValueError, match="offsets"):
        ham.ham_fp8_experts_linear(h, xc, xs, off[:2], y)
    with pytest.raises(ValueError, match="order"):
        ham.ham_fp8_experts_gated(g, xc, xs, off, order, 2, *empty_rows(8, 128))


def test_streams_share_a_handle():
    import torch
    rng = np.random.default_rng(11)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    h, args, y = run_linear(rng, [30, 0, 90], 256, 512, stream=a)
    ys = [torch.empty_like(y) for _ in range(8)]
    torch.cuda.synchronize()
    for i, z in enumerate(ys):
        ham.ham_fp8_experts_linear(h, *args, z, stream=(a, b)[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(z, y) for z in ys)

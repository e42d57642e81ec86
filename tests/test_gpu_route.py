"""The choice of experts and the weighted sum on the GPU against the fp64 oracle: the choices and the grouping equal,
weights within 2^-18 of themselves."""
import numpy as np
import pytest

from oracle import experts as ox
from paper_2505_20438_gb300 import ham
from tests.ops_helpers import check_bf16, dev

pytestmark = pytest.mark.gpu
INF = np.inf


def _logits(l, dtype="f32"):
    import torch
    t = torch.from_numpy(np.asarray(l, np.float32))
    t = t if dtype == "f32" else t.bfloat16()
    return t.cuda(), t.double().numpy()


def _outputs(t, k, experts):
    """Expert, weight, offsets, order and place, filled with what no call leaves."""
    import torch
    return (torch.full((t, k), -7, dtype=torch.int32, device="cuda"), torch.full((t, k), -7.0, device="cuda"),
            torch.full((experts + 1,), -7, dtype=torch.int32, device="cuda"),
            torch.full((t * k,), -7, dtype=torch.int32, device="cuda"),
            torch.full((t, k), -7, dtype=torch.int32, device="cuda"))


def _check(got, l, k, sigmoid=False, bias=None, rows=None, **kw):
    expert, weight, offsets, order, place = (g.cpu().numpy() for g in got)
    scale = kw.get("scale", 1.0)
    for t in range(len(l)) if rows is None else rows:
        e, w = ox.choose(l[t], k, sigmoid=sigmoid, bias=bias, **kw)
        assert expert[t].tolist() == e.tolist(), (t, expert[t], e)
        # (2^-140: a softmax's weight may be below fp32's normal numbers)
        assert (np.abs(weight[t] - w) <= 2.0 ** -18 * w + scale * 2.0 ** -140).all(), (t, weight[t], w)
    o, r, p = ox.group(expert, len(offsets) - 1)
    assert (offsets == o).all() and (order == r).all() and (place == p).all()


def _run(l, k, dtype="f32", sigmoid=False, bias=None, rows=None, stream=None, **kw):
    t, ref = _logits(l, dtype)
    b = None if bias is None else np.asarray(bias, np.float32)
    got = _outputs(len(ref), k, ref.shape[1])
    ham.ham_route(t, *got, bias=None if b is None else dev(b),
                  score=ham.HAM_SCORE_SIGMOID if sigmoid else ham.HAM_SCORE_SOFTMAX, stream=stream, **kw)
    _check(got, ref, k, sigmoid, None if b is None else b.astype(np.float64), rows, **kw)
    return got


@pytest.mark.parametrize("experts,k", [(1, 1), (2, 2), (7, 3), (32, 32), (33, 1), (60, 4), (64, 8), (65, 8), (128, 6),
                                       (200, 9), (256, 8), (257, 5), (512, 32)])
@pytest.mark.parametrize("dtype,sigmoid,with_bias,renorm", [
    ("f32", False, False, True), ("f32", True, True, True), ("bf16", False, True, False), ("bf16", True, False, False)])
def test_choice(experts, k, dtype, sigmoid, with_bias, renorm):
    rng = np.random.default_rng(experts * 100 + k)
    bias = 0.1 * rng.standard_normal(experts) if with_bias else None
    _run(2 * rng.standard_normal((19, experts)), k, dtype, sigmoid, bias, renorm=renorm, scale=2.5)


@pytest.mark.parametrize("experts,groups,top_groups,k", [
    (8, 2, 1, 4), (64, 8, 3, 8), (60, 4, 2, 7), (256, 8, 4, 8), (32, 32, 5, 5), (512, 32, 4, 32), (510, 30, 29, 8), (96, 3, 2, 6),
    (256, 1, 1, 8), (64, 8, 8, 8)])
@pytest.mark.parametrize("dtype,sigmoid,with_bias", [("f32", True, True), ("bf16", False, False), ("bf16", True, True)])
def test_groups(experts, groups, top_groups, k, dtype, sigmoid, with_bias):
    rng = np.random.default_rng(experts + groups)
    bias = 0.2 * rng.standard_normal(experts) if with_bias else None
    _run(1.5 * rng.standard_normal((41, experts)), k, dtype, sigmoid, bias, groups=groups, top_groups=top_groups)


@pytest.mark.parametrize("rows,experts,k", [(1, 64, 8), (5, 64, 8), (1023, 16, 1), (1025, 64, 8), (3001, 256, 5), (9000, 8, 2),
                                            (1024, 512, 32), (16384, 64, 8), (20001, 64, 7), (70000, 300, 3)])
def test_many_rows(rows, experts, k):
    rng = np.random.default_rng(rows)
    l = rng.standard_normal((rows, experts)) + 2 * rng.standard_normal(experts)  # some experts have most of the rows
    _run(l, k, rows=rng.integers(0, rows, 50))


@pytest.mark.parametrize("sigmoid", [False, True])
def test_values_that_fp32_cannot_tell_apart(sigmoid):
    """Biases that make up for the scores' differences to within 1e-9 .. 1e-7: the choice is the exact one."""
    rng = np.random.default_rng(9)
    experts = 64
    l = np.float32(rng.standard_normal((1, experts))).astype(np.float64)
    s = ox.scores(l[0], sigmoid)
    bias = np.float32(1.0 - s)              # every value within a rounding of 1
    v = np.sort(s + bias.astype(np.float64))
    assert 0 < np.diff(v).max() < 1e-6
    _run(l, 8, sigmoid=sigmoid, bias=bias)
    _run(l, 8, sigmoid=sigmoid, bias=bias, groups=8, top_groups=3)


@pytest.mark.parametrize("k", [1, 2, 7, 31, 32])
def test_pairs_of_near_values(k):
    """Here and there two values that differ by less than fp32 tells, among others that lie apart; the last chosen and the
    first that is not among them."""
    rng = np.random.default_rng(k)
    rows, experts = 64, 100
    l = np.float32(rng.standard_normal((rows, experts))).astype(np.float64)
    s = np.stack([ox.scores(r, True) for r in l])
    bias = np.zeros(experts)
    bias[:50] = 0.25
    # expert 50 + i of row i: the logit whose score is another's value, rounded to fp32
    for i in range(rows):
        v = np.sort(s[i] + bias)[::-1]
        target = v[min(k - 1 + i % 2, experts - 1)]
        if target < 0.999:
            l[i, 50 + i % 50] = np.float32(np.log(target / (1 - target)))
    _run(l, k, sigmoid=True, bias=bias)


@pytest.mark.parametrize("experts", [40, 64, 250, 345, 512])
@pytest.mark.parametrize("sigmoid,groups", [(True, 1), (False, 1), (True, 2)])
@pytest.mark.parametrize("k", [1, 2, 7, 20])
def test_a_larger_value_behind_equal_ones(experts, sigmoid, groups, k):
    """Many equal logits and, anywhere among them, one that is a unit larger: fp32 may give its value a place after all of
    theirs, or the same."""
    if experts % groups:
        groups = 3
    rng = np.random.default_rng(experts + k)
    l = np.empty((64, experts), np.float32)
    for t in range(len(l)):
        x = np.float32(rng.uniform(-2, 2))
        l[t] = x - 3
        some = rng.permutation(experts)[:int(rng.integers(k + 1, min(experts, k + 20)))]
        l[t, some] = x
        l[t, some[0]] = np.nextafter(x, np.float32(9))
    _run(l, min(k, experts // groups), sigmoid=sigmoid, bias=np.full(experts, 0.25), groups=groups, top_groups=1)


@pytest.mark.parametrize("experts", [40, 64, 96, 128, 250, 256, 500, 512])
@pytest.mark.parametrize("sigmoid,with_bias,groups", [(False, False, 1), (True, False, 1), (False, True, 1), (True, True, 1),
                                                      (True, True, 2), (False, False, 2)])
def test_chosen_experts_that_lie_together(experts, sigmoid, with_bias, groups):
    """The largest logits in one run of neighbours, rising, falling, equal and in few steps: all of a lane's are taken."""
    rng = np.random.default_rng(experts + groups)
    l = -3 + 0.5 * rng.integers(-2, 2, (48, experts))
    for t in range(len(l)):
        n = int(rng.integers(1, 33))
        at = int(rng.integers(0, experts - n + 1)) if t % 3 else (0 if t % 2 else experts - n)
        l[t, at:at + n] = [np.arange(n) / 16, -np.arange(n) / 16, np.zeros(n), rng.integers(0, 4, n) / 4][t % 4]
    bias = 0.125 * rng.integers(0, 2, experts) if with_bias else None
    for k in (8, 31, 32):
        _run(l, min(k, experts // groups), sigmoid=sigmoid, bias=bias, groups=groups, top_groups=1)


def test_equal_logits_and_equal_values():
    _run(np.zeros((3, 40)), 6)
    _run(np.zeros((3, 40)), 6, sigmoid=True, bias=np.full(40, 0.25), groups=5, top_groups=2)
    rng = np.random.default_rng(4)
    _run(rng.integers(0, 3, (200, 48)).astype(float), 10, dtype="bf16", sigmoid=True, bias=np.tile([0.5, 0.0, 0.0], 16))
    l = np.zeros((2, 8))
    l[:, 3], l[:, 5] = -0.0, 0.0
    _run(l, 8)


def test_ruled_out_experts_and_padding_rows():
    rng = np.random.default_rng(6)
    l = rng.standard_normal((50, 24))
    l[rng.random(l.shape) < 0.5] = -INF
    l[7, 3] = np.nan
    l[10:20] = -INF
    l[20, :], l[20, 13] = -INF, -3.0
    l[21, :] = np.nan
    for kw in (dict(), dict(sigmoid=True), dict(groups=6, top_groups=2), dict(sigmoid=True, bias=rng.standard_normal(24), groups=4, top_groups=3)):
        _run(l, 6, **kw)
        _run(l, 6, dtype="bf16", **kw)
    got = _run(np.full((9, 24), -INF), 2)
    assert (got[2].cpu() == 0).all() and (got[3].cpu() == -1).all()
    bias = rng.standard_normal(24)
    bias[[0, 5]], bias[9] = -INF, np.nan
    _run(l, 6, sigmoid=True, bias=bias)


def test_extreme_logits():
    l = np.zeros((8, 16))
    l[0, :4] = [INF, 3.4028234663852886e38, -3.4e38, 100.0]
    l[1] = -np.arange(16) * 20.0            # a sigmoid's end at -80
    l[2] = np.arange(16) * 20.0
    l[3] = -1000.0 - np.arange(16)
    l[4] = 3e38
    l[5] = 1e-40 * np.arange(16)
    l[6, 0], l[6, 1:] = 80.0, -30.0 - np.arange(15)  # the far ones' weights, 2^-18 of themselves
    for sigmoid in (False, True):
        _run(l, 4, sigmoid=sigmoid)
    _run(l, 4, sigmoid=True, bias=np.linspace(-1, 1, 16))
    # a far softmax's chosen experts, the likeliest one in another group: their weights are their own quotient
    l = np.full((1, 8), -300.0) + np.arange(8) * 0.5
    l[0, 0] = 50.0
    _run(l, 2, bias=np.array([-9.0, 0, 0, 0, 0, 0, 0.5, 0.4]))


def test_unaligned_views_streams_and_replays():
    """Buffers that start anywhere, another stream, and a captured call replayed on other logits."""
    import torch
    rng = np.random.default_rng(8)
    stream = torch.cuda.Stream()
    l = rng.standard_normal((33, 61))
    t, ref = _logits(l)
    pad = torch.empty(33 * 61 + 1, device="cuda")
    pad[1:] = t.reshape(-1)
    view = pad[1:].view(33, 61)
    got = _outputs(33, 3, 61)
    torch.cuda.synchronize()
    ham.ham_route(view, *got, stream=stream)
    stream.synchronize()
    _check(got, ref, 3)
    static = t.clone()
    with torch.cuda.stream(stream):
        ham.ham_route(static, *got)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ham.ham_route(static, *got)
    for seed in range(3):
        other, ref = _logits(np.random.default_rng(seed).standard_normal((33, 61)))
        static.copy_(other)
        graph.replay()
        torch.cuda.synchronize()
        _check(got, ref, 3)


@pytest.mark.parametrize("rows,k,n", [(1, 1, 1), (1, 8, 4096), (3, 2, 100), (7, 3, 1000), (130, 4, 264), (9, 32, 40), (65, 5, 4099)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("with_add", [False, True])
def test_combine(rows, k, n, dtype, with_add):
    import torch
    rng = np.random.default_rng(rows * n)
    y = torch.from_numpy(rng.standard_normal((rows * k, n)) * 2.0 ** rng.integers(-6, 7, (rows * k, 1)))
    y = y.float() if dtype == "f32" else y.bfloat16()
    weight = np.float32(rng.random((rows, k)))
    place = rng.permutation(rows * k).reshape(rows, k).astype(np.int32)
    place[rng.random(place.shape) < 0.2] = -1
    if rows > 2:
        place[1] = -1                        # nothing but what is added
        place[2, 0], place[2, -1] = rows * k, np.iinfo(np.int32).max   # (out of range adds nothing either)
    add = torch.from_numpy(rng.standard_normal((rows, n))).bfloat16() if with_add else None
    out = torch.full((rows, n), -7.0, dtype=torch.bfloat16, device="cuda")
    ham.ham_experts_combine(y.cuda(), dev(weight), dev(place), out, add=None if add is None else add.cuda())
    a = None if add is None else add.double().numpy()
    want = ox.combine(y.double().numpy(), weight.astype(np.float64), place, a)
    # k + 1 terms one after another: k roundings of sums that the terms' magnitudes bound (a product is rounded
    # with its sum)
    size = ox.combine(np.abs(y.double().numpy()), weight.astype(np.float64), place, None if a is None else np.abs(a))
    check_bf16(out, want, (k + 1) * 2.0 ** -24 * size)
    if with_add:                             # in place
        same = add.cuda()
        ham.ham_experts_combine(y.cuda(), dev(weight), dev(place), same, add=same)
        assert torch.equal(same, out)


def test_combine_passes_infinities_and_nan_on():
    import torch
    y = torch.ones((4, 16), dtype=torch.bfloat16, device="cuda")
    y[0, 0], y[1, 1], y[3] = INF, float("nan"), float("nan")
    out = torch.empty((2, 16), dtype=torch.bfloat16, device="cuda")
    ham.ham_experts_combine(y, dev(np.float32([[0.5, 0.5], [1.0, 0.0]])), dev(np.int32([[0, 1], [2, -1]])), out)
    got = out.float().cpu().numpy()
    assert got[0, 0] == INF and np.isnan(got[0, 1]) and (got[0, 2:] == 1).all() and (got[1] == 1).all()

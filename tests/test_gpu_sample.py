"""ham_sample against the fp64 oracle and, bit for bit, against its definition in whole numbers."""
import numpy as np
import pytest

from oracle import ops
from paper_2505_20438_gb300 import ham

pytestmark = pytest.mark.gpu


def sample(logits, u, **kw):
    import torch
    b = logits.shape[0]
    tokens = torch.full((b,), -7, dtype=torch.int32, device="cuda")
    probs = torch.full((b,), float("nan"), device="cuda")
    args = {}
    for name, v in kw.items():
        args[name] = torch.as_tensor(v, dtype=torch.int32 if name == "top_k" else torch.float32).expand(b) \
            .contiguous().cuda()
    ham.ham_sample(logits, torch.as_tensor(u, dtype=torch.float32).expand(b).contiguous().cuda(), tokens,
                   probs=probs, **args)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), probs.cpu().numpy()


def whole_number_definition(logits, u, temperature, top_k, top_p, min_p):
    """The documented formula in torch, whole numbers from the weights on."""
    import torch
    l = logits.float()
    l = torch.where(torch.isnan(l), -float("inf"), l)
    b, v = l.shape
    best = l.amax(1, keepdim=True)
    greedy = ~(temperature > 0)
    t = torch.where(greedy, 1.0, temperature)[:, None]
    w = (torch.exp(torch.where(l == best, 0.0, (l - best) / t)) * 2.0 ** 31).to(torch.int64)
    k = torch.where(greedy, 1, torch.where(top_k <= 0, v, top_k.clamp(max=v))).long()
    order = torch.sort(l, dim=1, descending=True, stable=True)[1]
    ws = w.gather(1, order)
    run = ws.cumsum(1)
    place = torch.arange(v, device=l.device)[None]
    mass = run.gather(1, (k - 1)[:, None]).double()
    p = top_p.double()[:, None]
    keep = (place < k[:, None]) & ((p >= 1) | (place == 0) | ((run - ws).double() < p * mass))
    keep &= ws.double() >= min_p.double().clamp(max=1)[:, None] * 2.0 ** 31
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0)).cumsum(1)
    total = kept[:, -1:]
    aim = torch.minimum((u.double()[:, None] * total.double()).floor().long(), total - 1)
    token = (kept <= aim).sum(1)
    prob = (w.gather(1, token[:, None].clamp(max=v - 1)).double() / total.double())[:, 0].float()
    none = best[:, 0] == -float("inf")
    return (torch.where(none, -1, token).int().cpu().numpy(), torch.where(none, 0.0, prob).cpu().numpy())


def check_exact(logits, u, temperature, top_k, top_p, min_p):
    import torch
    s = [torch.as_tensor(x).expand(logits.shape[0]).contiguous().cuda()
         for x in (np.float32(temperature), np.int32(top_k), np.float32(top_p), np.float32(min_p))] \
        if np.ndim(temperature) == 0 else [torch.as_tensor(x).cuda() for x in (temperature, top_k, top_p, min_p)]
    u = torch.as_tensor(u, dtype=torch.float32).cuda()
    tokens = torch.full((logits.shape[0],), -7, dtype=torch.int32, device="cuda")
    probs = torch.empty(logits.shape[0], device="cuda")
    ham.ham_sample(logits, u, tokens, temperature=s[0], top_k=s[1], top_p=s[2], min_p=s[3], probs=probs)
    torch.cuda.synchronize()
    want, prob = whole_number_definition(logits, u, *s)
    np.testing.assert_array_equal(tokens.cpu().numpy(), want)
    np.testing.assert_array_equal(probs.cpu().numpy(), prob)


def _logits(rng, b, v, spread, f32):
    import torch
    l = rng.standard_normal((b, v)) * spread
    l[np.arange(b), rng.integers(0, v, b)] += 6
    t = torch.from_numpy(l.astype(np.float32))
    return (t if f32 else t.bfloat16()).cuda()


SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.3, 50, 1.0, 0.0), (0.9, 50, 0.9, 0.02), (1.0, 3, 0.5, 0.0),
            (1.0, 0, 0.0, 0.0), (1.0, 0, 1.0, 0.3), (0.05, 0, 0.95, 0.0), (1.0, 1, 1.0, 0.0), (0.0, 7, 0.3, 0.1),
            (25.0, 1000, 0.99, 0.0), (1.0, 1 << 30, 0.37, 1e-4), (1.0, 7, 1.0, 2.0)]


# sizes: one token, below a vector, off every alignment (a row of 5003 bf16 values starts anywhere in
# 16 bytes), one CTA and clusters of 2, 4 and 8
@pytest.mark.parametrize("b,v", [(1, 1), (3, 7), (5, 33), (4, 1000), (9, 5003), (30, 20011), (200, 4097), (3, 128256)])
@pytest.mark.parametrize("f32", [True, False])
def test_sample_equals_its_definition(b, v, f32):
    rng = np.random.default_rng(b * 7919 + v)
    for i, s in enumerate(SETTINGS):
        for spread in (0.3, 2.5):
            check_exact(_logits(rng, b, v, spread, f32), rng.random(b).astype(np.float32), *s)


@pytest.mark.parametrize("f32", [True, False])
def test_every_row_its_own_settings(f32):
    rng = np.random.default_rng(5)
    b, v = 160, 32003
    pick = rng.integers(0, len(SETTINGS), b)
    t, k, p, m = (np.array([SETTINGS[i][j] for i in pick]) for j in range(4))
    check_exact(_logits(rng, b, v, 2.0, f32), rng.random(b).astype(np.float32), t.astype(np.float32),
                np.minimum(k, 2 ** 30).astype(np.int32), p.astype(np.float32), m.astype(np.float32))


@pytest.mark.parametrize("v", [17, 3000, 70001, 262144])
def test_equal_logits_are_kept_by_index(v):
    """Rows of equal logits, of two values, of steps: cuts that fall among equal tokens."""
    import torch
    rng = np.random.default_rng(v)
    rows = [np.zeros(v), np.where(np.arange(v) % 3 == 0, 1.0, 0.0), (np.arange(v) % 11) * 0.25,
            np.full(v, -np.inf), np.where(np.arange(v) < v - 1, -np.inf, 2.0)]
    l = torch.from_numpy(np.stack(rows).astype(np.float32)).cuda()
    for s in SETTINGS + [(1.0, v // 2, 1.0, 0.0), (1.0, v // 2 + 1, 0.73, 0.0), (1.0, v - 1, 1.0, 0.0)]:
        check_exact(l, rng.random(5).astype(np.float32), *s)
        check_exact(l.bfloat16(), rng.random(5).astype(np.float32), *s)


def test_near_equal_logits():
    """Thousands of tokens within a few units of the last place of one another."""
    import torch
    rng = np.random.default_rng(8)
    l = np.full((4, 40000), 5.0, np.float32).view(np.int32) + rng.integers(0, 5000, (4, 40000)).astype(np.int32)
    l = torch.from_numpy(l.view(np.float32)).cuda()
    for s in SETTINGS + [(1.0, 20000, 1.0, 0.0), (1.0, 0, 0.77, 0.0)]:
        check_exact(l, rng.random(4).astype(np.float32), *s)


@pytest.mark.parametrize("f32", [True, False])
def test_ruled_out_infinite_and_missing_logits(f32):
    import torch
    l = torch.randn(6, 5000)
    l[0, :] = -float("inf")
    l[1, :] = float("nan")
    l[2, 10:20] = float("inf")
    l[3, ::2] = -float("inf")
    l[4, 1::2] = float("nan")
    l[5, :] = -float("inf")
    l[5, 4321] = -3.0
    l = (l if f32 else l.bfloat16()).cuda()
    for s in SETTINGS:
        check_exact(l, np.linspace(0, 0.999, 6).astype(np.float32), *s)
    tokens, probs = sample(l, 0.5)
    assert list(tokens[:2]) == [-1, -1] and list(probs[:2]) == [0, 0] and tokens[5] == 4321
    assert 10 <= tokens[2] < 20 and probs[2] == np.float32(0.1) and tokens[3] % 2 == 1 and tokens[4] % 2 == 0


@pytest.mark.parametrize("v", [257, 50021])
def test_sample_against_the_oracle(v):
    """The fp64 oracle's running sum holds the aim at the chosen token.  A weight is off by at most
    2.6e-6 of itself (x up to 21.5 with two roundings of 2^-24, the exponential two units) and one unit
    of 2^31 by the truncation."""
    rng = np.random.default_rng(v)
    for s in (dict(), dict(temperature=0.8), dict(top_k=40), dict(top_p=0.9), dict(top_p=0.8, top_k=300, min_p=0.01)):
        l = _logits(rng, 6, v, 2.0, True)
        u = rng.random(6).astype(np.float32)
        tokens, probs = sample(l, u, **s)
        for b in range(6):
            kept = ops.kept_weights(l[b].cpu().numpy().astype(np.float64), **{n: np.float32(x) if n != "top_k" else x
                                                                              for n, x in s.items()})
            run = np.cumsum(kept)
            slack = 2 * (2.6e-6 * run[-1] + v)
            aim, t = u[b] * run[-1], tokens[b]
            assert kept[t] > 0
            assert run[t] - kept[t] - slack <= aim <= run[t] + slack
            assert abs(probs[b] - kept[t] / run[-1]) <= 1e-5 * probs[b] + 2.0 ** -31


def test_random_numbers_at_the_ends():
    l = _logits(np.random.default_rng(0), 3, 999, 1.0, True)
    tokens, _ = sample(l, [0.0, 1.0, float("nan")])
    assert list(tokens) == [0, 998, 0]


def test_frequencies_follow_the_weights():
    """4096 even steps of u over one row hit each token as often as its weight says, to one count."""
    import torch
    rng = np.random.default_rng(3)
    row = rng.standard_normal(37).astype(np.float32)
    n = 4096
    tokens, _ = sample(torch.from_numpy(row).cuda()[None].expand(n, 37).contiguous(), (np.arange(n) + 0.5) / n)
    w = np.exp(row - row.max())
    assert np.abs(np.bincount(tokens, minlength=37) - n * w / w.sum()).max() <= 1.001


def test_no_rows_and_refusals():
    import torch
    l = torch.zeros(2, 64, device="cuda")
    u, tok = torch.zeros(2, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ham.ham_sample(l[:0], u[:0], tok[:0])
    with pytest.raises(ValueError, match="top_k"):
        ham.ham_sample(l, u, tok, top_k=torch.zeros(2, device="cuda"))
    with pytest.raises(ValueError, match="logits"):
        ham.ham_sample(l.double(), u, tok)
    with pytest.raises(ham.HamError, match="vocab") as e:
        ham.ham_sample(torch.zeros(1, 262145, device="cuda"), u[:1], tok[:1])
    assert e.value.status == ham.HAM_EUNSUPPORTED


# Many rows of more logits than one CTA's shared memory holds: a CTA a row.  What its bounds may not hold, and
# lists that come near their 2048 tokens or pass them, beside the settings of the others.
MANY = SETTINGS + [(0.8, 300, 1.0, 0.0), (0.8, 2047, 1.0, 0.0), (1.5, 2045, 0.6, 0.0), (1.0, 5000, 0.9, 0.0),
                   (1.0, 0, 0.9999, 0.0), (1.0, 0, 0.99999, 0.05), (1.0, 0, 0.5, 0.2), (30.0, 0, 0.8, 0.0),
                   (1.0, 0, 1.0, 1e-5), (1e-6, 0, 0.9, 0.0), (1e6, 100, 0.9, 0.0)]


@pytest.mark.parametrize("b,v,f32", [(240, 20011, True), (160, 50001, True), (60, 262144, True), (240, 40003, False),
                                     (120, 130001, False)])
def test_many_rows(b, v, f32):
    rng = np.random.default_rng(b + v)
    for spread in (0.3, 2.5):
        pick = np.arange(b) % len(MANY)
        t, k, p, m = (np.array([MANY[i][j] for i in pick]) for j in range(4))
        check_exact(_logits(rng, b, v, spread, f32), rng.random(b).astype(np.float32), t.astype(np.float32),
                    np.minimum(k, 2 ** 30).astype(np.int32), p.astype(np.float32), m.astype(np.float32))


@pytest.mark.parametrize("f32", [True, False])
def test_many_rows_of_few_values(f32):
    """Equal, stepped, sorted, near-equal, ruled-out, infinite and missing logits, a row each."""
    import torch
    v = 40003
    rng = np.random.default_rng(21)
    at = np.arange(v)
    kinds = [np.zeros(v), np.where(at % 3 == 0, 1.0, 0.0), (at % 11) * 0.25, np.full(v, -np.inf),
             np.where(at < v - 1, -np.inf, 2.0), np.full(v, np.nan), np.where(at % 2 == 0, np.nan, at % 7),
             np.where((at > 100) & (at < 5000), np.inf, 1.0), np.where(at == 7, np.inf, rng.standard_normal(v)),
             8 - at * 1e-3, at * 1e-3 - 8, rng.standard_normal(v) * 1e6, rng.standard_normal(v) * 1e-6 + 1000,
             np.float32(5) + rng.integers(0, 5000, v) * np.float32(2.0 ** -21), np.where(at % 500 == 0, 0.0, -1e30)]
    settings = MANY + [(1.0, v // 2, 1.0, 0.0), (1.0, v // 2 + 1, 0.73, 0.0), (1.0, v - 1, 1.0, 0.0)]
    rows = [(x, s) for x in kinds for s in settings]
    assert len(rows) >= 240
    l = torch.from_numpy(np.stack([x for x, _ in rows]).astype(np.float32)).cuda()
    t, k, p, m = (np.array([s[j] for _, s in rows]) for j in range(4))
    check_exact(l if f32 else l.bfloat16(), rng.random(len(rows)).astype(np.float32), t.astype(np.float32),
                np.minimum(k, 2 ** 30).astype(np.int32), p.astype(np.float32), m.astype(np.float32))

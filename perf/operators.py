"""What follows a macro-step's attention, as a serving program calls it, for timing and comparison.

Four operators: the residual's addition with the root-mean-square norm and an output in 8 bits
("norm"), the product with 8-bit weights that have a scale for each block of 128 x 128 ("linear", from
8-bit rows or from bf16 rows that it encodes first), the first half of a gated feed-forward block in 8
bits ("gated"), and the choice of a token from its logits and a given random number ("sample").

8-bit rows: e4m3 codes and, for each 128 elements of a row, a scale byte s that stands for 2^(s - 127);
a row's scale bytes are padded to a multiple of four.  A block's scale is 2^(E - 8) for its largest
magnitude m 2^E (0.5 <= m < 1), E - 8 kept within -124..119, and 1 for a block of zeros.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
BLOCK = 128
FINE = 1 << 31          # a token's weight is counted in units of 1/FINE of the likeliest token's
MOST_FLOPS = 1.1e12     # a drawn product costs no more than the largest listed one
MOST_LOGITS = 256 * 128256
MOST_NORM = 16384 * 4096


# -------------------------------------------------------------------------------------------
# the cases
# -------------------------------------------------------------------------------------------
def _norm(name=None, **kw):
    c = dict(kind="norm", rows=8, hidden=4096, residual=True, out="fp8")
    c.update(kw)
    return dict(c, name=name) if name else c


def _linear(name=None, **kw):
    c = dict(kind="linear", rows=8, k=4096, n=4096, x="fp8", out="bf16")
    c.update(kw)
    return dict(c, name=name) if name else c


def _gated(name=None, **kw):
    c = dict(kind="gated", rows=8, k=4096, f=16384)
    c.update(kw)
    return dict(c, name=name) if name else c


def _sample(name=None, **kw):
    c = dict(kind="sample", rows=8, vocab=128256, dtype="f32", mode="all", spread=2.5)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The residual and norm after a layer's attention, for the small serving batch of 8 macro-steps:
        # the sum goes on to the next residual, the 8-bit rows to the feed-forward.
        _norm("norm_b8_h4096"),
        # The same for four prompts of 4096 tokens.
        _norm("norm_t16384_h4096", rows=16384),
        # A final norm of a ragged batch (no residual, bf16 rows out) at an uneven width.
        _norm("norm_t1333_h5136_bf16", rows=1333, hidden=5136, residual=False, out="bf16"),
        # One conversation: the output projection of one macro-step, its attention's bf16 output encoded
        # on the way.
        _linear("oproj_b1_h4096", rows=1, x="bf16"),
        # The head over the Llama-3 vocabulary for a batch of 64 macro-steps.
        _linear("head_b64_v128256", rows=64, n=128256, out="f32"),
        # An uneven product of a ragged batch: no size a multiple of a tile.
        _linear("linear_t777_k2064_n1000", rows=777, k=2064, n=1000),
        # A second feed-forward product of two prompts of 2048 tokens.
        _linear("down_t4096_k16384_n4096", rows=4096, k=16384),
        # The feed-forward's first half for the small serving batch.
        _gated("gated_b8_f16384"),
        # The same for four prompts of 1024 tokens.
        _gated("gated_t4096_f16384", rows=4096),
        # The first token of one conversation: top-k, top-p and min-p together.
        _sample("sample_b1_v128256", rows=1),
        # A batch of 256 macro-steps with every row's settings its own, greedy rows among them.
        _sample("sample_b256_v128256_mixed", rows=256, mode="mixed"),
        # A smaller vocabulary of uneven size in bf16, top-p alone, rather flat logits (many tokens kept).
        _sample("sample_b40_v50001_bf16", rows=40, vocab=50001, dtype="bf16", mode="top_p", spread=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _sixteens(rng, lo, hi):
    v = 16 * _log_int(rng, lo // 16, hi // 16)
    return v + 16 if v == 3 << 10 else v


def draw(rng):
    kind = rng.choice(["norm", "linear", "linear", "gated", "sample"])
    if kind == "norm":
        hidden = _sixteens(rng, 256, 16384)
        rows = min(_log_int(rng, 1, 16384), MOST_NORM // hidden)
        return _norm(rows=rows, hidden=hidden, residual=rng.random() < 0.7, out=rng.choice(["fp8", "fp8", "bf16"]))
    if kind == "sample":
        vocab = _log_int(rng, 1000, 200000)
        rows = min(_log_int(rng, 1, 256), MOST_LOGITS // vocab)
        return _sample(rows=rows, vocab=vocab, dtype=rng.choice(["f32", "bf16"]),
                       mode=rng.choice(["all", "mixed", "top_p", "top_k", "plain"]), spread=round(rng.uniform(0.5, 4.0), 3))
    rows, k = _log_int(rng, 1, 8192), _sixteens(rng, 256, 16384)
    n = _log_int(rng, 128, 16384) if rng.random() < 0.4 else _sixteens(rng, 128, 32768)
    if kind == "gated":
        f = max(16, n // 32 * 16)
        while 4.0 * rows * k * f > MOST_FLOPS:
            rows = rows // 2 + 1
        return _gated(rows=rows, k=k, f=f)
    while 2.0 * rows * k * n > MOST_FLOPS:
        rows = rows // 2 + 1
    return _linear(rows=rows, k=k, n=n, x=rng.choice(["fp8", "fp8", "bf16"]), out=rng.choice(["bf16", "bf16", "f32"]))


def work(case):
    c = case
    if c["kind"] == "norm":
        e = c["rows"] * c["hidden"]
        b = 2 * e + (4 * e if c["residual"] else 0) + (2 * e if c["out"] == "bf16" else e + e // BLOCK)
        return {"bytes": b + 2 * c["hidden"], "flops": 6 * e}
    if c["kind"] == "sample":
        e = c["rows"] * c["vocab"]
        return {"bytes": e * (4 if c["dtype"] == "f32" else 2) + 28 * c["rows"], "flops": 6 * e}
    t, k = c["rows"], c["k"]
    if c["kind"] == "gated":
        return {"bytes": (t * k + 2 * c["f"] * k + t * c["f"]) * (1 + 1 / BLOCK), "flops": 4 * t * k * c["f"]}
    x = 2 * t * k + t * k * (1 + 1 / BLOCK) if c["x"] == "bf16" else t * k * (1 + 1 / BLOCK)
    return {"bytes": x + c["n"] * k * (1 + 1 / BLOCK ** 2) + t * c["n"] * (4 if c["out"] == "f32" else 2),
            "flops": 2 * t * k * c["n"]}


# -------------------------------------------------------------------------------------------
# the inputs
# -------------------------------------------------------------------------------------------
def _gen(seed, what):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + what) & 0x7FFFFFFFFFFF)
    return g


def _scale_bytes(k):
    return 4 * (-(-k // (4 * BLOCK)))


def _hidden_rows(g, rows, width):
    """Rows as a residual stream has them: about N(0, 1), one channel in 256 eight times as large."""
    x = torch.randn((rows, width), generator=g, device="cuda")
    x[:, 7::256] *= 8.0
    return x


def _weight(g, n, k):
    """Codes and block scales of an n x k weight drawn N(0, 1/k)."""
    codes = torch.empty((n, k), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty((-(-n // BLOCK), _scale_bytes(k)), dtype=torch.uint8, device="cuda").fill_(127)
    for r in range(0, n, 8192):     # (in parts: the fp32 draw of a large weight is not held whole)
        w = torch.randn((min(8192, n - r), k), generator=g, device="cuda") * k ** -0.5
        rows, kb = -(-w.shape[0] // BLOCK), -(-k // BLOCK)
        p = torch.zeros((rows * BLOCK, kb * BLOCK), device="cuda")
        p[:w.shape[0], :k] = w
        p = p.view(rows, BLOCK, kb, BLOCK)
        e = _exponent(p.abs().amax(dim=(1, 3)))
        q = (p * _two_to(-e)[:, None, :, None]).reshape(rows * BLOCK, kb * BLOCK)
        codes[r:r + w.shape[0]] = q[:w.shape[0], :k].to(torch.float8_e4m3fn)
        scales[r // BLOCK:r // BLOCK + rows, :kb] = (e + 127).to(torch.uint8)
    return codes, scales


def _inputs(case, seed):
    c = case
    if c["kind"] == "norm":
        g = _gen(seed, 1)
        s = {"x": (0.5 * _hidden_rows(g, c["rows"], c["hidden"])).bfloat16(),
             "w": (1 + 0.1 * torch.randn((c["hidden"],), generator=g, device="cuda")).bfloat16()}
        s["r"] = _hidden_rows(g, c["rows"], c["hidden"]).bfloat16() if c["residual"] else None
        return s
    if c["kind"] == "sample":
        g = _gen(seed, 2)
        b, v = c["rows"], c["vocab"]
        logits = torch.randn((b, v), generator=g, device="cuda") * c["spread"]
        likely = torch.randint(0, v, (b, 16), generator=g, device="cuda")  # what the context makes likely
        logits.scatter_add_(1, likely, 4 + 3 * torch.rand((b, 16), generator=g, device="cuda"))
        logits[:, v // 3:v // 3 + 50] = -math.inf                          # tokens that a grammar rules out
        s = {"logits": logits if c["dtype"] == "f32" else logits.bfloat16(),
             "u": torch.rand((b,), generator=g, device="cuda"),
             "temperature": torch.full((b,), 0.8, device="cuda"),
             "top_k": torch.zeros((b,), dtype=torch.int32, device="cuda"),
             "top_p": torch.ones((b,), device="cuda"), "min_p": torch.zeros((b,), device="cuda")}
        if c["mode"] in ("all", "top_k"):
            s["top_k"].fill_(50)
        if c["mode"] in ("all", "top_p"):
            s["top_p"].fill_(0.9)
        if c["mode"] == "all":
            s["min_p"].fill_(0.02)
        if c["mode"] == "mixed":
            r = torch.rand((4, b), generator=g, device="cuda")
            s["temperature"] = torch.where(r[0] < 0.2, 0.0, 0.3 + 1.2 * r[0])
            s["top_k"] = torch.where(r[1] < 0.3, 0.0, r[1] * 2000).to(torch.int32)
            s["top_p"] = torch.where(r[2] < 0.3, 1.0, r[2])
            s["min_p"] = torch.where(r[3] < 0.5, 0.0, r[3] * 0.1)
        return s
    g = _gen(seed, 3)
    t, k = c["rows"], c["k"]
    s = {}
    x = _hidden_rows(g, t, k)
    if c.get("x") == "bf16":
        s["x"] = x.bfloat16()
    else:
        s["codes"], s["scales"] = _encode(x)
    if c["kind"] == "gated":
        s["w"], s["w_up"] = _weight(g, c["f"], k), _weight(g, c["f"], k)
    else:
        s["w"] = _weight(g, c["n"], k)
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if own:
        from paper_2505_20438_gb300 import ham
        s["ham"] = ham
        if case["kind"] in ("linear", "gated"):     # a program keeps the weights' handle
            n = case["f"] if case["kind"] == "gated" else case["n"]
            up = [t.view(torch.uint8) for t in s["w_up"]] if case["kind"] == "gated" else [None, None]
            w = [t.view(torch.uint8) for t in s["w"]]
            s["handle"] = ham.ham_fp8_weight_alloc(n, case["k"], w[0], w[1], up[0], up[1])
            s.pop("w"), s.pop("w_up", None)
    return s


# -------------------------------------------------------------------------------------------
# the plain forms
# -------------------------------------------------------------------------------------------
def _two_to(e):
    """2^e in fp32 for whole e in -126..127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(a):
    """The exponent of the scale of blocks whose largest magnitudes are `a`."""
    return torch.where(a > 0, (torch.frexp(a)[1] - 8).clamp(-124, 119), 0)


def _blocks(x):
    t, k = x.shape
    kb = -(-k // BLOCK)
    return torch.nn.functional.pad(x, (0, kb * BLOCK - k)).view(t, kb, BLOCK)


def _encode(x):
    """fp32 rows -> (e4m3 codes, scale bytes)."""
    t, k = x.shape
    b = _blocks(x)
    e = _exponent(b.abs().amax(dim=2))
    codes = (b * _two_to(-e)[:, :, None]).view(t, -1)[:, :k].to(torch.float8_e4m3fn)
    scales = torch.full((t, _scale_bytes(k)), 127, dtype=torch.uint8, device=x.device)
    scales[:, :e.shape[1]] = (e + 127).to(torch.uint8)
    return codes.contiguous(), scales


def _powers(scales, k):
    """The scales' fp32 values, for the blocks of a row of k."""
    return _two_to(scales[:, :-(-k // BLOCK)].to(torch.int32) - 127)


def _decode(codes, scales):
    p = _powers(scales, codes.shape[1]).repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]
    return codes.to(torch.float32) * p


def _decode_weight(w):
    codes, scales = w
    p = _powers(scales, codes.shape[1]).repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]
    return codes.to(torch.float32) * p.repeat_interleave(BLOCK, 0)[:codes.shape[0]]


def _as_values(codes, scales):
    """8-bit outputs as the values that they stand for (both views)."""
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}


def _plain_norm(s):
    h = s["x"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["w"].float()
    out = {"sum": h.bfloat16()} if s["r"] is not None else {}
    if s["case"]["out"] == "bf16":
        return dict(out, out=y.bfloat16())
    return dict(out, **_as_values(*_encode(y)))


def _plain_product(s):
    if "x" in s:
        codes, scales = _encode(s["x"].float())
    else:
        codes, scales = s["codes"], s["scales"]
    x = _decode(codes, scales)
    if s["case"]["kind"] == "gated":
        g, u = x @ _decode_weight(s["w"]).t(), x @ _decode_weight(s["w_up"]).t()
        return _as_values(*_encode(g / (1 + torch.exp(-g)) * u))
    y = x @ _decode_weight(s["w"]).t()
    out = {"y": y if s["case"]["out"] == "f32" else y.bfloat16()}
    return dict(out, **_as_values(codes, scales)) if "x" in s else out


def _plain_sample(s):
    logits = s["logits"].float()
    b, v = logits.shape
    logits = torch.where(torch.isnan(logits), -math.inf, logits)
    best = logits.amax(1, keepdim=True)
    greedy = ~(s["temperature"] > 0)
    t = torch.where(greedy, 1.0, s["temperature"])[:, None]
    x = torch.where(logits == best, 0.0, (logits - best) / t)
    w = (torch.exp(x) * FINE).to(torch.int64)
    k = torch.where(greedy, 1, torch.where(s["top_k"] <= 0, v, s["top_k"].clamp(max=v)))
    order = torch.sort(logits, dim=1, descending=True, stable=True)[1]
    ws = w.gather(1, order)
    run = ws.cumsum(1)
    place = torch.arange(v, device=logits.device)[None]
    mass = run.gather(1, (k.long() - 1)[:, None]).double()
    p = s["top_p"].double()[:, None]
    keep = (place < k[:, None]) & ((p >= 1) | (place == 0) | ((run - ws).double() < p * mass))
    keep &= ws.double() >= s["min_p"].double()[:, None] * FINE
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0)).cumsum(1)
    total = kept[:, -1:]
    target = torch.minimum((s["u"].double()[:, None] * total.double()).floor().long(), total - 1)
    token = (kept <= target).sum(1)
    prob = w.gather(1, token[:, None].clamp(max=v - 1))[:, 0].double() / total[:, 0].double()
    none = best[:, 0] == -math.inf
    return {"token": torch.where(none, -1, token).to(torch.int32), "prob": torch.where(none, 0.0, prob).float()}


# -------------------------------------------------------------------------------------------
# the framework's calls
# -------------------------------------------------------------------------------------------
def _own_norm(s):
    ham, c = s["ham"], s["case"]
    t, h = s["x"].shape
    total = torch.empty_like(s["x"]) if c["residual"] else None
    out = {"sum": total} if c["residual"] else {}
    if c["out"] == "bf16":
        y = torch.empty_like(s["x"])
        ham.ham_add_norm(s["x"], s["w"], EPS, residual=s["r"], sum_out=total, out=y)
        return dict(out, out=y)
    codes = torch.empty((t, h), dtype=torch.uint8, device="cuda")
    scales = torch.empty((t, _scale_bytes(h)), dtype=torch.uint8, device="cuda")
    ham.ham_add_norm(s["x"], s["w"], EPS, residual=s["r"], sum_out=total, codes=codes, scales=scales)
    return dict(out, **_as_values(codes, scales))


def _own_product(s):
    ham, c = s["ham"], s["case"]
    t, k, out = c["rows"], c["k"], {}
    if "x" in s:
        codes = torch.empty((t, k), dtype=torch.uint8, device="cuda")
        scales = torch.empty((t, _scale_bytes(k)), dtype=torch.uint8, device="cuda")
        ham.ham_fp8_encode(s["x"], codes, scales)
        out = _as_values(codes, scales)
    else:
        codes, scales = s["codes"].view(torch.uint8), s["scales"]
    if c["kind"] == "gated":
        h = torch.empty((t, c["f"]), dtype=torch.uint8, device="cuda")
        hs = torch.empty((t, _scale_bytes(c["f"])), dtype=torch.uint8, device="cuda")
        ham.ham_fp8_gated(s["handle"], codes, scales, h, hs)
        return _as_values(h, hs)
    y = torch.empty((t, c["n"]), dtype=torch.float32 if c["out"] == "f32" else torch.bfloat16, device="cuda")
    ham.ham_fp8_linear(s["handle"], codes, scales, y)
    return dict(out, y=y)


def _own_sample(s):
    b = s["logits"].shape[0]
    token = torch.empty((b,), dtype=torch.int32, device="cuda")
    prob = torch.empty((b,), dtype=torch.float32, device="cuda")
    s["ham"].ham_sample(s["logits"], s["u"], token, temperature=s["temperature"], top_k=s["top_k"],
                        top_p=s["top_p"], min_p=s["min_p"], probs=prob)
    return {"token": token, "prob": prob}


def run(state):
    kind = state["case"]["kind"]
    if kind == "norm":
        return _own_norm(state) if own else _plain_norm(state)
    if kind == "sample":
        return _own_sample(state) if own else _plain_sample(state)
    return _own_product(state) if own else _plain_product(state)


# -------------------------------------------------------------------------------------------
# the definitions in 64 bits
# -------------------------------------------------------------------------------------------
def _power(e):
    """2^e in fp64, exactly (a power function need not be exact)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_rows(v):
    """fp64 rows -> the values that their codes and scale bytes stand for."""
    t, k = v.shape
    codes, scales = torch.empty_like(v), torch.ones((t, _scale_bytes(k)), dtype=torch.float64, device=v.device)
    for i in range(-(-k // BLOCK)):
        part = v[:, i * BLOCK:(i + 1) * BLOCK]
        top = part.abs().max(1).values
        p = _power(torch.where(top > 0, torch.frexp(top).exponent - 8, 0).clamp(-124, 119))
        q = part / p[:, None]
        # e4m3: three bits after the leading one, none below 2^-9
        step = _power((torch.frexp(q).exponent - 4).clamp(min=-9))
        codes[:, i * BLOCK:(i + 1) * BLOCK] = torch.round(q / step) * step
        scales[:, i] = p
    return {"codes": codes, "scales": scales}


def _exact_operand(codes, scales, down):
    """The fp64 values of codes whose scales hold for `down` rows each."""
    v = codes.double()
    p = _power(scales.to(torch.int64) - 127)
    for i in range(-(-v.shape[1] // BLOCK)):
        v[:, i * BLOCK:(i + 1) * BLOCK] *= p[:, i].repeat_interleave(down)[:v.shape[0], None]
    return v


def _exact_prob(s):
    """The chosen tokens' probabilities among the kept ones, row by row in fp64."""
    at = {n: s[n].double().cpu().numpy() for n in s if n != "case"}
    prob = np.zeros(len(at["u"]))
    for b, l in enumerate(at["logits"]):
        l = np.where(np.isnan(l), -np.inf, l)
        top = l.max()
        if top == -np.inf:
            continue
        greedy = not at["temperature"][b] > 0
        with np.errstate(invalid="ignore"):
            x = np.where(l == top, 0.0, (l - top) / (1.0 if greedy else at["temperature"][b]))
        w = np.floor(np.exp(x) * FINE)
        first = np.lexsort((np.arange(len(l)), -l))
        k = 1 if greedy else int(at["top_k"][b]) if 0 < at["top_k"][b] < len(l) else len(l)
        run = np.cumsum(w[first[:k]])
        n = k if at["top_p"][b] >= 1 else min(k, 1 + int(np.searchsorted(run, at["top_p"][b] * run[-1], "left")))
        first = first[:n][w[first[:n]] >= at["min_p"][b] * FINE]
        kept = np.zeros_like(w)
        kept[first] = w[first]
        run = np.cumsum(kept)
        token = int(np.searchsorted(run, min(np.floor(at["u"][b] * run[-1]), run[-1] - 1), "right"))
        prob[b] = w[token] / run[-1]
    return torch.from_numpy(prob)


def exact(case, seed):
    c = case
    if 2.0 * c["rows"] * c.get("k", 0) * (c.get("n") or 2 * c.get("f", 0)) > 4e12:
        return None
    s = _inputs(case, seed)
    if c["kind"] == "norm":
        h = s["x"].double() if s["r"] is None else s["x"].double() + s["r"].double()
        y = s["w"].double() * h / torch.sqrt((h * h).sum(1, keepdim=True) / c["hidden"] + EPS)
        out = {"sum": h} if s["r"] is not None else {}
        return dict(out, out=y) if c["out"] == "bf16" else dict(out, **_exact_rows(y))
    if c["kind"] == "sample":
        return {"token": None, "prob": _exact_prob(s)}
    out = {}
    if "x" in s:
        out = _exact_rows(s["x"].double())
        x = out["codes"].clone()
        for i in range(-(-c["k"] // BLOCK)):
            x[:, i * BLOCK:(i + 1) * BLOCK] *= out["scales"][:, i:i + 1]
    else:
        x = _exact_operand(s["codes"], s["scales"], 1)
    y = x @ _exact_operand(*s["w"], BLOCK).T
    if c["kind"] == "gated":
        y = y / (1 + torch.exp(-y)) * (x @ _exact_operand(*s["w_up"], BLOCK).T)
        return _exact_rows(y)
    return dict(out, y=y)

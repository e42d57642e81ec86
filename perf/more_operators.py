"""A feed-forward block made of experts, as a serving program calls it, for timing and comparison.

Four operators: the choice of each row's experts with the grouping of the chosen (row, expert) pairs by
expert ("route"), the first half of the experts' gated blocks over the grouped rows, 8-bit rows and
weights ("gated"), their second product ("linear"), and the weighted sum of a row's results ("combine").

8-bit rows: e4m3 codes and, for each 128 elements of a row, a scale byte s that stands for 2^(s - 127);
a row's scale bytes are padded to a multiple of four.  A block's scale is 2^(E - 8) for its largest
magnitude m 2^E (0.5 <= m < 1), E - 8 kept within -124..119, and 1 for a block of zeros.  Weights have
one scale for each 128 x 128.

Route: scores are softmax(l), or 1 / (1 + exp(-max(l, -80))); an expert's value is its score plus its
bias; where experts come in groups, the best groups by the sum of their two largest values stay; of
what stays the top_k largest values are chosen, largest first, equal ones by index.  A logit of -inf
rules its expert out; a place that none is left for holds -1.  Slots are the chosen pairs in order of
(expert, row, place): `order` has each slot's pair row * top_k + place, `place` each pair's slot.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 128
MOST_FLOPS = 4.0 * 4096 * 8 * 4096 * 2048   # a drawn product costs no more than the largest listed one
MOST_WEIGHT = 64 * 2 * 4096 * 2048
MOST_LOGITS = 16384 * 256
MOST_SUMMED = 4096 * 8 * 4096


# -------------------------------------------------------------------------------------------
# the cases
# -------------------------------------------------------------------------------------------
def _route(name=None, **kw):
    c = dict(kind="route", rows=8, experts=64, top_k=8, dtype="f32", score="softmax", bias=False, groups=1,
             top_groups=1, renorm=True, scale=1.0, masked=0.0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _gated(name=None, **kw):
    c = dict(kind="gated", rows=8, experts=64, top_k=8, k=4096, f=2048)
    c.update(kw)
    return dict(c, name=name) if name else c


def _linear(name=None, **kw):
    c = dict(kind="linear", rows=8, experts=64, top_k=8, k=2048, n=4096, out="bf16")
    c.update(kw)
    return dict(c, name=name) if name else c


def _combine(name=None, **kw):
    c = dict(kind="combine", rows=8, top_k=8, n=4096, y="bf16", add=False, missing=0.0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The choice of 8 of 64 experts for the small serving batch of 8 macro-steps.
        _route("route_b8_e64"),
        # The same for four prompts of 4096 tokens and 256 experts in 8 groups, sigmoid scores and a bias that
        # balances the experts' load.
        _route("route_t16384_e256_groups", rows=16384, experts=256, score="sigmoid", bias=True, groups=8, top_groups=4,
               scale=2.5),
        # A ragged, padded batch of bf16 logits (equal ones among them), weights as the softmax has them.
        _route("route_t1333_e60_bf16", rows=1333, experts=60, top_k=4, dtype="bf16", renorm=False, masked=0.1),
        # One conversation: the first half of its macro-step's four experts.
        _gated("gated_b1_e32", rows=1, experts=32, top_k=4),
        # The small serving batch: about 40 of the 64 experts have a row or two each.
        _gated("gated_b8_e64"),
        # An uneven batch over few experts: no size a multiple of a tile.
        _gated("gated_t777_e24", rows=777, experts=24, top_k=3, k=2064, f=528),
        # Two prompts of 2048 tokens: some 512 rows an expert.
        _gated("gated_t4096_e64", rows=4096),
        # The second product for the small serving batch.
        _linear("linear_b8_e64"),
        # An uneven one with fp32 results.
        _linear("linear_t777_e24_f32", rows=777, experts=24, top_k=3, k=528, n=1000, out="f32"),
        # Two prompts of 2048 tokens.
        _linear("linear_t4096_e64", rows=4096),
        # The weighted sum for the same.
        _combine("combine_t4096_k8", rows=4096),
        # An uneven, padded batch of fp32 results with the residual added.
        _combine("combine_t1333_k3_f32", rows=1333, top_k=3, n=1000, y="f32", add=True, missing=0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _sixteens(rng, lo, hi):
    return 16 * _log_int(rng, lo // 16, hi // 16)


def draw(rng):
    kind = rng.choice(["route", "gated", "gated", "linear", "combine"])
    if kind == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * _log_int(rng, max(2, 8 // groups), 256 // groups)
        top_groups = rng.randint((groups + 1) // 2, groups)
        top_k = min(_log_int(rng, 1, 16), experts // groups * top_groups)
        rows = min(_log_int(rng, 1, 16384), MOST_LOGITS // experts)
        return _route(rows=rows, experts=experts, top_k=top_k, dtype=rng.choice(["f32", "bf16"]),
                      score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5, groups=groups,
                      top_groups=top_groups, renorm=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]),
                      masked=rng.choice([0.0, 0.0, 0.1]))
    if kind == "combine":
        n, top_k = _log_int(rng, 64, 8192), _log_int(rng, 1, 12)
        rows = min(_log_int(rng, 1, 8192), MOST_SUMMED // (n * top_k))
        return _combine(rows=max(rows, 1), top_k=top_k, n=n, y=rng.choice(["bf16", "bf16", "f32"]),
                        add=rng.random() < 0.5, missing=rng.choice([0.0, 0.0, 0.1]))
    experts = _log_int(rng, 4, 128)
    top_k = min(_log_int(rng, 1, 8), experts)
    rows, k = _log_int(rng, 1, 8192), _sixteens(rng, 256, 8192)
    n = _sixteens(rng, 128, 8192) if kind == "gated" or rng.random() < 0.6 else _log_int(rng, 128, 8192)
    parts = 2 if kind == "gated" else 1
    while parts * experts * k * n > MOST_WEIGHT:
        experts = max(experts // 2, 1)
        top_k = min(top_k, experts)
        if experts == 1:
            n = max(16, n // 32 * 16)
    while 2.0 * parts * rows * top_k * k * n > MOST_FLOPS:
        rows = rows // 2 + 1
    if kind == "gated":
        return _gated(rows=rows, experts=experts, top_k=top_k, k=k, f=n)
    return _linear(rows=rows, experts=experts, top_k=top_k, k=k, n=n, out=rng.choice(["bf16", "bf16", "f32"]))


def work(case):
    c = case
    t, top = c["rows"], c["top_k"]
    if c["kind"] == "route":
        e = t * c["experts"]
        return {"bytes": e * (4 if c["dtype"] == "f32" else 2) + 16 * t * top + 8 * c["experts"], "flops": 8 * e}
    if c["kind"] == "combine":
        live = 1 - c["missing"]
        return {"bytes": live * t * top * c["n"] * (4 if c["y"] == "f32" else 2) + t * c["n"] * (4 if c["add"] else 2)
                + 8 * t * top, "flops": 2 * t * top * c["n"]}
    # experts that have a row, of a uniform choice
    e = c["experts"] * (1 - (1 - top / c["experts"]) ** t)
    k, s = c["k"], t * top
    if c["kind"] == "gated":
        return {"bytes": t * k * (1 + 1 / BLOCK) + e * 2 * c["f"] * k * (1 + 1 / BLOCK ** 2)
                + s * c["f"] * (1 + 1 / BLOCK) + 4 * s, "flops": 4 * s * k * c["f"]}
    return {"bytes": s * k * (1 + 1 / BLOCK) + e * c["n"] * k * (1 + 1 / BLOCK ** 2)
            + s * c["n"] * (4 if c["out"] == "f32" else 2), "flops": 2 * s * k * c["n"]}


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


def _weights(g, experts, n, k):
    """Codes [experts][n][k] and block scales of weights drawn N(0, 1/k)."""
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    codes = torch.empty((experts, n, k), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.full((experts, nb, _scale_bytes(k)), 127, dtype=torch.uint8, device="cuda")
    for i in range(experts):
        p = torch.zeros((nb * BLOCK, kb * BLOCK), device="cuda")
        p[:n, :k] = torch.randn((n, k), generator=g, device="cuda") * k ** -0.5
        p = p.view(nb, BLOCK, kb, BLOCK)
        e = _exponent(p.abs().amax(dim=(1, 3)))
        q = (p * _two_to(-e)[:, None, :, None]).reshape(nb * BLOCK, kb * BLOCK)
        codes[i] = q[:n, :k].to(torch.float8_e4m3fn)
        scales[i, :, :kb] = (e + 127).to(torch.uint8)
    return codes, scales


def _grouped(expert, experts):
    """offsets, order and place of chosen experts [rows][top_k] (-1: none)."""
    flat = expert.reshape(-1).long()
    key = torch.where(flat < 0, experts, flat)
    counts = (key[:, None] == torch.arange(experts, device=flat.device)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    order = torch.sort(key, stable=True)[1]
    slots = torch.arange(flat.shape[0], device=flat.device)
    place = torch.empty_like(order)
    place[order] = slots
    place = torch.where(flat < 0, -1, place)
    order = torch.where(slots < offsets[-1], order, -1)
    return offsets.to(torch.int32), order.to(torch.int32), place.to(torch.int32)


def _inputs(case, seed):
    c = case
    t, top = c["rows"], c["top_k"]
    if c["kind"] == "route":
        g = _gen(seed, 11)
        l = torch.randn((t, c["experts"]), generator=g, device="cuda") * 1.5
        l += 0.5 * torch.randn((c["experts"],), generator=g, device="cuda")       # some are liked more
        if c["masked"]:
            l[torch.rand(l.shape, generator=g, device="cuda") < 0.02] = -math.inf  # experts that are full
            l[t - int(t * c["masked"]):] = -math.inf                               # the padding's rows
        bias = 0.1 * torch.randn((c["experts"],), generator=g, device="cuda") if c["bias"] else None
        return {"logits": l if c["dtype"] == "f32" else l.bfloat16(), "bias": bias}
    if c["kind"] == "combine":
        g = _gen(seed, 12)
        place = torch.randperm(t * top, generator=g, device="cuda").to(torch.int32).view(t, top)
        place[t - int(t * c["missing"]):] = -1
        w = torch.rand((t, top), generator=g, device="cuda")
        y = torch.randn((t * top, c["n"]), generator=g, device="cuda")
        add = torch.randn((t, c["n"]), generator=g, device="cuda").bfloat16() if c["add"] else None
        return {"place": place, "weight": w / w.sum(1, keepdim=True), "y": y if c["y"] == "f32" else y.bfloat16(),
                "add": add}
    g = _gen(seed, 13)
    liked = torch.rand((t, c["experts"]), generator=g, device="cuda")
    liked += 0.1 * torch.rand((c["experts"],), generator=g, device="cuda")
    expert = torch.sort(liked, dim=1, descending=True)[1][:, :top].to(torch.int32)
    offsets, order, _ = _grouped(expert, c["experts"])
    s = {"offsets": offsets, "order": order}
    n = c["f"] if c["kind"] == "gated" else c["n"]
    s["codes"], s["scales"] = _encode(_hidden_rows(g, t if c["kind"] == "gated" else t * top, c["k"]))
    s["w"] = _weights(g, c["experts"], n, c["k"])
    if c["kind"] == "gated":
        s["w_up"] = _weights(g, c["experts"], n, c["k"])
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if "offsets" in s and not own:
        s["parts"] = s["offsets"].tolist()          # the plain form's plan
    if own:
        from paper_2505_20438_gb300 import ham
        s["ham"] = ham
        if "w" in s:                                # a program keeps the weights' handle
            n = case["f"] if case["kind"] == "gated" else case["n"]
            w = [t.view(torch.uint8) for t in s.pop("w")]
            up = [t.view(torch.uint8) for t in s.pop("w_up")] if "w_up" in s else [None, None]
            s["handle"] = ham.ham_fp8_experts_alloc(case["experts"], n, case["k"], w[0], w[1], up[0], up[1])
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


def _decode_weight(codes, scales):
    p = _powers(scales, codes.shape[1]).repeat_interleave(BLOCK, 1)[:, :codes.shape[1]]
    return codes.to(torch.float32) * p.repeat_interleave(BLOCK, 0)[:codes.shape[0]]


def _as_values(codes, scales):
    """8-bit outputs as the values that they stand for (both views)."""
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}


def _plain_route(s):
    c = s["case"]
    t, e, top = c["rows"], c["experts"], c["top_k"]
    # in 64 bits: values next to one another decide which expert is chosen
    l = s["logits"].double()
    l = torch.where(torch.isnan(l), -math.inf, l)
    out = l == -math.inf
    if c["score"] == "sigmoid":
        l = torch.where(out, l, l.clamp(min=-80.0))
        score = 1 / (1 + torch.exp(-l))
    else:
        p = torch.exp(l - torch.where(out.all(1, keepdim=True), 0.0, l.amax(1, keepdim=True)))
        score = p / p.sum(1, keepdim=True)
    score = torch.where(out, 0.0, score)
    value = score if s["bias"] is None else score + s["bias"].double()
    value = torch.where(out, -math.inf, value)
    key = l if s["bias"] is None else value
    if c["groups"] > 1:
        best = torch.sort(value.view(t, c["groups"], -1), dim=2, descending=True)[0][:, :, :2]
        total = torch.where(best == -math.inf, 0.0, best).sum(2)
        total = torch.where(best[:, :, 0] == -math.inf, -math.inf, total)
        first = torch.sort(total, dim=1, descending=True, stable=True)[1][:, :c["top_groups"]]
        stays = torch.zeros_like(total, dtype=torch.bool).scatter_(1, first, True)
        key = torch.where(stays.repeat_interleave(e // c["groups"], 1), key, -math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True)[1][:, :top]
    none = key.gather(1, order) == -math.inf
    weight = torch.where(none, 0.0, score.gather(1, order))
    if c["renorm"]:
        total = weight.sum(1, keepdim=True)
        weight = weight / torch.where(total > 0, total, 1.0)
    expert = torch.where(none, -1, order).to(torch.int32)
    offsets, slots, place = _grouped(expert, e)
    return {"expert": expert, "weight": (weight * c["scale"]).float(), "offsets": offsets, "order": slots,
            "place": place.view(t, top)}


def _plain_gated(s):
    c, parts = s["case"], s["parts"]
    x = _decode(s["codes"], s["scales"])
    h = torch.empty((c["rows"] * c["top_k"], c["f"]), device="cuda")
    for e in range(c["experts"]):
        a, b = parts[e], parts[e + 1]
        if a == b:
            continue
        mine = x[(s["order"][a:b] // c["top_k"]).long()]
        g = mine @ _decode_weight(s["w"][0][e], s["w"][1][e]).t()
        u = mine @ _decode_weight(s["w_up"][0][e], s["w_up"][1][e]).t()
        h[a:b] = g / (1 + torch.exp(-g)) * u
    return _as_values(*_encode(h))


def _plain_linear(s):
    c, parts = s["case"], s["parts"]
    y = torch.empty((c["rows"] * c["top_k"], c["n"]), dtype=torch.float32 if c["out"] == "f32" else torch.bfloat16,
                    device="cuda")
    for e in range(c["experts"]):
        a, b = parts[e], parts[e + 1]
        if a < b:
            y[a:b] = _decode(s["codes"][a:b], s["scales"][a:b]) @ _decode_weight(s["w"][0][e], s["w"][1][e]).t()
    return {"y": y}


def _plain_combine(s):
    c = s["case"]
    total = s["add"].float() if c["add"] else torch.zeros((c["rows"], c["n"]), device="cuda")
    for j in range(c["top_k"]):
        at = s["place"][:, j]
        w = torch.where(at < 0, 0.0, s["weight"][:, j])
        total = total + w[:, None] * s["y"][at.clamp(min=0).long()].float()
    return {"out": total.bfloat16()}


# -------------------------------------------------------------------------------------------
# the framework's calls
# -------------------------------------------------------------------------------------------
def _own_route(s):
    ham, c = s["ham"], s["case"]
    t, top = c["rows"], c["top_k"]
    expert = torch.empty((t, top), dtype=torch.int32, device="cuda")
    weight = torch.empty((t, top), dtype=torch.float32, device="cuda")
    offsets = torch.empty((c["experts"] + 1,), dtype=torch.int32, device="cuda")
    order = torch.empty((t * top,), dtype=torch.int32, device="cuda")
    place = torch.empty((t, top), dtype=torch.int32, device="cuda")
    ham.ham_route(s["logits"], expert, weight, offsets, order, place, bias=s["bias"],
                  score=ham.HAM_SCORE_SIGMOID if c["score"] == "sigmoid" else ham.HAM_SCORE_SOFTMAX,
                  groups=c["groups"], top_groups=c["top_groups"], renorm=c["renorm"], scale=c["scale"])
    return {"expert": expert, "weight": weight, "offsets": offsets, "order": order, "place": place}


def _own_gated(s):
    ham, c = s["ham"], s["case"]
    slots = c["rows"] * c["top_k"]
    h = torch.empty((slots, c["f"]), dtype=torch.uint8, device="cuda")
    hs = torch.empty((slots, _scale_bytes(c["f"])), dtype=torch.uint8, device="cuda")
    ham.ham_fp8_experts_gated(s["handle"], s["codes"].view(torch.uint8), s["scales"], s["offsets"], s["order"],
                              c["top_k"], h, hs)
    return _as_values(h, hs)


def _own_linear(s):
    ham, c = s["ham"], s["case"]
    y = torch.empty((c["rows"] * c["top_k"], c["n"]), dtype=torch.float32 if c["out"] == "f32" else torch.bfloat16,
                    device="cuda")
    ham.ham_fp8_experts_linear(s["handle"], s["codes"].view(torch.uint8), s["scales"], s["offsets"], y)
    return {"y": y}


def _own_combine(s):
    ham, c = s["ham"], s["case"]
    out = torch.empty((c["rows"], c["n"]), dtype=torch.bfloat16, device="cuda")
    ham.ham_experts_combine(s["y"], s["weight"], s["place"], out, add=s["add"])
    return {"out": out}


def run(state):
    plain = {"route": _plain_route, "gated": _plain_gated, "linear": _plain_linear, "combine": _plain_combine}
    kernels = {"route": _own_route, "gated": _own_gated, "linear": _own_linear, "combine": _own_combine}
    return (kernels if own else plain)[state["case"]["kind"]](state)


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


def _exact_weights(c, s):
    """Each row's weights, row by row in fp64, in the order of their experts' values."""
    logits = s["logits"].double().cpu().numpy()
    bias = np.zeros(c["experts"]) if s["bias"] is None else s["bias"].double().cpu().numpy()
    weight = np.zeros((c["rows"], c["top_k"]))
    each = c["experts"] // c["groups"]
    for r, l in enumerate(logits):
        live = np.flatnonzero(l > -np.inf)
        if not len(live):
            continue
        score = np.zeros(c["experts"])
        if c["score"] == "sigmoid":
            score[live] = 1 / (1 + np.exp(-np.maximum(l[live], -80)))
        else:
            score[live] = np.exp(l[live] - l[live].max())
            score /= score.sum()
        value = score + bias
        if c["groups"] > 1:
            total = []
            for g in range(c["groups"]):
                mine = np.sort(value[live[live // each == g]])[::-1]
                total.append(mine[:2].sum() if len(mine) else -np.inf)
            first = np.lexsort((np.arange(c["groups"]), -np.array(total)))[:c["top_groups"]]
            live = live[np.isin(live // each, first)]
        by = value if s["bias"] is not None else l
        chosen = live[np.lexsort((live, -by[live]))][:c["top_k"]]
        w = score[chosen]
        if c["renorm"] and len(chosen):
            w = w / w.sum()
        weight[r, :len(chosen)] = c["scale"] * w
    return torch.from_numpy(weight)


def exact(case, seed):
    c = case
    if 2.0 * c["rows"] * c["top_k"] * c.get("k", 0) * (c.get("n") or 2 * c.get("f", 0)) > 4e12:
        return None
    s = _inputs(case, seed)
    if c["kind"] == "route":
        return {"expert": None, "weight": _exact_weights(c, s), "offsets": None, "order": None, "place": None}
    if c["kind"] == "combine":
        live = (s["place"] >= 0).double()
        rows = s["y"].double()[s["place"].clamp(min=0).long()]
        out = torch.einsum("tj,tjn->tn", s["weight"].double() * live, rows)
        return {"out": out + s["add"].double() if c["add"] else out}
    at = s["offsets"].tolist()
    n = c["f"] if c["kind"] == "gated" else c["n"]
    y = torch.zeros((c["rows"] * c["top_k"], n), dtype=torch.float64, device="cuda")
    x = _exact_operand(s["codes"], s["scales"], 1)
    for e in range(c["experts"]):
        a, b = at[e], at[e + 1]
        if a == b:
            continue
        if c["kind"] == "linear":
            y[a:b] = x[a:b] @ _exact_operand(s["w"][0][e], s["w"][1][e], BLOCK).T
            continue
        mine = x[s["order"][a:b].long() // c["top_k"]]
        g = mine @ _exact_operand(s["w"][0][e], s["w"][1][e], BLOCK).T
        y[a:b] = g / (1 + torch.exp(-g)) * (mine @ _exact_operand(s["w_up"][0][e], s["w_up"][1][e], BLOCK).T)
    return _exact_rows(y) if c["kind"] == "gated" else {"y": y}

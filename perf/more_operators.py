"""The operators around a mixture-of-experts layer that answers, as timed cases: the router's choice and its gradient,
matrices held in 4 bits, products with them for few rows, and a whole layer for a few tokens.

  kind "route"             the `slots` largest of a token's scores, largest first (ties: lowest expert), and their weights:
                           the softmax over those scores, or with "over_all" their part of the softmax over all.  A score of
                           minus infinity, or NaN, bars the expert; a slot for which none is left holds -1 and the weight 0
  kind "route_backward"    the gradient of the weights, brought back to all scores
  kind "hold"              a matrix brought into 4 bits and read back: codes of 2 exponent bits and 1 mantissa bit
                           (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) and a power of two for every 32 neighbours
  kind "product"           out[r, j] = sum over i of x[r, i] * w[j, i], w held in 4 bits, few rows
  kind "few"               y[t] = sum over s of weight[t, s] * w_out[e] (silu(g) * u), (g, u) the halves of w_in[e] x[t],
                           e = expert[t, s]; matrices in the type of x, or held in 4 bits

Values are what such layers see: normal activations with some large channels, matrices scaled by their width,
experts of uneven popularity, softmax weights.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_GROUP = 32                      # neighbours that share a scale
_LOWEST, _HIGHEST = -125, 125    # exponents a scale may have
_LARGEST_HELD = 1 << 27          # elements of a matrix that is brought into 4 bits
_LARGEST_FEW = 128 * 3 * 2048 * 1024 * 2    # bytes of the matrices that a few tokens meet


def _case(name, kind, **more):
    return {"name": name, "kind": kind, **more}


def listed():
    return [
        # the router of one decoding step of a few dozen requests
        _case("route_33x4_of_64_bf16", "route", tokens=33, slots=4, experts=64, over_all=False, barred=0.0, type="bf16"),
        # a training batch
        _case("route_65536x8_of_128_f32", "route", tokens=65536, slots=8, experts=128, over_all=False, barred=0.02, type="f32"),
        # its backward pass where weights are parts of a softmax over all experts, an odd number of them
        _case("route_backward_16384x6_of_101_f32", "route_backward", tokens=16384, slots=6, experts=101, over_all=True, barred=0.02, type="f32"),
        # one matrix of odd sizes in single precision
        _case("hold_1001x515_f32", "hold", rows=1001, width=515, type="f32"),
        # all first matrices of a layer of 32 experts, once when a model is loaded
        _case("hold_65536x2048_bf16", "hold", rows=65536, width=2048, type="bf16"),
        # one token through one matrix
        _case("product_1_2048x2048_bf16", "product", rows=1, k=2048, n=2048, type="bf16"),
        # a short prompt, odd sizes
        _case("product_37_1336x1003_f16", "product", rows=37, k=1336, n=1003, type="f16"),
        # a decoding step of some requests through a wide matrix
        _case("product_16_4096x32768_bf16", "product", rows=16, k=4096, n=32768, type="bf16"),
        # one token through a layer
        _case("few_1x4_of_32_2048x1024_bf16", "few", tokens=1, slots=4, experts=32, drop=0.0, width=2048, hidden=1024, type="bf16", bits=16),
        # some requests, odd sizes, slots that go nowhere
        _case("few_21x2_of_8_1001x515_f16", "few", tokens=21, slots=2, experts=8, drop=0.1, width=1001, hidden=515, type="f16", bits=16),
        # some requests through matrices in 4 bits
        _case("few_8x4_of_64_2048x1024_held4", "few", tokens=8, slots=4, experts=64, drop=0.0, width=2048, hidden=1024, type="bf16", bits=4),
        # the most tokens that still count as a few: every expert is met
        _case("few_64x8_of_128_2048x1024_bf16", "few", tokens=64, slots=8, experts=128, drop=0.0, width=2048, hidden=1024, type="bf16", bits=16),
    ]


def _spread(rng, low, high):
    """A whole number from low to high, spread over its logarithm: a power of two, a multiple of 8 or neither."""
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    form = rng.choice(["power", "eights", "any"])
    if form == "power":
        v = 2 ** round(math.log2(v))
    elif form == "eights" and v >= 8:
        v = int(v) // 64 * 64 + 8 * rng.randint(1, 7)
    else:
        v = int(v) + (int(v) % 64 == 0)
    return v if low <= v <= high else low if v < low else high


def draw(rng):
    kind = rng.choice(["route", "route_backward", "hold", "product", "product", "few", "few", "few"])
    case = {"kind": kind, "type": rng.choice(["bf16", "bf16", "f16", "f32"])}
    if kind == "hold":
        width = _spread(rng, 32, 8192)
        return {**case, "width": width, "rows": _spread(rng, 1, _LARGEST_HELD // width // (2 if case["type"] == "f32" else 1))}
    if kind == "product":
        return {**case, "rows": _spread(rng, 1, 64) if rng.random() < 0.7 else 1, "k": _spread(rng, 64, 8192), "n": _spread(rng, 64, 16384)}
    experts = _spread(rng, 2, 128)
    slots = rng.randint(1, min(8, experts))
    case.update(slots=slots, experts=experts)
    if kind != "few":
        return {**case, "tokens": _spread(rng, 1, min(131072, (65536 * 128) // experts)), "over_all": rng.random() < 0.5, "barred": rng.choice([0.0, 0.0, 0.02, 0.5])}
    width, hidden, bits = _spread(rng, 64, 4096), _spread(rng, 64, 4096), rng.choice([4, 8 * _BYTES[case["type"]]])
    experts = case["experts"] = max(slots, min(experts, _LARGEST_FEW // (3 * width * hidden * (4 if bits == 32 else 2))))
    return {**case, "tokens": _spread(rng, 1, 64) if rng.random() < 0.7 else 1, "drop": rng.choice([0.0, 0.0, 0.1]), "width": width, "hidden": hidden, "bits": bits}


def _held_bytes(rows, width):
    return rows * -(-width // _GROUP) * (_GROUP // 2 + 1)


def work(case):
    kind, b = case["kind"], _BYTES[case["type"]]
    if kind == "hold":
        rows, width = case["rows"], case["width"]
        return {"bytes": 2 * rows * width * b + _held_bytes(rows, width), "flops": 0}
    if kind == "product":
        rows, k, n = case["rows"], case["k"], case["n"]
        return {"bytes": _held_bytes(n, k) + rows * (k + n) * b, "flops": 2 * rows * k * n}
    tokens, slots, experts = case["tokens"], case["slots"], case["experts"]
    count = tokens * slots
    if kind == "route":
        return {"bytes": tokens * experts * b + 8 * count, "flops": tokens * experts}
    if kind == "route_backward":
        return {"bytes": tokens * experts * b * (2 if case["over_all"] else 1) + 12 * count, "flops": tokens * experts}
    width, hidden = case["width"], case["hidden"]
    used = count * (1 - case["drop"])
    met = experts * (1 - (1 - 1 / experts) ** used)
    matrix = _held_bytes(2 * hidden, width) + _held_bytes(width, hidden) if case["bits"] == 4 else 3 * hidden * width * b
    return {"bytes": met * matrix + 2 * tokens * width * b + 8 * count, "flops": 6 * used * width * hidden}


# --- inputs ---

def _activations(g, rows, width, dtype):
    x = torch.randn(rows, width, generator=g, device="cuda")
    loud = torch.rand(width, generator=g, device="cuda") < 0.01
    return (x * torch.where(loud, 20.0, 1.0)).to(dtype)


def _matrices(g, count, rows, width, dtype):
    w = torch.empty(count, rows, width, dtype=dtype, device="cuda")
    for part in w:
        part.copy_(torch.randn(rows, width, generator=g, device="cuda") / math.sqrt(width))
    return w


def _scores(g, case):
    """Scores of experts of uneven popularity, some of them barred; every fiftieth token has no expert at all where any are."""
    tokens, experts = case["tokens"], case["experts"]
    score = torch.randn(tokens, experts, generator=g, device="cuda") + 0.7 * torch.randn(experts, generator=g, device="cuda")
    barred = torch.rand(tokens, experts, generator=g, device="cuda") < case["barred"]
    if case["barred"]:
        barred[::50] = True
    return torch.where(barred, -math.inf, score).to(_TYPES[case["type"]])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, dtype = case["kind"], _TYPES[case["type"]]
    new = lambda *shape, dtype=dtype: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    u8 = torch.uint8
    s = {"case": case}
    if kind == "hold":
        rows, width = case["rows"], case["width"]
        groups = -(-width // _GROUP)
        s["x"], s["out"] = _matrices(g, 1, rows, width, dtype)[0], new(rows, width)
        s["codes"], s["scales"] = new(rows, groups * _GROUP // 2, dtype=u8), new(rows, groups, dtype=u8)
        return s
    if kind == "product":
        rows, k, n = case["rows"], case["k"], case["n"]
        s["x"], s["out"] = _activations(g, rows, k, dtype), new(rows, n)
        s["codes"], s["scales"] = _hold(_matrices(g, 1, n, k, dtype)[0])
        return s
    tokens, slots, experts = case["tokens"], case["slots"], case["experts"]
    if kind in ("route", "route_backward"):
        s["scores"] = _scores(g, case)
        if kind == "route":
            s["expert"], s["weights"] = new(tokens, slots, dtype=torch.int32), new(tokens, slots, dtype=torch.float32)
        else:
            s["expert"], s["weights"] = _route(s["scores"], slots, case["over_all"])
            s["grad"] = torch.randn(tokens, slots, generator=g, device="cuda")
            s["out"] = new(tokens, experts)
        return s
    width, hidden = case["width"], case["hidden"]
    s["expert"], s["weights"] = _route(_scores(g, {**case, "barred": 0.0}), slots, False)
    gone = torch.rand(tokens, slots, generator=g, device="cuda") < case["drop"]
    s["expert"] = torch.where(gone, -1, s["expert"])
    s["x"], s["out"] = _activations(g, tokens, width, dtype), new(tokens, width)
    s["w_in"], s["w_out"] = _matrices(g, experts, 2 * hidden, width, dtype), _matrices(g, experts, width, hidden, dtype)
    s["in_scales"] = s["out_scales"] = None
    if case["bits"] == 4:
        for w, scales in (("w_in", "in_scales"), ("w_out", "out_scales")):
            held = [_hold(m) for m in s[w]]
            s[w], s[scales] = torch.stack([c for c, _ in held]), torch.stack([c for _, c in held])
    if own:
        from paper_1705_01598_amd import binding as B
        s["workspace"] = new(B.expert_few_workspace_bytes(tokens, slots, experts, width, hidden, B.TYPES[case["type"]], case["bits"] == 4), dtype=u8)
    return s


# --- the operators in elementary steps ---

def _route(scores, slots, over_all):
    v = scores.float()
    v = torch.where(v.isnan(), -math.inf, v)
    top, at = torch.sort(v, dim=1, descending=True, stable=True)
    top, at = top[:, :slots], at[:, :slots]
    most = top[:, :1]
    part = lambda x: torch.where(x == -math.inf, 0.0, torch.where(x == most, 1.0, torch.exp(x - most)))  # noqa: E731
    p = part(top)
    total = part(v).sum(1, keepdim=True) if over_all else p.sum(1, keepdim=True)
    there = top > -math.inf
    return torch.where(there, at, -1).to(torch.int32), torch.where(there, p / total, 0.0)


def _hold(x):
    """x [rows, width] in 4 bits: codes [rows, groups * 16], two in a byte, the first in its low half, and biased exponents
    [rows, groups].  A group's scale is the least power of two 2^s with max |x| <= 6 * 2^s."""
    rows, width = x.shape
    groups = -(-width // _GROUP)
    v = torch.nn.functional.pad(x.float(), (0, groups * _GROUP - width)).reshape(rows, groups, _GROUP)
    most = v.abs().amax(-1)
    part, exponent = torch.frexp(most)          # most = part * 2^exponent, part in [0.5, 1)
    s = (exponent - 3 + (part > 0.75)).clamp(_LOWEST, _HIGHEST)
    s = torch.where(most > 0, s, _LOWEST)
    q = torch.ldexp(v, -s[..., None])
    a = q.abs()
    code = torch.zeros_like(q, dtype=torch.uint8)
    # halfway between two values the one with an even code
    for border, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= border) if up else (a > border)
    code |= torch.signbit(q).to(torch.uint8) << 3
    pairs = code.reshape(rows, groups * _GROUP // 2, 2)
    return pairs[..., 0] | pairs[..., 1] << 4, (s + 127).to(torch.uint8)


def _held(codes, scales, width):
    """The values that codes and scales stand for, in 32 bits."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).reshape(codes.shape[0], -1)
    e, m = ((c >> 1) & 3).float(), (c & 1).float()
    size = torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * torch.exp2(e - 1))
    size = torch.where(c >= 8, -size, size)
    s = torch.exp2(scales.float() - 127)
    return (size * s.repeat_interleave(_GROUP, dim=1))[:, :width]


def _plain(s):
    case = s["case"]
    kind, dtype = case["kind"], _TYPES[case["type"]]
    if kind == "route":
        return _route(s["scores"], case["slots"], case["over_all"])
    if kind == "route_backward":
        w, there = s["weights"], s["expert"] >= 0
        at = torch.where(there, s["expert"], 0).long()
        each = torch.where(there, w * s["grad"], 0.0)
        mean = each.sum(1, keepdim=True)
        out = torch.zeros(s["scores"].shape, device="cuda")
        if not case["over_all"]:
            return out.scatter_add(1, at, each - torch.where(there, w, 0.0) * mean).to(dtype)
        v = s["scores"].float()
        v = torch.where(v.isnan(), -math.inf, v)
        most = v.amax(1, keepdim=True)
        p = torch.where(v == -math.inf, 0.0, torch.where(v == most, 1.0, torch.exp(v - most)))
        p = p / p.sum(1, keepdim=True).clamp_min(1.0)
        return (out.scatter_add(1, at, each) - p * mean).to(dtype)
    if kind == "hold":
        codes, scales = _hold(s["x"])
        return _held(codes, scales, case["width"]).to(dtype), scales.view(torch.float8_e8m0fnu)
    if kind == "product":
        return (s["x"].float() @ _held(s["codes"], s["scales"], case["k"]).t()).to(dtype)
    x, hidden = s["x"].float(), case["hidden"]
    y = torch.zeros_like(x)
    for e in s["expert"].unique().tolist():
        if e < 0:
            continue
        token, slot = (s["expert"] == e).nonzero(as_tuple=True)
        if case["bits"] == 4:
            w_in, w_out = _held(s["w_in"][e], s["in_scales"][e], case["width"]), _held(s["w_out"][e], s["out_scales"][e], hidden)
        else:
            w_in, w_out = s["w_in"][e].float(), s["w_out"][e].float()
        g, u = (x[token] @ w_in.t()).split(hidden, dim=1)
        y[token] += s["weights"][token, slot, None] * ((g / (1 + torch.exp(-g)) * u) @ w_out.t())
    return y.to(dtype)


# --- the same through the library ---

def _library(s):
    from paper_1705_01598_amd import binding as B
    case = s["case"]
    kind, t = case["kind"], B.TYPES[case["type"]]
    stream = torch.cuda.current_stream().cuda_stream
    at = lambda name: None if s[name] is None else s[name].data_ptr()  # noqa: E731
    if kind == "hold":
        rows, width = case["rows"], case["width"]
        B.tperm_four_bit_store(at("x"), width, at("codes"), at("scales"), rows, width, t, stream)
        B.tperm_four_bit_load(at("codes"), at("scales"), at("out"), width, rows, width, t, stream)
        return s["out"], s["scales"].view(torch.float8_e8m0fnu)
    if kind == "product":
        k, n = case["k"], case["n"]
        B.tperm_four_bit_product(at("x"), k, at("codes"), at("scales"), at("out"), n, case["rows"], k, n, t, stream)
        return s["out"]
    tokens, slots, experts = case["tokens"], case["slots"], case["experts"]
    if kind == "route":
        B.tperm_expert_route(at("scores"), experts, at("expert"), at("weights"), tokens, slots, experts, case["over_all"], t, stream)
        return s["expert"], s["weights"]
    if kind == "route_backward":
        B.tperm_expert_route_backward(at("grad"), at("scores"), experts, at("expert"), at("weights"), at("out"), experts, tokens, slots, experts,
                                      case["over_all"], t, stream)
        return s["out"]
    width, hidden = case["width"], case["hidden"]
    B.tperm_expert_few(at("x"), width, at("expert"), at("weights"), at("w_in"), at("in_scales"), at("w_out"), at("out_scales"), at("out"), width,
                       at("workspace"), s["workspace"].numel(), tokens, slots, experts, width, hidden, t, stream)
    return s["out"]


def run(s):
    return _library(s) if own else _plain(s)


# --- from the definitions, in 64 bits ---

_CODES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _values_64(codes, scales, width):
    """Every code by its table of 16 numbers."""
    table = torch.tensor(_CODES + [-c for c in _CODES], dtype=torch.float64, device=codes.device)
    column = torch.arange(width, device=codes.device)
    byte = codes[:, column // 2].to(torch.int64)
    code = torch.where(column % 2 == 0, byte % 16, byte // 16)
    return table[code] * torch.pow(2.0, scales[:, column // _GROUP].double() - 127)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "hold":
        # the nearest of the 15 values to each, by its distance to all of them; at equal distance that of the even code
        x, width = s["x"].double(), case["width"]
        values = torch.tensor(_CODES, dtype=torch.float64, device="cuda")
        out = torch.empty_like(x)
        scales = torch.empty(x.shape[0], -(-width // _GROUP), dtype=torch.float64, device="cuda")
        for c in range(0, width, _GROUP):
            v = x[:, c:c + _GROUP]
            most = v.abs().amax(1, keepdim=True)
            e = torch.ceil(torch.log2(most.clamp_min(2.0 ** -149) / 6)).clamp(_LOWEST, _HIGHEST)
            e = torch.where(most > 6 * torch.pow(2.0, e), e + 1, e)
            e = torch.where(most <= 6 * torch.pow(2.0, e - 1), e - 1, e).clamp(_LOWEST, _HIGHEST)
            a = v.abs() / torch.pow(2.0, e)
            best, distance = torch.zeros_like(a), a.clone()
            for i in (2, 4, 6, 1, 3, 5, 7):
                d = (a - values[i]).abs()
                nearer = d < distance
                best, distance = torch.where(nearer, values[i], best), torch.where(nearer, d, distance)
            out[:, c:c + _GROUP] = torch.where(v < 0, -best, best) * torch.pow(2.0, e)
            scales[:, c // _GROUP] = torch.pow(2.0, e[:, 0])
        return out, scales
    if kind == "product":
        return s["x"].double() @ _values_64(s["codes"], s["scales"], case["k"]).t()
    if kind == "route":
        v = s["scores"].double()
        v = torch.where(v.isnan(), -math.inf, v)
        left, slots = v.clone(), case["slots"]
        weights = torch.zeros(v.shape[0], slots, dtype=torch.float64, device="cuda")
        chosen = torch.zeros_like(v, dtype=torch.bool)
        picked = []
        for _ in range(slots):
            at = left.argmax(1, keepdim=True)
            there = left.gather(1, at) > -math.inf
            picked.append((at, there))
            chosen.scatter_(1, at, chosen.gather(1, at) | there)
            left = left.scatter(1, at, -math.inf)
        total = torch.logsumexp(v if case["over_all"] else v.masked_fill(~chosen, -math.inf), 1, keepdim=True)
        for k, (at, there) in enumerate(picked):
            weights[:, k:k + 1] = torch.where(there, torch.exp(v.gather(1, at) - total), 0.0)
        return None, weights
    if kind == "route_backward":
        # from the definition with the scores: the weights that are given are these numbers rounded to 32 bits
        w, d = s["weights"].double(), s["grad"].double()
        mean = (w * d).sum(1)
        v = s["scores"].double()
        v = torch.where(v.isnan(), -math.inf, v)
        out = torch.zeros_like(v)
        if case["over_all"]:
            total = torch.logsumexp(v, 1, keepdim=True)
            out = torch.where(v > -math.inf, torch.exp(v - torch.where(total > -math.inf, total, 0.0)), 0.0) * -mean[:, None]
        for k in range(case["slots"]):
            t = (s["expert"][:, k] >= 0).nonzero()[:, 0]
            step = w[t, k] * d[t, k] if case["over_all"] else w[t, k] * (d[t, k] - mean[t])
            out[t, s["expert"][t, k].long()] += step
        return out
    hidden, width = case["hidden"], case["width"]
    x = s["x"].double()
    out = torch.zeros_like(x)
    expert = s["expert"].tolist()
    matrices = {}
    by_expert = sorted((e, t, k) for t, row in enumerate(expert) for k, e in enumerate(row) if e >= 0)
    for e, t, k in by_expert:
        if e not in matrices:
            matrices = {e: (_values_64(s["w_in"][e], s["in_scales"][e], width), _values_64(s["w_out"][e], s["out_scales"][e], hidden))
                        if case["bits"] == 4 else (s["w_in"][e].double(), s["w_out"][e].double())}
        w_in, w_out = matrices[e]
        both = w_in.mv(x[t])
        h = both[:hidden] * torch.special.expit(both[:hidden]) * both[hidden:]
        out[t] += s["weights"][t, k].double() * w_out.mv(h)
    return out

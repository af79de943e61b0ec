"""The operators of a mixture-of-experts layer, as timed cases: tokens brought into the order of their
experts and back, the experts' products and their gradients, activations kept in 8 bits for the backward pass.

Every token t has ``slots`` experts, expert[t, s]; a number outside 0 .. experts-1 is a slot that goes nowhere.
Assignment a = t * slots + s.  Row r of the sorted order belongs to assignment source[r], place is the inverse
map, offsets[e] is expert e's first row; rows from offsets[experts] on belong to slots that go nowhere.

  kind "sort"              offsets, source, place from the expert numbers (stable)
  kind "gather"            out[r] = weight[source[r]] * x[source[r] // slots]: tokens to their experts
  kind "combine"           out[t] = sum over s of weight[t, s] * rows[place[t, s]]: results back to the tokens
  kind "combine_backward"  the gradients of "combine" to rows and weights
  kind "product"           out[r] = x[source[r] // slots] times the matrix of row r's expert; "transposed" is the
                           product with the matrix's other index summed, which the gradient to x is
  kind "weight_gradient"   out[e][i, j] = sum over the rows r of expert e of x[source[r] // slots, i] * grad[r, j];
                           "held" is the number of bits that x was kept in
  kind "gated"             silu(g) * u of rows [g, u], which are kept in 8 bits: codes of 4 exponent and 3 mantissa bits
                           (finite, largest 448) and a power of two for every 32 neighbours
  kind "gated_backward"    from the gradient of the result and the 8-bit [g, u]: their gradient, and the result again

Values are what such layers see: normal activations with some large channels, matrices scaled by their width,
experts of uneven popularity, softmax weights.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_BLOCK = 32                  # neighbours that share a scale
_LOWEST, _HIGHEST = -117, 120    # exponents a scale may have


def _case(name, kind, **more):
    return {"name": name, "kind": kind, **more}


def listed():
    return [
        # the routing of one decoding step of a few dozen requests
        _case("sort_33x4_of_64", "sort", tokens=33, slots=4, experts=64, drop=0.0),
        # a training batch: half a million assignments, some over capacity
        _case("sort_65536x8_of_128", "sort", tokens=65536, slots=8, experts=128, drop=0.03),
        # a short prompt in single precision, rows of no round length
        _case("gather_1021x2_1000_f32", "gather", tokens=1021, slots=2, experts=16, drop=0.1, width=1000, type="f32", weighted=False),
        # results of a training batch back to its tokens
        _case("combine_8192x8_2048_bf16", "combine", tokens=8192, slots=8, experts=64, drop=0.02, width=2048, type="bf16", weighted=True),
        # the same step's backward pass, smaller batch
        _case("combine_backward_5000x4_1536_bf16", "combine_backward", tokens=5000, slots=4, experts=32, drop=0.02, width=1536, type="bf16", weighted=True),
        # one decoding step: every expert that is met costs its whole matrix
        _case("product_8x4_2048x1024_bf16", "product", tokens=8, slots=4, experts=64, drop=0.0, k=2048, n=1024, type="bf16", transposed=True),
        # prompts or a training batch through a wide layer
        _case("product_16384x4_2048x4096_bf16", "product", tokens=16384, slots=4, experts=32, drop=0.0, k=2048, n=4096, type="bf16", transposed=True),
        # gradient to the input: the same matrices, the other index summed
        _case("product_4001x2_1336x1000_f16", "product", tokens=4001, slots=2, experts=8, drop=0.05, k=1336, n=1000, type="f16", transposed=False),
        # gradient of the matrices from inputs kept in 8 bits
        _case("weight_gradient_8192x4_2048x2048_held8", "weight_gradient", tokens=8192, slots=4, experts=16, drop=0.0, k=2048, n=2048, type="bf16", held=8),
        # the same in single precision, odd sizes, few tokens
        _case("weight_gradient_777x2_515x260_f32", "weight_gradient", tokens=777, slots=2, experts=8, drop=0.1, k=515, n=260, type="f32", held=32),
        # between the two products of a training batch
        _case("gated_32768x2048_bf16", "gated", rows=32768, width=2048, type="bf16"),
        # its backward pass, odd number of rows, rows that end inside a block of 32
        _case("gated_backward_9001x1000_f16", "gated_backward", rows=9001, width=1000, type="f16"),
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
    kind = rng.choice(["sort", "gather", "combine", "combine_backward", "product", "product", "weight_gradient", "weight_gradient", "gated", "gated_backward"])
    kind_type = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("gated", "gated_backward"):
        width = _spread(rng, 32, 4096)
        return {"kind": kind, "rows": _spread(rng, 1, min(65536, (32768 * 2048) // width)), "width": width, "type": kind_type}
    experts = _spread(rng, 2, 128)
    slots = rng.randint(1, min(8, experts))
    case = {"kind": kind, "slots": slots, "experts": experts, "drop": rng.choice([0.0, 0.0, 0.05, 0.3])}
    if kind == "sort":
        return {**case, "tokens": _spread(rng, 1, 524288 // slots)}
    if kind in ("gather", "combine", "combine_backward"):
        width = _spread(rng, 16, 4096)
        return {**case, "tokens": _spread(rng, 1, min(16384, (65536 * 2048) // (slots * width))), "width": width, "type": kind_type,
                "weighted": kind == "combine_backward" or rng.random() < 0.6}
    k, n = _spread(rng, 64, 4096), _spread(rng, 64, 4096)
    experts = case["experts"] = max(slots, min(experts, (1 << 28) // (k * n)))
    most = (1 << 39) // (slots * k * n)
    if kind_type == "f32":
        most //= 8
    case = {**case, "tokens": _spread(rng, 1, max(1, min(16384, most))), "k": k, "n": n, "type": kind_type}
    if kind == "product":
        return {**case, "transposed": rng.random() < 0.5}
    return {**case, "held": rng.choice([8, 8 * _BYTES[kind_type]])}


def _dims(case):
    tokens, slots, experts = case["tokens"], case["slots"], case["experts"]
    return tokens, slots, experts, tokens * slots


def work(case):
    kind = case["kind"]
    if kind in ("gated", "gated_backward"):
        rows, width, b = case["rows"], case["width"], _BYTES[case["type"]]
        held = 2 * rows * (width + -(-width // _BLOCK))
        # gated: reads [g, u], writes the result and what is held; backward: reads the gradient and what is held,
        # writes the gradient of [g, u] and the result
        return {"bytes": 3 * rows * width * b + held if kind == "gated" else 4 * rows * width * b + held, "flops": 8 * rows * width}
    tokens, slots, experts, count = _dims(case)
    if kind == "sort":
        return {"bytes": 4 * (3 * count + experts + 1), "flops": 0}
    rows = count * (1 - case["drop"])
    b = _BYTES[case["type"]]
    maps, weights = 4 * (count + experts + 1), 4 * count
    if kind in ("gather", "combine"):
        moved = (tokens + (count if kind == "gather" else rows)) * case["width"] * b
        return {"bytes": moved + maps + (weights if case["weighted"] else 0), "flops": 2 * rows * case["width"]}
    if kind == "combine_backward":
        return {"bytes": (tokens + rows + count) * case["width"] * b + maps + 2 * weights, "flops": 3 * rows * case["width"]}
    k, n = case["k"], case["n"]
    flops = 2 * rows * k * n
    if kind == "product":
        met = experts * (1 - (1 - 1 / experts) ** rows)
        return {"bytes": b * (tokens * k + met * k * n + count * n) + maps, "flops": flops}
    x = tokens * (k + -(-k // _BLOCK)) if case["held"] == 8 else tokens * k * b
    return {"bytes": x + rows * n * b + experts * k * n * 4 + maps, "flops": flops}


# --- inputs ---

def _activations(g, rows, width, dtype):
    x = torch.randn(rows, width, generator=g, device="cuda")
    loud = torch.rand(width, generator=g, device="cuda") < 0.01
    return (x * torch.where(loud, 20.0, 1.0)).to(dtype)


def _routing(g, case):
    """Expert numbers of uneven popularity, different ones for one token, and softmax weights."""
    tokens, slots, experts, _ = _dims(case)
    score = torch.randn(tokens, experts, generator=g, device="cuda") + 0.7 * torch.randn(experts, generator=g, device="cuda")
    top, at = score.topk(slots, dim=1)
    gone = torch.rand(tokens, slots, generator=g, device="cuda") < case["drop"]
    return torch.where(gone, -1, at).to(torch.int32), torch.softmax(top, dim=1)


def _order(expert, experts):
    """offsets, source, place in elementary steps."""
    e = expert.reshape(-1).to(torch.int64)
    e = torch.where((e >= 0) & (e < experts), e, experts)
    source = torch.argsort(e, stable=True)
    place = torch.empty_like(source)
    place[source] = torch.arange(source.numel(), device=e.device)
    offsets = torch.searchsorted(e[source], torch.arange(experts + 1, device=e.device))
    return offsets.to(torch.int32), source.to(torch.int32), place.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    new = lambda *shape, dtype: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    s = {"case": case}
    if kind in ("gated", "gated_backward"):
        rows, width, dtype = case["rows"], case["width"], _TYPES[case["type"]]
        gates = _activations(g, rows, 2 * width, dtype)
        blocks = 2 * -(-width // _BLOCK)
        s["result"] = new(rows, width, dtype=dtype)
        if kind == "gated":
            s["gates"] = gates
            s["codes"], s["scales"] = new(rows, 2 * width, dtype=torch.uint8), new(rows, blocks, dtype=torch.uint8)
        else:
            s["grad"] = torch.randn(rows, width, generator=g, device="cuda").to(dtype)
            s["codes"], s["scales"] = _keep(gates.reshape(rows, 2, width))
            s["grad_gates"] = new(rows, 2 * width, dtype=dtype)
        return s
    tokens, slots, experts, count = _dims(case)
    expert, weights = _routing(g, case)
    if kind == "sort":
        s["expert"] = expert
        s["offsets"], s["source"], s["place"] = new(experts + 1, dtype=torch.int32), new(count, dtype=torch.int32), new(tokens, slots, dtype=torch.int32)
        s["workspace"] = new(1 << 20, dtype=torch.uint8)
        return s
    s["offsets"], s["source"], s["place"] = _order(expert, experts)
    dtype = _TYPES[case["type"]]
    if kind in ("gather", "combine", "combine_backward"):
        width = case["width"]
        s["weights"] = weights.contiguous() if case["weighted"] else None
        if kind != "combine":
            s["tokens"] = _activations(g, tokens, width, dtype)
        if kind != "gather":
            # what lies behind the last expert's rows is whatever the buffer held: here infinities
            there = torch.arange(count, device="cuda")[:, None] < s["offsets"][-1]
            s["rows"] = torch.where(there, _activations(g, count, width, dtype), math.inf)
        s["out"] = new(tokens if kind == "combine" else count, width, dtype=dtype)
        if kind == "combine_backward":
            s["grad_weights"] = new(tokens, slots, dtype=torch.float32)
        return s
    k, n = case["k"], case["n"]
    x = _activations(g, tokens, k, dtype)
    if kind == "product":
        s["x"] = x
        shape = (experts, n, k) if case["transposed"] else (experts, k, n)
        s["w"] = (torch.randn(*shape, generator=g, device="cuda") / math.sqrt(k)).to(dtype)
        s["out"] = new(count, n, dtype=dtype)
        return s
    s["grad"] = torch.randn(count, n, generator=g, device="cuda").to(dtype)
    s["x"], s["scales"] = _keep(x.reshape(tokens, 1, k)) if case["held"] == 8 else (x, None)
    s["out"] = new(experts, k, n, dtype=torch.float32)
    return s


# --- the operators in elementary steps ---

def _keep(x):
    """x [rows, parts, width] in 8 bits: codes [rows, parts * width] and biased exponents [rows, parts * blocks].

    A block's scale is the least power of two 2^s with max |x| <= 448 * 2^s over its finite values."""
    rows, parts, width = x.shape
    blocks = -(-width // _BLOCK)
    v = torch.nn.functional.pad(x.float(), (0, blocks * _BLOCK - width)).reshape(rows, parts, blocks, _BLOCK)
    most = torch.where(v.isfinite(), v.abs(), 0.0).amax(-1)
    part, exponent = torch.frexp(most)          # most = part * 2^exponent, part in [0.5, 1)
    s = (exponent - 9 + (part > 0.875)).clamp(_LOWEST, _HIGHEST)
    s = torch.where(most > 0, s, _LOWEST)
    q = torch.ldexp(v, -s[..., None])
    codes = torch.where(v.isfinite(), q, math.nan).to(torch.float8_e4m3fn).reshape(rows, parts, -1)[..., :width]
    return codes.contiguous().view(torch.uint8).reshape(rows, parts * width), (s + 127).to(torch.uint8).reshape(rows, parts * blocks)


def _kept(codes, scales, parts):
    """The values that codes and scales stand for, in 32 bits: [rows, parts, width]."""
    rows = codes.shape[0]
    q = codes.view(torch.float8_e4m3fn).float().reshape(rows, parts, -1)
    s = torch.exp2(scales.float() - 127).reshape(rows, parts, -1)
    return q * s.repeat_interleave(_BLOCK, dim=2)[..., :q.shape[2]]


def _stands_for(codes, scales):
    """Codes and scales as the numbers that they stand for: the same bytes under their own types."""
    return codes.view(torch.float8_e4m3fn), scales.view(torch.float8_e8m0fnu)


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "gated":
        rows, width = case["rows"], case["width"]
        g, u = s["gates"].float().split(width, dim=1)
        codes, scales = _keep(s["gates"].reshape(rows, 2, width))
        return ((g / (1 + torch.exp(-g))) * u).to(s["gates"].dtype), *_stands_for(codes, scales)
    if kind == "gated_backward":
        g, u = _kept(s["codes"], s["scales"], 2).unbind(1)
        d, dtype = s["grad"].float(), s["grad"].dtype
        sig = 1 / (1 + torch.exp(-g))
        return torch.cat([d * u * sig * (1 + g * (1 - sig)), d * g * sig], dim=1).to(dtype), (g * sig * u).to(dtype)
    if kind == "sort":
        offsets, source, place = _order(s["expert"], case["experts"])
        return offsets, source, place.reshape(s["expert"].shape)
    tokens, slots, experts, count = _dims(case)
    source = s["source"].long()
    there = torch.arange(count, device=source.device) < s["offsets"][-1]       # by row
    if kind == "gather":
        rows = s["tokens"].float()[source // slots]
        if s["weights"] is not None:
            rows = rows * s["weights"].reshape(-1)[source, None]
        return torch.where(there[:, None], rows, 0.0).to(s["out"].dtype)
    if kind in ("combine", "combine_backward"):
        place = s["place"].long().reshape(tokens, slots)
        back = s["rows"].float()[place]                                        # tokens, slots, width
        used = (place < s["offsets"][-1])
        if kind == "combine":
            if s["weights"] is not None:
                back = back * s["weights"][..., None]
            return torch.where(used[..., None], back, 0.0).sum(1).to(s["out"].dtype)
        grad = s["tokens"].float()
        grad_weights = torch.where(used, (back * grad[:, None]).sum(-1), 0.0)
        grad_rows = torch.where(there[:, None], s["weights"].reshape(-1)[source, None] * grad[source // slots], 0.0)
        return grad_rows.to(s["out"].dtype), grad_weights
    sizes = s["offsets"].diff().tolist()        # one matrix product for each expert: its rows have to be known here
    met = sum(sizes)
    token = source[:met] // slots
    if kind == "product":
        dtype = s["x"].dtype
        parts = s["x"].float()[token].split(sizes)
        matrices = (w.float().t() if case["transposed"] else w.float() for w in s["w"])
        out = torch.cat([a @ w for a, w in zip(parts, matrices)])
        return torch.nn.functional.pad(out, (0, 0, 0, count - met)).to(dtype)
    x = _kept(s["x"], s["scales"], 1)[:, 0] if s["scales"] is not None else s["x"].float()
    pairs = zip(x[token].split(sizes), s["grad"][:met].float().split(sizes))
    return torch.stack([a.t() @ d for a, d in pairs])


# --- the same through the library ---

def _library(s):
    from paper_1705_01598_amd import binding as B
    case = s["case"]
    kind = case["kind"]
    stream = torch.cuda.current_stream().cuda_stream
    at = lambda name: None if s[name] is None else s[name].data_ptr()  # noqa: E731
    if kind == "gated":
        rows, width, t = case["rows"], case["width"], B.TYPES[case["type"]]
        B.tperm_gated_forward(at("gates"), 2 * width, at("result"), width, at("codes"), at("scales"), rows, width, t, stream)
        return s["result"], *_stands_for(s["codes"], s["scales"])
    if kind == "gated_backward":
        rows, width, t = case["rows"], case["width"], B.TYPES[case["type"]]
        B.tperm_gated_backward(at("grad"), width, at("codes"), at("scales"), at("grad_gates"), 2 * width, at("result"), width, rows, width, t, stream)
        return s["grad_gates"], s["result"]
    tokens, slots, experts, count = _dims(case)
    if kind == "sort":
        B.tperm_expert_sort(at("expert"), tokens, slots, experts, at("offsets"), at("source"), at("place"), at("workspace"),
                            s["workspace"].numel(), stream)
        return s["offsets"], s["source"], s["place"]
    t = B.TYPES[case["type"]]
    if kind in ("gather", "combine", "combine_backward"):
        width = case["width"]
        if kind == "gather":
            B.tperm_expert_gather(at("tokens"), width, at("source"), at("offsets"), at("weights"), at("out"), width,
                                  tokens, slots, experts, width, t, stream)
            return s["out"]
        if kind == "combine":
            B.tperm_expert_combine(at("rows"), width, at("place"), at("offsets"), at("weights"), at("out"), width,
                                   tokens, slots, experts, width, t, stream)
            return s["out"]
        B.tperm_expert_combine_backward(at("tokens"), width, at("rows"), width, at("place"), at("offsets"), at("weights"), at("out"), width,
                                        at("grad_weights"), tokens, slots, experts, width, t, stream)
        return s["out"], s["grad_weights"]
    k, n = case["k"], case["n"]
    if kind == "product":
        B.tperm_expert_product(at("x"), k, tokens, at("source"), slots, at("offsets"), at("w"), case["transposed"], at("out"), n,
                               count, experts, k, n, t, stream)
        return s["out"]
    B.tperm_expert_weight_gradient(at("x"), k, at("scales"), tokens, at("source"), slots, at("grad"), n, at("offsets"), at("out"), B.TYPES["f32"],
                                   False, False, count, experts, k, n, t, stream)
    return s["out"]


def run(s):
    return _library(s) if own else _plain(s)


# --- from the definitions, in 64 bits ---

def _held_64(codes, scales, parts):
    """Every code from its bits: sign, 4 exponent bits of bias 7, 3 mantissa bits."""
    c = codes.to(torch.int64)
    e, m = (c >> 3) & 15, (c & 7).double()
    size = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.pow(2.0, (e - 10).double()))
    size = torch.where((c & 127) == 127, math.nan, size) * torch.where(c >= 128, -1.0, 1.0)
    width, blocks = codes.shape[1] // parts, scales.shape[1] // parts
    column = torch.arange(codes.shape[1], device=codes.device)
    block = column // width * blocks + column % width // _BLOCK
    return size * torch.pow(2.0, scales.double() - 127)[:, block]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "gated":
        # the codes are the nearest to the values by the definition of the type, and nothing nearer in 64 bits
        width = case["width"]
        g, u = s["gates"][:, :width].double(), s["gates"][:, width:].double()
        return g * torch.special.expit(g) * u, None, None
    if kind == "gated_backward":
        v, width, d = _held_64(s["codes"], s["scales"], 2), case["width"], s["grad"].double()
        g, u, p = v[:, :width], v[:, width:], torch.special.expit(v[:, :width])
        grad = torch.empty_like(v)
        grad[:, :width] = (p + g * p * torch.special.expit(-g)) * u * d
        grad[:, width:] = p * g * d
        return grad, p * g * u
    tokens, slots, experts, count = _dims(case)
    if kind == "sort":
        return None
    offsets = s["offsets"].tolist()
    assigned = torch.full((count,), -1, dtype=torch.int64, device="cuda")       # expert of each assignment
    rows_of = [s["source"][a:b].long() for a, b in zip(offsets, offsets[1:])]   # assignments of each expert, in row order
    for e, a in enumerate(rows_of):
        assigned[a] = e
    if kind == "gather":
        x = s["tokens"].double()
        out = torch.zeros(count, case["width"], dtype=torch.float64, device="cuda")
        for e, a in enumerate(rows_of):
            w = torch.ones_like(a, dtype=torch.float64) if s["weights"] is None else s["weights"].reshape(-1)[a].double()
            out[offsets[e]:offsets[e + 1]] = w[:, None] * x[torch.div(a, slots, rounding_mode="floor")]
        return out
    if kind in ("combine", "combine_backward"):
        place = s["place"].reshape(-1).long()
        w = torch.ones(count, dtype=torch.float64, device="cuda") if s["weights"] is None else s["weights"].reshape(-1).double()
        out = torch.zeros(tokens if kind == "combine" else count, case["width"], dtype=torch.float64, device="cuda")
        grad_w = torch.zeros(count, dtype=torch.float64, device="cuda")
        for slot in range(slots):
            a = torch.arange(slot, count, slots, device="cuda")
            a = a[assigned[a] >= 0]
            token, row = a // slots, place[a]
            if kind == "combine":
                out[token] += w[a, None] * s["rows"][row].double()
            else:
                d = s["tokens"][token].double()
                out[row] = w[a, None] * d
                grad_w[a] = (d * s["rows"][row].double()).sum(1)
        return out if kind == "combine" else (out, grad_w.reshape(tokens, slots))
    k, n = case["k"], case["n"]
    if kind == "product":
        out = torch.zeros(count, n, dtype=torch.float64, device="cuda")
        for e, a in enumerate(rows_of):
            w = s["w"][e].double()
            out[offsets[e]:offsets[e + 1]] = s["x"][a // slots].double().matmul(w.t() if case["transposed"] else w)
        return out
    out = torch.zeros(experts, k, n, dtype=torch.float64, device="cuda")
    for e, a in enumerate(rows_of):
        x = s["x"][a // slots]
        x = _held_64(x, s["scales"][a // slots], 1) if s["scales"] is not None else x.double()
        out[e] = x.t().matmul(s["grad"][offsets[e]:offsets[e + 1]].double())
    return out

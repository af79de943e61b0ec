"""Router, matrices in 4 bits, products with them and the layer for a few tokens on the GPU, against plain
implementations in 64 bits.

Tolerances, fixed before the first run, elementwise: `rounding` for the rounding to the element type, and for a sum of n
products in binary32 n * 2^-23 times the sum of their magnitudes, as in test_gpu_experts.

Softmax: exp is right to 2^-23 of itself and its argument v - max, rounded to 24 bits, adds |v - max| * 2^-24; a sum of n
positive terms adds n * 2^-24, the division 2^-24.  So a weight is within (4 + |v - max| + n) * 2^-23 of itself.

Layer: a hidden row is held in 16 bits at least (two bfloat16 parts, each rounding to 2^-9 of what is left: 2^-17 with room
to spare), in binary16 to 2^-22 or 2^-25, in binary32 as it is.  The activation's slope is at most 1.1 in g."""
import math

import pytest

from paper_1705_01598_amd import binding as B

torch = pytest.importorskip("torch")
from test_gpu_experts import SUM, TYPES, Matrix, near, rounding, stream  # noqa: E402

pytestmark = pytest.mark.gpu

VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def generator(seed):
    return torch.Generator().manual_seed(seed)


# --- the router ---

def plain_route(scores, slots, over_all):
    """expert, weights and their tolerance, row by row; scores are doubles."""
    tokens, experts = scores.shape
    v = torch.where(scores.isnan(), -math.inf, scores)
    at = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :slots]
    expert = torch.full((tokens, slots), -1, dtype=torch.int32)
    weights, off = torch.zeros(tokens, slots, dtype=torch.float64), torch.zeros(tokens, slots, dtype=torch.float64)
    p = torch.zeros(tokens, experts, dtype=torch.float64)
    for t in range(tokens):
        chosen = [int(e) for e in at[t] if v[t, e] > -math.inf]
        if not chosen:
            continue
        most = v[t, chosen[0]]
        part = torch.where(v[t] == most, 1.0, torch.exp(v[t] - most)) if math.isfinite(most) else (v[t] == most).double()
        p[t] = part / part.sum()
        total = part.sum() if over_all else part[chosen].sum()
        for s, e in enumerate(chosen):
            far = float(most - v[t, e]) if math.isfinite(most) and part[e] > 0 else 0.0
            expert[t, s], weights[t, s] = e, part[e] / total
            off[t, s] = (4 + far + experts) * SUM * weights[t, s] + 2.0 ** -126
    return expert, weights, off, p


def scores_of(kind, tokens, experts, g):
    v = torch.randn(tokens, experts, generator=g, dtype=torch.float64) * 3
    if kind == "ties":
        v = v.round()
    elif kind == "barred":
        v[torch.rand(v.shape, generator=g) < 0.6] = -math.inf
        v[torch.rand(v.shape, generator=g) < 0.1] = math.nan
        v[::5] = -math.inf
    elif kind == "wide":
        v *= 40
    elif kind == "odd":
        v[torch.rand(v.shape, generator=g) < 0.2] = math.inf
        v[torch.rand(v.shape, generator=g) < 0.3] = 0.0
        v[torch.rand(v.shape, generator=g) < 0.3] *= 0.0        # zeros of both signs are equal
        v[::3] = torch.finfo(torch.float32).min
    return v


ROUTES = [(1, 1, 1), (1, 1, 3), (7, 5, 2), (33, 16, 4), (70, 17, 17), (19, 32, 8), (40, 33, 5), (9, 64, 64), (21, 100, 6), (130, 128, 8), (5, 129, 8),
          (6, 256, 16), (3, 257, 20), (4, 1000, 64), (2, 1024, 10), (3, 5, 40)]


@pytest.mark.parametrize("over_all", [False, True])
@pytest.mark.parametrize("kind", ["plain", "ties", "barred", "wide", "odd"])
@pytest.mark.parametrize("t", list(TYPES))
def test_route(t, kind, over_all):
    g = generator(11)
    for i, (tokens, experts, slots) in enumerate(ROUTES):
        m = Matrix(tokens, experts, TYPES[t], scores_of(kind, tokens, experts, g).float(), pad=i % 3, offset=i % 5)
        expert, weights = Matrix(tokens, slots, torch.int32), Matrix(tokens, slots, torch.float32)
        B.tperm_expert_route(m.ptr, m.stride, expert.ptr, weights.ptr, tokens, slots, experts, over_all, B.TYPES[t], stream())
        torch.cuda.synchronize()
        want, w, off, _ = plain_route(m.values(), slots, over_all)
        assert torch.equal(expert.view().cpu(), want), (tokens, experts, slots)
        near(weights.view(), w, off)
        assert expert.outside_untouched() and weights.outside_untouched()


@pytest.mark.parametrize("over_all", [False, True])
@pytest.mark.parametrize("tokens,experts,slots", [(8192, 32, 4), (8200, 30, 3), (9001, 64, 8), (8192, 61, 7), (10007, 128, 8), (8192, 101, 6), (8195, 200, 5)])
@pytest.mark.parametrize("t", list(TYPES))
def test_route_of_many_tokens(t, tokens, experts, slots, over_all):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    v = torch.randn(tokens, experts, generator=g, device="cuda") * 3
    v[torch.rand(v.shape, generator=g, device="cuda") < 0.2] = -math.inf
    v[::100] = -math.inf
    v[1::100] = v[1::100].round()
    scores = v.to(TYPES[t])
    expert, weights = torch.empty(tokens, slots, dtype=torch.int32, device="cuda"), torch.empty(tokens, slots, device="cuda")
    B.tperm_expert_route(scores.data_ptr(), experts, expert.data_ptr(), weights.data_ptr(), tokens, slots, experts, over_all, B.TYPES[t], stream())
    v = scores.double()
    top, at = torch.sort(v, dim=1, descending=True, stable=True)
    top, at = top[:, :slots], at[:, :slots]
    there = top > -math.inf
    assert torch.equal(expert, torch.where(there, at, -1).to(torch.int32))
    total = torch.logsumexp(v if over_all else top, 1, keepdim=True)
    want = torch.where(there, torch.exp(top - total), 0.0)
    far = torch.where(there, top[:, :1] - top, 0.0)
    near(weights, want.cpu(), ((4 + far + experts) * SUM * want).cpu())


@pytest.mark.parametrize("over_all", [False, True])
@pytest.mark.parametrize("kind", ["plain", "barred", "wide"])
@pytest.mark.parametrize("t", list(TYPES))
def test_route_backward(t, kind, over_all):
    g = generator(12)
    for i, (tokens, experts, slots) in enumerate(ROUTES):
        m = Matrix(tokens, experts, TYPES[t], scores_of(kind, tokens, experts, g).float(), pad=i % 3, offset=i % 5)
        v = m.values()
        expert, weights, _, p = plain_route(v, slots, over_all)
        weights = weights.float()
        if i % 2:       # an order that no router makes: the same expert twice, entries outside, whose weights are not looked at
            expert = torch.randint(-2, experts + 2, expert.shape, generator=g).to(torch.int32)
            weights = torch.where((expert >= 0) & (expert < experts), torch.rand(weights.shape, generator=g), math.nan)
        d = torch.randn(tokens, slots, generator=g)
        out = Matrix(tokens, experts, TYPES[t], pad=i % 2, offset=i % 3)
        on = [a.cuda() for a in (d, expert, weights)]
        B.tperm_expert_route_backward(on[0].data_ptr(), m.ptr if over_all else None, m.stride if over_all else 0, on[1].data_ptr(), on[2].data_ptr(), out.ptr, out.stride, tokens, slots, experts, over_all, B.TYPES[t], stream())
        torch.cuda.synchronize()
        there = (expert >= 0) & (expert < experts)
        w = torch.where(there, weights.double(), 0.0)
        each = w * d.double()
        mean, size = each.sum(1, keepdim=True), each.abs().sum(1, keepdim=True)
        step = each if over_all else each - w * mean
        bound = (slots + 4) * SUM * (each.abs() + (0 if over_all else w * size))
        want, off = torch.zeros(tokens, experts, dtype=torch.float64), torch.zeros(tokens, experts, dtype=torch.float64)
        for s in range(slots):
            hit = there[:, s].nonzero()[:, 0]
            want[hit, expert[hit, s].long()] += step[hit, s]
            off[hit, expert[hit, s].long()] += bound[hit, s] + (slots + 1) * SUM * step[hit, s].abs()
        if over_all:
            known = torch.where(v.isnan() | (v == -math.inf), 0.0, v)
            far = known.amax(1, keepdim=True) - known       # at least the distance to the largest
            want -= p * mean
            off += p * size * (4 + experts + slots + far.clamp_max(200)) * SUM + (slots + 1) * SUM * p * mean.abs() + 2.0 ** -126 * size
        near(out.view(), want, off + rounding(t, want) + 2.0 ** -126)
        assert out.outside_untouched()


@pytest.mark.parametrize("over_all", [False, True])
def test_route_backward_is_the_slope_of_route(over_all):
    """Differences of the forward call's weights, in binary32, against the gradient."""
    tokens, experts, slots, step = 8, 24, 5, 2.0 ** -7
    g = generator(5)
    v = torch.randperm(tokens * experts, generator=g).reshape(tokens, experts).float() / 64        # no step changes the choice: 2^-6 apart
    d = torch.randn(tokens, slots, generator=g)

    def loss(v):
        expert, w = torch.empty(tokens, slots, dtype=torch.int32, device="cuda"), torch.empty(tokens, slots, device="cuda")
        v = v.cuda()
        B.tperm_expert_route(v.data_ptr(), experts, expert.data_ptr(), w.data_ptr(), tokens, slots, experts, over_all, B.TYPE_F32, stream())
        return expert, w, (w.double().cpu() * d.double()).sum(1)

    expert, w, _ = loss(v)
    out, scores, grad = torch.empty(tokens, experts, device="cuda"), v.cuda(), d.cuda()
    B.tperm_expert_route_backward(grad.data_ptr(), scores.data_ptr(), experts, expert.data_ptr(), w.data_ptr(), out.data_ptr(), experts, tokens, slots,
                                  experts, over_all, B.TYPE_F32, stream())
    got = out.double().cpu()
    for e in range(experts):
        a, b = v.clone(), v.clone()
        a[:, e] += step / 2
        b[:, e] -= step / 2
        (ea, _, la), (eb, _, lb) = loss(a), loss(b)
        assert torch.equal(ea, expert) and torch.equal(eb, expert)
        # a central difference is off by step^2 / 24 of the third derivative, at most 6 times the gradients' sum here, and by two roundings
        # of each of 5 weights, each (4 + 3 + 24) * 2^-23 of it
        size = d.abs().double().sum(1)
        assert bool(((la - lb) / step - got[:, e]).abs().le(size * (step ** 2 / 4 + 2 * 31 * SUM / step)).all()), e


# --- 4 bits ---

def plain_hold(x):
    """codes (one a number), scales (biased) and values of a matrix of doubles, by distances."""
    rows, width = x.shape
    groups = B.four_bit_groups(width)
    codes, scales = torch.zeros(rows, groups * 32, dtype=torch.int64), torch.zeros(rows, groups, dtype=torch.int64)
    values = torch.zeros(rows, groups * 32, dtype=torch.float64)
    table = torch.tensor(VALUES, dtype=torch.float64)
    for r in range(rows):
        for c in range(groups):
            v = x[r, c * 32:(c + 1) * 32]
            if not bool(v.isfinite().all()):
                scales[r, c], values[r, c * 32:(c + 1) * 32] = 255, math.nan
                continue
            s, most = -125, float(v.abs().max())
            while most > 6 * 2.0 ** s and s < 125:
                s += 1
            a = v.abs() / 2.0 ** s
            distance = (a[:, None] - table).abs()
            # of two at the same distance the even one
            code = torch.tensor([min(range(8), key=lambda i: (float(row[i]), i % 2)) for row in distance])
            codes[r, c * 32:c * 32 + v.numel()] = code + 8 * torch.signbit(v).long()
            values[r, c * 32:c * 32 + v.numel()] = torch.where(torch.signbit(v), -table[code], table[code]) * 2.0 ** s
            scales[r, c] = s + 127
    return codes, scales, values[:, :width]


def held(m, t):
    """Matrix m by the library: codes and scales."""
    groups = B.four_bit_groups(m.width)
    codes, scales = Matrix(m.rows, groups * 16, torch.uint8), Matrix(m.rows, groups, torch.uint8)
    B.tperm_four_bit_store(m.ptr, m.stride, codes.ptr, scales.ptr, m.rows, m.width, B.TYPES[t], stream())
    return codes, scales


def edge_values(t, width, g):
    """Rows at the borders of codes and scales, small and large, and one with numbers that are none."""
    kind = torch.finfo(TYPES[t])
    rows = [torch.randn(width, generator=g, dtype=torch.float64) for _ in range(3)]
    borders = torch.tensor([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 0.25 + 2 ** -9, 5 - 2 ** -6, 6 + 2 ** -5, 0.5, 1.5, 3, 4], dtype=torch.float64)
    at = torch.arange(width)
    rows.append(borders[at % 16] * torch.where(at // 16 % 2 == 0, 1.0, -1.0))
    rows.append(borders[at % 16].clamp_max(6) * torch.where(at % 2 == 0, -1.0, 1.0) * 2.0 ** -3)
    rows.append(torch.zeros(width, dtype=torch.float64))
    rows.append(-torch.zeros(width, dtype=torch.float64))
    rows.append(torch.randn(width, generator=g, dtype=torch.float64) * float(kind.tiny) * 8)
    rows.append((torch.rand(width, generator=g, dtype=torch.float64) * 2 - 1) * float(kind.max))
    rows.append(torch.full((width,), float(kind.max), dtype=torch.float64))
    for bad in (math.nan, math.inf, -math.inf):
        v = torch.randn(width, generator=g, dtype=torch.float64)
        v[width // 2] = bad
        rows.append(v)
    v = torch.randn(width, generator=g, dtype=torch.float64)
    v[::32] = float(kind.smallest_normal)
    v[1::32] = 2.0 ** 9
    rows.append(v)
    return torch.stack(rows)


@pytest.mark.parametrize("width", [1, 7, 8, 31, 32, 33, 40, 64, 100, 259])
@pytest.mark.parametrize("t", list(TYPES))
def test_four_bits(t, width):
    g = generator(width)
    v = edge_values(t, width, g).to(TYPES[t])
    for pad, offset in ((0, 0), (8, 8), (3, 1)):
        m = Matrix(v.shape[0], width, TYPES[t], v, pad=pad, offset=offset)
        codes, scales = held(m, t)
        out = Matrix(m.rows, width, TYPES[t], pad=pad, offset=offset)
        B.tperm_four_bit_load(codes.ptr, scales.ptr, out.ptr, out.stride, m.rows, width, B.TYPES[t], stream())
        torch.cuda.synchronize()
        c, s, values = plain_hold(m.values())
        got = codes.view().cpu().long()
        assert torch.equal(torch.stack([got & 15, got >> 4], dim=2).reshape(m.rows, -1), c)
        assert torch.equal(scales.view().cpu().long(), s)
        most = float(torch.finfo(TYPES[t]).max)
        near(out.view(), values.clamp(-most, most).to(TYPES[t]), torch.zeros(()))
        assert codes.outside_untouched() and scales.outside_untouched() and out.outside_untouched()


@pytest.mark.parametrize("t", list(TYPES))
def test_every_code_at_every_scale(t):
    scales = torch.tensor([*range(2, 253), 255], dtype=torch.uint8)
    codes = torch.tensor([(2 * i) | (2 * i + 1) << 4 for i in range(8)] * 2, dtype=torch.uint8).repeat(len(scales), 1)
    out = torch.empty(len(scales), 32, dtype=TYPES[t], device="cuda")
    on = codes.cuda(), scales.cuda()
    B.tperm_four_bit_load(on[0].data_ptr(), on[1].data_ptr(), out.data_ptr(), 32, len(scales), 32, B.TYPES[t], stream())
    table = torch.tensor(VALUES + [-v for v in VALUES], dtype=torch.float64).repeat(2)
    want = table * torch.where(scales == 255, math.nan, torch.exp2(scales.double() - 127))[:, None]
    most = float(torch.finfo(TYPES[t]).max)
    near(out, want.clamp(-most, most).to(TYPES[t]), torch.zeros(()))


def test_four_bits_in_long_rows_and_many():
    for rows, width in ((1, 1 << 20), (70001, 33)):
        x = torch.randn(rows, width, device="cuda").bfloat16()
        groups = B.four_bit_groups(width)
        codes, scales, out = torch.empty(rows, groups * 16, dtype=torch.uint8, device="cuda"), torch.empty(rows, groups, dtype=torch.uint8, device="cuda"), torch.empty_like(x)
        B.tperm_four_bit_store(x.data_ptr(), width, codes.data_ptr(), scales.data_ptr(), rows, width, B.TYPE_BF16, stream())
        B.tperm_four_bit_load(codes.data_ptr(), scales.data_ptr(), out.data_ptr(), width, rows, width, B.TYPE_BF16, stream())
        a, b = x.float(), out.float()
        scale = torch.exp2(scales.float() - 127).repeat_interleave(32, dim=1)[:, :width]
        assert bool(((a - b).abs() <= torch.maximum(a.abs() / 4, scale / 4)).all())


# --- products ---

def product(x, codes, scales, n, t, out):
    B.tperm_four_bit_product(x.ptr, x.stride, codes.ptr, scales.ptr, out.ptr, out.stride, x.rows, x.width, n, B.TYPES[t], stream())
    torch.cuda.synchronize()


PRODUCTS = [(1, 1, 1), (1, 32, 16), (1, 31, 17), (2, 33, 33), (3, 128, 48), (5, 100, 100), (16, 256, 64), (17, 257, 31), (32, 640, 96), (33, 1000, 35),
            (64, 2048, 130), (65, 2056, 40), (130, 515, 260), (1, 8192, 1003), (7, 4104, 33),
            # the tiles of wide matrices
            (1, 96, 8200), (2, 300, 16400), (12, 100, 8193), (16, 264, 16390), (16, 128, 32776), (20, 264, 8200), (40, 130, 8200), (50, 264, 8200)]


@pytest.mark.parametrize("rows,k,n", PRODUCTS)
@pytest.mark.parametrize("t", list(TYPES))
def test_product(t, rows, k, n):
    g = generator(rows + k + n)
    w = Matrix(n, k, TYPES[t], torch.randn(n, k, generator=g) / math.sqrt(k))
    codes, scales = held(w, t)
    values = Matrix(n, k, torch.float32)
    B.tperm_four_bit_load(codes.ptr, scales.ptr, values.ptr, k, n, k, B.TYPE_F32, stream())
    for pad, offset in ((0, 0), (8, 16), (1, 3)):
        x = Matrix(rows, k, TYPES[t], torch.randn(rows, k, generator=g) * torch.where(torch.rand(k, generator=g) < 0.05, 20.0, 1.0), pad=pad, offset=offset)
        # what lies beside the rows is never part of a sum
        x.buf[:x.lead] = math.nan
        x.buf[x.lead + rows * x.stride:] = math.nan
        if pad:
            x.buf[x.lead:x.lead + rows * x.stride].view(rows, x.stride)[:, k:] = math.inf
        out = Matrix(rows, n, TYPES[t], pad=pad, offset=offset)
        product(x, codes, scales, n, t, out)
        a, b = x.values(), values.values()
        want = a @ b.t()
        near(out.view(), want, rounding(t, want) + k * SUM * (a.abs() @ b.abs().t()))
        assert out.outside_untouched()


@pytest.mark.parametrize("t", list(TYPES))
def test_product_keeps_every_bit_of_its_rows(t):
    """One element of a row against a matrix of ones: the parts that it is multiplied in sum up to it."""
    k = 96
    g = generator(3)
    kind = torch.finfo(TYPES[t])
    v = torch.randn(200, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-40 if t != "f16" else -12, 40 if t != "f16" else 12, (200,), generator=g).double())
    v[:6] = torch.tensor([0.0, float(kind.max), -float(kind.max), math.inf, -math.inf, math.nan], dtype=torch.float64)
    v[6] = float(kind.smallest_normal) if t != "f32" else 2.0 ** -100
    w = Matrix(1, k, TYPES[t], torch.ones(1, k))
    codes, scales = held(w, t)
    x = torch.zeros(200, k, dtype=torch.float64)
    x[torch.arange(200), torch.arange(200) % k] = v
    x = Matrix(200, k, TYPES[t], x)
    out = Matrix(200, 1, TYPES[t])
    product(x, codes, scales, 1, t, out)
    near(out.view()[:, 0], x.values()[torch.arange(200), torch.arange(200) % k], torch.zeros(()))


def test_product_of_nan_groups_and_of_largest_scales():
    w = torch.ones(48, 64)
    w[3, 40] = math.nan
    w[5, 0] = math.inf
    w[7] = 2.0 ** 127
    w[9] = 2.0 ** -120
    m = Matrix(48, 64, torch.float32, w)
    codes, scales = held(m, "f32")
    x = Matrix(2, 64, torch.float32, torch.stack([torch.full((64,), 2.0 ** -8), torch.full((64,), 2.0 ** 8)]))
    out = Matrix(2, 48, torch.float32)
    product(x, codes, scales, 48, "f32", out)
    want = x.values() @ w.double().t()
    want[:, 5] = math.nan
    near(out.view(), torch.where(want > 2.0 ** 128, math.inf, want), torch.zeros(()))


def test_product_of_many_rows():
    """More rows than one launch takes workgroups for along its second dimension, in three columns."""
    rows, k = 65535 * 64 + 70, 8
    x = torch.randint(-4, 5, (rows, k), device="cuda").bfloat16()
    w = torch.randint(-2, 3, (3, k), device="cuda").bfloat16()
    codes, scales, out = torch.empty(3, 16, dtype=torch.uint8, device="cuda"), torch.empty(3, 1, dtype=torch.uint8, device="cuda"), torch.empty(rows, 3, dtype=torch.bfloat16, device="cuda")
    B.tperm_four_bit_store(w.data_ptr(), k, codes.data_ptr(), scales.data_ptr(), 3, k, B.TYPE_BF16, stream())
    B.tperm_four_bit_product(x.data_ptr(), k, codes.data_ptr(), scales.data_ptr(), out.data_ptr(), 3, rows, k, 3, B.TYPE_BF16, stream())
    assert torch.equal(out.float(), x.float() @ w.float().t())      # whole numbers below 2^8


# --- a layer for a few tokens ---

def numbers(tokens, slots, experts, g, drop=0.0, twice=False):
    """Expert numbers, different ones for a token unless `twice`; some outside."""
    e = torch.randint(0, experts, (tokens, slots), generator=g) if twice or slots > experts else \
        torch.stack([torch.randperm(experts, generator=g)[:slots] for _ in range(tokens)])
    gone = torch.rand(tokens, slots, generator=g) < drop
    return torch.where(gone, torch.tensor([-1, experts, -2 ** 31, 2 ** 31 - 1])[torch.randint(0, 4, e.shape, generator=g)], e).to(torch.int32)


HELD = {"f32": 0.0, "f16": 2.0 ** -22, "bf16": 2.0 ** -16}


def plain_few(x, expert, weights, w_in, w_out, t, four):
    """Result and tolerance; everything in doubles."""
    tokens, width = x.shape
    experts, hidden = w_in.shape[0], w_out.shape[2]
    want, off = torch.zeros(tokens, width, dtype=torch.float64), torch.zeros(tokens, width, dtype=torch.float64)
    size = torch.zeros_like(want)
    keep = (2.0 ** -16 if t != "f32" else 0.0) if four else HELD[t]
    for i in range(tokens):
        for s in range(expert.shape[1]):
            e = int(expert[i, s])
            if not 0 <= e < experts:
                continue
            both, both_size = w_in[e] @ x[i], w_in[e].abs() @ x[i].abs()
            g, u, off_g, off_u = both[:hidden], both[hidden:], width * SUM * both_size[:hidden], width * SUM * both_size[hidden:]
            h = g * torch.special.expit(g) * u
            silu = (g * torch.special.expit(g)).abs()
            off_h = 1.1 * off_g * (u.abs() + off_u) + silu * off_u + (keep + 12 * SUM) * h.abs()
            w = float(weights[i, s])
            off_h = abs(w) * off_h + (2.0 ** -25 if t == "f16" and not four else 2.0 ** -120)
            want[i] += w * (w_out[e] @ h)
            size[i] += w_out[e].abs() @ (abs(w) * h.abs())
            off[i] += w_out[e].abs() @ off_h
    return want, off + (hidden + expert.shape[1]) * SUM * size + rounding(t, want)


class Layer:
    def __init__(self, t, four, experts, width, hidden, g, offset=0):
        self.t, self.four, self.experts, self.width, self.hidden = t, four, experts, width, hidden
        shapes = [(experts * 2 * hidden, width), (experts * width, hidden)]
        self.w = [Matrix(r, c, TYPES[t], torch.randn(r, c, generator=g) / math.sqrt(c), offset=offset) for r, c in shapes]
        self.values = [m.values() for m in self.w]
        self.ptrs = [self.w[0].ptr, None, self.w[1].ptr, None]
        if four:
            self.held = [held(m, t) for m in self.w]
            self.ptrs = [a.ptr for pair in self.held for a in pair]
            for i, (m, (codes, scales)) in enumerate(zip(self.w, self.held)):
                v = torch.empty(m.rows, m.width, device="cuda")
                B.tperm_four_bit_load(codes.ptr, scales.ptr, v.data_ptr(), m.width, m.rows, m.width, B.TYPE_F32, stream())
                self.values[i] = v.double().cpu()
        self.values = [self.values[0].reshape(experts, 2 * hidden, width), self.values[1].reshape(experts, width, hidden)]

    def room(self, tokens, slots):
        return Matrix(1, B.expert_few_workspace_bytes(tokens, slots, self.experts, self.width, self.hidden, B.TYPES[self.t], self.four), torch.uint8)

    def __call__(self, x, expert, weights, out, room):
        w_in, in_scales, w_out, out_scales = self.ptrs
        B.tperm_expert_few(x.ptr, x.stride, expert.data_ptr(), None if weights is None else weights.data_ptr(), w_in, in_scales, w_out, out_scales, out.ptr, out.stride,
                           room.ptr, room.width, expert.shape[0], expert.shape[1], self.experts, self.width, self.hidden, B.TYPES[self.t], stream())


#        tokens, slots, experts, width, hidden, drop, pad, offset
LAYERS = [(1, 1, 1, 1, 1, 0.0, 0, 0), (1, 2, 4, 64, 32, 0.0, 0, 0), (1, 4, 8, 512, 256, 0.0, 8, 0), (2, 3, 5, 100, 33, 0.3, 1, 0), (7, 2, 3, 33, 100, 0.0, 3, 1),
          (16, 4, 16, 128, 128, 0.1, 0, 0), (17, 1, 1, 136, 72, 0.0, 0, 0), (33, 2, 3, 257, 65, 0.2, 0, 0), (40, 1, 1, 48, 520, 0.0, 0, 8), (64, 4, 40, 96, 64, 0.0, 0, 0),
          (64, 2, 2, 72, 40, 0.0, 8, 8), (5, 64, 70, 24, 16, 0.5, 0, 0), (64, 64, 1024, 8, 8, 0.1, 0, 0), (3, 2, 4, 1001, 515, 0.0, 0, 3), (9, 8, 6, 40, 48, 0.0, 0, 0)]


@pytest.mark.parametrize("tokens,slots,experts,width,hidden,drop,pad,offset", LAYERS)
@pytest.mark.parametrize("four", [False, True], ids=["own", "four"])
@pytest.mark.parametrize("t", list(TYPES))
def test_few(t, four, tokens, slots, experts, width, hidden, drop, pad, offset):
    g = generator(tokens * 1000 + width)
    layer = Layer(t, four, experts, width, hidden, g, offset)
    x = Matrix(tokens, width, TYPES[t], torch.randn(tokens, width, generator=g), pad=pad, offset=offset)
    if pad:
        x.buf[x.lead:x.lead + tokens * x.stride].view(tokens, x.stride)[:, width:] = math.nan
    expert = numbers(tokens, slots, experts, g, drop)
    inside = (expert >= 0) & (expert < experts)
    weights = torch.where(inside, torch.randn(tokens, slots, generator=g), math.nan)
    out, room = Matrix(tokens, width, TYPES[t], pad=pad, offset=offset), layer.room(tokens, slots)
    room.view()[:] = 255        # whatever a workspace holds
    layer(x, expert.cuda(), weights.cuda(), out, room)
    torch.cuda.synchronize()
    want, off = plain_few(x.values(), expert, weights.double(), *layer.values, t, four)
    near(out.view(), want, off)
    room.before[room.lead:room.lead + room.width] = 0
    room.buf[room.lead:room.lead + room.width] = 0
    assert out.outside_untouched() and torch.equal(room.buf, room.before)


@pytest.mark.parametrize("four", [False, True], ids=["own", "four"])
def test_few_without_weights_without_experts_and_with_one_twice(four):
    t, tokens, slots, experts, width, hidden = "bf16", 6, 4, 5, 80, 48
    g = generator(8)
    layer = Layer(t, four, experts, width, hidden, g)
    x = Matrix(tokens, width, TYPES[t], torch.randn(tokens, width, generator=g))
    room = layer.room(tokens, slots)
    for expert, weights in ((numbers(tokens, slots, experts, g), None), (torch.full((tokens, slots), -1, dtype=torch.int32), None),
                            (torch.full((tokens, slots), 3, dtype=torch.int32), torch.randn(tokens, slots, generator=g)),
                            (torch.tensor([[0, 0, 1, 0]] * tokens, dtype=torch.int32), torch.randn(tokens, slots, generator=g)),
                            (torch.where(torch.arange(tokens)[:, None] == 2, numbers(tokens, slots, experts, g), -1), torch.randn(tokens, slots, generator=g))):
        out = Matrix(tokens, width, TYPES[t])
        layer(x, expert.cuda(), None if weights is None else weights.cuda(), out, room)
        torch.cuda.synchronize()
        want, off = plain_few(x.values(), expert, torch.ones(tokens, slots).double() if weights is None else weights.double(), *layer.values, t, four)
        near(out.view(), want, off)


@pytest.mark.parametrize("four", [False, True], ids=["own", "four"])
@pytest.mark.parametrize("t", list(TYPES))
def test_tokens_do_not_touch_each_other(t, four):
    """NaN and infinities of one token stay there, and so do those of an expert that nobody names."""
    tokens, slots, experts, width, hidden = 20, 2, 6, 136, 72
    g = generator(9)
    layer = Layer(t, four, experts, width, hidden, g)
    x = Matrix(tokens, width, TYPES[t], torch.randn(tokens, width, generator=g))
    expert = numbers(tokens, slots, experts - 1, g)
    weights = torch.rand(tokens, slots, generator=g).cuda()
    room, clean, out = layer.room(tokens, slots), Matrix(tokens, width, TYPES[t]), Matrix(tokens, width, TYPES[t])
    layer(x, expert.cuda(), weights, clean, room)
    bad = {3: math.nan, 11: math.inf, 19: -math.inf}
    for i, v in bad.items():
        x.view()[i, 5] = v
    if four:
        for (_, scales), rows in zip(layer.held, (2 * hidden, width)):
            scales.view()[(experts - 1) * rows:] = 255
    else:
        for w, rows in zip(layer.w, (2 * hidden, width)):
            w.view()[(experts - 1) * rows:] = math.nan
    layer(x, expert.cuda(), weights, out, room)
    torch.cuda.synchronize()
    for i in range(tokens):
        if i not in bad:
            assert torch.equal(out.view()[i], clean.view()[i])
        else:
            assert not bool(out.view()[i].isfinite().all())


def few_on_the_gpu(x, expert, weights, w_in, w_out, t, four):
    """plain_few, by expert; matrices are what the call takes, or what their codes stand for."""
    tokens, width = x.shape
    hidden = w_out.shape[2]
    want, off, size = (torch.zeros(tokens, width, dtype=torch.float64, device="cuda") for _ in range(3))
    keep = (2.0 ** -16 if t != "f32" else 0.0) if four else HELD[t]
    for e in range(w_in.shape[0]):
        token, slot = (expert == e).nonzero(as_tuple=True)
        a, w, b, c = x[token], weights[token, slot, None].double(), w_in[e].double(), w_out[e].double()
        both, both_size = a @ b.t(), a.abs() @ b.abs().t()
        g, u, off_g, off_u = both[:, :hidden], both[:, hidden:], width * SUM * both_size[:, :hidden], width * SUM * both_size[:, hidden:]
        silu = g * torch.special.expit(g)
        h = silu * u
        off_h = 1.1 * off_g * (u.abs() + off_u) + silu.abs() * off_u + (keep + 12 * SUM) * h.abs()
        off_h = w.abs() * off_h + (2.0 ** -25 if t == "f16" and not four else 2.0 ** -120)
        want.index_add_(0, token, w * (h @ c.t()))
        size.index_add_(0, token, (w.abs() * h.abs()) @ c.abs().t())
        off.index_add_(0, token, off_h @ c.abs().t())
    return want, off + (hidden + expert.shape[1]) * SUM * size + rounding(t, want)


# Sizes that take four tiles to an item, shares of results, tokens from LDS, entries of more than 8, 16 and 32 tokens.
WIDE = [(64, 2, 24, 72, 1024), (64, 2, 24, 75, 1027), (64, 2, 4, 1208, 4104), (64, 2, 4, 1203, 4101), (8, 4, 40, 520, 1024), (7, 4, 40, 523, 1021),
        (16, 4, 64, 1536, 1544), (40, 3, 64, 1541, 1537), (1, 8, 64, 1536, 4096)]


@pytest.mark.parametrize("tokens,slots,experts,width,hidden", WIDE)
@pytest.mark.parametrize("four", [False, True], ids=["own", "four"])
@pytest.mark.parametrize("t", list(TYPES))
def test_few_of_wide_layers(t, four, tokens, slots, experts, width, hidden):
    g = torch.Generator(device="cuda").manual_seed(width)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, w_in, w_out = randn(tokens, width).to(TYPES[t]), (randn(experts, 2 * hidden, width) / width ** 0.5).to(TYPES[t]), (randn(experts, width, hidden) / hidden ** 0.5).to(TYPES[t])
    expert = torch.argsort(randn(tokens, experts), dim=1)[:, :slots].to(torch.int32)
    expert = torch.where(torch.rand(tokens, slots, generator=g, device="cuda") < 0.05, -1, expert)
    weights = torch.rand(tokens, slots, generator=g, device="cuda")
    matrices, stands, keep = [], [], []
    for w in (w_in, w_out):
        rows, k = w.shape[0] * w.shape[1], w.shape[2]
        if four:
            codes, scales = (torch.empty(rows * B.four_bit_groups(k) * n, dtype=torch.uint8, device="cuda") for n in (16, 1))
            B.tperm_four_bit_store(w.data_ptr(), k, codes.data_ptr(), scales.data_ptr(), rows, k, B.TYPES[t], stream())
            v = torch.empty(w.shape, device="cuda")
            B.tperm_four_bit_load(codes.data_ptr(), scales.data_ptr(), v.data_ptr(), k, rows, k, B.TYPE_F32, stream())
            matrices += [codes.data_ptr(), scales.data_ptr()]
            keep += [codes, scales]
            stands.append(v)
        else:
            matrices += [w.data_ptr(), None]
            stands.append(w)
    out = Matrix(tokens, width, TYPES[t], pad=1)
    need = B.expert_few_workspace_bytes(tokens, slots, experts, width, hidden, B.TYPES[t], four)
    room = Matrix(1, need, torch.uint8)

    def few():
        B.tperm_expert_few(x.data_ptr(), width, expert.data_ptr(), weights.data_ptr(), *matrices, out.ptr, out.stride, room.ptr, need, tokens, slots, experts, width,
                           hidden, B.TYPES[t], stream())
        torch.cuda.synchronize()
        return out.view().clone()

    got = few()
    want, off = few_on_the_gpu(x.double(), expert, weights, *stands, t, four)
    near(got, want.cpu(), off.cpu())
    assert torch.equal(few(), got) and out.outside_untouched()
    room.before[room.lead:room.lead + need] = 0
    room.buf[room.lead:room.lead + need] = 0
    assert torch.equal(room.buf, room.before)


def test_large_matrices():
    """An expert's matrix behind 4 GiB: the same bits as from the first place (how a sum is split goes by the sizes, number of experts among them)."""
    experts, width, hidden, tokens, slots = 5, 16384, 16384, 3, 2
    t = B.TYPE_BF16
    g = torch.Generator(device="cuda").manual_seed(4)
    w_in = torch.empty(experts, 2 * hidden, width, dtype=torch.bfloat16, device="cuda").normal_(generator=g).mul_(width ** -0.5)
    w_out = torch.empty(experts, width, hidden, dtype=torch.bfloat16, device="cuda").normal_(generator=g).mul_(hidden ** -0.5)
    x = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    room = torch.empty(B.expert_few_workspace_bytes(tokens, slots, experts, width, hidden, t), dtype=torch.uint8, device="cuda")

    def few(expert, a, b, experts, scales=(None, None)):
        out = torch.empty_like(x)
        expert = torch.tensor([[expert, -1]] * tokens, dtype=torch.int32, device="cuda")
        B.tperm_expert_few(x.data_ptr(), width, expert.data_ptr(), None, a.data_ptr(), scales[0], b.data_ptr(), scales[1], out.data_ptr(), width, room.data_ptr(),
                           room.numel(), tokens, slots, experts, width, hidden, t, stream())
        torch.cuda.synchronize()
        return out

    got = few(4, w_in, w_out, experts)
    w_in[0].copy_(w_in[4])
    w_out[0].copy_(w_out[4])
    assert torch.equal(got, few(0, w_in, w_out, experts))
    g_, u = (x.float() @ w_in[4].float().t()).split(hidden, dim=1)
    want = (torch.nn.functional.silu(g_) * u) @ w_out[4].float().t()
    assert float((got.float() - want).norm() / want.norm()) < 2.0 ** -8
    assert bool(got.isfinite().all())


# --- streams, graphs, repetition ---

def test_same_bits_again_on_another_stream_and_in_a_graph():
    t, tokens, slots, experts, width, hidden = "bf16", 24, 3, 12, 200, 136
    g = generator(2)
    layers = [Layer(t, four, experts, width, hidden, g) for four in (False, True)]
    x, other = (Matrix(tokens, width, TYPES[t], torch.randn(tokens, width, generator=g)) for _ in range(2))
    scores = torch.randn(tokens, experts, generator=g).bfloat16().cuda()
    d = torch.randn(tokens, slots, generator=g).cuda()
    expert, weights = torch.empty(tokens, slots, dtype=torch.int32, device="cuda"), torch.empty(tokens, slots, device="cuda")
    grad = torch.empty_like(scores)
    outs = [Matrix(tokens, width, TYPES[t]) for _ in range(3)]
    room = layers[1].room(tokens, slots)
    assert room.width >= layers[0].room(tokens, slots).width
    codes, scales = layers[1].held[1]

    def all_of_them(x):
        s = stream()
        B.tperm_expert_route(scores.data_ptr(), experts, expert.data_ptr(), weights.data_ptr(), tokens, slots, experts, True, B.TYPES[t], s)
        for layer, out in zip(layers, outs):
            layer(x, expert, weights, out, room)
        B.tperm_expert_route_backward(d.data_ptr(), scores.data_ptr(), experts, expert.data_ptr(), weights.data_ptr(), grad.data_ptr(), experts, tokens, slots,
                                      experts, True, B.TYPES[t], s)
        # of the last expert's second matrix: the first `hidden` channels of the tokens
        B.tperm_four_bit_product(x.ptr, x.stride, codes.ptr + (experts - 1) * width * 16 * B.four_bit_groups(hidden),
                                 scales.ptr + (experts - 1) * width * B.four_bit_groups(hidden), outs[2].ptr, outs[2].stride, tokens, hidden, width, B.TYPES[t], s)

    def results():
        torch.cuda.synchronize()
        return [expert.clone(), weights.clone(), grad.clone(), *(o.view().clone() for o in outs)]

    all_of_them(x)
    want = results()
    all_of_them(other)
    assert not torch.equal(results()[3], want[3])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        all_of_them(x)
    assert all(torch.equal(a, b) for a, b in zip(results(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_of_them(x)
    for _ in range(4):
        all_of_them(other)
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(results(), want))

"""What lies between the two products of the layer for a few tokens, weight * g * sigmoid(g) * u, keeps the bits and the range of binary32 whatever
the types of the matrices are.

Bounds, fixed before the first run, elementwise.  A sum of n terms in binary32 is off by n * 2^-23 times the sum of their magnitudes at most (three products to a
hidden value, which meets a matrix of 16 or 4 bits in three parts); the activation's slope is at most 1.1 in g, g * sigmoid(g) * u * weight is right
to 12 * 2^-23 of itself, and holding it adds nothing; the result is rounded to its type."""
import math

import pytest

from paper_1705_01598_amd import binding as B

torch = pytest.importorskip("torch")
from test_gpu_decode import held  # noqa: E402
from test_gpu_experts import SUM, TYPES, Matrix, near, rounding, stream  # noqa: E402

pytestmark = pytest.mark.gpu


class Layer:
    """Matrices w_in [experts, 2 * hidden, width] and w_out [experts, width, hidden], as they are or in 4 bits."""

    def __init__(self, t, four, w_in, w_out):
        self.t, self.experts, self.width, self.hidden = t, w_in.shape[0], w_in.shape[2], w_out.shape[2]
        self.four, self.values, self.keep, self.at = four, [], [], []
        for w in (w_in, w_out):
            m = Matrix(w.shape[0] * w.shape[1], w.shape[2], TYPES[t], w.reshape(-1, w.shape[2]))
            values = m.values()
            if four:
                codes, scales = held(m, t)
                v = torch.empty(m.rows, m.width, device="cuda")
                B.tperm_four_bit_load(codes.ptr, scales.ptr, v.data_ptr(), m.width, m.rows, m.width, B.TYPE_F32, stream())
                values = v.double().cpu()
                self.keep += [codes, scales]
                self.at += [codes.ptr, scales.ptr]
            else:
                self.keep.append(m)
                self.at += [m.ptr, None]
            self.values.append(values.reshape(w.shape))

    def __call__(self, x, expert, weights):
        out = Matrix(x.rows, self.width, TYPES[self.t])
        need = B.expert_few_workspace_bytes(x.rows, expert.shape[1], self.experts, self.width, self.hidden, B.TYPES[self.t], self.four)
        room = Matrix(1, need, torch.uint8)
        expert, weights = expert.to(torch.int32).cuda(), weights.float().cuda()
        B.tperm_expert_few(x.ptr, x.stride, expert.data_ptr(), weights.data_ptr(), *self.at, out.ptr, out.stride, room.ptr, need, x.rows, expert.shape[1], self.experts,
                           self.width, self.hidden, B.TYPES[self.t], stream())
        torch.cuda.synchronize()
        assert out.outside_untouched()
        return out.view()


def plain(layer, x, expert, weights):
    """Result and bound, in doubles."""
    w_in, w_out = layer.values
    width, hidden = layer.width, layer.hidden
    want, off, size = (torch.zeros(x.shape, dtype=torch.float64) for _ in range(3))
    for i in range(x.shape[0]):
        for e, w in zip(expert[i].tolist(), weights[i].double().tolist()):
            both, both_size = w_in[e] @ x[i], w_in[e].abs() @ x[i].abs()
            g, u, off_g, off_u = both[:hidden], both[hidden:], width * SUM * both_size[:hidden], width * SUM * both_size[hidden:]
            silu = g * torch.special.expit(g)
            h = silu * u
            off_h = abs(w) * (1.1 * off_g * (u.abs() + off_u) + silu.abs() * off_u + 12 * SUM * h.abs()) + 2.0 ** -120
            want[i] += w * (w_out[e] @ h)
            size[i] += w_out[e].abs() @ (abs(w) * h.abs())
            off[i] += w_out[e].abs() @ off_h
    return want, off + (3 * hidden + expert.shape[1]) * SUM * size + rounding(layer.t, want)


# size of x * sqrt(width), of both matrices' elements, and of the weights: hidden values near the sizes of the second column
#       type    x, w_in, w_out, weight          hidden
SIZES = {"small": {"f16": (2.0 ** -5, 2.0 ** -5, 2.0 ** 10, 2.0 ** -3),          # 2^-24
                   "bf16": (2.0 ** -20, 2.0 ** -15, 2.0 ** 60, 2.0 ** -10),      # 2^-81
                   "f32": (2.0 ** -20, 2.0 ** -15, 2.0 ** 60, 2.0 ** -10)},
         "large": {"f16": (2.0 ** 6, 2.0 ** 4, 2.0 ** -12, 1.0),                 # 2^20
                   "bf16": (2.0 ** 30, 2.0 ** 29, 2.0 ** -100, 1.0),             # 2^118
                   "f32": (2.0 ** 30, 2.0 ** 29, 2.0 ** -100, 1.0)}}


@pytest.mark.parametrize("tokens,slots,experts,width,hidden", [(1, 2, 3, 64, 96), (7, 2, 5, 33, 50), (23, 1, 1, 40, 72), (40, 2, 3, 96, 40)])
@pytest.mark.parametrize("size", list(SIZES))
@pytest.mark.parametrize("four", [False, True], ids=["own", "four"])
@pytest.mark.parametrize("t", list(TYPES))
def test_range(t, four, size, tokens, slots, experts, width, hidden):
    g = torch.Generator().manual_seed(tokens)
    randn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x_size, in_size, out_size, weight_size = SIZES[size][t]
    layer = Layer(t, four, randn(experts, 2 * hidden, width) * in_size / math.sqrt(width), randn(experts, width, hidden) * out_size)
    x = Matrix(tokens, width, TYPES[t], randn(tokens, width) * x_size)
    expert = torch.stack([torch.randperm(experts, generator=g)[:slots] for _ in range(tokens)])
    weights = ((0.5 + torch.rand(tokens, slots, generator=g)) * weight_size).float()
    want, off = plain(layer, x.values(), expert, weights)
    assert bool((want.abs() > 0).all()) and float(want.abs().max()) < torch.finfo(TYPES[t]).max
    near(layer(x, expert, weights), want, off)


@pytest.mark.parametrize("four", [False, True], ids=["own", "four"])
@pytest.mark.parametrize("t", list(TYPES))
def test_bits(t, four):
    """Two experts of the same diagonal matrices, with weights that cancel but for some 2^-12: what is left shows the bits that were held.  Products with zeros are
    exact, and so is that of two diagonal elements, which have 8 bits each; so the bound is that of g * sigmoid(g) * u * weight, of the
    three parts' sum and of the sum over the slots."""
    tokens, n = 64, 32
    g = torch.Generator().manual_seed(6)
    few_bits = lambda *s: (1 + torch.rand(*s, generator=g)).bfloat16().double()  # noqa: E731
    w_g, w_u, w_o = (torch.diag(few_bits(n)) for _ in range(3))
    layer = Layer(t, four, torch.cat([w_g, w_u]).expand(2, -1, -1), w_o.expand(2, -1, -1))
    x = Matrix(tokens, n, TYPES[t], few_bits(tokens, n) * 2)
    expert = torch.tensor([[0, 1]] * tokens)
    first = 0.5 + torch.rand(tokens, generator=g)
    weights = torch.stack([first, -first * (1 + 2.0 ** -12 * (1 + torch.rand(tokens, generator=g)))], 1).float()
    (w_in, w_out), v = layer.values, x.values()
    gate, up, last = v * w_in[0, :n].diagonal(), v * w_in[0, n:].diagonal(), w_out[0].diagonal()
    y = gate * torch.special.expit(gate) * up * last
    want, size = y * weights.double().sum(1, keepdim=True), y.abs() * weights.double().abs().sum(1, keepdim=True)
    near(layer(x, expert, weights), want, 13 * SUM * size + rounding(t, want))


@pytest.mark.parametrize("tokens,width,hidden", [(3, 40, 72), (12, 33, 75), (40, 48, 40), (30, 1600, 24)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("four", [False, True], ids=["own", "four"])
@pytest.mark.parametrize("t", list(TYPES))
def test_an_infinite_hidden_value(t, four, bad, tokens, width, hidden):
    """One channel of one token leaves binary32's range: its products are infinite with the signs of that channel's elements, NaN where those are zero; other
    tokens of the same expert keep their bits."""
    g = torch.Generator().manual_seed(width)
    randn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    w_in, w_out, channel = randn(1, 2 * hidden, width) / math.sqrt(width), randn(1, width, hidden) / math.sqrt(hidden), hidden - 2
    large = 2.0 ** 15 if t == "f16" else 2.0 ** 40
    w_in[:, :, 0] = 0.0
    w_in[0, channel] = w_in[0, hidden + channel] = 0.0
    w_in[0, channel, 0], w_in[0, hidden + channel, 0] = large, math.copysign(large, bad)
    w_out[0, ::7, channel] = 0.0
    layer = Layer(t, four, w_in, w_out)
    v, weights = randn(tokens, width), torch.rand(tokens, 1, generator=g)
    v[:, 0] = 0.0
    expert = torch.zeros(tokens, 1)
    clean = layer(Matrix(tokens, width, TYPES[t], v), expert, weights)
    v[1, 0] = large if not math.isnan(bad) else bad
    if t == "f16":
        weights[1] = 2.0 ** 80
    got = layer(Matrix(tokens, width, TYPES[t], v), expert, weights)
    last = layer.values[1][0, :, channel]
    want = torch.where((last == 0) | math.isnan(bad), math.nan, torch.sign(last) * bad)
    near(got[1], want, torch.zeros(()))
    others = torch.arange(tokens) != 1
    assert torch.equal(got.cpu()[others], clean.cpu()[others]) and bool(clean.isfinite().all())


@pytest.mark.parametrize("tokens", [6, 14, 40])
@pytest.mark.parametrize("four", [False, True], ids=["own", "four"])
@pytest.mark.parametrize("t", ["f16", "bf16"])
def test_an_infinite_hidden_value_where_results_are_shared(t, four, tokens):
    """The same in a layer whose second matrix is large enough for workgroups to share its experts, in tiles of every kind: 8, 16 and 32 tokens to an expert."""
    width = hidden = 8192
    g = torch.Generator(device="cuda").manual_seed(tokens)
    randn = lambda *s: (torch.randn(*s, generator=g, device="cuda") / 64).to(TYPES[t])  # noqa: E731
    w_in, w_out, x, channel = randn(2, 2 * hidden, width), randn(2, width, hidden), randn(tokens, width), 4099
    large = 2.0 ** 15 if t == "f16" else 2.0 ** 40
    w_in[:, :, 0] = 0.0
    w_in[0, channel] = w_in[0, hidden + channel] = 0.0
    w_in[0, channel, 0] = w_in[0, hidden + channel, 0] = large
    w_out[0, ::7, channel] = 0.0
    x[:, 0] = 0.0
    at, keep, last = [], [], w_out[0, :, channel].float()
    for w in (w_in, w_out):
        rows, k = 2 * w.shape[1], w.shape[2]
        if four:
            codes, scales = (torch.empty(rows * B.four_bit_groups(k) * n, dtype=torch.uint8, device="cuda") for n in (16, 1))
            B.tperm_four_bit_store(w.data_ptr(), k, codes.data_ptr(), scales.data_ptr(), rows, k, B.TYPES[t], stream())
            keep += [codes, scales]
            at += [codes.data_ptr(), scales.data_ptr()]
        else:
            at += [w.data_ptr(), None]
    if four:
        stands = torch.empty(2, width, hidden, device="cuda")
        B.tperm_four_bit_load(at[2], at[3], stands.data_ptr(), hidden, 2 * width, hidden, B.TYPE_F32, stream())
        last = stands[0, :, channel]
    weights = torch.rand(tokens, 2, generator=g, device="cuda")
    expert = torch.tensor([[0, -1]] * tokens, dtype=torch.int32, device="cuda")
    need = B.expert_few_workspace_bytes(tokens, 2, 2, width, hidden, B.TYPES[t], four)
    assert need > 2 * tokens * hidden * 4      # there are shares behind the hidden rows
    room = torch.empty(need, dtype=torch.uint8, device="cuda")

    def few():
        out = torch.empty_like(x)
        B.tperm_expert_few(x.data_ptr(), width, expert.data_ptr(), weights.data_ptr(), *at, out.data_ptr(), width, room.data_ptr(), need, tokens, 2, 2, width, hidden,
                           B.TYPES[t], stream())
        torch.cuda.synchronize()
        return out

    clean = few()
    x[1, 0] = large
    if t == "f16":
        weights[1] = 2.0 ** 80
    got = few()
    near(got[1], torch.where(last == 0, math.nan, torch.sign(last) * math.inf).cpu(), torch.zeros(()))
    others = torch.arange(tokens, device="cuda") != 1
    assert torch.equal(got[others], clean[others]) and bool(clean.isfinite().all())


def test_shared_results_in_a_graph_between_eager_passes():
    """The third kernel in a captured pass: replays between eager passes of other tokens through the same workspace give the eager bits."""
    tokens, slots, experts, width, hidden, t = 12, 4, 48, 1001, 1030, "bf16"
    g = torch.Generator(device="cuda").manual_seed(3)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    keep, at = [], []
    for rows, k in ((experts * 2 * hidden, width), (experts * width, hidden)):
        w = (randn(rows, k) / k ** 0.5).to(TYPES[t])
        codes, scales = (torch.empty(rows * B.four_bit_groups(k) * n, dtype=torch.uint8, device="cuda") for n in (16, 1))
        B.tperm_four_bit_store(w.data_ptr(), k, codes.data_ptr(), scales.data_ptr(), rows, k, B.TYPES[t], stream())
        keep += [codes, scales]
        at += [codes.data_ptr(), scales.data_ptr()]
    expert, weights = torch.argsort(randn(tokens, experts), dim=1)[:, :slots].to(torch.int32), torch.rand(tokens, slots, generator=g, device="cuda")
    need = B.expert_few_workspace_bytes(tokens, slots, experts, width, hidden, B.TYPES[t], True)
    assert need > tokens * slots * 1280 * 4      # there are shares behind the hidden rows
    room = torch.empty(need, dtype=torch.uint8, device="cuda")
    x, other, out = randn(tokens, width).to(TYPES[t]), randn(tokens, width).to(TYPES[t]), torch.empty(tokens, width, dtype=TYPES[t], device="cuda")

    def few(x):
        B.tperm_expert_few(x.data_ptr(), width, expert.data_ptr(), weights.data_ptr(), *at, out.data_ptr(), width, room.data_ptr(), need, tokens, slots, experts, width,
                           hidden, B.TYPES[t], stream())

    few(x)
    torch.cuda.synchronize()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        few(x)
    for _ in range(4):
        few(other)
        torch.cuda.synchronize()
        assert not torch.equal(out, want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("t", list(TYPES))
def test_an_infinite_element_of_the_second_matrix(t):
    """Diagonal matrices, the second one's elements infinite: results are infinite with the sign of the hidden value, whatever bits that has."""
    tokens, n = 64, 32
    g = torch.Generator().manual_seed(7)
    randn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    layer = Layer(t, False, torch.cat([torch.diag(1 + randn(n).abs()) for _ in range(2)])[None], torch.diag(torch.full((n,), math.inf))[None].nan_to_num(nan=0.0, posinf=math.inf))
    x = Matrix(tokens, n, TYPES[t], randn(tokens, n))
    x.view()[x.view().abs() < 0.01] = 0.5
    got = layer(x, torch.zeros(tokens, 1), torch.rand(tokens, 1, generator=g) + 0.5)
    gate = x.values() * layer.values[0][0, :n].diagonal()
    up = x.values() * layer.values[0][0, n:].diagonal()
    near(got, torch.sign(gate * torch.special.expit(gate) * up) * math.inf, torch.zeros(()))

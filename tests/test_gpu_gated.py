"""The gated activation far from zero and at values that are no numbers, against its formulas in 64 bits.

Tolerances, fixed before the first run.  exp2 and reciprocal are right to 2^-23 of their result, an operation to 2^-24.  With
E = exp(-|g| / 2) off by 1.5 * 2^-23, squared in the sigmoid of a negative g (3), the denominator 1 + E^2 off by 1.75 + 0.5 of
2^-23 and its reciprocal by 1 more, and four products (2): 8.25 * 2^-23 of the result, at most 9, whatever g is, in
binary32; types of 16 bits add |g| * 2^-24, the rounding of |g| * log2(e).  The gradient's 1 + g (1 - p) is a sum: its
error is held against 1 + |g (1 - p)|, with 6 * 2^-23 for the sum's own terms."""
import pytest

from paper_1705_01598_amd import binding as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -148, "f16": 2.0 ** -25, "bf16": 2.0 ** -133}     # a step of the smallest numbers
SUM = 2.0 ** -23


def stream():
    return torch.cuda.current_stream().cuda_stream


def near(got, want, bound):
    got, want = got.double().cpu(), want.double()
    same = (torch.isnan(got) & torch.isnan(want)) | (got == want)
    bad = ~same & ~((got - want).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:4], want[bad][:4])


def forward(gates, t):
    rows, width = gates.shape[0], gates.shape[1] // 2
    out = torch.empty(rows, width, dtype=TYPES[t], device="cuda")
    B.tperm_gated_forward(gates.data_ptr(), 2 * width, out.data_ptr(), width, None, None, rows, width, B.TYPES[t], stream())
    return out


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("width", [1024, 1023])
def test_forward_far_from_zero(t, width):
    g = torch.linspace(-104, 104, 16 * width).view(width, 16).t().contiguous()
    u = torch.linspace(0.5, 2.0, 16 * width).view(16, width)
    gates = torch.cat([g, u], 1).to(TYPES[t]).cuda()
    g, u = gates.double().cpu().split(width, dim=1)
    want = g * torch.special.expit(g) * u
    near(forward(gates, t), want, UNIT[t] * want.abs() + TINY[t] + (9 + (0 if t == "f32" else g.abs() / 2)) * SUM * want.abs())


@pytest.mark.parametrize("t", TYPES)
def test_forward_of_what_is_no_number(t):
    inf, nan = float("inf"), float("nan")
    pairs = [(inf, 1.0), (inf, -2.0), (inf, 0.0), (-inf, 1.0), (nan, 1.0), (1.0, nan), (1.0, inf), (-1.0, inf), (0.0, inf), (-0.0, 3.0), (0.0, -3.0), (-1e4, 1.0),
             (1e4, 0.5), (-1e4, inf), (inf, inf), (-60000.0, -1.0), (60000.0, 0.0)]
    g, u = (torch.tensor(v) for v in zip(*pairs))
    gates = torch.cat([g, u]).view(1, -1).to(TYPES[t]).cuda()
    g, u = gates.double().cpu().view(2, -1)
    want = g * torch.special.expit(g) * u
    limit = torch.finfo(TYPES[t]).max
    assert bool((want.isnan() | want.isinf() | (want.abs() <= limit)).all())
    near(forward(gates, t).view(-1), want, (UNIT[t] + 9 * SUM + (0 if t == "f32" else g.abs() * SUM / 2)) * want.abs())


def backward(g, u, d, t, again=True):
    """Through codes: g and u have to be values that 8 bits hold exactly."""
    rows, width = g.shape
    gates = torch.cat([g, u], 1).float().cuda()
    codes = torch.empty(rows, 2 * width, dtype=torch.uint8, device="cuda")
    scales = torch.empty(rows, 2 * B.checkpoint_blocks(width), dtype=torch.uint8, device="cuda")
    B.tperm_gated_forward(gates.data_ptr(), 2 * width, torch.empty(rows, width, device="cuda").data_ptr(), width, codes.data_ptr(), scales.data_ptr(), rows, width,
                          B.TYPE_F32, stream())
    held = torch.empty(2 * rows, width, device="cuda")
    B.tperm_checkpoint_load(codes.data_ptr(), scales.data_ptr(), held.data_ptr(), width, 2 * rows, width, B.TYPE_F32, stream())
    assert torch.equal(held.view(rows, 2 * width).nan_to_num(7.0), gates.nan_to_num(7.0, 7.0, 7.0))
    d = d.to(TYPES[t]).cuda()
    grad, out = torch.empty(rows, 2 * width, dtype=TYPES[t], device="cuda"), torch.empty(rows, width, dtype=TYPES[t], device="cuda")
    B.tperm_gated_backward(d.data_ptr(), width, codes.data_ptr(), scales.data_ptr(), grad.data_ptr(), 2 * width, out.data_ptr(), width, rows, width, B.TYPES[t], stream())
    return d.double().cpu(), *grad.split(width, dim=1), out


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("width", [32, 64, 31])
def test_backward_far_from_zero(t, width):
    gen = torch.Generator().manual_seed(width)
    steps = torch.tensor([0.5, 1, 4, 8, 16, 30, 40, 52, 60, 72, 80, 88, 96, 104, 0, 2], dtype=torch.float64)
    g = steps[torch.randint(0, 16, (64, width), generator=gen)] * (2.0 * torch.randint(0, 2, (64, width), generator=gen) - 1)
    u = torch.randint(1, 9, (64, width), generator=gen).double() / 4
    d, dg, du, h = backward(g, u, torch.randn(64, width, generator=gen), t)
    p, q = torch.special.expit(g), torch.special.expit(-g)
    more = 0 if t == "f32" else g.abs() / 2
    parts = (d * u * p).abs() * (1 + (g * q).abs())
    want = d * u * p * (1 + g * q)
    near(dg, want, UNIT[t] * want.abs() + TINY[t] + (15 + more * 2) * SUM * parts)
    want = d * g * p
    near(du, want, UNIT[t] * want.abs() + TINY[t] + (9 + more) * SUM * want.abs())
    want = g * p * u
    near(h, want, UNIT[t] * want.abs() + TINY[t] + (9 + more) * SUM * want.abs())


@pytest.mark.parametrize("t", TYPES)
def test_backward_of_what_is_no_number(t):
    inf, nan = float("inf"), float("nan")
    cases = [(nan, 1.0, 1.0), (1.0, nan, 1.0), (1.0, 1.0, nan), (1.0, 1.0, inf), (-1.0, 1.0, -inf), (0.0, 1.0, 1.0), (-88.0, 1.0, inf), (88.0, 1.0, inf), (0.0, 0.0, 1.0),
             (30.0, 0.0, inf)]
    g, u, d = (torch.tensor(v, dtype=torch.float64).view(1, -1) for v in zip(*cases))
    d, dg, du, h = backward(g, u, d, t)
    p, q = torch.special.expit(g), torch.special.expit(-g)
    for got, want, size in ((dg, d * u * p * (1 + g * q), (d * u * p).abs() * (1 + (g * q).abs())), (du, d * g * p, (d * g * p).abs()), (h, g * p * u, (g * p * u).abs())):
        near(got, want, UNIT[t] * want.abs() + TINY[t] + (15 + g.abs()) * SUM * size)

"""Operators of a mixture-of-experts layer on the GPU, against plain implementations in 64 bits.

Tolerances, fixed before the first run, elementwise: u * |result| for the rounding to the element type
(u = 2^-24, 2^-11, 2^-8 for binary32, binary16, bfloat16, and half the smallest subnormal number, 2^-25, for
binary16), and for a sum of n products in binary32 n * 2^-23 times the sum of the products' magnitudes.  What is
moved or counted is compared for equality.
"""
import numpy as np
import pytest

from paper_1705_01598_amd import binding as B

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}
SUM = 2.0 ** -23
GUARD = 119


def stream():
    return torch.cuda.current_stream().cuda_stream


class Matrix:
    """rows x width elements with a stride, an offset (elements) from an aligned start, and sentinels around."""

    def __init__(self, rows, width, dtype, values=None, pad=0, offset=0):
        self.rows, self.width, self.stride = rows, width, width + pad
        self.lead = 64 + offset
        self.buf = torch.full((self.lead + rows * self.stride + 64,), GUARD, dtype=dtype, device="cuda")
        if values is not None:
            self.view().copy_(values.to(dtype))
        self.before = self.buf.clone()

    def view(self):
        return self.buf[self.lead:self.lead + self.rows * self.stride].view(self.rows, self.stride)[:, :self.width] if self.rows else \
            self.buf[:0].view(0, self.width)

    @property
    def ptr(self):
        return self.buf.data_ptr() + self.lead * self.buf.element_size()

    def values(self):
        return self.view().double().cpu()

    def outside_untouched(self):
        now, was = self.buf.clone(), self.before.clone()
        for b in (now, was):
            if self.rows:
                b[self.lead:self.lead + self.rows * self.stride].view(self.rows, self.stride)[:, :self.width] = 0
        return torch.equal(now, was)


def near(got, want, bound):
    got, want = got.double().cpu(), want.double()
    assert got.shape == want.shape
    same = (torch.isnan(got) & torch.isnan(want)) | (got == want)
    bad = ~same & ~((got - want).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:3], want[bad][:3])


def rounding(t, want):
    return UNIT[t] * want.abs() + TINY[t]


# --- the order ---

def plain_order(expert, experts):
    e = np.where((expert < 0) | (expert >= experts), experts, expert).reshape(-1)
    source = np.argsort(e, kind="stable").astype(np.int32)
    place = np.empty_like(source)
    place[source] = np.arange(source.size, dtype=np.int32)
    return np.searchsorted(e[source], np.arange(experts + 1)).astype(np.int32), source, place


def order_on_gpu(expert, tokens, slots, experts):
    n = tokens * slots
    d = torch.from_numpy(np.ascontiguousarray(expert.astype(np.int32).reshape(-1))).cuda()
    out = [torch.full((k + 8,), -7, dtype=torch.int32, device="cuda") for k in (experts + 1, n, n)]
    need = B.expert_sort_workspace_bytes(n, experts)
    ws = torch.full((need // 4 + 1,), -9, dtype=torch.int32, device="cuda")
    B.tperm_expert_sort(d.data_ptr(), tokens, slots, experts, *(o.data_ptr() for o in out), ws.data_ptr(), need, stream())
    torch.cuda.synchronize()
    for o, k in zip(out, (experts + 1, n, n)):
        assert bool((o[k:] == -7).all())
    assert int(ws[-1]) == -9
    return [o[:k].cpu().numpy() for o, k in zip(out, (experts + 1, n, n))]


def routing(rng, tokens, slots, experts, drop=0.0, skew=True):
    p = rng.gamma(0.5, size=experts) + 1e-3 if skew else np.ones(experts)
    e = rng.choice(experts, size=(tokens, slots), p=p / p.sum()).astype(np.int32)
    e[rng.random((tokens, slots)) < drop] = -1
    return e


@pytest.mark.parametrize("tokens,slots,experts,drop", [
    (0, 1, 1, 0), (1, 1, 1, 0), (1, 1, 1, 1.0), (1, 8, 1024, 0), (63, 1, 2, 0), (64, 1, 3, 0.2), (65, 1, 3, 0.2), (257, 3, 64, 0), (1024, 1, 1024, 0.1),
    (1025, 1, 1, 0), (4096, 2, 256, 0.5), (8191, 1, 7, 0), (4097, 2, 7, 0), (8193, 1, 1024, 0.01), (10001, 8, 128, 0.03), (65536, 8, 128, 0), (300000, 2, 1000, 1.0),
    (524289, 1, 2, 0.1), (140000, 8, 901, 0.0), (9001, 64, 1023, 0.0)])
def test_sort(tokens, slots, experts, drop):
    rng = np.random.default_rng(tokens * 31 + slots * 7 + experts)
    e = routing(rng, tokens, slots, experts, drop)
    if drop:
        e[rng.random(e.shape) < 0.01] = experts          # and other numbers that name none
        e[rng.random(e.shape) < 0.01] = 2 ** 31 - 1
        e[rng.random(e.shape) < 0.01] = -2 ** 31
    for got, want in zip(order_on_gpu(e, tokens, slots, experts), plain_order(e, experts)):
        assert np.array_equal(got, want)


def test_sort_of_one_expert_and_of_runs():
    for e in (np.zeros(20000, np.int32), np.repeat(np.arange(40, dtype=np.int32), 500)[::-1].copy(), np.full(20000, 39, np.int32)):
        for got, want in zip(order_on_gpu(e, 20000, 1, 40), plain_order(e, 40)):
            assert np.array_equal(got, want)


class Order:
    def __init__(self, seed, tokens, slots, experts, drop):
        rng = np.random.default_rng(seed)
        self.tokens, self.slots, self.experts, self.rows = tokens, slots, experts, tokens * slots
        maps = plain_order(routing(rng, tokens, slots, experts, drop), experts)
        self.offsets, self.source, self.place = (torch.from_numpy(m).long() for m in maps)
        self.d_offsets, self.d_source, self.d_place = (torch.from_numpy(m).cuda() for m in maps)
        self.used = int(self.offsets[-1])
        self.weights = torch.from_numpy(rng.random((tokens, slots)).astype(np.float32))
        self.d_weights = self.weights.cuda()
        self.g = torch.Generator().manual_seed(seed)

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g)


ROWS = [  # tokens, slots, experts, drop, width, pad, offset
    (1, 1, 1, 0, 1, 0, 0), (1, 4, 8, 0, 16, 0, 0), (5, 2, 3, 0.4, 7, 1, 1), (33, 8, 16, 0.1, 64, 0, 0), (19, 1, 4, 0, 65, 3, 5), (130, 3, 5, 1.0, 72, 8, 8),
    (40, 2, 6, 0.2, 512, 0, 0), (41, 5, 6, 0.2, 1000, 0, 4), (12, 9, 6, 0.2, 1032, 8, 0), (7, 64, 3, 0.1, 2048, 0, 0), (3, 2, 4, 0, 4097, 0, 1), (2, 17, 4, 0, 8200, 0, 0)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,slots,experts,drop,width,pad,offset", ROWS)
def test_rows(t, tokens, slots, experts, drop, width, pad, offset):
    o = Order(tokens + width, tokens, slots, experts, drop)
    dtype = TYPES[t]
    a = dict(tokens=tokens, slots=slots, experts=experts, width=width, dtype=B.TYPES[t], stream=stream())
    used = torch.arange(o.rows) < o.used
    token = o.source // slots
    x = Matrix(tokens, width, dtype, o.randn(tokens, width), pad, offset)
    rows = Matrix(o.rows, width, dtype, o.randn(o.rows, width), pad, offset)
    rows.view()[o.used:] = float("nan")                    # unused rows are not read
    place = o.place.view(tokens, slots)
    w = o.weights.double()
    for weighted in (False, True):
        wp, wd = (o.d_weights.data_ptr(), w) if weighted else (None, torch.ones_like(w))
        out = Matrix(o.rows, width, dtype, None, pad, offset)
        B.tperm_expert_gather(x.ptr, x.stride, o.d_source.data_ptr(), o.d_offsets.data_ptr(), wp, out.ptr, out.stride, **a)
        want = torch.where(used[:, None], wd.view(-1)[o.source, None] * x.values()[token], 0.0)
        near(out.view(), want, rounding(t, want) + SUM * want.abs() if weighted else torch.zeros_like(want))
        assert out.outside_untouched()
        out = Matrix(tokens, width, dtype, None, pad, offset)
        B.tperm_expert_combine(rows.ptr, rows.stride, o.d_place.data_ptr(), o.d_offsets.data_ptr(), wp, out.ptr, out.stride, **a)
        terms = torch.where((place < o.used)[..., None], wd[..., None] * rows.values()[place], 0.0)
        want = terms.sum(1)
        near(out.view(), want, rounding(t, want) + (slots + 1) * SUM * terms.abs().sum(1))
        assert out.outside_untouched()
    grad_rows = Matrix(o.rows, width, dtype, None, pad, offset)
    grad_weights = Matrix(tokens, slots, torch.float32)
    B.tperm_expert_combine_backward(x.ptr, x.stride, rows.ptr, rows.stride, o.d_place.data_ptr(), o.d_offsets.data_ptr(), o.d_weights.data_ptr(),
                                    grad_rows.ptr, grad_rows.stride, grad_weights.ptr, **a)
    want = torch.where(used[:, None], w.view(-1)[o.source, None] * x.values()[token], 0.0)
    near(grad_rows.view(), want, rounding(t, want) + SUM * want.abs())
    products = torch.where((place < o.used)[..., None], x.values()[:, None] * rows.values()[place], 0.0)
    want = products.sum(-1)
    near(grad_weights.view(), want, (width + 1) * SUM * products.abs().sum(-1))
    assert grad_rows.outside_untouched() and grad_weights.outside_untouched()


def test_entries_outside_the_maps_are_unused():
    o = Order(3, 20, 2, 4, 0.0)
    x, rows = Matrix(20, 40, torch.float32, o.randn(20, 40)), Matrix(40, 40, torch.float32, o.randn(40, 40))
    source, place = o.d_source.clone(), o.d_place.clone()
    source[5], source[6], place[9], place[10] = -1, 40, 40, -2 ** 31
    a = dict(tokens=20, slots=2, experts=4, width=40, dtype=B.TYPE_F32, stream=stream())
    out, back = Matrix(40, 40, torch.float32), Matrix(20, 40, torch.float32)
    B.tperm_expert_gather(x.ptr, 40, source.data_ptr(), o.d_offsets.data_ptr(), None, out.ptr, 40, **a)
    want = x.values()[o.source // 2]
    want[5:7] = 0
    near(out.view(), want, torch.zeros_like(want))
    B.tperm_expert_combine(rows.ptr, 40, place.data_ptr(), o.d_offsets.data_ptr(), None, back.ptr, 40, **a)
    terms = rows.values()[o.place.view(20, 2)]
    terms[4, 1] = terms[5, 0] = 0
    near(back.view(), terms.sum(1), 4 * SUM * terms.abs().sum(1))
    grad_rows, grad_w = Matrix(40, 40, torch.float32), Matrix(20, 2, torch.float32)
    B.tperm_expert_combine_backward(x.ptr, 40, rows.ptr, 40, place.data_ptr(), o.d_offsets.data_ptr(), o.d_weights.data_ptr(), grad_rows.ptr, 40, grad_w.ptr, **a)
    assert float(grad_w.view()[4, 1]) == 0 and float(grad_w.view()[5, 0]) == 0
    w = torch.randn(4, 40, 8).cuda()
    product = Matrix(40, 8, torch.float32)
    B.tperm_expert_product(x.ptr, 40, 20, source.data_ptr(), 2, o.d_offsets.data_ptr(), w.data_ptr(), False, product.ptr, 8, 40, 4, 40, 8, B.TYPE_F32, stream())
    assert bool((product.view()[5:7] == 0).all()) and bool((product.view()[4] != 0).any())
    for m in (out, back, grad_rows, grad_w, product):
        assert m.outside_untouched()


def test_gradients_of_rows_against_differences():
    """combine is linear in the rows and in the weights, so a difference over any step is its derivative: the loss
    <combine(rows, weights), grad> along random directions, binary32, steps of the values' own size."""
    o = Order(11, 300, 3, 8, 0.1)
    width = 96
    a = dict(tokens=300, slots=3, experts=8, width=width, dtype=B.TYPE_F32, stream=stream())
    rows, grad = o.randn(o.rows, width).cuda(), o.randn(300, width).cuda()
    out = torch.empty(300, width, device="cuda")

    def loss(rows, weights):
        B.tperm_expert_combine(rows.data_ptr(), width, o.d_place.data_ptr(), o.d_offsets.data_ptr(), weights.data_ptr(), out.data_ptr(), width, **a)
        return float((out.double() * grad.double()).sum())

    g_rows, g_w = torch.empty_like(rows), torch.empty(300, 3, device="cuda")
    B.tperm_expert_combine_backward(grad.data_ptr(), width, rows.data_ptr(), width, o.d_place.data_ptr(), o.d_offsets.data_ptr(), o.d_weights.data_ptr(),
                                    g_rows.data_ptr(), width, g_w.data_ptr(), **a)
    for along_rows in (True, False):
        step = (o.randn(o.rows, width) if along_rows else o.randn(300, 3)).cuda()
        difference = loss(rows + step, o.d_weights) - loss(rows - step, o.d_weights) if along_rows else loss(rows, o.d_weights + step) - loss(rows, o.d_weights - step)
        derivative = 2 * float((step.double() * (g_rows if along_rows else g_w).double()).sum())
        # 300 * 96 results of three terms of size about 4 at most, each 2^-22 off, against grad of size 1
        assert abs(difference - derivative) <= 300 * width * 3 * 4 * 2.0 ** -22


# --- products ---

PRODUCTS = [  # tokens, slots, experts, drop, k, n, pad, offset
    (1, 1, 1, 0, 1, 1, 0, 0), (1, 2, 4, 0, 64, 32, 0, 0), (3, 1, 2, 1.0, 40, 24, 0, 0), (17, 2, 3, 0.2, 33, 65, 1, 1), (100, 2, 4, 0.1, 128, 136, 8, 8),
    (129, 1, 1, 0, 200, 128, 0, 0), (300, 2, 70, 0.3, 72, 264, 0, 0), (257, 3, 2, 0, 515, 130, 0, 3), (700, 2, 5, 0.05, 384, 320, 0, 0), (1300, 1, 3, 0.0, 1024, 520, 16, 0)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens,slots,experts,drop,k,n,pad,offset", PRODUCTS)
def test_products(t, tokens, slots, experts, drop, k, n, pad, offset):
    o = Order(tokens + k + n, tokens, slots, experts, drop)
    dtype = TYPES[t]
    x = Matrix(tokens, k, dtype, o.randn(tokens, k), pad, offset)
    xs = Matrix(o.rows, k, dtype, x.view()[(o.source // slots).cuda()], pad, offset)
    xs.view()[o.used:] = float("inf")
    w = Matrix(experts, k * n, dtype, o.randn(experts, k * n) / k ** 0.5, 0, offset)
    wd = w.values().view(experts, k, n)
    rows = x.values()[o.source // slots]
    want, size = torch.zeros(o.rows, n, dtype=torch.float64), torch.zeros(o.rows, n, dtype=torch.float64)
    for e in range(experts):
        s = slice(int(o.offsets[e]), int(o.offsets[e + 1]))
        want[s], size[s] = rows[s] @ wd[e], rows[s].abs() @ wd[e].abs()
    bound = rounding(t, want) + k * SUM * size
    wt = Matrix(experts, k * n, dtype, w.view().view(experts, k, n).transpose(1, 2).reshape(experts, k * n), 0, offset)
    for gathered in (True, False):
        for k_first in (True, False):
            out = Matrix(o.rows, n, dtype, None, pad, offset)
            m, source = (x, o.d_source.data_ptr()) if gathered else (xs, None)
            B.tperm_expert_product(m.ptr, m.stride, m.rows, source, slots, o.d_offsets.data_ptr(), (wt if k_first else w).ptr, k_first, out.ptr, out.stride,
                                   o.rows, experts, k, n, B.TYPES[t], stream())
            near(out.view(), want, bound)
            assert out.outside_untouched()


def grid(rows, width, g):
    """Values that 8-bit codes hold exactly, whatever the block: largest magnitude 448 * 2^-8 in every 32 neighbours."""
    v = torch.randint(-8, 9, (rows, width), generator=g).float() * 2.0 ** torch.randint(-8, -3, (rows, width), generator=g).float()
    v[:, ::32] = 1.75
    return v


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("held", ["own", "codes"])
@pytest.mark.parametrize("tokens,slots,experts,drop,k,n,pad,offset", PRODUCTS)
def test_weight_gradients(t, held, tokens, slots, experts, drop, k, n, pad, offset):
    o = Order(tokens + k + n, tokens, slots, experts, drop)
    dtype = TYPES[t]
    gathered = (tokens + k) % 2 == 0
    x = Matrix(tokens, k, dtype, grid(tokens, k, o.g), pad, offset)
    grad = Matrix(o.rows, n, dtype, o.randn(o.rows, n), pad, offset)
    grad.view()[o.used:] = float("nan")
    rows = x.values()[o.source // slots]
    if not gathered:
        x = Matrix(o.rows, k, dtype, rows, pad, offset)
    want, size = torch.zeros(experts, k, n, dtype=torch.float64), torch.zeros(experts, k, n, dtype=torch.float64)
    count = torch.zeros(experts, 1, 1, dtype=torch.float64)
    for e in range(experts):
        s = slice(int(o.offsets[e]), int(o.offsets[e + 1]))
        want[e], size[e] = rows[s].T @ grad.values()[s], rows[s].abs().T @ grad.values()[s].abs()
        count[e] = s.stop - s.start
    ptr, stride, scales = x.ptr, x.stride, None
    if held == "codes":
        codes = torch.empty(x.rows * k, dtype=torch.uint8, device="cuda")
        scales = torch.empty(x.rows * B.checkpoint_blocks(k), dtype=torch.uint8, device="cuda")
        B.tperm_checkpoint_store(x.ptr, x.stride, codes.data_ptr(), scales.data_ptr(), x.rows, k, B.TYPES[t], stream())
        ptr, stride = codes.data_ptr(), 0
    for out_t in ("f32", t):
        for k_first in (False, True):
            for accumulate in (False, True):
                start = o.randn(experts, k * n)
                out = Matrix(experts, k * n, TYPES[out_t], start)
                old = out.values().view(experts, n, k).transpose(1, 2) if k_first else out.values().view(experts, k, n)
                B.tperm_expert_weight_gradient(ptr, stride, None if scales is None else scales.data_ptr(), x.rows, o.d_source.data_ptr() if gathered else None,
                                               slots, grad.ptr, grad.stride, o.d_offsets.data_ptr(), out.ptr, B.TYPES[out_t], k_first, accumulate,
                                               o.rows, experts, k, n, B.TYPES[t], stream())
                got = out.view().view(experts, n, k).transpose(1, 2) if k_first else out.view().view(experts, k, n)
                total = want + old if accumulate else want
                near(got, total, rounding(out_t, total) + (count + 1) * SUM * (size + (old.abs() if accumulate else 0)))
                assert out.outside_untouched()


def test_weight_gradient_without_rows_writes_zeros():
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    out = Matrix(3, 40 * 24, torch.float32)
    B.tperm_expert_weight_gradient(None, 40, None, 0, None, 1, None, 24, offsets.data_ptr(), out.ptr, B.TYPE_F32, False, False, 0, 3, 40, 24, B.TYPE_BF16, stream())
    assert bool((out.view() == 0).all()) and out.outside_untouched()


def test_gradients_of_products_against_differences():
    """The product is linear in x and in w: differences of <product(x, w), grad> over steps of any size."""
    o = Order(5, 200, 2, 6, 0.1)
    k, n = 72, 88
    x, w, grad = o.randn(200, k).cuda(), o.randn(6, n, k).cuda() / k ** 0.5, o.randn(o.rows, n).cuda()
    grad[o.used:] = 0

    def loss(x, w):
        out = torch.empty(o.rows, n, device="cuda")
        B.tperm_expert_product(x.data_ptr(), k, 200, o.d_source.data_ptr(), 2, o.d_offsets.data_ptr(), w.data_ptr(), True, out.data_ptr(), n, o.rows, 6, k, n,
                               B.TYPE_F32, stream())
        return float((out.double() * grad.double()).sum())

    g_rows, g_x, g_w = torch.empty(o.rows, k, device="cuda"), torch.empty(200, k, device="cuda"), torch.empty(6, n, k, device="cuda")
    B.tperm_expert_product(grad.data_ptr(), n, o.rows, None, 1, o.d_offsets.data_ptr(), w.data_ptr(), False, g_rows.data_ptr(), k, o.rows, 6, n, k, B.TYPE_F32, stream())
    B.tperm_expert_combine(g_rows.data_ptr(), k, o.d_place.data_ptr(), o.d_offsets.data_ptr(), None, g_x.data_ptr(), k, 200, 2, 6, k, B.TYPE_F32, stream())
    B.tperm_expert_weight_gradient(x.data_ptr(), k, None, 200, o.d_source.data_ptr(), 2, grad.data_ptr(), n, o.d_offsets.data_ptr(), g_w.data_ptr(), B.TYPE_F32,
                                   True, False, o.rows, 6, k, n, B.TYPE_F32, stream())
    for at, g, f in ((x, g_x, lambda d: loss(x + d, w) - loss(x - d, w)), (w, g_w, lambda d: loss(x, w + d) - loss(x, w - d))):
        step = o.randn(*at.shape).cuda()
        derivative = 2 * float((step.double() * g.double()).sum())
        # 400 * 88 results, each a sum of 72 products of size 4 / sqrt(72) at most on average, 72 * 2^-23 off
        assert abs(f(step) - derivative) <= o.rows * n * 72 * 0.5 * 72 * 2.0 ** -23


# --- 8 bits ---

def plain_codes(x):
    """(values, scales) of rows of doubles: every finite value to the nearest number of the 8-bit type, ties to even."""
    rows, width = x.shape
    blocks = -(-width // 32)
    values, scales = np.zeros_like(x), np.zeros((rows, blocks), np.uint8)
    for b in range(blocks):
        v = x[:, 32 * b:32 * b + 32]
        most = np.where(np.isfinite(v), np.abs(v), 0).max(1)
        s = np.full(rows, -117)
        for i in range(rows):
            while s[i] < 120 and most[i] > 448.0 * 2.0 ** s[i]:
                s[i] += 1
        q = v / 2.0 ** s[:, None].astype(np.float64)
        with np.errstate(divide="ignore", invalid="ignore"):
            step = 2.0 ** np.maximum(np.floor(np.log2(np.abs(np.where(q == 0, 1, q)))) - 3, -9)
        r = np.rint(q / step) * step                          # rint: ties to even
        values[:, 32 * b:32 * b + 32] = np.where(np.isfinite(v), r, np.nan) * 2.0 ** s[:, None].astype(np.float64)
        scales[:, b] = s + 127
    return values, scales


WIDTHS = [(1, 1, 0, 0), (3, 31, 0, 0), (5, 32, 0, 1), (4, 33, 7, 0), (9, 64, 0, 0), (7, 100, 4, 4), (2, 1000, 0, 0), (3, 1025, 1, 0), (33, 256, 8, 8)]


def loud(g, rows, width, t):
    x = torch.randn(rows, width, generator=g) * 2.0 ** torch.randint(-12, 9, (rows, 1), generator=g).float()
    x[torch.rand(rows, width, generator=g) < 0.05] *= 30
    x[torch.rand(rows, width, generator=g) < 0.05] = 0
    x = x.to(TYPES[t])
    flat = x.view(-1)
    for i, v in enumerate((float("inf"), float("nan"), float("-inf"), 448.0, 464.0, 480.0, 1.75, 1.7578125, -0.0)):
        if flat.numel() > 40 * i + 11:
            flat[40 * i + 11] = v
    return x


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,width,pad,offset", WIDTHS)
def test_checkpoint(t, rows, width, pad, offset):
    g = torch.Generator().manual_seed(rows * width)
    x = Matrix(rows, width, TYPES[t], loud(g, rows, width, t), pad, offset)
    codes, scales = Matrix(rows, width, torch.uint8), Matrix(rows, B.checkpoint_blocks(width), torch.uint8)
    B.tperm_checkpoint_store(x.ptr, x.stride, codes.ptr, scales.ptr, rows, width, B.TYPES[t], stream())
    want, want_scales = plain_codes(x.values().numpy())
    assert np.array_equal(scales.view().cpu().numpy(), want_scales)
    held = codes.view().view(torch.float8_e4m3fn).double().cpu().numpy() * 2.0 ** (np.repeat(want_scales, 32, 1)[:, :width].astype(np.float64) - 127)
    assert np.array_equal(held, want, equal_nan=True)
    assert codes.outside_untouched() and scales.outside_untouched()
    for out_t in TYPES:
        out = Matrix(rows, width, TYPES[out_t], None, pad, offset)
        B.tperm_checkpoint_load(codes.ptr, scales.ptr, out.ptr, out.stride, rows, width, B.TYPES[out_t], stream())
        limit = float(torch.finfo(TYPES[out_t]).max)
        back = torch.from_numpy(np.clip(want, -limit, limit))
        near(out.view(), back, torch.zeros_like(back) if out_t == "f32" else rounding(out_t, back))
        assert out.outside_untouched()
    finite = np.isfinite(x.values().numpy())
    error = np.abs(want - x.values().numpy())[finite]
    step = (2.0 ** (np.repeat(want_scales, 32, 1)[:, :width].astype(np.float64) - 127))[finite]
    assert np.all(error <= np.maximum(2.0 ** -4 * np.abs(x.values().numpy()[finite]), 2.0 ** -10 * step))


@pytest.mark.parametrize("value", [0.0, 2.0 ** -149, 2.0 ** -126, 1e-38, 3.3e38, 2.0 ** 127, float(np.finfo(np.float32).max)])
def test_checkpoint_at_the_ends_of_the_range(value):
    x = torch.full((2, 70), value, dtype=torch.float32)
    x[1, 1::2] *= -0.37
    d = x.cuda()
    codes, scales = torch.empty(2, 70, dtype=torch.uint8, device="cuda"), torch.empty(2, 3, dtype=torch.uint8, device="cuda")
    B.tperm_checkpoint_store(d.data_ptr(), 70, codes.data_ptr(), scales.data_ptr(), 2, 70, B.TYPE_F32, stream())
    out = torch.empty_like(d)
    B.tperm_checkpoint_load(codes.data_ptr(), scales.data_ptr(), out.data_ptr(), 70, 2, 70, B.TYPE_F32, stream())
    want, want_scales = plain_codes(x.double().numpy())
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    limit = float(np.finfo(np.float32).max)
    near(out, torch.from_numpy(np.clip(want, -limit, limit)), torch.zeros(2, 70, dtype=torch.float64))


def test_largest_binary16_values_stay_finite():
    x = torch.full((1, 64), 65504.0, dtype=torch.float16, device="cuda")
    codes, scales, out = torch.empty(1, 64, dtype=torch.uint8, device="cuda"), torch.empty(1, 2, dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    B.tperm_checkpoint_store(x.data_ptr(), 64, codes.data_ptr(), scales.data_ptr(), 1, 64, B.TYPE_F16, stream())
    B.tperm_checkpoint_load(codes.data_ptr(), scales.data_ptr(), out.data_ptr(), 64, 1, 64, B.TYPE_F16, stream())
    assert bool((out == 65504).all())


def silu_parts(g):
    p = torch.special.expit(g)
    return p, g * p


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,width,pad,offset", WIDTHS)
def test_gated(t, rows, width, pad, offset):
    gen = torch.Generator().manual_seed(rows + width)
    gates = Matrix(rows, 2 * width, TYPES[t], torch.randn(rows, 2 * width, generator=gen) * 4, pad, offset)
    blocks = B.checkpoint_blocks(width)
    v = gates.values()
    g, u = v[:, :width], v[:, width:]
    p, silu = silu_parts(g)
    want = silu * u
    for keep in (True, False):
        out = Matrix(rows, width, TYPES[t], None, pad, offset)
        codes, scales = Matrix(rows, 2 * width, torch.uint8), Matrix(rows, 2 * blocks, torch.uint8)
        B.tperm_gated_forward(gates.ptr, gates.stride, out.ptr, out.stride, codes.ptr if keep else None, scales.ptr if keep else None, rows, width,
                              B.TYPES[t], stream())
        # exp2 of an argument of size 1.45 |g| rounded to 24 bits, then four operations of 2^-23 each
        near(out.view(), want, rounding(t, want) + (g.abs() + 8) * SUM * want.abs())
        assert out.outside_untouched() and codes.outside_untouched() and scales.outside_untouched()
        if keep:
            for part, c0, s0 in ((g, 0, 0), (u, width, blocks)):
                values, biased = plain_codes(part.numpy())
                assert np.array_equal(scales.view()[:, s0:s0 + blocks].cpu().numpy(), biased)
                held = codes.view()[:, c0:c0 + width].contiguous().view(torch.float8_e4m3fn).double().cpu().numpy()
                assert np.array_equal(held * 2.0 ** (np.repeat(biased, 32, 1)[:, :width].astype(np.float64) - 127), values)
            kept = codes, scales
    g, u = (torch.from_numpy(plain_codes(part.numpy())[0]) for part in (g, u))
    p, silu = silu_parts(g)
    grad = Matrix(rows, width, TYPES[t], torch.randn(rows, width, generator=gen), pad, offset)
    d = grad.values()
    for again in (True, False):
        out, grad_gates = Matrix(rows, width, TYPES[t], None, pad, offset), Matrix(rows, 2 * width, TYPES[t], None, pad, offset)
        B.tperm_gated_backward(grad.ptr, grad.stride, kept[0].ptr, kept[1].ptr, grad_gates.ptr, grad_gates.stride, out.ptr if again else None, out.stride,
                               rows, width, B.TYPES[t], stream())
        dg, du, h = d * u * p * (1 + g * (1 - p)), d * silu, silu * u
        near(grad_gates.view()[:, :width], dg, rounding(t, dg) + (g.abs() + 12) * SUM * (d * u * p).abs() * (1 + g.abs()))
        near(grad_gates.view()[:, width:], du, rounding(t, du) + (g.abs() + 8) * SUM * du.abs())
        if again:
            near(out.view(), h, rounding(t, h) + (g.abs() + 8) * SUM * h.abs())
        assert grad_gates.outside_untouched() and out.outside_untouched()


def test_gated_gradient_against_differences():
    """Central differences of tperm_gated_forward in binary32, at values that 8 bits hold exactly."""
    gen = torch.Generator().manual_seed(2)
    rows, width, h = 64, 96, 2.0 ** -6
    v = torch.cat([grid(rows, width, gen), grid(rows, width, gen)], 1).cuda()
    grad = torch.randn(rows, width, generator=gen).cuda()
    codes, scales = torch.empty(rows, 2 * width, dtype=torch.uint8, device="cuda"), torch.empty(rows, 6, dtype=torch.uint8, device="cuda")

    def forward(v, keep=False):
        out = torch.empty(rows, width, device="cuda")
        B.tperm_gated_forward(v.data_ptr(), 2 * width, out.data_ptr(), width, codes.data_ptr() if keep else None, scales.data_ptr() if keep else None, rows, width,
                              B.TYPE_F32, stream())
        return out.double()

    forward(v, True)
    got = torch.empty(rows, 2 * width, device="cuda")
    B.tperm_gated_backward(grad.data_ptr(), width, codes.data_ptr(), scales.data_ptr(), got.data_ptr(), 2 * width, None, width, rows, width, B.TYPE_F32, stream())
    for part in (0, 1):
        step = torch.zeros_like(v)
        step[:, part * width:(part + 1) * width] = h
        difference = (forward(v + step) - forward(v - step)) / (2 * h) * grad.double()
        # |silu'''| < 1 and |u| <= 1.75: h^2 / 6 * 1.75; values of size 4 at most that are 12 * 2^-23 off, over h
        bound = (h * h / 6 * 1.75 + 12 * 2.0 ** -23 * 4 / h) * grad.double().abs() + 1e-6
        assert bool(((difference - got[:, part * width:(part + 1) * width].double()).abs() <= bound).all())


# --- streams, graphs, repetition ---

def test_same_bits_on_another_stream_and_in_a_graph():
    o = Order(8, 500, 2, 12, 0.1)
    k, n = 256, 192
    x, w = o.randn(500, k).cuda().bfloat16(), o.randn(12, 2 * n, k).cuda().bfloat16()
    rows = torch.empty(o.rows, 2 * n, dtype=torch.bfloat16, device="cuda")
    h, back = torch.empty(o.rows, n, dtype=torch.bfloat16, device="cuda"), torch.empty(500, n, dtype=torch.bfloat16, device="cuda")
    codes, scales = torch.empty(o.rows, 2 * n, dtype=torch.uint8, device="cuda"), torch.empty(o.rows, 12, dtype=torch.uint8, device="cuda")
    grad_w = torch.empty(12, k, 2 * n, device="cuda")
    expert = torch.from_numpy(routing(np.random.default_rng(8), 500, 2, 12, 0.1)).cuda()
    maps = [torch.empty(c, dtype=torch.int32, device="cuda") for c in (13, o.rows, o.rows)]

    def all_calls():
        s = stream()
        off, src, plc = (m.data_ptr() for m in maps)
        B.tperm_expert_sort(expert.data_ptr(), 500, 2, 12, off, src, plc, None, 0, s)
        B.tperm_expert_product(x.data_ptr(), k, 500, src, 2, off, w.data_ptr(), True, rows.data_ptr(), 2 * n, o.rows, 12, k, 2 * n, B.TYPE_BF16, s)
        B.tperm_gated_forward(rows.data_ptr(), 2 * n, h.data_ptr(), n, codes.data_ptr(), scales.data_ptr(), o.rows, n, B.TYPE_BF16, s)
        B.tperm_expert_combine(h.data_ptr(), n, plc, off, o.d_weights.data_ptr(), back.data_ptr(), n, 500, 2, 12, n, B.TYPE_BF16, s)
        B.tperm_expert_weight_gradient(x.data_ptr(), k, None, 500, src, 2, rows.data_ptr(), 2 * n, off, grad_w.data_ptr(), B.TYPE_F32, False, False, o.rows, 12, k, 2 * n,
                                       B.TYPE_BF16, s)

    outputs = [*maps, rows, h, codes, scales, back, grad_w]
    all_calls()
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]

    def check():
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outputs, want))
        for t in outputs:
            t.view(torch.uint8).fill_(0x55)
        torch.cuda.synchronize()

    check()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        all_calls()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_calls()
    for _ in range(4):
        graph.replay()
        check()
        all_calls()
        check()


def test_rows_beyond_32_bits():
    """Rows whose bytes lie beyond 4 GiB: a wide stride over a small number of them."""
    tokens, width, stride = 40, 256, 1 << 26
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough memory")
    o = Order(9, tokens, 1, 3, 0.1)
    far = torch.empty(tokens * stride, dtype=torch.bfloat16, device="cuda")
    x = o.randn(tokens, width).bfloat16().cuda()
    rows = far.as_strided((tokens, width), (stride, 1))
    a = dict(tokens=tokens, slots=1, experts=3, width=width, dtype=B.TYPE_BF16, stream=stream())
    B.tperm_expert_gather(x.data_ptr(), width, o.d_source.data_ptr(), o.d_offsets.data_ptr(), None, far.data_ptr(), stride, **a)
    want = torch.where((torch.arange(tokens) < o.used)[:, None], x.cpu()[o.source], torch.zeros(1, dtype=torch.bfloat16))
    assert torch.equal(rows.cpu(), want)
    w = o.randn(3, width, 64).bfloat16().cuda()
    out = torch.empty(tokens, 64, dtype=torch.bfloat16, device="cuda")
    B.tperm_expert_product(far.data_ptr(), stride, tokens, None, 1, o.d_offsets.data_ptr(), w.data_ptr(), False, out.data_ptr(), 64, tokens, 3, width, 64, B.TYPE_BF16, stream())
    grad_w = torch.empty(3, width, 64, device="cuda")
    B.tperm_expert_weight_gradient(far.data_ptr(), stride, None, tokens, None, 1, out.data_ptr(), 64, o.d_offsets.data_ptr(), grad_w.data_ptr(), B.TYPE_F32, False, False,
                                   tokens, 3, width, 64, B.TYPE_BF16, stream())
    for e in range(3):
        s = slice(int(o.offsets[e]), int(o.offsets[e + 1]))
        r = want[s].double()
        exact = r @ w[e].double().cpu()
        near(out[s], exact, rounding("bf16", exact) + width * SUM * (r.abs() @ w[e].double().cpu().abs()))
        d = out[s].double().cpu()
        near(grad_w[e], r.T @ d, (s.stop - s.start + 1) * SUM * (r.abs().T @ d.abs()) + 2.0 ** -126)

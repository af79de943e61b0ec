"""The experts' products in tiles of every size, elementwise against products in 64 bits, and the operators where their
tensors are large.

tperm_expert_tile says which tile a call takes, and every case asserts its own, so that sizes follow when the
choice changes.  Tolerances as in test_gpu_experts: the rounding to the element type, and for a sum of n
products in binary32 n * 2^-23 times the sum of their magnitudes."""
import pytest

from paper_1705_01598_amd import binding as B

torch = pytest.importorskip("torch")
from test_gpu_experts import SUM, TYPES, Matrix, Order, grid, rounding, stream  # noqa: E402

pytestmark = pytest.mark.gpu


def near(got, want, bound):
    """As there, on the GPU."""
    got = got.double()
    assert got.shape == want.shape
    bad = ~((torch.isnan(got) & torch.isnan(want)) | (got == want) | ((got - want).abs() <= bound))
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist(), got[bad][:3].tolist(), want[bad][:3].tolist())


WRONG = (-1, 2 ** 31 - 1, -2 ** 31)


def spoilt(source, slots, x_rows):
    """Some entries of the map outside the rows that there are; (map, which)."""
    bad = torch.zeros(source.numel(), dtype=torch.bool, device="cuda")
    source = source.clone()
    for i, at in enumerate(range(3, source.numel(), 61)):
        source[at] = (*WRONG, x_rows * slots)[i % 4]
        bad[at] = True
    return source, bad


# tile, types, tokens, slots, experts, k, n
PRODUCTS = {"small": ((128, 128), ("f16", "bf16"), 521, 2, 8, 264, 1032), "wide": ((256, 256), ("f16", "bf16"), 1201, 2, 8, 328, 2056),
            "narrow": ((128, 64), ("f32",), 560, 2, 16, 100, 4100), "split": ((64, 64), ("f16", "bf16", "f32"), 333, 2, 8, 520, 264)}


@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("name,t", [(name, t) for name, case in PRODUCTS.items() for t in case[1]])
def test_product_tiles(name, aligned, t):
    tile, _, tokens, slots, experts, k, n = PRODUCTS[name]
    pad, offset = (0, 0) if aligned else (3, 1)
    k, n = (k, n) if aligned else (k + 5, n + 3)
    o = Order(tokens + n, tokens, slots, experts, 0.05)
    dtype = TYPES[t]
    assert B.tperm_expert_tile(False, B.TYPES[t], False, o.rows, experts, k, n) == tile
    x = Matrix(tokens, k, dtype, o.randn(tokens, k), pad, offset)
    token = (o.source // slots).cuda()
    xs = Matrix(o.rows, k, dtype, x.view()[token], pad, offset)
    xs.view()[o.used:] = float("inf")
    w = Matrix(experts, k * n, dtype, o.randn(experts, k * n) / k ** 0.5, 0, offset)
    wt = Matrix(experts, k * n, dtype, w.view().view(experts, k, n).transpose(1, 2).reshape(experts, k * n), 0, offset)
    rows, wd = x.view().double()[token], w.view().double().view(experts, k, n)
    want, size = torch.zeros(o.rows, n, dtype=torch.float64, device="cuda"), torch.zeros(o.rows, n, dtype=torch.float64, device="cuda")
    for e in range(experts):
        s = slice(int(o.offsets[e]), int(o.offsets[e + 1]))
        want[s], size[s] = rows[s] @ wd[e], rows[s].abs() @ wd[e].abs()
    bound = rounding(t, want) + k * SUM * size
    source, bad = spoilt(o.d_source, slots, tokens)
    for m, maps, expected in ((x, o.d_source, want), (xs, None, want), (x, source, torch.where(bad[:, None], 0.0, want))):
        for k_first in (True, False):
            out = Matrix(o.rows, n, dtype, None, pad, offset)
            B.tperm_expert_product(m.ptr, m.stride, m.rows, None if maps is None else maps.data_ptr(), slots, o.d_offsets.data_ptr(), (wt if k_first else w).ptr, k_first,
                                   out.ptr, out.stride, o.rows, experts, k, n, B.TYPES[t], stream())
            near(out.view(), expected, bound)
            assert out.outside_untouched()


# tile, types, tokens, slots, experts, k, n
GRADIENTS = {"small": ((128, 128), ("f16", "bf16"), 333, 2, 8, 704, 696), "wide": ((256, 256), ("f16", "bf16"), 411, 2, 8, 1040, 1048),
             "narrow": ((128, 64), ("f32",), 211, 2, 8, 1028, 1032), "split": ((64, 64), ("f16", "bf16", "f32"), 333, 2, 5, 304, 272)}


@pytest.mark.parametrize("held", ["own", "codes"])
@pytest.mark.parametrize("aligned", [True, False])
@pytest.mark.parametrize("name,t", [(name, t) for name, case in GRADIENTS.items() for t in case[1]])
def test_gradient_tiles(name, aligned, held, t):
    tile, _, tokens, slots, experts, k, n = GRADIENTS[name]
    pad, offset = (0, 0) if aligned else (3, 1)
    k, n = (k // 16 * 16 if held == "codes" else k, n) if aligned else (k + 5, n + 3)
    o = Order(tokens + n, tokens, slots, experts, 0.05)
    dtype = TYPES[t]
    token = (o.source // slots).cuda()
    x = Matrix(tokens, k, dtype, grid(tokens, k, o.g), pad, offset)
    xs = Matrix(o.rows, k, dtype, x.view()[token], pad, offset)
    grad = Matrix(o.rows, n, dtype, o.randn(o.rows, n), pad, offset)
    source, bad = spoilt(o.d_source, slots, tokens)
    rows, d = x.view().double()[token], grad.view().double()
    grad.view()[o.used:] = float("nan")
    codes = {}
    for m in (x, xs) if held == "codes" else ():
        c = torch.empty(m.rows * k, dtype=torch.uint8, device="cuda"), torch.empty(m.rows * B.checkpoint_blocks(k), dtype=torch.uint8, device="cuda")
        B.tperm_checkpoint_store(m.ptr, m.stride, c[0].data_ptr(), c[1].data_ptr(), m.rows, k, B.TYPES[t], stream())
        codes[m] = c
    for m, maps in ((x, o.d_source), (xs, None), (x, source)):
        there = torch.where(bad[:, None], 0.0, rows) if maps is source else rows
        want, size = torch.empty(experts, k, n, dtype=torch.float64, device="cuda"), torch.empty(experts, k, n, dtype=torch.float64, device="cuda")
        count = torch.empty(experts, 1, 1, dtype=torch.float64, device="cuda")
        for e in range(experts):
            s = slice(int(o.offsets[e]), int(o.offsets[e + 1]))
            want[e], size[e], count[e] = there[s].t() @ d[s], there[s].abs().t() @ d[s].abs(), s.stop - s.start
        for k_first in (False, True):
            assert B.tperm_expert_tile(True, B.TYPES[t], k_first, o.rows, experts, k, n) == tile
            for out_t, accumulate in (("f32", False), ("f32", True), (t, False), (t, True)):
                out = Matrix(experts, k * n, TYPES[out_t], o.randn(experts, k * n), 0, 0 if aligned else 1)
                old = out.view().double()
                old = old.view(experts, n, k).transpose(1, 2) if k_first else old.view(experts, k, n)
                ptr, stride, scales = (m.ptr, m.stride, None) if held == "own" else (codes[m][0].data_ptr(), 0, codes[m][1].data_ptr())
                B.tperm_expert_weight_gradient(ptr, stride, scales, m.rows, None if maps is None else maps.data_ptr(), slots, grad.ptr, grad.stride, o.d_offsets.data_ptr(),
                                               out.ptr, B.TYPES[out_t], k_first, accumulate, o.rows, experts, k, n, B.TYPES[t], stream())
                got = out.view().view(experts, n, k).transpose(1, 2) if k_first else out.view().view(experts, k, n)
                total, extra = (want + old, old.abs()) if accumulate else (want, 0)
                near(got, total, rounding(out_t, total) + (count + 1) * SUM * (size + extra))
                assert out.outside_untouched()


def test_a_map_entry_outside_its_range_adds_nothing_to_a_small_gradient():
    """Row r of a call with one row of x to a row and none else, all types: no row of x, so zeros."""
    for t, dtype in TYPES.items():
        x, grad = torch.ones(4, 32, dtype=dtype, device="cuda"), torch.ones(4, 24, dtype=dtype, device="cuda")
        source = torch.tensor([0, -1, 4, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
        offsets = torch.tensor([0, 1, 4], dtype=torch.int32, device="cuda")
        out = torch.full((2, 32, 24), 7.0, device="cuda")
        B.tperm_expert_weight_gradient(x.data_ptr(), 32, None, 4, source.data_ptr(), 1, grad.data_ptr(), 24, offsets.data_ptr(), out.data_ptr(), B.TYPE_F32, False, False,
                                       4, 2, 32, 24, B.TYPES[t], stream())
        assert bool((out[0] == 1).all()) and bool((out[1] == 0).all())


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("k", [256, 255])
@pytest.mark.parametrize("k_first", [False, True])
def test_gradient_multiplies_what_checkpoint_load_gives(t, k, k_first):
    """Every code at every scale, one row of an expert times ones: the value itself, whatever way the codes take."""
    rows, n, dtype = 247 - 10 + 1, 16, TYPES[t]
    codes = torch.arange(256, dtype=torch.uint8)[:k].repeat(rows, 1).contiguous().cuda()
    scales = torch.arange(10, 248, dtype=torch.uint8)[:, None].repeat(1, 8).contiguous().cuda()
    held = torch.empty(rows, k, dtype=dtype, device="cuda")
    B.tperm_checkpoint_load(codes.data_ptr(), scales.data_ptr(), held.data_ptr(), k, rows, k, B.TYPES[t], stream())
    grad, offsets = torch.ones(rows, n, dtype=dtype, device="cuda"), torch.arange(rows + 1, dtype=torch.int32, device="cuda")
    out = torch.empty(rows, k * n, device="cuda")
    B.tperm_expert_weight_gradient(codes.data_ptr(), 0, scales.data_ptr(), rows, None, 1, grad.data_ptr(), n, offsets.data_ptr(), out.data_ptr(), B.TYPE_F32, k_first, False,
                                   rows, rows, k, n, B.TYPES[t], stream())
    out = out.view(rows, n, k) if k_first else out.view(rows, k, n).transpose(1, 2)
    want = held.float()[:, None].expand(rows, n, k)
    assert torch.equal(out.nan_to_num(7.0), want.nan_to_num(7.0)) and torch.equal(out.isnan(), want.isnan())


# --- rows that are read past the caches, and large tensors ---

@pytest.mark.parametrize("t,tokens,slots,width", [("bf16", 9001, 3, 2048), ("f32", 6007, 2, 2052)])
def test_rows_that_fill_a_third_of_the_memory_side_cache(t, tokens, slots, width):
    o = Order(tokens, tokens, slots, 16, 0.05)
    dtype = TYPES[t]
    assert o.rows * width * dtype.itemsize * 3 > 256 << 20
    a = dict(tokens=tokens, slots=slots, experts=16, width=width, dtype=B.TYPES[t], stream=stream())
    rows, grad = torch.randn(o.rows, width, device="cuda").to(dtype), torch.randn(tokens, width, device="cuda").to(dtype)
    rows[o.used:] = float("nan")
    place, w = o.place.view(tokens, slots).cuda(), o.d_weights.double()
    there = place < o.used
    out = torch.empty(tokens, width, dtype=dtype, device="cuda")
    B.tperm_expert_combine(rows.data_ptr(), width, o.d_place.data_ptr(), o.d_offsets.data_ptr(), o.d_weights.data_ptr(), out.data_ptr(), width, **a)
    want, size = torch.zeros(2, tokens, width, dtype=torch.float64, device="cuda")
    grad_rows, grad_w = torch.empty_like(rows), torch.empty(tokens, slots, device="cuda")
    B.tperm_expert_combine_backward(grad.data_ptr(), width, rows.data_ptr(), width, o.d_place.data_ptr(), o.d_offsets.data_ptr(), o.d_weights.data_ptr(),
                                    grad_rows.data_ptr(), width, grad_w.data_ptr(), **a)
    d = grad.double()
    for s in range(slots):
        term = torch.where(there[:, s, None], rows[place[:, s]].double(), 0.0)
        want += w[:, s, None] * term
        size += (w[:, s, None] * term).abs()
        near(grad_w[:, s], (d * term).sum(1), (width + 1) * SUM * (d * term).abs().sum(1))
        back = torch.where(there[:, s, None], w[:, s, None] * d, 0.0)
        near(grad_rows[place[:, s]], back, rounding(t, back) + SUM * back.abs())
    near(out, want, rounding(t, want) + (slots + 1) * SUM * size)


def room(gib):
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip("not enough memory")


def test_more_workgroups_than_one_dimension_of_a_grid_takes():
    """2^22 workgroups lie along the first dimension, further ones along the second; thread numbers beyond 2^31 are
    divided in 64 bits.  Values are exact, so results are compared for equality."""
    room(24)
    # gather: 64 rows a workgroup
    tokens, slots = (1 << 23) + 1, 32
    rows = tokens * slots
    source = torch.arange(rows - 1, -1, -1, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, rows - 5], dtype=torch.int32, device="cuda")
    x = torch.arange(tokens, device="cuda").remainder(251).to(torch.bfloat16).view(tokens, 1)
    out = torch.full((rows, 1), 3.0, dtype=torch.bfloat16, device="cuda")
    B.tperm_expert_gather(x.data_ptr(), 1, source.data_ptr(), offsets.data_ptr(), None, out.data_ptr(), 1, tokens, slots, 1, 1, B.TYPE_BF16, stream())
    assert torch.equal(out[:rows - 5].view(-1), x.view(-1).flip(0).repeat_interleave(slots)[:rows - 5]) and not bool(out[rows - 5:].any())
    del source, x, out
    # 8 bits: 64 rows a workgroup, 4 threads a row
    rows = (1 << 29) + 3
    x = (torch.arange(rows, dtype=torch.int32, device="cuda").remainder(15) + 1).to(torch.bfloat16)
    codes, scales, back = (torch.empty(rows, dtype=d, device="cuda") for d in (torch.uint8, torch.uint8, torch.bfloat16))
    B.tperm_checkpoint_store(x.data_ptr(), 1, codes.data_ptr(), scales.data_ptr(), rows, 1, B.TYPE_BF16, stream())
    B.tperm_checkpoint_load(codes.data_ptr(), scales.data_ptr(), back.data_ptr(), 1, rows, 1, B.TYPE_BF16, stream())
    assert torch.equal(back, x)
    del codes, scales, back
    # product: 256 rows a workgroup
    rows = (1 << 30) + 5
    x = (torch.arange(rows, dtype=torch.int32, device="cuda").remainder(15) + 1).to(torch.bfloat16)
    ends = [0, 77, rows // 2, rows - 9]
    offsets, w = torch.tensor(ends, dtype=torch.int32, device="cuda"), torch.tensor([2.0, -1.0, 0.5], dtype=torch.bfloat16, device="cuda")
    out = torch.full((rows,), 3.0, dtype=torch.bfloat16, device="cuda")
    B.tperm_expert_product(x.data_ptr(), 1, rows, None, 1, offsets.data_ptr(), w.data_ptr(), False, out.data_ptr(), 1, rows, 3, 1, 1, B.TYPE_BF16, stream())
    for e in range(3):
        assert torch.equal(out[ends[e]:ends[e + 1]], x[ends[e]:ends[e + 1]] * w[e])
    assert not bool(out[ends[3]:].any())


def test_operands_beyond_4_gib_without_a_map():
    """Dense rows that are reached from a stage's first one: the last expert's lie beyond 2^32 bytes."""
    room(24)
    before, last, wide, narrow = (1 << 22) + 1, 300, 512, 64
    rows = before + last
    offsets = torch.tensor([0, before, rows], dtype=torch.int32, device="cuda")
    far, thin = torch.randn(rows, wide, device="cuda", dtype=torch.bfloat16), torch.randn(rows, narrow, device="cuda", dtype=torch.bfloat16)
    f, t = far[before:].double(), thin[before:].double()
    out = torch.empty(2, wide, narrow, device="cuda")
    args = (offsets.data_ptr(), out.data_ptr(), B.TYPE_F32, False, False, rows, 2)
    B.tperm_expert_weight_gradient(far.data_ptr(), wide, None, rows, None, 1, thin.data_ptr(), narrow, *args, wide, narrow, B.TYPE_BF16, stream())
    near(out[1], f.t() @ t, (last + 1) * SUM * (f.abs().t() @ t.abs()))
    out = out.view(2, narrow, wide)
    B.tperm_expert_weight_gradient(thin.data_ptr(), narrow, None, rows, None, 1, far.data_ptr(), wide, *args, narrow, wide, B.TYPE_BF16, stream())
    near(out[1], t.t() @ f, (last + 1) * SUM * (t.abs().t() @ f.abs()))
    w = (torch.randn(2, wide, narrow, device="cuda") / 16).bfloat16()
    back = torch.empty(rows, narrow, dtype=torch.bfloat16, device="cuda")
    B.tperm_expert_product(far.data_ptr(), wide, rows, None, 1, offsets.data_ptr(), w.data_ptr(), False, back.data_ptr(), narrow, rows, 2, wide, narrow, B.TYPE_BF16, stream())
    want = f @ w[1].double()
    near(back[before:], want, rounding("bf16", want) + wide * SUM * (f.abs() @ w[1].double().abs()))
    B.tperm_expert_product(thin.data_ptr(), narrow, rows, None, 1, offsets.data_ptr(), w.data_ptr(), True, far.data_ptr(), wide, rows, 2, narrow, wide, B.TYPE_BF16, stream())
    want = t @ w[1].double().t()
    near(far[before:], want, rounding("bf16", want) + narrow * SUM * (t.abs() @ w[1].double().abs().t()))
    del far
    wide = 1024
    codes = torch.randint(0, 0x78, (rows, wide), dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, wide // 32), 120, dtype=torch.uint8, device="cuda")
    c = codes[before:].view(torch.float8_e4m3fn).double() * 2.0 ** -7
    out = torch.empty(2, wide, narrow, device="cuda")
    B.tperm_expert_weight_gradient(codes.data_ptr(), 0, scales.data_ptr(), rows, None, 1, thin.data_ptr(), narrow, offsets.data_ptr(), out.data_ptr(), B.TYPE_F32, False,
                                   False, rows, 2, wide, narrow, B.TYPE_BF16, stream())
    near(out[1], c.t() @ t, (last + 1) * SUM * (c.abs().t() @ t.abs()))

"""Router and matrices in 4 bits at sizes whose thread numbers, workgroups or offsets pass 32 bits or one dimension of a grid.  Inputs are such that results are known
exactly, for every row."""
import pytest

from paper_1705_01598_amd import binding as B

torch = pytest.importorskip("torch")
from test_gpu_experts import stream  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def memory_goes_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t,dtype", [("bf16", torch.bfloat16), ("f32", torch.float32)])
def test_four_bits_of_more_threads_than_31_bits_count(t, dtype):
    """Rows of one element, four threads or more each: +-1 and +-1.5 times powers of two, which 4 bits hold."""
    rows = (1 << 29) + 1000003
    x = torch.empty(rows, dtype=dtype, device="cuda")
    for first in range(0, rows, 1 << 27):
        r = torch.arange(first, min(first + (1 << 27), rows), dtype=torch.int32, device="cuda")
        x[first:first + (1 << 27)] = (1 - r % 2 * 2) * (1 + r // 2 % 2 * 0.5) * torch.exp2((r % 61 - 30).float())
        del r
    codes, scales = torch.empty(rows, 16, dtype=torch.uint8, device="cuda"), torch.full((rows,), 7, dtype=torch.uint8, device="cuda")
    B.tperm_four_bit_store(x.data_ptr(), 1, codes.data_ptr(), scales.data_ptr(), rows, 1, B.TYPES[t], stream())
    out = torch.zeros_like(x)
    B.tperm_four_bit_load(codes.data_ptr(), scales.data_ptr(), out.data_ptr(), 1, rows, 1, B.TYPES[t], stream())
    assert torch.equal(out, x)
    words = codes.view(torch.int64)
    assert not bool((words[:, 1] != 0).any()) and int(words[:, 0].max()) <= 15 and int(words[:, 0].min()) >= 0      # zeros behind a row's end


@pytest.mark.parametrize("experts,slots", [(513, 2), (130, 9)])
def test_router_of_more_workgroups_than_a_row_of_the_grid(experts, slots):
    """A wavefront to a token, four to a workgroup: every token has one expert, the others are barred."""
    tokens = (1 << 24) + 12345
    t = B.TYPE_BF16
    scores = torch.full((tokens, experts), -torch.inf, dtype=torch.bfloat16, device="cuda")
    at = (torch.arange(tokens, device="cuda") * 7) % experts
    scores.scatter_(1, at[:, None], 1.5)
    expert, weights = torch.full((tokens, slots), 9, dtype=torch.int32, device="cuda"), torch.full((tokens, slots), 9.0, device="cuda")
    B.tperm_expert_route(scores.data_ptr(), experts, expert.data_ptr(), weights.data_ptr(), tokens, slots, experts, False, t, stream())
    assert torch.equal(expert[:, 0].long(), at) and bool((expert[:, 1:] == -1).all())
    assert bool((weights[:, 0] == 1.0).all()) and not bool(weights[:, 1:].any())
    weights[:, 0] = 0.5
    grad_weights = torch.ones(tokens, slots, device="cuda")
    grad = torch.full_like(scores, 3.0)
    B.tperm_expert_route_backward(grad_weights.data_ptr(), None, 0, expert.data_ptr(), weights.data_ptr(), grad.data_ptr(), experts, tokens, slots, experts, False, t, stream())
    want = torch.zeros_like(scores)
    want.scatter_(1, at[:, None], 0.25)        # w (g - m) = 0.5 (1 - 0.5)
    assert torch.equal(grad, want)


def test_four_bit_matrices_of_experts_behind_4_gib():
    """Codes of the last expert lie behind 4 GiB in both matrices: the same bits as from the first place, and the formula's result."""
    experts, width, hidden, tokens, slots = 33, 16384, 16384, 3, 2
    t = B.TYPE_BF16
    g = torch.Generator(device="cuda").manual_seed(4)
    groups = width // 32
    made = lambda rows: (torch.randint(0, 256, (experts, rows, groups * 16), generator=g, dtype=torch.uint8, device="cuda"),  # noqa: E731
                         torch.randint(117, 120, (experts, rows, groups), generator=g, dtype=torch.uint8, device="cuda"))
    (w_in, in_scales), (w_out, out_scales) = made(2 * hidden), made(width)
    assert w_out[-1].data_ptr() - w_out.data_ptr() >= 1 << 32
    x = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    room = torch.empty(B.expert_few_workspace_bytes(tokens, slots, experts, width, hidden, t, True), dtype=torch.uint8, device="cuda")

    def few(e):
        out = torch.empty_like(x)
        expert = torch.tensor([[e, -1]] * tokens, dtype=torch.int32, device="cuda")
        B.tperm_expert_few(x.data_ptr(), width, expert.data_ptr(), None, w_in.data_ptr(), in_scales.data_ptr(), w_out.data_ptr(), out_scales.data_ptr(),
                           out.data_ptr(), width, room.data_ptr(), room.numel(), tokens, slots, experts, width, hidden, t, stream())
        torch.cuda.synchronize()
        return out

    got = few(experts - 1)
    for m in (w_in, in_scales, w_out, out_scales):
        m[0].copy_(m[-1])
    assert torch.equal(got, few(0))

    def stands(codes, scales, rows):
        v = torch.empty(rows, width, device="cuda")
        B.tperm_four_bit_load(codes[-1].data_ptr(), scales[-1].data_ptr(), v.data_ptr(), width, rows, width, B.TYPE_F32, stream())
        return v

    both = x.float() @ stands(w_in, in_scales, 2 * hidden).t()
    want = (torch.nn.functional.silu(both[:, :hidden]) * both[:, hidden:]) @ stands(w_out, out_scales, width).t()
    # bfloat16 results, and sums of 16384 products in binary32 on both sides: a bound of norms, 2^-8 as in the test of matrices in 16 bits
    assert bool(got.isfinite().all()) and float((got.float() - want).norm() / want.norm()) < 2.0 ** -8

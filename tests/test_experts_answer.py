"""The mixture-of-experts layer that answers: router, matrices in 4 bits, few tokens and many, together as a program uses them.

Bounds as in test_experts_layer: 2-norms of differences against formulas in 64 bits, 1e-5 in binary32, where every intermediate
is rounded to 24 bits and sums have at most a few thousand terms, 2e-2 and 4e-3 in bfloat16 and binary16, where two to four
intermediates are rounded to 8 and 11 bits."""
import json

import pytest

from paper_1705_01598_amd import binding as B
from paper_1705_01598_amd import experts as E
from paper_1705_01598_amd.experts import ExpertLayer, HeldMatrices

torch = pytest.importorskip("torch")
BOUND = {torch.float32: 1e-5, torch.float16: 4e-3, torch.bfloat16: 2e-2}


def test_arguments_are_checked():
    layer = ExpertLayer(4, 2, 8, 40, torch.float32, device="cpu")
    scores = torch.zeros(3, 4)
    for bad in (torch.zeros(3, 5), torch.zeros(3, 4, dtype=torch.float64), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(4, 3).t()):
        with pytest.raises(ValueError):
            layer.route(bad)
        with pytest.raises(ValueError):
            layer.route_backward(torch.zeros(3, 2), bad, torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2))
    good = [torch.zeros(3, 2), scores, torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)]
    for i, bad in ((0, torch.zeros(3, 3)), (0, torch.zeros(3, 2).half()), (2, torch.zeros(3, 2, dtype=torch.int64)), (3, torch.zeros(2, 2))):
        with pytest.raises(ValueError):
            layer.route_backward(*(bad if j == i else g for j, g in enumerate(good)))
    w_in, w_out = torch.zeros(4, 80, 8), torch.zeros(4, 8, 40)
    with pytest.raises(ValueError):
        layer.hold(w_in, w_out.half())
    with pytest.raises(ValueError):
        layer.hold(w_out, w_in)
    u8 = torch.uint8
    held = HeldMatrices(torch.zeros(4, 80, 16, dtype=u8), torch.zeros(4, 80, 1, dtype=u8), torch.zeros(4, 8, 32, dtype=u8), torch.zeros(4, 8, 2, dtype=u8))
    x, expert, weights = torch.zeros(3, 8), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2)
    for matrices in ((held, w_out), (w_in,), (w_in, w_out.half()), (held._replace(w_out=torch.zeros(4, 8, 16, dtype=u8)),), (held._replace(in_scales=held.in_scales.float()),)):
        with pytest.raises(ValueError):
            layer.answer(x, expert, weights, *matrices)
    for call in (lambda: layer.route(scores), lambda: layer.hold(w_in, w_out), lambda: layer.answer(x, expert, weights, held), lambda: layer.answer(x, expert, weights, w_in, w_out)):
        with pytest.raises(ValueError, match="GPU"):     # a layer made for the host computes nothing
            call()


def test_command_refuses_bits_without_an_answer(capsys):
    if torch.cuda.is_available():
        pytest.skip("on a GPU it is tested by running it")
    with pytest.raises(SystemExit):
        E._bench(["--answer", "--bits", "3"])


def off(got, want):
    got, want = got.double().cpu(), want.detach().double().cpu()
    return float((got - want).norm() / want.norm()) if float(want.norm()) else float(got.norm())


def plain(x, expert, weights, w_in, w_out):
    """The layer in doubles, differentiable in x and weights."""
    hidden = w_out.shape[2]
    rows = []
    for t in range(x.shape[0]):
        y = torch.zeros_like(x[t])
        for s, e in enumerate(expert[t].tolist()):
            if 0 <= e < w_in.shape[0]:
                both = w_in[e] @ x[t]
                y = y + weights[t, s] * (w_out[e] @ (torch.nn.functional.silu(both[:hidden]) * both[hidden:]))
        rows.append(y)
    return torch.stack(rows)


def made(tokens, experts, width, hidden, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return [t.to(dtype).cuda() for t in (randn(tokens, width), randn(tokens, experts), randn(experts, 2 * hidden, width) / width ** 0.5, randn(experts, width, hidden) / hidden ** 0.5)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("tokens,experts,slots,width,hidden", [(1, 4, 2, 64, 96), (17, 5, 3, 100, 33), (64, 8, 2, 96, 160), (65, 8, 2, 96, 160), (130, 3, 1, 40, 72)])
def test_route_and_answer(dtype, tokens, experts, slots, width, hidden):
    x, scores, w_in, w_out = made(tokens, experts, width, hidden, dtype, tokens)
    scores[0] = -float("inf")
    layer = ExpertLayer(experts, slots, width, hidden, dtype)
    expert, weights = layer.route(scores, over_all=True)
    assert expert[0].tolist() == [-1] * slots and not bool(weights[0].any())
    y = layer.answer(x, expert, weights, w_in, w_out)
    held = layer.hold(w_in, w_out)
    z = layer.answer(x, expert, weights, held)
    assert not bool(y[0].any()) and not bool(z[0].any())
    stands = [torch.empty(m.shape, device="cuda") for m in (w_in, w_out)]
    for (codes, scales), m in zip((held[:2], held[2:]), stands):
        B.tperm_four_bit_load(codes.data_ptr(), scales.data_ptr(), m.data_ptr(), m.shape[2], m.shape[0] * m.shape[1], m.shape[2], B.TYPE_F32, torch.cuda.current_stream().cuda_stream)
    d = lambda t: t.double().cpu()  # noqa: E731
    assert off(y, plain(d(x), expert, d(weights), d(w_in), d(w_out))) < BOUND[dtype]
    assert off(z, plain(d(x), expert, d(weights), *(d(m) for m in stands))) < BOUND[dtype]
    if dtype == torch.float32:
        assert off(y, layer.forward(x, expert, weights, w_in, w_out)) < 2 * BOUND[dtype]


@pytest.mark.gpu
def test_gradients_from_the_result_to_the_scores():
    """Router, layer and their backward passes against autograd in doubles, at the input that the layer kept in 8 bits or near it: the scores'
    gradient passes through the weights alone."""
    tokens, experts, slots, width, hidden = 23, 6, 3, 64, 48
    x, scores, w_in, w_out = made(tokens, experts, width, hidden, torch.float32, 3)
    grad = torch.randn(tokens, width, generator=torch.Generator().manual_seed(4)).cuda()
    for over_all in (False, True):
        layer = ExpertLayer(experts, slots, width, hidden, torch.float32)
        expert, weights = layer.route(scores, over_all)
        layer.forward(x, expert, weights, w_in, w_out)
        _, grad_weights = layer.backward(grad, torch.zeros(w_in.shape, device="cuda"), torch.zeros(w_out.shape, device="cuda"))
        got = layer.route_backward(grad_weights, scores, expert, weights, over_all)
        s = scores.double().cpu().requires_grad_()
        at = expert.long().cpu()
        w = torch.softmax(s, 1).gather(1, at) if over_all else torch.softmax(s.gather(1, at), 1)
        y = plain(x.double().cpu(), expert, w, w_in.double().cpu(), w_out.double().cpu())
        (y * grad.double().cpu()).sum().backward()
        assert off(got, s.grad) < 2e-5


@pytest.mark.gpu
def test_answers_between_the_passes_leave_them_alone():
    tokens, experts, slots, width, hidden = 70, 5, 2, 64, 40
    x, scores, w_in, w_out = made(tokens, experts, width, hidden, torch.bfloat16, 5)
    layer = ExpertLayer(experts, slots, width, hidden, torch.bfloat16)
    expert, weights = layer.route(scores)
    grad = x.flip(0).contiguous()

    def backward():
        a, b = torch.empty(w_in.shape, device="cuda"), torch.empty(w_out.shape, device="cuda")
        return [*layer.backward(grad, a, b, accumulate=False), a, b]

    layer.forward(x, expert, weights, w_in, w_out)
    want = backward()
    layer.forward(x, expert, weights, w_in, w_out)
    for n in (1, 64, 70):
        layer.answer(grad[:n], expert[:n], weights[:n], w_in, w_out)
        layer.answer(grad[:n], expert[:n], weights[:n], layer.hold(w_in, w_out))
    assert all(torch.equal(a, b) for a, b in zip(backward(), want))


@pytest.mark.gpu
def test_no_tokens():
    layer = ExpertLayer(4, 2, 16, 16, torch.float16)
    w_in, w_out = torch.ones(4, 32, 16, device="cuda").half(), torch.ones(4, 16, 16, device="cuda").half()
    expert, weights = layer.route(torch.empty(0, 4, device="cuda"))
    assert expert.shape == (0, 2) and weights.shape == (0, 2)
    assert layer.answer(torch.empty(0, 16, device="cuda").half(), expert, weights, w_in, w_out).shape == (0, 16)
    assert layer.answer(torch.empty(0, 16, device="cuda").half(), expert, weights, layer.hold(w_in, w_out)).shape == (0, 16)
    assert layer.route_backward(weights, torch.empty(0, 4, device="cuda"), expert, weights).shape == (0, 4)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [3, 90])
def test_answers_in_a_graph(tokens):
    """Router and both kinds of answer captured, replayed between eager ones of other tokens: the same bits every time."""
    experts, slots, width, hidden = 6, 2, 96, 72
    x, scores, w_in, w_out = made(tokens, experts, width, hidden, torch.bfloat16, 6)
    layer = ExpertLayer(experts, slots, width, hidden, torch.bfloat16)
    held = layer.hold(w_in, w_out)

    def both(x):
        expert, weights = layer.route(scores)
        return [expert, weights, layer.answer(x, expert, weights, w_in, w_out), layer.answer(x, expert, weights, held)]

    want = [t.clone() for t in both(x)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = both(x)
    for _ in range(4):
        both(x.flip(0).contiguous())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want))


@pytest.mark.gpu
@pytest.mark.parametrize("more", [["--tokens", "2"], ["--tokens", "2", "--bits", "4"], ["--tokens", "100", "--bits", "4", "--dtype", "f16"]])
def test_command(more, capsys):
    E._bench(["--answer", "--experts", "4", "--slots", "2", "--width", "64", "--hidden", "32", "--reps", "2", *more])
    got = json.loads(capsys.readouterr().out)
    assert got["answer_ms"] > 0 and got["experts_named"] <= 4 and got["bits"] in (4, 16)

"""What the mixture-of-experts layer does around its calls, with stand-ins for torch and the library that record
them: on which GPU and stream they are enqueued, and what is left of a pass that fails.  No GPU is needed."""
import contextlib
import gc
import weakref

import pytest

from paper_1705_01598_amd import binding
from paper_1705_01598_amd.experts import ExpertLayer

torch = pytest.importorskip("torch")
EXPERTS, SLOTS, WIDTH, HIDDEN = 4, 2, 16, 24


class Tensor:
    _next = 1 << 20

    def __init__(self, *shape, dtype, device):
        self.shape, self.dtype, self.device = tuple(shape), dtype, torch.device(device)
        self._at, Tensor._next = Tensor._next, Tensor._next + (1 << 24)

    def is_contiguous(self):
        return True

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def data_ptr(self):
        return self._at

    def element_size(self):
        return self.dtype.itemsize

    def zero_(self):
        return self


class Torch:
    """Two GPUs, of which number 0 is the current one; stream 1000 + d is the current stream of GPU d."""

    def __init__(self):
        self.current = 0
        self.cuda = self

    def __getattr__(self, name):
        return getattr(torch, name)     # dtypes

    def empty(self, *shape, dtype, device):
        return Tensor(*(shape[0] if len(shape) == 1 and not isinstance(shape[0], int) else shape), dtype=dtype, device=device)

    def empty_like(self, t):
        return Tensor(*t.shape, dtype=t.dtype, device=t.device)

    def current_device(self):
        return self.current

    def device(self, d):
        d = torch.device(d)

        @contextlib.contextmanager
        def current():
            before, self.current = self.current, d.index
            yield
            self.current = before
        return current()

    def current_stream(self, device=None):
        index = self.current if device is None or torch.device(device).index is None else torch.device(device).index
        return type("Stream", (), {"cuda_stream": 1000 + index})


class Library:
    """The binding, whose calls are recorded; the call named `failing` raises."""

    def __init__(self, gpus):
        self.calls, self.gpus, self.failing = [], gpus, None

    def __getattr__(self, name):
        if not name.startswith("tperm_"):
            return getattr(binding, name)

        def call(*args):
            if name == self.failing:
                raise binding.TpermError(binding.ERR_TOO_LARGE, name)
            self.calls.append((name, args[-1], self.gpus.current))
        return call


def layer_on(device):
    layer = ExpertLayer(EXPERTS, SLOTS, WIDTH, HIDDEN, torch.bfloat16, device=device)
    layer._torch = Torch()
    layer._B = Library(layer._torch)
    return layer


def inputs(device, tokens=5):
    new = lambda *s, dtype=torch.bfloat16: Tensor(*s, dtype=dtype, device=device)  # noqa: E731
    return [new(tokens, WIDTH), new(tokens, SLOTS, dtype=torch.int32), new(tokens, SLOTS, dtype=torch.float32),
            new(EXPERTS, 2 * HIDDEN, WIDTH), new(EXPERTS, WIDTH, HIDDEN)]


def gradients(device, tokens=5):
    new = lambda *s, dtype=torch.float32: Tensor(*s, dtype=dtype, device=device)  # noqa: E731
    return [new(tokens, WIDTH, dtype=torch.bfloat16), new(EXPERTS, 2 * HIDDEN, WIDTH), new(EXPERTS, WIDTH, HIDDEN)]


@pytest.mark.parametrize("made_for", ["cuda:1", "cuda"])
def test_calls_go_to_the_gpu_and_the_stream_of_the_tensors(made_for):
    layer = layer_on(made_for)
    layer.forward(*inputs("cuda:1"))
    layer.kept_gates()
    layer.backward(*gradients("cuda:1"))
    assert len(layer._B.calls) == 6 + 1 + 7
    assert {(stream, gpu) for _, stream, gpu in layer._B.calls} == {(1001, 1)}
    assert layer._torch.current == 0


@pytest.mark.parametrize("made_for,given", [("cuda:1", "cuda:0"), ("cuda:0", "cuda:1"), ("cuda", "cpu"), ("cpu", "cuda:0")])
def test_tensors_of_another_device_are_refused(made_for, given):
    layer = layer_on(made_for)
    with pytest.raises(ValueError):
        layer.forward(*inputs(given))
    assert not layer._B.calls


def test_a_device_without_a_number_is_that_of_the_first_tensors():
    layer = layer_on("cuda")
    layer.forward(*inputs("cuda:1"))
    for i in range(5):
        mixed = inputs("cuda:1")
        mixed[i] = inputs("cuda:0")[i]
        with pytest.raises(ValueError):
            layer.forward(*mixed)
    for i in range(3):
        mixed = gradients("cuda:1")
        mixed[i] = gradients("cuda:0")[i]
        with pytest.raises(ValueError):
            layer.backward(*mixed)


def test_host_memory_goes_to_no_kernel():
    layer = layer_on("cpu")
    with pytest.raises(ValueError):
        layer.forward(*inputs("cpu"))
    assert not layer._B.calls


def test_nothing_is_left_of_a_forward_pass_that_fails():
    """Its first calls, or larger buffers, have taken the place of what the pass before it kept."""
    for failing in ("tperm_expert_sort", "tperm_expert_product", "tperm_expert_combine"):
        for tokens in (5, 50):
            layer = layer_on("cuda:1")
            layer.forward(*inputs("cuda:1"))
            layer._B.failing = failing
            with pytest.raises(binding.TpermError):
                layer.forward(*inputs("cuda:1", tokens))
            layer._B.failing = None
            for late in (lambda: layer.backward(*gradients("cuda:1")), lambda: layer.backward(*gradients("cuda:1", tokens)), layer.kept_gates):
                with pytest.raises(RuntimeError, match="forward"):
                    late()


def test_a_refused_forward_pass_leaves_the_one_before():
    layer = layer_on("cuda:1")
    layer.forward(*inputs("cuda:1"))
    with pytest.raises(ValueError):
        layer.forward(*inputs("cuda:0"))
    layer.backward(*gradients("cuda:1"))


def test_a_backward_pass_that_fails_is_not_run_again():
    """It has written over the kept rows, and may have added to the gradients."""
    for failing in ("tperm_expert_combine_backward", "tperm_expert_weight_gradient", "tperm_expert_combine"):
        layer = layer_on("cuda:1")
        layer.forward(*inputs("cuda:1"))
        layer._B.failing = failing
        with pytest.raises(binding.TpermError):
            layer.backward(*gradients("cuda:1"))
        layer._B.failing = None
        with pytest.raises(RuntimeError, match="forward"):
            layer.backward(*gradients("cuda:1"))
    layer.forward(*inputs("cuda:1"))
    with pytest.raises(ValueError):             # arguments are looked at first: this one may be run again
        layer.backward(*gradients("cuda:0"))
    layer.backward(*gradients("cuda:1"))


def test_one_backward_pass_to_a_forward_pass_without_tokens_too():
    layer = layer_on("cuda:1")
    layer.forward(*inputs("cuda:1", 0))
    layer.backward(*gradients("cuda:1", 0))
    with pytest.raises(RuntimeError, match="forward"):
        layer.backward(*gradients("cuda:1", 0))


def test_kept_gates_of_no_tokens():
    layer = layer_on("cuda:1")
    layer.forward(*inputs("cuda:1", 0))
    assert layer.kept_gates().shape == (0, 2 * HIDDEN)


def test_what_stays_between_the_passes_is_in_8_bits():
    """Input and gates stay as codes and scales, the rows that the experts gave and the maps as they are; the input itself,
    the gates and the hidden rows go back to the allocator."""
    tokens = 500
    layer = layer_on("cuda:1")
    made = []
    empty = layer._torch.empty

    def recorded(*shape, dtype, device):
        t = empty(*shape, dtype=dtype, device=device)
        made.append(weakref.ref(t))
        return t

    layer._torch.empty = recorded
    given = inputs("cuda:1", tokens)
    x = weakref.ref(given[0])
    layer.forward(*given)
    del given
    gc.collect()
    assert x() is None
    alive = sum(t().numel() * t().element_size() for t in made if t() is not None)
    rows, blocks = tokens * SLOTS, binding.checkpoint_blocks
    kept = tokens * (WIDTH + blocks(WIDTH)) + rows * 2 * (HIDDEN + blocks(HIDDEN)) + rows * WIDTH * 2 + (2 * rows + EXPERTS + 1) * 4
    assert alive == kept == layer.kept_bytes()
    layer.backward(*gradients("cuda:1", tokens))
    gc.collect()
    assert sum(t().numel() * t().element_size() for t in made if t() is not None) == kept

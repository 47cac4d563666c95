"""What the example layer keeps: its calls of the library recorded on the CPU in place of a GPU."""
import importlib.util
import os

import pytest
import torch

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")
N, H, F, E, K = 5, 8, 4, 3, 2


class Calls:
    """The library's functions by shape alone; `kept` records what a forward pass asked to keep."""

    def __init__(self):
        self.kept = {}

    def do_fused(self, scores, k, want_bits):
        return torch.zeros(1, 1, E, 8, dtype=torch.int64), torch.zeros(1, E, E, dtype=torch.int32), None

    class ExpertRows(tuple):
        def __new__(cls, *lists):
            return super().__new__(cls, lists)

    def do_expert_rows(self, bits, n, k):
        return self.ExpertRows(*(torch.zeros(i + 1, dtype=torch.int32) for i in range(4)))

    def do_expert_swiglu(self, x, w1, rows, p=None, checkpoint=False):
        self.kept["checkpoint"] = checkpoint
        q = (torch.zeros(N * K, 2, F, dtype=torch.int8), torch.zeros(N * K, 2, 1, dtype=torch.uint8))
        return torch.zeros(N * K, F), self.Act8(*q) if checkpoint else None

    class Act8(tuple):
        def __new__(cls, q, e):
            return super().__new__(cls, (q, e))

    def do_expert_matmul(self, x, w, rows, transposed=False):
        return torch.zeros(N * K, H)

    def do_expert_combine(self, o, rows):
        return torch.ones(N, H)

    def do_surrogate(self, p, k, bits, D, want_grad):
        self.kept["gradient"] = want_grad
        return torch.zeros(1, dtype=torch.float64), torch.zeros(1, N, E) if want_grad else None

    def do_expert_swiglu_grad(self, dy, w2, rows, kept, p):
        assert isinstance(kept, self.Act8) and kept[0].shape == (N * K, 2, F) and kept[1].dtype == torch.uint8
        assert [t.numel() for t in rows] == [1, 2, 3, 4]
        return torch.zeros(N * K, 2 * F), torch.zeros(N * K, F), torch.ones(N, E)

    def do_expert_weight_grad(self, dy, x, rows, gather_dy=False, gather_x=False):
        return torch.ones((E, H, F) if gather_dy else (E, 2 * F, H))


@pytest.fixture()
def layer_and_calls(monkeypatch):
    spec = importlib.util.spec_from_file_location("moe_layer_serving", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    calls = Calls()
    monkeypatch.setattr(m, "dl", calls)
    return m.MoELayer(H, F, E, K, torch.float32, device="cpu"), calls


def test_serving_keeps_nothing(layer_and_calls):
    layer, calls = layer_and_calls
    with torch.no_grad():
        layer(torch.randn(N, H))
    assert calls.kept == {"checkpoint": False, "gradient": False}
    for q in layer.parameters():
        q.requires_grad_(False)
    layer(torch.randn(N, H))
    assert calls.kept == {"checkpoint": False, "gradient": False}


def test_training_keeps_the_checkpoint(layer_and_calls):
    layer, calls = layer_and_calls
    y, loss = layer(torch.randn(N, H))
    assert calls.kept == {"checkpoint": True, "gradient": True}
    (y.sum() + loss).backward()
    assert all(q.grad is not None for q in layer.parameters())


def test_what_is_kept_goes_through_saved_tensors(layer_and_calls):
    # so that hooks (to offload, to count) see the 8-bit values too
    layer, _ = layer_and_calls
    seen = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: seen.append(t.dtype) or t, lambda t: t):
        layer(torch.randn(N, H))
    assert torch.int8 in seen and torch.uint8 in seen


def test_a_second_derivative_is_refused(layer_and_calls):
    layer, _ = layer_and_calls
    x = torch.randn(N, H, requires_grad=True)
    y, _ = layer(x)
    with pytest.raises(RuntimeError):
        (g,) = torch.autograd.grad(y.sum(), x, create_graph=True)
        g.sum().backward()

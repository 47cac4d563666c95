"""The example layer: its outputs and gradients against the same layer in 64 bits, and a few steps of training."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("moe_layer_example", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _reference(x, router, w1, w2, k, dtype):
    """y by the definition; the selection from the scores in the layer's own types."""
    scores = torch.nn.functional.linear(x.detach().to(dtype), router.detach().to(dtype)).float()
    pick = torch.zeros_like(scores, dtype=torch.bool).scatter_(1, scores.topk(k, dim=1).indices, True)
    p = torch.softmax(torch.nn.functional.linear(x, router), dim=1)
    y = 0.0
    F = w2.shape[2]
    for e in range(w1.shape[0]):
        a = x @ w1[e].t()
        h = p[:, e:e + 1] * torch.nn.functional.silu(a[:, :F]) * a[:, F:]
        y = y + (h @ w2[e].t()) * pick[:, e:e + 1]
    return y


def _off(got, ref):
    """Relative distance in the root mean square."""
    return ((got.double() - ref).norm() / ref.norm()).item()


@pytest.mark.parametrize("N,H,F,E,k", [(300, 64, 96, 8, 2), (1, 64, 32, 8, 2), (513, 40, 33, 12, 3)])
def test_layer_against_64_bits(example, N, H, F, E, k):
    print(f"[case] layer N={N} H={H} F={F} E={E} k={k}", flush=True)
    layer = example.MoELayer(H, F, E, k, torch.float32, seed=N)
    g = torch.Generator()
    g.manual_seed(N + 1)
    x = torch.randn(N, H, generator=g).cuda().requires_grad_()
    dy = torch.randn(N, H, generator=g).cuda()
    y, _ = layer(x)
    y.backward(dy)
    ref = [t.detach().double().requires_grad_() for t in (x, layer.router, layer.w1, layer.w2)]
    yr = _reference(*ref, k, torch.float32)
    yr.backward(dy.double())
    # sums of at most a few hundred fp32 products, the router's scores by the library
    assert _off(y, yr) < 1e-4
    # g and u return in 8 bits, off by 2^e / sqrt(12) in the root mean square where the largest of 32
    # values is above 63.5 2^e: at most 1 % of the root mean square of normal values.  Three factors of the
    # gradients carry that, with slopes of about one.
    for got, want, name in zip((x.grad, layer.router.grad, layer.w1.grad, layer.w2.grad), ref,
                               ("x", "router", "w1", "w2")):
        off = _off(got, want.grad)
        print(f"  gradient of {name}: {off:.2e}", flush=True)
        assert off < 0.05, name
    with torch.no_grad():  # serving keeps nothing, and computes the same
        assert torch.equal(layer(x)[0], y)


def test_surrogate_reaches_the_router(example):
    layer = example.MoELayer(64, 32, 8, 2, torch.float32)
    g = torch.Generator()
    g.manual_seed(5)
    x = torch.randn(256, 64, generator=g).cuda()
    _, loss = layer(x)
    loss.backward()
    assert layer.router.grad.abs().max() > 0 and not layer.w1.grad.any() and not layer.w2.grad.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_fits(example, dtype):
    _, losses = example.train(steps=30, tokens=1024, H=64, F=64, E=8, k=2, dtype=dtype, log=None)
    print(f"  mean square {losses[0]:.3f} -> {losses[-1]:.3f}", flush=True)
    assert losses[-1] < 0.8 * losses[0]

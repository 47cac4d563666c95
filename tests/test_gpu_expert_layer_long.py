"""The layer of a few tokens where its waves refill their loads many times, where up to 16 blocks share a column tile, and
on 8-bit weights at both ends of their exponents; against its definition in 64 bits."""
import pytest
import torch

from fp8_util import E4M3, lattice
from test_gpu_expert_layer import BF16, F32, _check, _gen, _inputs, dl  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

FORMS = [(F32, False), (F32, True), (BF16, False), (BF16, True)]
# N, E, k, H, F: one tile of tokens and two, contractions of at least two rounds of loads and a remainder in both kernels,
# whole steps and a last one that ends inside
LONG = [(1, 16, 4, 2304, 800), (40, 2, 2, 2304, 1100), (64, 3, 2, 2309, 1105)]
# the second kernel's column tiles split over blocks: with 8-bit weights for one tile of tokens and two, 16 ways, and
# with more blocks' waves than experts
SPLIT = [(16, 64, 8, 256, 768), (24, 64, 8, 64, 1040), (40, 32, 4, 136, 1100), (1, 8, 4, 48, 8200), (33, 2, 2, 40, 16400)]


@pytest.mark.parametrize("N,E,k,H,F", LONG + SPLIT)
@pytest.mark.parametrize("dtype,w8", FORMS)
def test_layer_of_long_contractions(dl, N, E, k, H, F, dtype, w8):  # noqa: F811
    print(f"[case] long layer N={N} E={E} k={k} H={H} F={F} {dtype} w8={w8}", flush=True)
    x, scores, w1, w2, p = _inputs(dl, _gen(N + E + F), N, E, k, H, F, dtype, w8)
    y = _check(dl, x, scores, k, w1, w2, p)
    assert torch.equal(dl.do_expert_layer(x, scores, k, w1, w2, p), y)  # whatever the order its blocks arrive in


@pytest.mark.parametrize("N,E,k,H,F", SPLIT[:2])
@pytest.mark.parametrize("dtype,w8", FORMS)
def test_split_layer_streams_and_replays(dl, N, E, k, H, F, dtype, w8):  # noqa: F811
    # the blocks' counters are cleared by each call: three streams at once, two graphs replayed beside eager calls
    gen = _gen(50)
    x, scores, w1, w2, p = _inputs(dl, gen, N, E, k, H, F, dtype, w8)
    inputs = [(torch.randn(N, H, generator=gen).to(dtype).cuda(), torch.randn(N, E, generator=gen).cuda(),
               torch.rand(N, E, generator=gen).cuda()) for _ in range(3)]
    print(f"[case] split layer streams and graphs N={N} {dtype} w8={w8}", flush=True)
    want = [_check(dl, a, b, k, w1, w2, c) for a, b, c in inputs]
    got = []
    for a, b, c in inputs:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(dl.do_expert_layer(a, b, k, w1, w2, c))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = dl.do_expert_layer(x, scores, k, w1, w2, p)
        graphs.append((g, y))
    for i in (2, 0, 1, 2):
        for dst, src in zip((x, scores, p), inputs[i]):
            dst.copy_(src)
        for g, _ in graphs:
            g.replay()
        eager = dl.do_expert_layer(x, scores, k, w1, w2, p)
        torch.cuda.synchronize()
        assert all(torch.equal(t, want[i]) for t in (graphs[0][1], graphs[1][1], eager))


def _below_one_step(dl, gen, *shape):
    """Weights of e4m3's subnormal values k 2^-9, |k| <= 7, times 2^-120 to 2^-118."""
    q = torch.randint(0, 8, shape, generator=gen) + 128 * torch.randint(0, 2, shape, generator=gen)
    e = torch.randint(7, 10, (*shape[:-2], -(-shape[-2] // 128), -(-shape[-1] // 128)), generator=gen, dtype=torch.uint8)
    return dl.Fp8(q.to(torch.uint8).view(E4M3).cuda(), e.cuda())


@pytest.mark.parametrize("N", [5, 40])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ends", [(-119, 119), (119, -119), ("least", 100), (100, "least")])
def test_layer_of_weights_at_the_ends_of_their_exponents(dl, N, dtype, ends):  # noqa: F811
    # whole numbers times powers of two, so that no product of the first contraction is rounded; tokens and probabilities
    # bring the activations and the outputs back to where the bound is not below its least
    E, k, H, F = 4, 2, 272, 144
    gen = _gen(60)
    print(f"[case] layer exponents N={N} {dtype} {ends}", flush=True)

    def made(end, *shape):
        return _below_one_step(dl, gen, *shape) if end == "least" else lattice(dl, gen, *shape, weights=True, scale=end)

    w1, w2 = made(ends[0], E, 2 * F, H), made(ends[1], E, H, F)
    up = -{"least": -128}.get(ends[0], ends[0]) - 4
    x = (torch.randint(-7, 8, (N, H), generator=gen).double() * 2.0 ** min(up, 115)).to(dtype).cuda()
    scores = torch.randn(N, E, generator=gen).cuda()
    back = -{"least": -128}.get(ends[1], ends[1])
    p = (torch.rand(N, E, generator=gen).double() * 2.0 ** max(-60, min(60, back))).float().cuda()
    y = _check(dl, x, scores, k, w1, w2, p)
    assert (y != 0).any(1).all()

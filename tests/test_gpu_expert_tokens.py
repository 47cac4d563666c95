"""Token indices outside [0, N): every kernel of the experts takes the nearest token, as the header says.

Each call is compared bit for bit with the same call on the clamped list.
"""
import pytest
import torch

from expert_util import choose, device_rows

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dl():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_32398_amd as p

    p.lib()
    return p


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def _normal(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=gen) * scale).to(dtype).cuda()


def _lists(dl, gen, N, E, k):
    """The rows with every fifth token out of range, and with those clamped."""
    rows = device_rows(dl, choose(gen, N, E, k), k)
    tok = rows.row_token.clone()
    bad = torch.tensor([-1, -N - 7, -(1 << 31), N, N + 5, (1 << 31) - 1], dtype=torch.int32, device="cuda")
    at = torch.arange(0, N * k, 5, device="cuda")
    tok[at] = bad[torch.arange(at.numel(), device="cuda") % bad.numel()]
    return rows._replace(row_token=tok), rows._replace(row_token=tok.clamp(0, N - 1))


# N, E, k, H, F: one tile size each (one token, 16 or fewer rows an expert, more of them, 128 or more), and
# widths that are not whole pieces
SHAPES = [(3, 8, 4, 64, 32), (300, 64, 2, 128, 1056), (90, 4, 2, 64, 96), (700, 4, 2, 136, 264), (700, 4, 2, 33, 41),
          (90, 4, 2, 31, 37)]


@pytest.mark.parametrize("N,E,k,H,F", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products(dl, N, E, k, H, F, dtype):
    print(f"[case] tokens out of range, products N={N} E={E} H={H} F={F} {dtype}", flush=True)
    gen = _gen(N + H)
    given, clamped = _lists(dl, gen, N, E, k)
    x, w = _normal(gen, N, H, dtype=dtype), _normal(gen, E, F, H, dtype=dtype)
    wt = _normal(gen, E, H, F, dtype=dtype)
    for ww, t in ((w, False), (wt, True)):
        got = dl.do_expert_matmul(x, ww, given, gather=True, transposed=t)
        assert torch.equal(got, dl.do_expert_matmul(x, ww, clamped, gather=True, transposed=t))


@pytest.mark.parametrize("N,E,k,H,F", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gated_activation(dl, N, E, k, H, F, dtype):
    print(f"[case] tokens out of range, gated N={N} E={E} H={H} F={F} {dtype}", flush=True)
    gen = _gen(N + H + 1)
    given, clamped = _lists(dl, gen, N, E, k)
    x, w1 = _normal(gen, N, H, dtype=dtype), _normal(gen, E, 2 * F, H, dtype=dtype, scale=H ** -0.5)
    w2, dy = _normal(gen, E, H, F, dtype=dtype, scale=F ** -0.5), _normal(gen, N, H, dtype=dtype)
    p = torch.rand(N, E, generator=gen).cuda()
    out = []
    for rows in (given, clamped):
        h, kept = dl.do_expert_swiglu(x, w1, rows, p, checkpoint=True)
        out.append([h, *kept, *dl.do_expert_swiglu_grad(dy, w2, rows, kept, p)])
    for a, b in zip(*out):
        assert torch.equal(a, b)


@pytest.mark.parametrize("N,E,O,I", [(700, 4, 96, 264), (700, 4, 41, 33), (700, 16, 1032, 1048), (700, 16, 1031, 1049)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gdy,gx", [(True, False), (False, True), (True, True)])
def test_weight_grad(dl, N, E, O, I, dtype, gdy, gx):
    print(f"[case] tokens out of range, weight grad N={N} E={E} O={O} I={I} {dtype} {gdy} {gx}", flush=True)
    gen = _gen(N + O)
    given, clamped = _lists(dl, gen, N, E, 2)
    dy = _normal(gen, N if gdy else 2 * N, O, dtype=dtype)
    x = _normal(gen, N if gx else 2 * N, I, dtype=dtype)
    got = dl.do_expert_weight_grad(dy, x, given, gather_dy=gdy, gather_x=gx)
    assert torch.equal(got, dl.do_expert_weight_grad(dy, x, clamped, gather_dy=gdy, gather_x=gx))

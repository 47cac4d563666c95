"""Each tile of the grouped products at shapes that reach it, against the definitions in 64 bits.

The bars are those of test_gpu_experts, whose checks run here on the shapes below; test_expert_launches holds
the shapes to the kernels that they are meant for.
"""
import pytest
import torch

import test_gpu_experts as base
from expert_util import EPS32, choose, device_rows, product_tol, spans, within

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

# N, E, k, O, I of a product, O outputs: at most 16 rows an expert and too many tiles for the kernel of few
FEW = [(128, 64, 8, 1056, 200), (128, 64, 8, 1050, 1032), (100, 70, 8, 1032, 40), (128, 128, 8, 600, 2048)]
# N, E, k, H, F of the gated activation, likewise
FEW_GATED = [(128, 64, 8, 200, 552), (128, 64, 8, 1032, 549), (100, 70, 8, 72, 1000), (96, 64, 8, 2048, 528)]
# Few tiles: contractions of several lines for each wave, whole and not, one token and more
SKINNY = [(1, 128, 8, 300, 2048), (1, 8, 2, 64, 1096), (3, 128, 2, 129, 520), (40, 8, 1, 70, 776), (2, 5, 5, 520, 264)]
SKINNY_GATED = [(1, 128, 8, 2048, 96), (1, 8, 2, 1096, 33), (3, 128, 2, 520, 200), (40, 8, 1, 776, 40), (2, 5, 5, 264, 65)]
# E, O, I of weight gradients of the large tile: whole pieces, and not
LARGE = [(16, 1032, 1048), (16, 1031, 1049)]


@pytest.fixture(scope="module")
def dl():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_32398_amd as p

    p.lib()
    return p


@pytest.mark.parametrize("N,E,k,O,I", FEW + SKINNY)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dist,gather", [("even", True), ("idle", False)])
def test_products_of_few_rows(dl, N, E, k, O, I, dtype, transposed, dist, gather):
    # transposed: I outputs, so the sizes change places
    a, b = (I, O) if transposed else (O, I)
    base.test_matmul(dl, N, E, k, a, b, dtype, transposed, dist, gather)


@pytest.mark.parametrize("N,E,k,H,F", FEW_GATED + SKINNY_GATED)
@pytest.mark.parametrize("dtype,pdtype", [(F32, F32), (BF16, BF16), (BF16, None)])
@pytest.mark.parametrize("dist", ["even", "idle"])
def test_gated_activation_of_few_rows(dl, N, E, k, H, F, dtype, pdtype, dist):
    base.test_swiglu(dl, N, E, k, H, F, dtype, pdtype, dist)


@pytest.mark.parametrize("N,E,k,H,F", FEW_GATED)
@pytest.mark.parametrize("dtype,pdtype", [(F32, F32), (BF16, BF16)])
def test_gated_gradient_of_few_rows(dl, N, E, k, H, F, dtype, pdtype):
    base.test_swiglu_grad(dl, N, E, k, H, F, dtype, pdtype, "idle")


def _uneven(N, E):
    """[N][E], two experts a token: every token in expert 2, the other one by its number; experts 0 and the last
    two have none, expert 1 has one row, experts 3 and 4 have 64 and 65."""
    m = torch.zeros(N, E, dtype=torch.bool)
    m[:, 2] = True
    other = 5 + torch.arange(N) * 7 % (E - 7)
    other[0], other[1:65], other[65:130] = 1, 3, 4
    m[torch.arange(N), other] = True
    return m


@pytest.mark.parametrize("E,O,I", LARGE)
@pytest.mark.parametrize("N", [2600, 150])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("gdy,gx", [(False, False), (False, True), (True, False), (True, True)])
def test_weight_grad_of_the_large_tile(dl, E, O, I, N, dtype, gdy, gx):
    print(f"[case] large weight grad N={N} E={E} O={O} I={I} {dtype} {gdy} {gx}", flush=True)
    gen = base._gen(N + O + I)
    mask = _uneven(N, E)
    rows = device_rows(dl, mask, 2)
    R = 2 * N
    assert int(rows.offsets[-1]) == R and int(rows.offsets[-3]) == R  # the last two begin past the last row
    dy = base._normal(gen, N if gdy else R, O, dtype=dtype)
    x = base._normal(gen, N if gx else R, I, dtype=dtype)
    before = base._normal(gen, E, O, I)
    out = torch.full((E, O, I), float("nan"), device="cuda")
    dw = dl.do_expert_weight_grad(dy, x, rows, gather_dy=gdy, gather_x=gx, out=out)
    acc = dl.do_expert_weight_grad(dy, x, rows, gather_dy=gdy, gather_x=gx, out=before.clone(), accumulate=True)
    used = set()
    for e, a, b, tok in spans(mask, 2):
        used.add(e)
        d, v = (dy[tok] if gdy else dy[a:b]).double(), (x[tok] if gx else x[a:b]).double()
        ref = d.t() @ v
        tol = product_tol(d.abs().t() @ v.abs(), b - a, ref, F32)
        within(dw[e], ref, tol, f"dw of expert {e}")
        total = before[e].double() + ref
        within(acc[e], total, tol + EPS32 * total.abs() + EPS32 * ref.abs(), f"accumulated, expert {e}")
    idle = [e for e in range(E) if e not in used]
    assert idle == [0, E - 2, E - 1]
    assert not dw[idle].any() and torch.equal(acc[idle], before[idle])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_weight_grad_where_no_expert_has_rows(dl, dtype):
    # every block's tiles are empty
    E, O, I, N = 16, 1032, 1048, 3
    rows = device_rows(dl, torch.zeros(N, E, dtype=torch.bool), 1)
    dy, x = torch.ones(N, O, dtype=dtype, device="cuda"), torch.ones(N, I, dtype=dtype, device="cuda")
    out = torch.full((E, O, I), 7.0, device="cuda")
    print(f"[case] weight grad without rows {dtype}", flush=True)
    dl.do_expert_weight_grad(dy, x, rows, gather_x=True, out=out, accumulate=True)
    assert (out == 7.0).all()
    dl.do_expert_weight_grad(dy, x, rows, gather_x=True, out=out)
    assert not out.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_tiles_repeat_bit_for_bit(dl, dtype):
    # a layer of large tiles, twice, with other work on the same memory in between
    N, E, k, H, F = 6000, 8, 2, 1024, 1056
    print(f"[case] large tiles twice {dtype}", flush=True)
    gen = base._gen(31)
    rows = device_rows(dl, choose(gen, N, E, k, "idle"), k)
    x, dy = base._normal(gen, N, H, dtype=dtype), base._normal(gen, N, H, dtype=dtype)
    w1 = base._normal(gen, E, 2 * F, H, dtype=dtype, scale=H ** -0.5)
    w2 = base._normal(gen, E, H, F, dtype=dtype, scale=F ** -0.5)
    p = torch.rand(N, E, generator=gen).cuda()
    runs = []
    for _ in range(3):
        h, kept = dl.do_expert_swiglu(x, w1, rows, p, checkpoint=True)
        y = dl.do_expert_matmul(h, w2, rows)
        da, h2, dp = dl.do_expert_swiglu_grad(dy, w2, rows, kept, p)
        dw1 = dl.do_expert_weight_grad(da, x, rows, gather_x=True)
        dw2 = dl.do_expert_weight_grad(dy, h2, rows, gather_dy=True)
        dx = dl.do_expert_matmul(da, w1, rows, transposed=True)
        runs.append([h, *kept, y, da, h2, dp, dw1, dw2, dx])
        torch.full((1 << 28,), float("nan"), device="cuda")  # another tenant of the caches
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert torch.equal(a, b)


# --- rows by token past 4 GiB, fp32, and both sides by token ---------------------------------------------------------

N_LONG, H_LONG, E_LONG, SMALL = 530_003, 2048, 40, 64


@pytest.fixture(scope="module")
def long32():
    g = torch.Generator("cuda")
    g.manual_seed(3)
    x = torch.empty(N_LONG, H_LONG, device="cuda").normal_(generator=g)
    assert x.numel() * 4 > 1 << 32
    return x


@pytest.fixture(scope="module")
def routed32(dl):
    """(rows, expert of each row, sampled rows): token t to expert (t * 7919 >> 4) % 39; the last expert has none."""
    t = torch.arange(N_LONG, device="cuda")
    expert = (t * 7919 >> 4) % (E_LONG - 1)
    order = torch.argsort(expert, stable=True)
    offsets = torch.zeros(E_LONG + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.bincount(expert, minlength=E_LONG).cumsum(0)
    back = torch.empty_like(order)
    back[order] = t
    rows = dl.ExpertRows(offsets.int(), order.int(), back.int()[:, None].contiguous(), expert.int()[:, None].contiguous())
    sample = torch.cat([torch.arange(0, N_LONG, 4001, device="cuda"), back[-3:], torch.tensor([N_LONG - 1], device="cuda")])
    return rows, expert[order], sample.unique()


def _small(*shape, scale=1.0, seed=2):
    return base._normal(base._gen(seed), *shape, scale=scale)


def _rowwise(v, w):
    """v[r] times w[r] (one matrix a row), and the sum of the magnitudes, in 64 bits, some rows at a time."""
    ref, size = [], []
    for a, b in zip(v.double().split(64), w.split(64)):
        b = b.double()
        ref.append(torch.bmm(b, a[:, :, None])[:, :, 0])
        size.append(torch.bmm(b.abs(), a.abs()[:, :, None])[:, :, 0])
    return torch.cat(ref), torch.cat(size)


@pytest.mark.parametrize("transposed", [False, True])
def test_long_fp32_products(dl, long32, routed32, transposed):
    rows, expert, sample = routed32
    w = _small(*((E_LONG, H_LONG, SMALL) if transposed else (E_LONG, SMALL, H_LONG)))
    print(f"[case] long fp32 product t={transposed}", flush=True)
    y = dl.do_expert_matmul(long32, w, rows, gather=True, transposed=transposed)
    v, we = long32[rows.row_token[sample].long()], w[expert[sample]]
    ref, size = _rowwise(v, we.transpose(1, 2).contiguous() if transposed else we)
    within(y[sample], ref, product_tol(size, H_LONG, ref, F32), "y")


@pytest.mark.parametrize("gdy", [False, True])
@pytest.mark.parametrize("long_x", [False, True])
def test_long_fp32_weight_grad(dl, long32, routed32, long_x, gdy):
    # the short operand is zero but for the sample; it is by row, or by token too
    rows, expert, sample = routed32
    tok = rows.row_token.long()
    other = torch.zeros(N_LONG, SMALL, device="cuda")
    other[tok[sample] if gdy else sample] = _small(sample.numel(), SMALL)
    print(f"[case] long fp32 weight grad long_x={long_x} both by token={gdy}", flush=True)
    if long_x:
        dw = dl.do_expert_weight_grad(other, long32, rows, gather_x=True, gather_dy=gdy)
    else:
        dw = dl.do_expert_weight_grad(long32, other, rows, gather_dy=True, gather_x=gdy)
    most = int(rows.offsets.diff().max())
    for e in (0, E_LONG // 2, E_LONG - 2):
        at = sample[expert[sample] == e]
        a, b = other[tok[at] if gdy else at].double(), long32[tok[at]].double()
        if not long_x:
            a, b = b, a
        ref = a.t() @ b
        within(dw[e], ref, product_tol(a.abs().t() @ b.abs(), most, ref, F32), f"dw of expert {e}")
    assert not dw[E_LONG - 1].any()


def test_long_fp32_gated_activation_and_its_gradient(dl, long32, routed32):
    rows, expert, sample = routed32
    F = SMALL
    w1 = _small(E_LONG, 2 * F, H_LONG, scale=H_LONG ** -0.5)
    print("[case] long fp32 gated activation", flush=True)
    h, kept = dl.do_expert_swiglu(long32, w1, rows, checkpoint=True)
    v = long32[rows.row_token[sample].long()]
    a, size = _rowwise(v, w1[expert[sample]])
    off = 4 * (H_LONG + 2) * EPS32 * size
    g, u, dg, du = a[:, :F], a[:, F:], off[:, :F], off[:, F:]
    silu = g * torch.sigmoid(g)
    ref = silu * u
    tol = 1.1 * dg * u.abs() + silu.abs() * du + 1.1 * dg * du + ref.abs() * (g.abs() + 8) * 4 * EPS32
    within(h[sample], ref, tol + EPS32 * (ref.abs() + tol) + 1e-30, "h")

    w2 = _small(E_LONG, H_LONG, F, scale=F ** -0.5, seed=3)
    print("[case] long fp32 gated gradient", flush=True)
    grad, h2, none = dl.do_expert_swiglu_grad(long32, w2, rows, kept)
    assert none is None
    scale = torch.ldexp(torch.ones(kept.e[sample].shape, dtype=torch.float64, device="cuda"), kept.e[sample].int() - 127)
    a = kept.q[sample].double() * scale.repeat_interleave(32, 2)
    g, u = a[:, 0], a[:, 1]
    dh, size = _rowwise(v, w2[expert[sample]].transpose(1, 2).contiguous())
    err = 4 * (H_LONG + 2) * EPS32 * size
    z = torch.sigmoid(g)
    slope, fn = z * (1 + g * (1 - z)), (g.abs() + 8) * 4 * EPS32

    def close(got, ref, tol, what):
        within(got, ref, tol + EPS32 * (ref.abs() + tol) + 1e-30, what)

    close(h2[sample], g * z * u, (g * z * u).abs() * fn, "h again")
    rg, ru = dh * u * slope, dh * g * z
    close(grad[sample][:, :F], rg, err * (u * slope).abs() + (dh * u).abs() * (z + 2 * g.abs() * z) * fn
          + rg.abs() * 8 * EPS32, "dg")
    close(grad[sample][:, F:], ru, err * (g * z).abs() + ru.abs() * (fn + 8 * EPS32), "du")

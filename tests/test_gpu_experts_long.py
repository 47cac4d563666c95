"""The experts' operators where an operand or output passes 4 GiB and 2^31 elements.

One expert a token, so that the rows are as many as the tokens.  The bars are
those of the short cases; the reference is computed for a sample of rows spread
over the whole length, first and last among them.
"""
import pytest
import torch

from expert_util import EPS16, EPS32, product_tol, within

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
N, H, E = 1_060_003, 2048, 40
SMALL = 64


@pytest.fixture(scope="module")
def dl():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_32398_amd as p

    p.lib()
    return p


@pytest.fixture(scope="module")
def long():
    """[N][H] bf16, 4.3 GB."""
    g = torch.Generator("cuda")
    g.manual_seed(1)
    x = torch.empty(N, H, dtype=BF16, device="cuda").normal_(generator=g)
    assert x.numel() > 1 << 31 and x.numel() * 2 > 1 << 32
    return x


@pytest.fixture(scope="module")
def routed(dl):
    """(rows, expert of each row, sampled rows): token t to expert (t * 7919 >> 4) % E."""
    t = torch.arange(N, device="cuda")
    expert = (t * 7919 >> 4) % E
    order = torch.argsort(expert, stable=True)
    offsets = torch.zeros(E + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = torch.bincount(expert, minlength=E).cumsum(0)
    back = torch.empty_like(order)
    back[order] = t
    rows = dl.ExpertRows(offsets.int(), order.int(), back.int()[:, None].contiguous(), expert.int()[:, None].contiguous())
    sample = torch.cat([torch.arange(0, N, 4001, device="cuda"), back[-3:], torch.tensor([N - 1], device="cuda")]).unique()
    return rows, expert[order], sample


def _small(*shape, dtype=BF16, scale=1.0, seed=2):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def _rowwise(v, w):
    """v[r] times w[r] (one matrix a row), and the sum of the magnitudes; in 64 bits, some rows at a time."""
    ref, size = [], []
    for a, b in zip(v.double().split(64), w.split(64)):
        b = b.double()
        ref.append(torch.bmm(b, a[:, :, None])[:, :, 0])
        size.append(torch.bmm(b.abs(), a.abs()[:, :, None])[:, :, 0])
    return torch.cat(ref), torch.cat(size)


@pytest.mark.parametrize("transposed", [False, True])
def test_matmul_of_long_rows_by_token(dl, long, routed, transposed):
    rows, expert, sample = routed
    w = _small(*((E, H, SMALL) if transposed else (E, SMALL, H)))
    print(f"[case] long matmul, gathered, t={transposed}", flush=True)
    y = dl.do_expert_matmul(long, w, rows, gather=True, transposed=transposed)
    v, we = long[rows.row_token[sample].long()], w[expert[sample]]
    ref, size = _rowwise(v, we.transpose(1, 2).contiguous() if transposed else we)
    within(y[sample], ref, product_tol(size, H, ref, BF16), "y")


@pytest.mark.parametrize("transposed", [False, True])
def test_matmul_to_long_rows_and_their_sum(dl, routed, transposed):
    rows, expert, sample = routed
    w = _small(*((E, SMALL, H) if transposed else (E, H, SMALL)))
    x = _small(N, SMALL)
    print(f"[case] long matmul output, t={transposed}", flush=True)
    y = dl.do_expert_matmul(x, w, rows, transposed=transposed)
    we = w[expert[sample]]
    ref, size = _rowwise(x[sample], we.transpose(1, 2).contiguous() if transposed else we)
    within(y[sample], ref, product_tol(size, SMALL, ref, BF16), "y")
    # from long rows in the experts' order: nothing by token
    if not transposed:
        back = dl.do_expert_matmul(y, w, rows, transposed=True)
        ref, size = _rowwise(y[sample], we.transpose(1, 2).contiguous())
        within(back[sample], ref, product_tol(size, H, ref, BF16), "back")
        s = dl.do_expert_combine(y, rows)
        assert torch.equal(s[rows.row_token[sample].long()], y[sample])


@pytest.mark.parametrize("of_x", [False, True])
def test_weight_grad_of_long_rows_by_token(dl, long, routed, of_x):
    # the other operand is zero but for the sample, which makes the gradient a sum over it
    rows, expert, sample = routed
    other = torch.zeros(N, SMALL, dtype=BF16, device="cuda")
    other[sample] = _small(sample.numel(), SMALL)
    print(f"[case] long weight grad, of_x={of_x}", flush=True)
    dw = dl.do_expert_weight_grad(other, long, rows, gather_x=True) if of_x else \
        dl.do_expert_weight_grad(long, other, rows, gather_dy=True)
    most = int(rows.offsets.diff().max())
    for e in (0, E // 2, E - 1):
        at = sample[expert[sample] == e]
        a, b = other[at].double(), long[rows.row_token[at].long()].double()
        if not of_x:
            a, b = b, a
        ref = a.t() @ b
        within(dw[e], ref, product_tol(a.abs().t() @ b.abs(), most, ref, F32), f"dw of expert {e}")


def test_swiglu_and_its_gradient_of_long_rows(dl, long, routed):
    rows, expert, sample = routed
    F = SMALL
    w1 = _small(E, 2 * F, H, scale=H ** -0.5)
    print("[case] long swiglu", flush=True)
    h, kept = dl.do_expert_swiglu(long, w1, rows, checkpoint=True)
    v = long[rows.row_token[sample].long()]
    a, size = _rowwise(v, w1[expert[sample]])
    da = 4 * (H + 2) * EPS32 * size
    g, u, dg, du = a[:, :F], a[:, F:], da[:, :F], da[:, F:]
    silu = g * torch.sigmoid(g)
    ref = silu * u
    tol = 1.1 * dg * u.abs() + silu.abs() * du + 1.1 * dg * du + ref.abs() * (g.abs() + 8) * 4 * EPS32
    within(h[sample], ref, tol + EPS16 * (ref.abs() + tol) + 1e-30, "h")

    w2 = _small(E, H, F, scale=F ** -0.5, seed=3)
    print("[case] long swiglu grad", flush=True)
    grad, h2, none = dl.do_expert_swiglu_grad(long, w2, rows, kept)
    assert none is None
    scale = torch.ldexp(torch.ones(kept.e[sample].shape, dtype=torch.float64, device="cuda"), kept.e[sample].int() - 127)
    a = kept.q[sample].double() * scale.repeat_interleave(32, 2)
    g, u = a[:, 0], a[:, 1]
    dh, size = _rowwise(v, w2[expert[sample]].transpose(1, 2).contiguous())
    err = 4 * (H + 2) * EPS32 * size
    z = torch.sigmoid(g)
    slope, fn = z * (1 + g * (1 - z)), (g.abs() + 8) * 4 * EPS32

    def close(got, ref, tol, what):
        within(got, ref, tol + EPS16 * (ref.abs() + tol) + 1e-30, what)

    close(h2[sample], g * z * u, (g * z * u).abs() * fn, "h again")
    rg, ru = dh * u * slope, dh * g * z
    close(grad[sample][:, :F], rg, err * (u * slope).abs() + (dh * u).abs() * (z + 2 * g.abs() * z) * fn
          + rg.abs() * 8 * EPS32, "dg")
    close(grad[sample][:, F:], ru, err * (g * z).abs() + ru.abs() * (fn + 8 * EPS32), "du")


def test_act8_of_long_rows(dl, long):
    print("[case] long act8", flush=True)
    a = dl.do_act8_pack(long)
    at = torch.cat([torch.arange(0, N, 4001), torch.tensor([N - 1])]).cuda()
    part = dl.do_act8_pack(long[at])
    assert torch.equal(a.q[at], part.q) and torch.equal(a.e[at], part.e)
    assert torch.equal(dl.do_act8_unpack(a, BF16)[at], dl.do_act8_unpack(part, BF16))


def test_matmul_of_an_experts_weights_past_4_gib(dl):
    # one expert of two has 65,536 x 36,864 bf16, 4.5 GiB: forward with weight rows on both sides of 4 GiB, and transposed
    O, I, n = 65536, 36864, 20
    w = torch.zeros(2, O, I, dtype=BF16, device="cuda")
    for o in (0, 1, 31000, 59000, O - 2, O - 1):
        w[1, o] = _small(I, seed=o)
    mask_expert = torch.ones(n, 1, dtype=torch.int32, device="cuda")
    t = torch.arange(n, dtype=torch.int32, device="cuda")
    rows = dl.ExpertRows(torch.tensor([0, 0, n], dtype=torch.int32, device="cuda"), t, t[:, None].contiguous(), mask_expert)
    x = _small(n, I, scale=I ** -0.5, seed=4)
    print("[case] matmul of 4.5 GiB of weights", flush=True)
    y = dl.do_expert_matmul(x, w, rows)
    hit = torch.tensor([0, 1, 31000, 59000, O - 2, O - 1], device="cuda")
    some = w[1, hit].double()
    ref = x.double() @ some.t()
    within(y[:, hit], ref, product_tol(x.double().abs() @ some.abs().t(), I, ref, BF16), "y")
    rest = torch.ones(O, dtype=torch.bool, device="cuda")
    rest[hit] = False
    assert not y[:, rest].any()
    dy = torch.zeros(n, O, dtype=BF16, device="cuda")
    dy[:, hit] = _small(n, 6, seed=5)
    dx = dl.do_expert_matmul(dy, w, rows, transposed=True)
    d = dy[:, hit].double()
    ref = d @ some
    within(dx, ref, product_tol(d.abs() @ some.abs(), O, ref, BF16), "dx")

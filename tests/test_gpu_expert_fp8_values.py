"""What the 8-bit products keep of ordinary operands, that their powers of two are applied as such from the least to the
largest, and a training step whose operands' roundings are all accounted for."""
import pytest
import torch

from expert_util import EPS16, choose, device_rows, spans
from fp8_util import E4M3, lattice, pack_ref, power, spread, values
from test_gpu_expert_fp8 import BF16, F32, _act8_ref, _gen, _layer_step, _products, _scale, dl  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def _off(got, ref):
    return ((got.double() - ref.double()).norm() / ref.double().norm()).item()


@pytest.mark.parametrize("N,E,k,O,I", [(700, 4, 2, 300, 72), (1500, 4, 2, 1296, 1024), (64, 32, 4, 768, 2048),
                                       (900, 2, 1, 512, 2048)])
@pytest.mark.parametrize("transposed", [False, True])
def test_products_of_normal_operands_keep_what_is_stated(dl, N, E, k, O, I, transposed):  # noqa: F811
    # Sums off by s of a result in norm carry those that lie within s of a border between two bf16 values across it: a
    # part of about 2 s / step, each by a step, 2^-8 to 2^-7 of the value, so sqrt(2 s 2^-7) in norm at most.  The stated
    # s = 1.3e-5 makes 4.5e-4; 1e-3 would take s = 6.4e-5, five times as much.
    print(f"[case] fp8 products' bits N={N} E={E} O={O} I={I} t={transposed}", flush=True)
    gen = _gen(N + I)
    mask = choose(gen, N, E, k)
    rows = device_rows(dl, mask, k)
    w = dl.do_fp8_pack((torch.randn(E, O, I, generator=gen) * I ** -0.5).cuda(), weights=True)
    x = dl.do_fp8_pack(torch.randn(N * k, O if transposed else I, generator=gen).cuda())
    y = dl.do_expert_matmul_fp8(x, w, rows, transposed=transposed)
    ref, _ = _products(values(x), values(w, True), mask, k, transposed, N * k)
    assert _off(y, ref.to(BF16)) <= 1e-3


def _times(dl, a, by):  # noqa: F811
    e = a.e.int() + by
    assert int(e.min()) >= 7 and int(e.max()) <= 247
    return dl.Fp8(a.q, e.to(torch.uint8))


# powers of two moved from one operand to the other, to both ends of what the format holds: the same bits
@pytest.mark.parametrize("by", [-119, 119])
@pytest.mark.parametrize("N", [30, 400, 2600])
@pytest.mark.parametrize("whole", [True, False])
def test_products_carry_powers_of_two_at_their_ends(dl, by, N, whole):  # noqa: F811
    E, k, H, F = 4, 2, (272, 267)[not whole], (144, 139)[not whole]
    gen = _gen(70)
    mask = choose(gen, N, E, k)
    rows = device_rows(dl, mask, k)
    R = N * k
    print(f"[case] fp8 exponents N={N} by={by} whole={whole}", flush=True)
    w1, w2 = lattice(dl, gen, E, 2 * F, H, weights=True), lattice(dl, gen, E, H, F, weights=True)
    x, h, dy = lattice(dl, gen, N, H), lattice(dl, gen, R, F), lattice(dl, gen, N, H)
    p = torch.rand(N, E, generator=gen).cuda()
    kept = dl.do_act8_pack(torch.randn(R, 2, F, generator=gen).cuda())

    def calls(up, down):
        a, b = (lambda t: _times(dl, t, up)), (lambda t: _times(dl, t, down))
        act, c = dl.do_expert_swiglu_fp8(a(x), b(w1), rows, p, checkpoint=True)
        y = dl.do_expert_matmul_fp8(a(h), b(w2), rows)
        return [y, dl.do_expert_matmul_fp8(a(dy), b(w2), rows, gather=True, transposed=True), act.q.view(torch.uint8),
                act.e, *c, *dl.do_expert_swiglu_grad_fp8(a(dy), b(w2), rows, kept, p)]

    for got, want in zip(calls(by, -by), calls(0, 0)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("R", [9, 300, 2600])
def test_products_of_the_least_values(dl, R, transposed):  # noqa: F811
    # e4m3's subnormal values k 2^-9, |k| <= 7, times 2^-120: 2^-129 to 2^-127, beside rows that bring them back
    O, I = 528, 272
    gen = _gen(71)
    q = torch.randint(0, 8, (1, O, I), generator=gen) + 128 * torch.randint(0, 2, (1, O, I), generator=gen)
    e = torch.full((1, -(-O // 128), -(-I // 128)), 7, dtype=torch.uint8)
    w = dl.Fp8(q.to(torch.uint8).view(E4M3).cuda(), e.cuda())
    x = lattice(dl, gen, R, O if transposed else I, scale=119)
    print(f"[case] fp8 least values R={R} t={transposed}", flush=True)
    y = dl.do_expert_matmul_fp8(x, w, None, transposed=transposed)
    m = values(w, True)[0]
    ref = (values(x) @ (m if transposed else m.t())).to(BF16)
    assert torch.equal(y, ref) and bool(ref.any())


def _packed(v, weights=False):
    q, e = pack_ref(v, weights)
    return q * spread(power(e), v.shape, weights)


def _kept(a):
    q, e = _act8_ref(a)
    return q * power(e).repeat_interleave(32, -1)[..., : a.shape[-1]]


@pytest.mark.parametrize("N,E,k,H,F", [(50, 8, 2, 136, 72), (600, 4, 2, 256, 384), (300, 4, 2, 129, 141)])
def test_a_training_step_with_every_rounding(dl, N, E, k, H, F):  # noqa: F811
    # Against the step in 64 bits whose operands are rounded where the calls round them.  What is left: results in bf16
    # (at most EPS16 = 2^-8 of each), and operands whose sums lie so near a border that they are rounded across it.  With sums
    # off by s (2^-10 of the magnitudes at most) and a step of t, that is sqrt(2 s t) in norm: 2^-6 for e4m3 (t = 2^-3),
    # 2^-8 for the checkpoint (t = 2^-7 of a group's largest).  Operands and what is off are random here, so a product
    # keeps their ratio in norm.  y: one packed operand and two results; dw1, dw2, dp: the checkpoint's two halves,
    # slopes up to 1.1, and two results; dx: both kinds and three results.
    print(f"[case] a step in fp8 with every rounding N={N} E={E} H={H} F={F}", flush=True)
    gen = _gen(N + 80)
    mask = choose(gen, N, E, k)
    rows = device_rows(dl, mask, k)
    x, dy = (torch.randn(N, H, generator=gen).bfloat16().cuda() for _ in range(2))
    w1 = dl.do_fp8_pack((torch.randn(E, 2 * F, H, generator=gen) * H ** -0.5).cuda(), weights=True)
    w2 = dl.do_fp8_pack((torch.randn(E, H, F, generator=gen) * F ** -0.5).cuda(), weights=True)
    p = torch.rand(N, E, generator=gen).cuda()
    y, dp, dw1, dw2, dx = _layer_step(dl, x, dy, w1, w2, rows, p)
    v1, v2, xq, dyq = values(w1, True), values(w2, True), _packed(x.double()), _packed(dy.double())
    ry, rdx = (torch.zeros(N, H, dtype=torch.float64, device="cuda") for _ in range(2))
    rp, r1, r2 = torch.zeros(N, E, dtype=torch.float64, device="cuda"), torch.zeros_like(v1), torch.zeros_like(v2)
    for e, lo, hi, tok in spans(mask, k):
        pe = p[tok, e].double()[:, None]
        a = (xq[tok] @ v1[e].t()).view(-1, 2, F)
        g, u = a[:, 0], a[:, 1]
        ry[tok] += _packed(pe * g * torch.sigmoid(g) * u) @ v2[e].t()
        c = _kept(a)
        g, u = c[:, 0], c[:, 1]
        z = torch.sigmoid(g)
        dh = dyq[tok] @ v2[e]
        rp[tok, e] = (dh * g * z * u).sum(1)
        da = torch.cat([pe * dh * u * z * (1 + g * (1 - z)), pe * dh * g * z], 1)
        r2[e] = dy[tok].double().t() @ (pe * g * z * u)
        r1[e] = da.t() @ x[tok].double()
        rdx[tok] += _packed(da.to(BF16).double()) @ v1[e]
    most = {"y": 2.0 ** -6 + 2 * EPS16, "dp": 2.2 * 2.0 ** -8 + EPS16, "dw1": 2.2 * 2.0 ** -8 + 2 * EPS16,
            "dw2": 2.2 * 2.0 ** -8 + 2 * EPS16, "dx": 2.0 ** -6 + 2.2 * 2.0 ** -8 + 3 * EPS16}
    for what, got, ref in (("y", y, ry), ("dp", dp, rp), ("dw1", dw1, r1), ("dw2", dw2, r2), ("dx", dx, rdx)):
        off = _off(got, ref)
        print(f"  {what} {off:.2e}", flush=True)
        assert off <= most[what], (what, off, most[what])

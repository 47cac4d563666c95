"""The experts' operators against their definitions in 64 bits.

Bars: whole numbers exactly; a sum of K products within 4 (K + 2) 2^-24 of the
sum of the products' magnitudes plus the rounding of the stored type (2^-8 of
the value for bf16, 2^-24 for fp32); what follows from such sums by the bound
of its formula, given at each test.
"""
import math

import pytest
import torch

from expert_util import EPS16, EPS32, choose, device_rows, product_tol, rows_of, signatures, spans, within

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


# --- rows and their sum ----------------------------------------------------------------------------------------------


@pytest.mark.parametrize("N,E,k", [(1, 1, 1), (1, 8, 2), (1, 1024, 16), (63, 2, 2), (64, 8, 1), (65, 100, 6),
                                   (511, 128, 8), (512, 128, 8), (513, 128, 8), (1025, 256, 8), (5000, 64, 6),
                                   (2000, 1024, 12), (40000, 33, 3)])
@pytest.mark.parametrize("dist", ["even", "idle", "one"])
def test_rows(dl, N, E, k, dist):
    print(f"[case] rows N={N} E={E} k={k} {dist}", flush=True)
    mask = choose(_gen(N + E + k), N, E, k, dist)
    got = dl.do_expert_rows(signatures(mask.cuda()), N, k)
    for name, g, r in zip(got._fields, got, rows_of(mask, k)):
        assert g.dtype == torch.int32
        assert torch.equal(g.cpu().long(), r), name


def test_rows_many_units_per_block(dl):
    # 600 units: more than there are blocks
    N, E, k = 600 * 512 - 77, 9, 3
    mask = choose(_gen(5), N, E, k)
    print("[case] rows of 600 units", flush=True)
    got = dl.do_expert_rows(signatures(mask.cuda()), N, k)
    for name, g, r in zip(got._fields, got, rows_of(mask, k)):
        assert torch.equal(g.cpu().long(), r), name


@pytest.mark.parametrize("N,E,k", [(700, 40, 4), (130, 256, 8), (77, 5, 5)])
def test_rows_of_any_signatures(dl, N, E, k):
    # tokens with no expert, with fewer than k and with more; garbage in the bits past N
    gen = _gen(N)
    mask = torch.rand(N, E, generator=gen) < torch.rand(N, 1, generator=gen)
    mask[3], mask[4] = False, True
    bits = signatures(mask.cuda())
    pad = torch.ones(bits.shape[0] * 512, E, dtype=torch.bool)
    pad[:N] = False
    bits |= signatures(pad.cuda())
    print(f"[case] rows of any signatures N={N} E={E} k={k}", flush=True)
    got = dl.do_expert_rows(bits, N, k)
    ref = rows_of(mask, k)
    rows = int(ref[0][-1])
    assert torch.equal(got.offsets.cpu().long(), ref[0])
    assert torch.equal(got.row_token[:rows].cpu().long(), ref[1])
    assert torch.equal(got.token_row.cpu().long(), ref[2])
    assert torch.equal(got.token_expert.cpu().long(), ref[3])


def test_rows_of_the_top_k_kernel(dl):
    N, E, k = 3000, 128, 8
    scores = torch.randn(N, E, generator=_gen(1)).cuda()
    got = dl.do_expert_rows(dl.do_topk_signature(scores, k), N, k)
    mask = torch.zeros(N, E, dtype=torch.bool)
    mask.scatter_(1, scores.topk(k, dim=1).indices.cpu(), True)
    for g, r in zip(got, rows_of(mask, k)):
        assert torch.equal(g.cpu().long(), r)


@pytest.mark.parametrize("N,k,H", [(1, 1, 1), (1, 8, 2048), (33, 6, 7), (100, 2, 520), (257, 16, 1028), (1000, 8, 64)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_combine(dl, N, k, H, dtype):
    print(f"[case] combine N={N} k={k} H={H} {dtype}", flush=True)
    gen = _gen(H)
    E = max(16, k)
    mask = choose(gen, N, E, k)
    mask[N // 2, :] = False  # a token without rows
    rows = device_rows(dl, mask, k)
    o = _normal(gen, N * k, H, dtype=dtype)
    o[int(rows.offsets[-1]):] = float("nan")  # rows past the last are not read
    y = dl.do_expert_combine(o, rows)
    at = rows.token_row.long()
    v = o.double()[at.clamp(min=0)] * (at >= 0)[..., None].double()
    v = torch.where((at >= 0)[..., None], v, torch.zeros_like(v))
    ref = v.sum(1)
    within(y, ref, product_tol(v.abs().sum(1), k, ref, dtype), "y")
    assert y.dtype == dtype and not y[N // 2].any()


# --- products --------------------------------------------------------------------------------------------------------

# N, E, k, O, I: small and large tiles, widths of whole pieces and not, single tokens, contractions below,
# at and past a stage, experts with no row, with one and with most of them
SHAPES = [(1, 8, 2, 64, 64), (1, 128, 8, 96, 40), (3, 4, 1, 1, 1), (70, 8, 2, 33, 7), (200, 16, 4, 130, 96),
          (129, 8, 3, 200, 264), (700, 4, 2, 256, 128), (700, 4, 2, 300, 72), (1000, 3, 2, 257, 129),
          (900, 5, 2, 520, 136), (64, 256, 8, 72, 200), (2500, 2, 1, 64, 512)]


def _matmul_ref(x, w, mask, k, transposed, dtype, R):
    O, I = w.shape[1:]
    out = I if transposed else O
    ref = torch.zeros(R, out, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(ref)
    for e, a, b, _ in spans(mask, k):
        we = w[e].double() if transposed else w[e].double().t()
        ref[a:b] = x[a:b].double() @ we
        size[a:b] = x[a:b].double().abs() @ we.abs()
    return ref, size


@pytest.mark.parametrize("N,E,k,O,I", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dist,gather", [("even", False), ("idle", True), ("one", True)])
def test_matmul(dl, N, E, k, O, I, dtype, transposed, dist, gather):
    print(f"[case] matmul N={N} E={E} k={k} O={O} I={I} {dtype} t={transposed} {dist} gather={gather}", flush=True)
    gen = _gen(N + O + I)
    mask = choose(gen, N, E, k, dist)
    rows = device_rows(dl, mask, k)
    R, inner = N * k, O if transposed else I
    w = _normal(gen, E, O, I, dtype=dtype)
    x = _normal(gen, N if gather else R, inner, dtype=dtype)
    y = dl.do_expert_matmul(x, w, rows, gather=gather, transposed=transposed)
    xr = x[rows.row_token.long()] if gather else x
    ref, size = _matmul_ref(xr, w, mask, k, transposed, dtype, R)
    assert y.dtype == dtype
    within(y, ref, product_tol(size, inner, ref, dtype), "y")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("O,I", [(64, 64), (40, 33)])
def test_matmul_rows_past_the_last_are_left(dl, dtype, O, I):
    # tokens with fewer than k experts: the rows past offsets[E] are neither read nor written
    N, E, k = 90, 8, 4
    mask = choose(_gen(1), N, E, k)
    mask[::2, 1:] = False
    rows = device_rows(dl, mask, k)
    used = int(rows.offsets[-1])
    gen = _gen(2)
    w, x = _normal(gen, E, O, I, dtype=dtype), _normal(gen, N * k, I, dtype=dtype)
    x[used:] = float("nan")
    out = torch.full((N * k, O), 7.0, dtype=dtype, device="cuda")
    print(f"[case] matmul with {used} of {N * k} rows", flush=True)
    dl.do_expert_matmul(x, w, rows, out=out)
    ref, size = _matmul_ref(x, w, mask, k, False, dtype, N * k)
    within(out[:used], ref[:used], product_tol(size, I, ref, dtype)[:used], "y")
    assert (out[used:] == 7.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift", [0, 1])
def test_matmul_element_alignment(dl, dtype, shift):
    # operands and output that start one element past a 16-byte boundary
    N, E, k, O, I = 300, 2, 1, 64, 128
    mask = choose(_gen(3), N, E, k)
    rows = device_rows(dl, mask, k)
    gen = _gen(4)
    w = _normal(gen, E * O * I + shift, dtype=dtype)[shift:].view(E, O, I)
    x = _normal(gen, N * I + shift, dtype=dtype)[shift:].view(N, I)
    buf = torch.full((N * O + 2,), 7.0, dtype=dtype, device="cuda")
    out = buf[shift:shift + N * O].view(N, O)
    print(f"[case] matmul shift={shift} {dtype}", flush=True)
    dl.do_expert_matmul(x, w, rows, out=out)
    ref, size = _matmul_ref(x, w, mask, k, False, dtype, N)
    within(out, ref, product_tol(size, I, ref, dtype), "y")
    assert (buf[:shift] == 7.0).all() and (buf[shift + N * O:] == 7.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_matmul_infinite_and_nan_rows_stay_in_their_row(dl, dtype):
    N, E, k, O, I = 500, 3, 1, 128, 72
    mask = choose(_gen(6), N, E, k)
    rows = device_rows(dl, mask, k)
    gen = _gen(7)
    w, x = _normal(gen, E, O, I, dtype=dtype), _normal(gen, N, I, dtype=dtype)
    clean = dl.do_expert_matmul(x, w, rows)
    x[5, 3], x[40, 71], x[N - 1, 0] = float("inf"), float("nan"), float("-inf")
    got = dl.do_expert_matmul(x, w, rows)
    hit = torch.zeros(N, dtype=torch.bool, device="cuda")
    hit[[5, 40, N - 1]] = True
    assert torch.equal(got[~hit], clean[~hit])
    assert not got[hit].isfinite().any()


@pytest.mark.parametrize("N,E,k,O,I", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dist,gdy,gx", [("even", False, False), ("idle", False, True), ("one", True, False)])
def test_weight_grad(dl, N, E, k, O, I, dtype, dist, gdy, gx):
    print(f"[case] weight grad N={N} E={E} k={k} O={O} I={I} {dtype} {dist} {gdy} {gx}", flush=True)
    gen = _gen(N + O + I + 1)
    mask = choose(gen, N, E, k, dist)
    rows = device_rows(dl, mask, k)
    R = N * k
    dy = _normal(gen, N if gdy else R, O, dtype=dtype)
    x = _normal(gen, N if gx else R, I, dtype=dtype)
    before = _normal(gen, E, O, I)
    dw = dl.do_expert_weight_grad(dy, x, rows, gather_dy=gdy, gather_x=gx)
    acc = dl.do_expert_weight_grad(dy, x, rows, gather_dy=gdy, gather_x=gx, out=before.clone(), accumulate=True)
    ref = torch.zeros(E, O, I, dtype=torch.float64, device="cuda")
    tol = torch.full_like(ref, 1e-30)
    for e, a, b, tok in spans(mask, k):
        d, v = (dy[tok] if gdy else dy[a:b]).double(), (x[tok] if gx else x[a:b]).double()
        ref[e] = d.t() @ v
        tol[e] = product_tol(d.abs().t() @ v.abs(), b - a, ref[e], F32)
    assert dw.dtype == F32
    within(dw, ref, tol, "dw")
    total = before.double() + ref
    within(acc, total, tol + EPS32 * total.abs() + EPS32 * ref.abs(), "accumulated")
    idle = [e for e in range(E) if e not in {s[0] for s in spans(mask, k)}]
    assert not dw[idle].any() and torch.equal(acc[idle], before[idle])


# --- the gated activation --------------------------------------------------------------------------------------------

# N, E, k, H, F
GATED = [(1, 8, 2, 64, 32), (1, 128, 8, 72, 96), (5, 4, 1, 1, 1), (60, 8, 2, 40, 33), (200, 16, 4, 128, 96),
         (700, 4, 2, 136, 256), (700, 4, 2, 64, 200), (1000, 3, 2, 129, 129), (600, 3, 2, 72, 40), (64, 64, 8, 96, 160)]


def _silu64(g):
    return g * torch.sigmoid(g)


def _first_product(x, w1, mask, k, R):
    """a [R][2 F] and the bound on its fp32 sums."""
    a = torch.zeros(R, w1.shape[1], dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(a)
    for e, lo, hi, tok in spans(mask, k):
        v, we = x[tok].double(), w1[e].double().t()
        a[lo:hi] = v @ we
        tol[lo:hi] = 4 * (x.shape[1] + 2) * EPS32 * (v.abs() @ we.abs())
    return a, tol


def _row_probs(p, mask, k, R):
    out = torch.zeros(R, dtype=torch.float64, device="cuda")
    for e, lo, hi, tok in spans(mask, k):
        out[lo:hi] = 1.0 if p is None else p[tok, e].double()
    return out[:, None]


@pytest.mark.parametrize("N,E,k,H,F", GATED)
@pytest.mark.parametrize("dtype,pdtype", [(F32, F32), (BF16, F32), (BF16, BF16), (BF16, None)])
@pytest.mark.parametrize("dist", ["even", "idle"])
def test_swiglu(dl, N, E, k, H, F, dtype, pdtype, dist):
    print(f"[case] swiglu N={N} E={E} k={k} H={H} F={F} {dtype} p={pdtype} {dist}", flush=True)
    gen = _gen(H + F)
    mask = choose(gen, N, E, k, dist)
    rows = device_rows(dl, mask, k)
    R = N * k
    x, w1 = _normal(gen, N, H, dtype=dtype), _normal(gen, E, 2 * F, H, dtype=dtype, scale=H ** -0.5)
    p = None if pdtype is None else torch.rand(N, E, generator=gen).to(pdtype).cuda()
    h, none = dl.do_expert_swiglu(x, w1, rows, p)
    h2, kept = dl.do_expert_swiglu(x, w1, rows, p, checkpoint=True)
    assert none is None and torch.equal(h, h2)
    a, da = _first_product(x, w1, mask, k, R)
    g, u, dg, du = a[:, :F], a[:, F:], da[:, :F], da[:, F:]
    pr = _row_probs(p, mask, k, R)
    ref = pr * _silu64(g) * u
    # |silu'| < 1.1; exp and the quotient are off by (|g| + 8) 2^-22 relative
    tol = pr * (1.1 * dg * u.abs() + _silu64(g).abs() * du + 1.1 * dg * du) + ref.abs() * (g.abs() + 8) * 4 * EPS32
    tol = tol + (EPS16 if dtype == BF16 else EPS32) * (ref.abs() + tol) + 1e-30
    assert h.dtype == dtype
    within(h, ref, tol, "h")
    # the checkpoint: each value within half a step of 2^e, e the least that fits
    v = dl.do_act8_unpack(kept, F32).double()
    step = torch.ldexp(torch.ones(kept.e.shape, dtype=torch.float64, device="cuda"), kept.e.int() - 127)
    wide = step.repeat_interleave(32, 2)[..., :F]
    a3, da3 = a.view(R, 2, F), da.view(R, 2, F)
    within(v, a3, 0.5 * wide + da3, "checkpoint")
    pad = -F % 32
    top = torch.nn.functional.pad(a3.abs(), (0, pad)).view(R, 2, -1, 32).amax(3)
    dtop = torch.nn.functional.pad(da3, (0, pad)).view(R, 2, -1, 32).amax(3)
    assert (top <= 127 * step + dtop).all()
    assert ((top + dtop > 63.5 * step) | (kept.e == 1)).all()


@pytest.mark.parametrize("N,E,k,H,F", GATED)
@pytest.mark.parametrize("dtype,pdtype", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, None)])
@pytest.mark.parametrize("dist", ["even", "idle"])
def test_swiglu_grad(dl, N, E, k, H, F, dtype, pdtype, dist):
    print(f"[case] swiglu grad N={N} E={E} k={k} H={H} F={F} {dtype} p={pdtype} {dist}", flush=True)
    gen = _gen(H + F + 1)
    mask = choose(gen, N, E, k, dist)
    rows = device_rows(dl, mask, k)
    R = N * k
    dy, w2 = _normal(gen, N, H, dtype=dtype), _normal(gen, E, H, F, dtype=dtype, scale=F ** -0.5)
    p = None if pdtype is None else torch.rand(N, E, generator=gen).to(pdtype).cuda()
    kept = dl.Act8(torch.randint(-127, 128, (R, 2, F), generator=gen, dtype=torch.int8).cuda(),
                   torch.randint(118, 124, (R, 2, -(-F // 32)), generator=gen, dtype=torch.uint8).cuda())
    da, h, dp = dl.do_expert_swiglu_grad(dy, w2, rows, kept, p)
    scale = torch.ldexp(torch.ones(kept.e.shape, dtype=torch.float64, device="cuda"), kept.e.int() - 127)
    a = kept.q.double() * scale.repeat_interleave(32, 2)[..., :F]
    g, u = a[:, 0], a[:, 1]
    pr = _row_probs(p, mask, k, R)
    dh = torch.zeros(R, F, dtype=torch.float64, device="cuda")
    err = torch.zeros_like(dh)
    for e, lo, hi, tok in spans(mask, k):
        d, we = dy[tok].double(), w2[e].double()
        dh[lo:hi] = d @ we
        err[lo:hi] = 4 * (H + 2) * EPS32 * (d.abs() @ we.abs())
    z = torch.sigmoid(g)
    s, slope = g * z * u, z * (1 + g * (1 - z))
    fn = (g.abs() + 8) * 4 * EPS32  # exp and the quotient, relative to z
    eps = EPS16 if dtype == BF16 else EPS32

    def close(got, ref, tol, what):
        within(got, ref, tol + eps * (ref.abs() + tol) + 1e-30, what)

    close(h, pr * s, (pr * s).abs() * fn, "h")
    rg, ru = pr * dh * u * slope, pr * dh * g * z
    # the slope's terms z and g z (1 - z) carry the error of z each
    slope_err = (z + 2 * g.abs() * z) * fn
    close(da[:, :F], rg, pr * (err * (u * slope).abs() + (dh * u).abs() * slope_err) + rg.abs() * 8 * EPS32, "dg")
    close(da[:, F:], ru, pr * (err * (g * z).abs()) + ru.abs() * (fn + 8 * EPS32), "du")
    if p is None:
        assert dp is None
        return
    assert dp.dtype == p.dtype
    ref = torch.zeros(N, E, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(ref)
    for e, lo, hi, tok in spans(mask, k):
        ref[tok, e] = (dh * s)[lo:hi].sum(1)
        tol[tok, e] = (err * s.abs() + (dh * s).abs() * (fn + 4 * (F + 4) * EPS32))[lo:hi].sum(1)
    assert not dp[~mask.cuda()].any()
    within(dp, ref, tol + (EPS16 if pdtype == BF16 else EPS32) * (ref.abs() + tol) + 1e-30, "dp")


def test_swiglu_grad_against_differences(dl):
    # the loss sum(dy * y) of the fp32 layer y_t = sum_e p_te W2_e (silu(g) u), g and u as checkpointed: central
    # differences of it in 64 bits along random directions of g, u and p against the gradients
    N, E, k, H, F = 40, 6, 2, 24, 48
    gen = _gen(11)
    mask = choose(gen, N, E, k)
    rows = device_rows(dl, mask, k)
    x, w1 = _normal(gen, N, H), _normal(gen, E, 2 * F, H, scale=H ** -0.5)
    w2, dy = _normal(gen, E, H, F, scale=F ** -0.5), _normal(gen, N, H)
    p = torch.rand(N, E, generator=gen).cuda()
    _, kept = dl.do_expert_swiglu(x, w1, rows, p, checkpoint=True)
    da, h, dp = dl.do_expert_swiglu_grad(dy, w2, rows, kept, p)
    a = dl.do_act8_unpack(kept, F32).double().view(N * k, 2 * F)
    ev = torch.empty(N * k, dtype=torch.long)
    for e, lo, hi, _ in spans(mask, k):
        ev[lo:hi] = e
    ev, tok = ev.cuda(), rows.row_token.long()

    def loss(a, p):
        s = p[tok, ev][:, None] * _silu64(a[:, :F]) * a[:, F:]
        o = torch.bmm(w2[ev].double(), s[:, :, None])[:, :, 0]
        return (dy.double()[tok] * o).sum()

    for seed in range(3):
        va = torch.randn(N * k, 2 * F, generator=_gen(seed), dtype=torch.float64).cuda()
        vp = torch.randn(N, E, generator=_gen(seed + 9), dtype=torch.float64).cuda()
        t = 1e-4
        fd = (loss(a + t * va, p.double() + t * vp) - loss(a - t * va, p.double() - t * vp)) / (2 * t)
        an = (da.double() * va).sum() + (dp.double() * vp).sum()
        # third derivatives are of order one: the difference is off by about t^2 of the terms' magnitudes
        size = ((da.double() * va).abs().sum() + (dp.double() * vp).abs().sum()).item()
        assert abs(fd.item() - an.item()) <= (10 * t * t + 1e-6) * size, (fd.item(), an.item(), size)


# --- 8 bits ----------------------------------------------------------------------------------------------------------


def _act8_ref(x):
    """q, e of x [rows][W] in Python's exact arithmetic by element."""
    rows, W = x.shape
    v = x.double().cpu()
    q = torch.zeros(rows, W, dtype=torch.int8)
    e = torch.zeros(rows, -(-W // 32), dtype=torch.uint8)
    for r in range(rows):
        for c in range(0, W, 32):
            part = v[r, c:c + 32]
            if not part.isfinite().all():
                e[r, c // 32] = 255
                continue
            top = part.abs().max().item()
            m, ex = math.frexp(top)
            b = max(-126, ex - 7 + (1 if m > 127 / 128 else 0)) if top else -126
            assert top <= 127 * 2.0 ** b and (b == -126 or top > 127 * 2.0 ** (b - 1))
            e[r, c // 32] = b + 127
            q[r, c:c + 32] = torch.tensor([round(t * 2.0 ** -b) for t in part.tolist()], dtype=torch.int8)
    return q, e


@pytest.mark.parametrize("rows,W", [(1, 1), (3, 31), (5, 32), (4, 33), (7, 96), (6, 1001), (40, 64), (2, 2048)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_act8(dl, rows, W, dtype):
    print(f"[case] act8 rows={rows} W={W} {dtype}", flush=True)
    gen = _gen(rows + W)
    x = torch.randn(rows, W, generator=gen) * torch.exp2(torch.randint(-140, 120, (rows, 1), generator=gen).float())
    x[:, ::7] = 0.0
    x[0, 0] = 127.0 * 2.0 ** 3
    if rows > 2:
        x[1] = 0.0
        x[2, 0] = 127.5  # just past 127 2^0
    if rows > 3:
        x[3, W - 1] = 3.3e38
    x = x.to(dtype)
    a = dl.do_act8_pack(x.cuda())
    q, e = _act8_ref(x)
    assert torch.equal(a.e.cpu(), e)
    assert torch.equal(a.q.cpu(), q)
    for out in (F32, BF16):
        back = dl.do_act8_unpack(a, out)
        ref = q.double() * torch.exp2(e.double() - 127).repeat_interleave(32, 1)[:, :W]
        assert back.dtype == out and torch.equal(back.cpu().double(), ref)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_act8_not_finite(dl, dtype, bad):
    x = torch.randn(4, 72, generator=_gen(1)).to(dtype)
    x[1, 40] = bad
    x[3, 71] = bad
    a = dl.do_act8_pack(x.cuda())
    back = dl.do_act8_unpack(a, F32).cpu()
    lost = torch.zeros(4, 72, dtype=torch.bool)
    lost[1, 32:64] = lost[3, 64:] = True
    assert torch.equal(back.isnan(), lost)
    assert (a.e.cpu() == 255).sum() == 2


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_act8_element_alignment(dl, dtype):
    x = torch.randn(9 * 64 + 1, generator=_gen(2)).to(dtype).cuda()[1:].view(9, 64)
    a = dl.do_act8_pack(x)
    q, e = _act8_ref(x)
    assert torch.equal(a.q.cpu(), q) and torch.equal(a.e.cpu(), e)
    buf = torch.zeros(9 * 64 + 1, dtype=dtype, device="cuda")
    back = dl.do_act8_unpack(a, dtype, out=buf[1:].view(9, 64))
    assert torch.equal(back, dl.do_act8_unpack(a, dtype)) and buf[0] == 0


def test_not_finite_checkpoint_reaches_only_its_group(dl):
    # an infinite pre-activation: its group of 32 reads back as NaN, nothing else does
    N, E, k, H, F = 20, 2, 1, 8, 64
    mask = choose(_gen(1), N, E, k)
    rows = device_rows(dl, mask, k)
    gen = _gen(2)
    x, w1 = _normal(gen, N, H), _normal(gen, E, 2 * F, H)
    tok = 7
    w1[:, 5, :] = 1e38
    x[tok] = 100.0
    _, kept = dl.do_expert_swiglu(x, w1, rows, checkpoint=True)
    back = dl.do_act8_unpack(kept, F32)
    # of the other tokens, those whose product passes fp32's largest value are lost too
    terms = x.double()[rows.row_token.long()] * 1e38
    sure, possible = terms.sum(1).abs() > 3.5e38, terms.abs().sum(1) > 3.4e38
    assert sure[rows.row_token == tok].all()
    nan = back.isnan()
    assert nan[sure, 0, :32].all() and not nan[~possible].any()
    assert not nan[:, 0, 32:].any() and not nan[:, 1].any()


# --- streams, graphs and repeats -------------------------------------------------------------------------------------


def _layer(dl, bits, x, p, w1, w2, dy):
    N, k = x.shape[0], 2
    rows = dl.do_expert_rows(bits, N, k)
    h, kept = dl.do_expert_swiglu(x, w1, rows, p, checkpoint=True)
    y = dl.do_expert_combine(dl.do_expert_matmul(h, w2, rows), rows)
    da, h2, dp = dl.do_expert_swiglu_grad(dy, w2, rows, kept, p)
    dw2 = dl.do_expert_weight_grad(dy, h2, rows, gather_dy=True)
    dw1 = dl.do_expert_weight_grad(da, x, rows, gather_x=True)
    dx = dl.do_expert_combine(dl.do_expert_matmul(da, w1, rows, transposed=True), rows)
    return [y, dp, dw1, dw2, dx, dl.do_act8_unpack(dl.do_act8_pack(x), BF16)]


def _layer_inputs(seed, N=900, E=6, H=128, F=96):
    gen = _gen(seed)
    mask = choose(gen, N, E, 2)
    return [signatures(mask.cuda()), _normal(gen, N, H, dtype=BF16), torch.rand(N, E, generator=gen).cuda(),
            _normal(gen, E, 2 * F, H, dtype=BF16, scale=H ** -0.5),
            _normal(gen, E, H, F, dtype=BF16, scale=F ** -0.5), _normal(gen, N, H, dtype=BF16)]


def test_layer_repeats_bit_for_bit_on_another_stream(dl):
    args = _layer_inputs(21)
    first = _layer(dl, *args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = _layer(dl, *args)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_layer_in_a_graph(dl):
    args = _layer_inputs(22)
    others = [_layer_inputs(s) for s in (23, 24, 25)]
    eager = [_layer(dl, *o) for o in others]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _layer(dl, *args)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _layer(dl, *args)
    for o, want in zip(others, eager):
        for dst, src in zip(args, o):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)

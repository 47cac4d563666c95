"""The whole layer of a few tokens against its definition in 64 bits."""
import numpy as np
import pytest
import torch

from expert_util import EPS16, EPS32, device_rows, within
from fp8_util import values

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def dl():
    import paper_2609_32398_amd as p

    return p


def _gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def chosen(scores, k):
    """[N][E] truth values: each token's k best, larger scores first, equal ones by the lower expert, NaN last."""
    s = scores.double().cpu().numpy()
    N, E = s.shape
    mask = torch.zeros(N, E, dtype=torch.bool)
    for t in range(N):
        nan = np.isnan(s[t])
        order = np.lexsort((np.arange(E), -np.where(nan, 0, s[t]), nan))
        mask[t, torch.from_numpy(order[:k].copy())] = True
    return mask


def _layer64(x, w1, w2, p, mask, dtype):
    """y, and the bound on what fp32 sums, the activations' rounding to dtype and y's own leave."""
    F, H = w2.shape[2], w1.shape[2]
    eps = EPS16 if dtype == BF16 else EPS32
    y = torch.zeros(x.shape[0], H, dtype=torch.float64, device="cuda")
    tol, size = torch.zeros_like(y), torch.zeros_like(y)
    for e in mask.any(0).nonzero()[:, 0].tolist():
        tok = mask[:, e].nonzero()[:, 0].cuda()
        v, a1, a2 = x[tok].double(), w1[e].double(), w2[e].double()
        a, da = v @ a1.t(), 4 * (H + 2) * EPS32 * (v.abs() @ a1.abs().t())
        g, u, dg, du = a[:, :F], a[:, F:], da[:, :F], da[:, F:]
        pr = (p[tok, e].double() if p is not None else torch.ones(tok.numel(), dtype=torch.float64, device="cuda"))[:, None]
        s = g * torch.sigmoid(g)
        h = pr * s * u
        # |silu'| < 1.1; exp and the quotient are off by (|g| + 8) 2^-22 relative
        dh = pr.abs() * (1.1 * dg * u.abs() + s.abs() * du + 1.1 * dg * du) + h.abs() * (g.abs() + 8) * 4 * EPS32
        dh = dh + eps * (h.abs() + dh)
        y[tok] += h @ a2.t()
        tol[tok] += dh @ a2.abs().t()
        size[tok] += (h.abs() + dh) @ a2.abs().t()
    k = int(mask.sum(1).max())
    tol = tol + 4 * (F + k + 16) * EPS32 * size
    return y, tol + eps * (y.abs() + tol) + 1e-30


def _inputs(dl, gen, N, E, k, H, F, dtype, w8, pdtype=F32, sdtype=F32):
    scores = torch.randn(N, E, generator=gen).to(sdtype).cuda()
    x = torch.randn(N, H, generator=gen).to(dtype).cuda()
    w1 = (torch.randn(E, 2 * F, H, generator=gen) * H ** -0.5).to(dtype).cuda()
    w2 = (torch.randn(E, H, F, generator=gen) * F ** -0.5).to(dtype).cuda()
    if w8:
        w1, w2 = dl.do_fp8_pack(w1, weights=True), dl.do_fp8_pack(w2, weights=True)
    p = None if pdtype is None else torch.rand(N, E, generator=gen).to(pdtype).cuda()
    return x, scores, w1, w2, p


def _weights(w):
    return w.double() if torch.is_tensor(w) else values(w, True)


def _check(dl, x, scores, k, w1, w2, p, **kw):
    y = dl.do_expert_layer(x, scores, k, w1, w2, p, **kw)
    ref, tol = _layer64(x, _weights(w1), _weights(w2), p, chosen(scores, k), x.dtype)
    assert y.dtype == x.dtype
    within(y, ref, tol, "y")
    return y


# N, E, k, H, F: one token to 64, one expert to 1,024, widths below, at and past a step, a block of 128 and four waves'
# shares, odd ones, more rows than a matrix tile holds, every expert chosen
SIZES = [(1, 1, 1, 1, 1), (1, 8, 2, 64, 32), (1, 128, 8, 256, 96), (2, 3, 3, 7, 5), (3, 16, 1, 130, 40),
         (5, 64, 6, 200, 33), (16, 32, 4, 128, 128), (17, 8, 2, 136, 72), (33, 4, 3, 100, 17), (37, 64, 6, 333, 100),
         (64, 2, 1, 96, 48), (64, 1, 1, 80, 64), (64, 256, 8, 72, 24), (64, 300, 9, 40, 16), (9, 1024, 16, 48, 8),
         (48, 5, 5, 257, 129), (1, 16, 16, 640, 272), (20, 6, 2, 1040, 336)]


@pytest.mark.parametrize("N,E,k,H,F", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("w8", [False, True])
@pytest.mark.parametrize("pdtype,sdtype", [(F32, F32), (BF16, BF16), (None, F32)])
def test_layer(dl, N, E, k, H, F, dtype, w8, pdtype, sdtype):
    print(f"[case] layer N={N} E={E} k={k} H={H} F={F} {dtype} w8={w8} p={pdtype} scores={sdtype}", flush=True)
    x, scores, w1, w2, p = _inputs(dl, _gen(N + E + H), N, E, k, H, F, dtype, w8, pdtype, sdtype)
    _check(dl, x, scores, k, w1, w2, p)


@pytest.mark.parametrize("E,k", [(12, 5), (300, 40), (64, 64)])
@pytest.mark.parametrize("sdtype", [F32, BF16])
def test_layer_takes_ties_infinities_and_nan_as_the_ranking_does(dl, E, k, sdtype):
    N, H, F = 24, 64, 16
    x, scores, w1, w2, p = _inputs(dl, _gen(E), N, E, k, H, F, F32, False)
    scores = scores.round().to(sdtype)  # many ties, both zeros
    scores[1], scores[2, 1:] = 0.0, float("nan")
    scores[3], scores[4, ::2], scores[5, ::3], scores[6, 1::2] = float("nan"), float("inf"), float("-inf"), -0.0
    scores[7], scores[8, : E // 2], scores[8, E // 2:] = float("-inf"), float("nan"), float("-inf")
    print(f"[case] layer ranking E={E} k={k} {sdtype}", flush=True)
    _check(dl, x, scores, k, w1, w2, p)
    bits = dl.do_topk_signature(scores, k)
    word = bits.view(-1, E, 8)[0, :, 0].cpu()
    mask = torch.stack([(word >> t) & 1 for t in range(N)]).bool()
    assert torch.equal(mask, chosen(scores, k))


@pytest.mark.parametrize("N", [1, 13, 40])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("w8", [False, True])
def test_layer_is_untouched_by_what_it_does_not_choose(dl, N, dtype, w8):
    E, k, H, F = 8, 2, 272, 144
    x, scores, w1, w2, p = _inputs(dl, _gen(N), N, E, k, H, F, dtype, w8)
    scores[:, 3], scores[:, 6] = float("-inf"), float("-inf")
    print(f"[case] layer unchosen N={N} {dtype} w8={w8}", flush=True)
    clean = _check(dl, x, scores, k, w1, w2, p)
    if w8:
        w1.e[3], w2.e[6] = 255, 255
        w1.q.view(torch.uint8)[6], w2.q.view(torch.uint8)[3] = 0x7F, 0x7F
    else:
        w1[3], w2[3], w1[6], w2[6] = float("nan"), float("inf"), float("-inf"), float("nan")
    p = p.masked_fill(~chosen(scores, k).cuda(), float("nan"))
    assert torch.equal(dl.do_expert_layer(x, scores, k, w1, w2, p), clean)
    # a token's NaN, and an expert's for those who chose it, reach their rows alone
    mask = chosen(scores, k)
    if N > 1:
        x2 = x.clone()
        x2[N // 2, 5] = float("nan")
        got = dl.do_expert_layer(x2, scores, k, w1, w2, p)
        rest = torch.arange(N) != N // 2
        assert torch.equal(got[rest], clean[rest]) and got[N // 2].isnan().all()
    e = int(mask.sum(0).argmax())
    hit = mask[:, e].cuda()
    if w8:
        w2.e[e, 1] = 255  # output columns 128 to 255
        got = dl.do_expert_layer(x, scores, k, w1, w2, p)
        assert got[hit][:, 128:256].isnan().all() and torch.equal(got[:, :128], clean[:, :128])
        w1.e[e, 0, 0] = 255
    else:
        w1[e, 0, 3] = float("nan")
    got = dl.do_expert_layer(x, scores, k, w1, w2, p)
    assert got[hit].isnan().all() and torch.equal(got[~hit], clean[~hit])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("w8", [False, True])
def test_layer_alignment_and_out(dl, dtype, w8):
    N, E, k, H, F = 6, 8, 2, 64, 48
    x, scores, w1, w2, p = _inputs(dl, _gen(5), N, E, k, H, F, dtype, w8)

    def moved(t):
        b = torch.zeros(t.numel() + 1, dtype=torch.uint8 if t.element_size() == 1 else t.dtype, device="cuda")
        b[1:] = (t.view(torch.uint8) if t.element_size() == 1 else t).flatten()
        return b[1:].view(t.dtype).view(t.shape)

    y = _check(dl, x, scores, k, w1, w2, p)
    buf = torch.full((N * H + 2,), 7.0, dtype=dtype, device="cuda")
    out = buf[1:-1].view(N, H)
    m1, m2 = (dl.Fp8(moved(w1.q), moved(w1.e)), dl.Fp8(moved(w2.q), moved(w2.e))) if w8 else (moved(w1), moved(w2))
    print(f"[case] layer alignment {dtype} w8={w8}", flush=True)
    assert dl.do_expert_layer(moved(x), moved(scores), k, m1, m2, moved(p), out=out) is out
    assert torch.equal(out, y) and buf[0] == 7.0 and buf[-1] == 7.0


def test_layer_far_weights(dl):
    # an expert whose weights lie past 2^31 and 2^32 elements
    N, E, k, H, F = 3, 40, 2, 8192, 4096
    gen = _gen(8)
    w1 = torch.empty(E, 2 * F, H, dtype=torch.uint8, device="cuda")
    w1.view(-1).view(torch.int64).random_(0, 1 << 62)
    w1 &= 0xBF  # finite, within 1.875
    w2 = torch.empty(E, H, F, dtype=torch.uint8, device="cuda")
    w2.view(-1).view(torch.int64).random_(0, 1 << 62)
    w2 &= 0xBF
    f8 = torch.float8_e4m3fn
    w1 = dl.Fp8(w1.view(f8), torch.full((E, 2 * F // 128, H // 128), 120, dtype=torch.uint8, device="cuda"))
    w2 = dl.Fp8(w2.view(f8), torch.full((E, H // 128, F // 128), 120, dtype=torch.uint8, device="cuda"))
    x = torch.randn(N, H, generator=gen).bfloat16().cuda()
    scores = torch.zeros(N, E, device="cuda")
    scores[0, 39], scores[1, 38], scores[2, 20] = 2.0, 2.0, 2.0
    scores[:, 33] = 1.0
    print("[case] layer far weights", flush=True)
    y = dl.do_expert_layer(x, scores, k, w1, w2)
    mask = chosen(scores, k)
    use = mask.any(0).nonzero()[:, 0]
    a1 = torch.zeros(E, dtype=torch.long)
    a1[use] = torch.arange(use.numel())
    part1 = values(dl.Fp8(w1.q[use.cuda()], w1.e[use.cuda()]), True)
    part2 = values(dl.Fp8(w2.q[use.cuda()], w2.e[use.cuda()]), True)
    ref, tol = _layer64(x, part1, part2, None, mask[:, use], BF16)
    within(y, ref, tol, "y")


@pytest.mark.parametrize("dtype,w8", [(F32, False), (BF16, True)])
def test_layer_beside_the_operators_it_stands_for(dl, dtype, w8):
    # the same weights, packed or not, through do_expert_rows, do_expert_swiglu, do_expert_matmul and do_expert_combine
    N, E, k, H, F = 40, 16, 4, 256, 128
    x, scores, w1, w2, p = _inputs(dl, _gen(12), N, E, k, H, F, dtype, w8)
    print(f"[case] layer beside the chain {dtype} w8={w8}", flush=True)
    y = dl.do_expert_layer(x, scores, k, w1, w2, p)
    u1, u2 = (dl.do_fp8_unpack(w, dtype) if w8 else w for w in (w1, w2))
    rows = dl.do_expert_rows(dl.do_topk_signature(scores, k), N, k)
    want = device_rows(dl, chosen(scores, k), k)
    assert all(torch.equal(a, b) for a, b in zip(rows, want))
    h, _ = dl.do_expert_swiglu(x, u1, rows, p)
    o = dl.do_expert_matmul(h, u2, rows)
    chain = dl.do_expert_combine(o, rows)
    ref, tol = _layer64(x, _weights(w1), _weights(w2), p, chosen(scores, k), dtype)
    within(y, ref, tol, "layer")
    at = rows.token_row.long()
    # the chain rounds each expert's output as well
    within(chain, ref, tol + (EPS16 if dtype == BF16 else EPS32) * 1.01 * o.double()[at].abs().sum(1), "chain")


def test_layer_streams_and_replays(dl):
    N, E, k, H, F = 16, 32, 4, 256, 160
    gen = _gen(30)
    x, scores, w1, w2, p = _inputs(dl, gen, N, E, k, H, F, BF16, True)
    inputs = [(torch.randn(N, H, generator=gen).bfloat16().cuda(), torch.randn(N, E, generator=gen).cuda(),
               torch.rand(N, E, generator=gen).cuda()) for _ in range(4)]
    print("[case] layer streams and graphs", flush=True)
    want = [dl.do_expert_layer(a, b, k, w1, w2, c) for a, b, c in inputs]
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s, (a, b, c) in zip(streams, inputs):  # calls on three streams at once
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
    for i in (2, 0, 3, 1):
        for dst, src in zip((x, scores, p), inputs[i]):
            dst.copy_(src)
        for g, _ in graphs:
            g.replay()
        eager = dl.do_expert_layer(x, scores, k, w1, w2, p)
        torch.cuda.synchronize()
        assert torch.equal(graphs[0][1], want[i]) and torch.equal(graphs[1][1], want[i]) and torch.equal(eager, want[i])

"""Routed rows and 64-bit references for the experts' tests."""
import torch

EPS32 = 2.0 ** -24  # relative rounding of one fp32 operation
EPS16 = 2.0 ** -8   # half a unit in the last place of bf16, relative


def signatures(mask: torch.Tensor) -> torch.Tensor:
    """[N][E] truth values -> the library's signatures [U, E, 8] (int64 words)."""
    N, E = mask.shape
    U = (N + 511) // 512
    m = torch.zeros(U * 512, E, dtype=torch.bool, device=mask.device)
    m[:N] = mask
    bit = torch.ones(64, dtype=torch.int64, device=mask.device) << torch.arange(64, device=mask.device)
    return (m.view(U, 8, 64, E) * bit.view(1, 1, 64, 1)).sum(2).permute(0, 2, 1).contiguous()


def choose(gen, N, E, k, dist="even") -> torch.Tensor:
    """[N][E]: k experts of each token.  dist "even", "idle" (every third expert unused where k are left) or
    "one" (the first k experts take every token)."""
    s = torch.rand(N, E, generator=gen)
    if dist == "idle" and E - (E + 2) // 3 >= k:
        s[:, ::3] -= 2.0
    if dist == "one":
        s[:, :k] += 2.0
    m = torch.zeros(N, E, dtype=torch.bool)
    return m.scatter_(1, s.topk(k, dim=1).indices, True)


def rows_of(mask: torch.Tensor, k: int):
    """(offsets, row_token, token_row, token_expert) by loops' definition: token choices past the k-th left out."""
    N, E = mask.shape
    take = mask & (mask.int().cumsum(1) <= k)
    load = take.sum(0)
    offsets = torch.zeros(E + 1, dtype=torch.int64)
    offsets[1:] = load.cumsum(0)
    et = take.t().nonzero()
    row_token = et[:, 1].clone()
    row_of = torch.full((N, E), -1, dtype=torch.int64)
    row_of[et[:, 1], et[:, 0]] = torch.arange(et.shape[0])
    token_row = torch.full((N, k), -1, dtype=torch.int64)
    token_expert = torch.full((N, k), -1, dtype=torch.int64)
    te = take.nonzero()
    place = (take.int().cumsum(1) - 1)[te[:, 0], te[:, 1]]
    token_row[te[:, 0], place] = row_of[te[:, 0], te[:, 1]]
    token_expert[te[:, 0], place] = te[:, 1]
    return offsets, row_token, token_row, token_expert


def device_rows(dl, mask, k):
    """The reference rows as an ExpertRows on the device (entries past the last row are zero)."""
    offsets, row_token, token_row, token_expert = rows_of(mask, k)
    full = torch.zeros(mask.shape[0] * k, dtype=torch.int64)
    full[: row_token.numel()] = row_token
    return dl.ExpertRows(*(t.int().cuda() for t in (offsets, full, token_row, token_expert)))


def spans(mask, k):
    """[(expert, first row, last row + 1, tokens)] of the experts that have rows."""
    offsets, row_token, _, _ = rows_of(mask, k)
    o = offsets.tolist()
    return [(e, o[e], o[e + 1], row_token[o[e]:o[e + 1]].cuda()) for e in range(len(o) - 1) if o[e + 1] > o[e]]


def within(got: torch.Tensor, ref: torch.Tensor, tol: torch.Tensor, what: str):
    """Every element within its tolerance (all float64)."""
    err = (got.double() - ref).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: "
                           f"got {got.double()[bad][0].item()}, expected {ref[bad][0].item()} "
                           f"+- {tol[bad][0].item()}")


def product_tol(size: torch.Tensor, K: int, ref: torch.Tensor, dtype):
    """Bound on a K-term fp32 sum of products whose magnitudes sum to `size` (each of K sums and products
    may be off by EPS32 of the running magnitude, twice that where the hardware truncates), and the
    rounding of the stored result."""
    return 4 * (K + 2) * EPS32 * size + (EPS16 if dtype == torch.bfloat16 else EPS32) * ref.abs() + 1e-30

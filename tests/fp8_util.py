"""The 8-bit floating point format in 64 bits, and operands whose products are exact, for the experts' tests."""
import torch

BLOCK = 128
E4M3 = torch.float8_e4m3fn
HALF = 2.0 ** -4   # a rounding to e4m3, relative to the value, from 2^-6 on
TINY = 2.0 ** -10  # and below: half of the step 2^-9


def blocks(n):
    return -(-n // BLOCK)


def power(e):
    """2^e in float64, exactly (torch.ldexp goes through pow, which is off by a unit), for -1022 <= e <= 1023."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def spread(e, shape, weights):
    """Exponents of blocks, one for each element of `shape`."""
    e = e.repeat_interleave(BLOCK, -1)[..., : shape[-1]]
    return e.repeat_interleave(BLOCK, -2)[..., : shape[-2], :] if weights else e


def round_fp8(v):
    """e4m3 values of v (float64, within 448), ties to even."""
    e = torch.frexp(v)[1].clamp(min=-5) - 4  # 2^(floor(log2 |v|) - 3), 2^-9 at least
    step = power(e)
    return torch.round(v / step) * step


def pack_ref(x, weights=False):
    """(values, exponents) of finite x by the definition, in float64."""
    x = x.double()
    v = torch.nn.functional.pad(x.abs(), (0, -x.shape[-1] % BLOCK)).unflatten(-1, (-1, BLOCK)).amax(-1)
    if weights:
        v = torch.nn.functional.pad(v, (0, 0, 0, -v.shape[-2] % BLOCK)).unflatten(-2, (-1, BLOCK)).amax(-2)
    m, ex = torch.frexp(v)  # m 2^ex <= 448 2^e = 0.875 2^(9 + e)
    e = torch.where(v > 0, ex - 9 + (m > 0.875).int(), torch.full_like(ex, -120)).clamp(min=-120)
    return round_fp8(x * spread(power(-e), x.shape, weights)), e


def values(a, weights=False):
    """What an Fp8 stands for, in float64."""
    f = power(a.e.int() - 127)
    f = torch.where(a.e == 255, torch.full_like(f, float("nan")), f)
    return a.q.double() * spread(f, a.q.shape, weights)


def lattice(dl, gen, *shape, weights=False, scale=0):
    """An Fp8 of whole numbers up to 7 times 2^-1, 2^0 or 2^1 (times 2^scale) a block: the product of two of them is a
    multiple of a quarter, at most 196, so that sums of 2^15 such products are exact in fp32's 24 bits, and no bit of
    one is below 2^-13 of another's."""
    q = torch.randint(-7, 8, shape, generator=gen).float()
    eshape = (*shape[:-2], blocks(shape[-2]), blocks(shape[-1])) if weights else (*shape[:-1], blocks(shape[-1]))
    e = torch.randint(126, 129, eshape, generator=gen) + scale
    return dl.Fp8(q.to(E4M3).cuda(), e.to(torch.uint8).cuda())


def eight_bit_tol(size):
    """Bound on what the matrix instructions drop: below 2^-13 of the largest of each eight products, so 2^-10 of the
    eight's magnitudes at most, which sum to `size`."""
    return 2.0 ** -10 * size


def same(got, ref, what):
    """Equal element by element (NaN to nothing), with a short account of what is not."""
    assert got.shape == ref.shape and got.dtype == ref.dtype, (what, got.shape, ref.shape, got.dtype, ref.dtype)
    bad = ~(got == ref)
    n = int(bad.sum())
    assert n == 0, (f"{what}: {n} of {bad.numel()} differ, first at {bad.nonzero()[0].tolist()}: "
                    f"{got[bad][0].item()!r}, expected {ref[bad][0].item()!r}")

"""Plain 64-bit forms of 8-bit cache rows: e4m3 codes with a power of two a row."""
import torch

import paged_util as pu

LEAST = 16      # the least scale byte: 2^-111


def scale_bytes(x):
    """x float64 [..., hd]: the byte of the least power of two s >= 2^-111 with max |x| <= 448 s, over the values that are finite."""
    most = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    frac, exp = torch.frexp(most / 448.0)                     # (exact: 448 = 7 x 64 divides without changing on which side of a power of two the quotient lies)
    e = torch.where(frac == 0.5, exp - 1, exp) + 127
    return torch.where(most > 0, e, LEAST).clamp(min=LEAST).to(torch.uint8)


def power(e):
    return torch.exp2(e.double() - 127).unsqueeze(-1)


def half_step(x, e):
    """Half a step of the codes at x, under scale byte e: 2^-4 of the power of two below |x| / s, at least half of the smallest code, 2^-10."""
    y = (x / power(e)).abs()
    return torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 4) * power(e)


def codes(x, e):
    """Nearest codes of x / s, ties to the even one, as values (float64) and as bytes; what is not finite is NaN."""
    y = x / power(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    q = torch.round(y / step) * step
    q = torch.where(torch.isfinite(y), q, torch.full_like(q, float("nan")))
    return q, q.float().to(torch.float8_e4m3fn).view(torch.uint8)


def stored(x):
    """Bytes, scale bytes and the values they stand for (float64) of rows x."""
    e = scale_bytes(x.double())
    q, b = codes(x.double(), e)
    return b, e, q * power(e)


def values(b, e):
    """float64 values of code bytes and scale bytes; a scale of 255 is NaN."""
    v = b.view(torch.float8_e4m3fn).double() * power(e)
    return torch.where((e == 255).unsqueeze(-1), torch.full_like(v, float("nan")), v)


def attention(qkv, nq, k, v, *rest):
    """paged_util.attention over the bf16 values that the codes stand for, queries in two bf16 parts (the last argument), and what one bf16 part of a probability adds to how far a
    kernel's may be off: each enters its product rounded by at most 2^-8 of itself, so the output is off by at most 2^-8 of sum p |v| (its divisor sums the probabilities unrounded)."""
    out, tol = pu.attention(qkv, nq, k, v, *rest)
    size, _ = pu.attention(qkv, nq, k, v.abs(), *rest)
    return out, tol + 2.0 ** -8 * size

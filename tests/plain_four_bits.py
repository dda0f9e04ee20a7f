"""K and V in 4 bits written out in 64 bits, and how far an attention over them may lie from the formula.

A rounding is off by at most half a step: 2^-8 of the value in bf16, 2^-24 in fp32."""
import math

import torch

import plain_operators as plain

GROUP = 32
NUMBERS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]   # e2m1
_two_to = plain._two_to


def _least_exponent(m, most, lo, hi):
    """The least e in [lo, hi] with m <= most * 2^e, as fp64."""
    e = torch.frexp(m)[1].double() - 5
    for _ in range(5):
        e = torch.where(m > most * _two_to(e.clamp(-900, 900)), e + 1, e)
    return e.clamp(lo, hi)


def exponents(x):
    """x [..., D] -> the exponent of each group, fp64 [..., D / 32, 1]."""
    m = x.double().unflatten(-1, (-1, GROUP)).abs().amax(dim=-1, keepdim=True)
    return _least_exponent(m, 7.0, -100, 125)


def held(x):
    """x [..., D] as 4 bits hold it, fp64."""
    y = x.double().unflatten(-1, (-1, GROUP))
    scale = _two_to(exponents(x))
    numbers = torch.tensor(NUMBERS, dtype=torch.float64, device=x.device)
    z = (y.abs() / scale).clamp(max=6.0)
    hi = torch.searchsorted(numbers, z.contiguous()).clamp(max=7)
    lo = (hi - 1).clamp(min=0)
    up, down = numbers[hi] - z, z - numbers[lo]
    out = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), numbers[hi], numbers[lo])
    return (out * scale * torch.sign(y)).flatten(-2)


def attention(q, k, v, scale):
    """As plain.attention, over held k and v, with the products' rounding of Q: y = q * scale * log2(e), whose group's largest is m, 2^a the
    least power with m <= 7.5 * 2^a, is held as the number of 4 significant bits next to y * 2^-a, times 2^a, and the number of 4 significant
    bits (steps of 1/8 at least, up to 7.5) next to 2^5 times what is left, r.  r is at most 1/4, 1/8 or 1/16 where |y| * 2^-a is 4, 2 or less than
    2, the second number then at most 8, 4 or 2 with steps of 1/2, 1/4 or 1/8: half of them are 2^(a - 7), 2^(a - 8), 2^(a - 9), but beyond
    7.75, for which 7.5 stands, up to 2^(a - 6).  (A y on the grid that the two have there is off by its roundings in fp32 alone, 2^-20 of it at
    most.)  That moves a score, as a power of
    two, by at most the sum of these times |k|, and a weight, relative to the others', by a factor of 2 to twice that.

    Weights of 2^-120 of the largest and less may vanish: a reference that is up to 2^6 below the largest weight of its time is left for
    one more than 2^126 above it by a factor that fp32 flushes to 0 (held values may be 0 where the weight is 1, so that this shows)."""
    q, k, v = (x.double() for x in (q, k, v))
    o, bound = plain.attention(q, k, v, scale)
    y = (q * (scale * math.log2(math.e))).unflatten(-1, (-1, GROUP))
    one = _two_to(_least_exponent(y.abs().amax(dim=-1, keepdim=True), 7.5, -110, 130))
    size = y.abs() / one
    grid = one * torch.where(size >= 3.99, 2.0 ** -6, torch.where(size >= 1.99, 2.0 ** -7, 2.0 ** -8))
    ends = (size >= 3.9) & ((size - torch.round(size * 2) / 2).abs() > 7.7 / 32)
    on_it = ((y - torch.round(y / grid) * grid).abs() <= 2.0 ** -20 * y.abs()) & ~ends
    step = torch.where(ends, 2.0 ** -6, torch.where(size >= 3.9, 2.0 ** -7, torch.where(size >= 1.9, 2.0 ** -8, 2.0 ** -9)))
    off = torch.where(on_it, 2.0 ** -20 * y.abs(), one * step).flatten(-2)
    far = (off @ k.abs().transpose(-1, -2)).amax(dim=-1, keepdim=True) * math.log(2)
    s = q @ k.transpose(-1, -2) * scale
    p, rel = torch.softmax(s, dim=-1), torch.exp(s - s.amax(dim=-1, keepdim=True))
    size, lost = p @ v.abs(), torch.where(rel <= 1.01 * 2.0 ** -120, p, torch.zeros_like(p)) @ v.abs()
    return o, bound * torch.exp(2 * far) + torch.expm1(2 * far) * (size + o.abs()) + lost

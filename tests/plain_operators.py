"""The operators written out in 64 bits, and how far results in fewer bits may lie from them.

A rounding is off by at most half a step: 2^-8 of the value in bf16, 2^-24 in fp32, 2^-4 in e4m3 (2^-10 below 2^-6)."""
import math

import torch

BF16, F32 = 2.0 ** -8, 2.0 ** -24


def attention(q, k, v, scale):
    """q [..., Tq, D], k, v [..., Tk, D] in any type -> (O, bound), fp64.  Bound, element by element: the weights are rounded to
    bf16 and O is, 2^-8 each; a score is a sum of D products in fp32 (D + 2 roundings of 2^-24 of the sum of magnitudes, with the
    scale), and a weight's exponent is rounded once more, relative to itself (below 2^8 here): 2^-16, with the sum and the
    quotient a few 2^-24 more.

    The weights may be added up as they are rounded.  With p_i (1 + d_i), |d_i| <= 2^-8, in the sum of the products and in the sum
    that divides it, O is off by sum p_i d_i (v_i - o) / (1 + sum p_i d_i): at most 2^-8 sum p_i |v_i - o| <= 2^-8 (sum p_i |v_i| +
    |o|) to first order.  Two keys, p = (0.9, 0.1) and v = (0, a), show that the second term is needed: 0.18 a 2^-8 where sum
    p_i |v_i| = 0.1 a.  The division by 1 + sum p_i d_i >= 1 - 2^-8 is the factor of 1.004."""
    q, k, v = (x.double() for x in (q, k, v))
    s = q @ k.transpose(-1, -2) * scale
    p = torch.softmax(s, dim=-1)
    o = p @ v
    size = p @ v.abs()
    err = (q.shape[-1] + 2) * F32 * (q.abs() @ k.abs().transpose(-1, -2)).amax(dim=-1, keepdim=True) * scale + 2.0 ** -16
    return o, size * (BF16 * 1.004 + 2 * err) + o.abs() * 2.004 * BF16 + 1e-37


def frequencies(rot_dim, axes, base=10000.0, factor=1.0, original=0.0, low=0.0, high=0.0):
    out = []
    n = rot_dim // 2 // axes
    for i in range(n):
        f = base ** (-i / n)
        g = 0.0
        if low or high:
            g = min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low)))
        out.append(f * (g + (1 - g) / factor))
    return out


def table(positions, rot_dim, amplitude=1.0, **k):
    """positions fp64 [n][axes] -> fp64 [n][rot_dim/2][2]."""
    f = torch.tensor(frequencies(rot_dim, positions.shape[-1], **k), dtype=torch.float64, device=positions.device)
    angle = (positions[..., None] * f).flatten(-2)
    return amplitude * torch.stack((torch.cos(angle), torch.sin(angle)), dim=-1)


def turn(x, tab, pairing, back=False):
    """x [..., T, D], tab [..., T, pairs, 2] in one type, every product and sum rounded by itself in it."""
    c, s = tab[..., 0], tab[..., 1] * (-1 if back else 1)
    n = c.shape[-1]
    a = torch.arange(n, device=x.device) if pairing == "half" else torch.arange(0, 2 * n, 2, device=x.device)
    b = a + (n if pairing == "half" else 1)
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def e4m3_numbers():
    """All of them that are not negative, ascending."""
    return [m * 2.0 ** -9 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8) if (e, m) != (8, 7)]


def _two_to(e):
    """2^e, fp64, from its bits: torch's pow on the GPU is off by a unit in the last place at some whole e (-4 and 11 among them)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def held(x):
    """x [..., T, D] (a scale) as a cache of 8 bits holds it, fp64: block of 16 tokens by block.  (The next number above 1.875 *
    2^127 would be 2^128, which is not a bf16 number.)"""
    top = 1.875 * 2.0 ** 127
    n = x.shape[-2]
    x = x.double()
    y = torch.cat((x, x.new_zeros(*x.shape[:-2], -n % 16, x.shape[-1])), dim=-2).unflatten(-2, (-1, 16))
    m = y.abs().amax(dim=(-1, -2), keepdim=True)
    e = (torch.frexp(m)[1].double() - 10).clamp(min=-100)            # too small by two at most
    for _ in range(2):
        e = torch.where(m > 448 * _two_to(e), e + 1, e)
    assert bool(((m <= 448 * _two_to(e)) & ((m > 448 * _two_to(e - 1)) | (e == -100) | (m == 0))).all())
    numbers = torch.tensor(e4m3_numbers(), dtype=torch.float64, device=x.device)
    z = y.abs() / _two_to(e)
    hi = torch.searchsorted(numbers, z).clamp(max=len(numbers) - 1)       # the first number not below z
    lo = (hi - 1).clamp(min=0)
    up, down = numbers[hi] - z, z - numbers[lo]
    take_hi = (up < down) | ((up == down) & (hi % 2 == 0))                # ties to the even code
    out = torch.where(take_hi, numbers[hi], numbers[lo]) * _two_to(e) * torch.sign(y)
    return out.flatten(-3, -2)[..., :n, :].clamp(-top, top)

"""The 8-bit moments of the AdamW step from their definition, in 64 bits: what the tests compare with."""
import numpy as np
import torch

import oracle

BLOCK = 256


def blocks_of(numels):
    """First block of each tensor, and their number."""
    first = [0]
    for n in numels:
        first.append(first[-1] + (n + BLOCK - 1) // BLOCK)
    return first


def padded(xs, numels):
    """The tensors as blocks of 64 bits with zeros behind each one's last element."""
    first = blocks_of(numels)
    out = torch.zeros(first[-1], BLOCK, dtype=torch.float64)
    for x, n, b in zip(xs, numels, first):
        out.view(-1)[b * BLOCK: b * BLOCK + n] = x.detach().cpu().double().view(-1)
    return out


def chances(n_blocks, seed, t):
    """(blocks, 256): the 16 random bits of each element, over 2^16."""
    words = oracle.philox_draws(seed, t & 0xFFFFFFFF, t >> 32, 32, 4 * n_blocks).transpose(1, 0, 2)
    halves = np.stack([words & 0xFFFF, words >> 16], -1).reshape(n_blocks, BLOCK)
    return torch.from_numpy(halves.astype(np.float64)) / 65536


def exponent(top, binades):
    """The exponent byte of a block whose largest magnitude is `top`."""
    _, e = torch.frexp(top)
    up = top > (1 - 2.0 ** -4) * torch.exp2(e.double())                   # it may be rounded up to the next power of two
    field = torch.where(top > 0, e + 126 + up.int(), 0).clamp(min=0)
    return (field - (binades - 1)).clamp(0, 256 - binades)


def code(x, k, chance, binades):
    """The codes of blocks x >= 0 (normal numbers of fp32, or 0) with exponent bytes k."""
    _, e = torch.frexp(torch.where(x > 0, x, 1.0))
    unit = torch.exp2((e - 4).double())
    y = torch.floor(x / unit + chance) * unit                             # a multiple of an eighth of its power of two
    frac, e = torch.frexp(torch.where(y > 0, y, 1.0))
    c = (e + 126 - k[:, None]) * 8 + (frac * 16).int() - 8
    return torch.where(y > 0, c, 0).clamp(0, 8 * binades - 1)


def value(c, k, zero):
    """The values of codes; zero: code 0 is zero (m)."""
    field = k[:, None].int() + c // 8
    normal = (1 + (c % 8) / 8.0).double() * torch.exp2((field - 127).double())
    v = torch.where(field == 0, (c % 8) / 8.0 * 2.0 ** -126, normal)
    return torch.where(c == 0, 0.0, v) if zero else v


def read(state, n_blocks):
    """(m, v, codes of |m|, codes of v, exponents of both) of an 8-bit state."""
    s = state.cpu().int()
    n = n_blocks * BLOCK
    cm, cv, k = s[:n].view(-1, BLOCK), s[n: 2 * n].view(-1, BLOCK), s[2 * n:].view(-1, 2)
    m = value(cm & 127, k[:, 0], True)
    return torch.where(cm > 127, -m, m), value(cv, k[:, 1], False), cm & 127, cv, k

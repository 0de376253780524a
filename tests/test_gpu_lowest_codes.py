"""The 8-bit moments at and below their lowest codes."""
import pytest
import torch

import adamw8 as Q
from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_moments_around_their_lowest_codes():
    """beta 0: m is g, v is g^2.  The largest of a block is 1 (k = 112 for m, 96 for v: code 0 stands for 2^-15 and 2^-31)."""
    n = 1 << 16
    x = torch.zeros(n // 256, 256)
    x[:, 0] = 1.0
    steps = [0.0, 2.0 ** -40, 2.0 ** -16, 2.0 ** -15 * 0.999, 2.0 ** -15, 2.0 ** -15 * 1.0625, 2.0 ** -15 * 1.125, 2.0 ** -15 * 1.1875]
    for i, s in enumerate(steps):
        x[:, 1 + i * 31: 32 + i * 31] = -s if i % 2 else s
    p = torch.zeros(n, device="cuda")
    opt = B.AdamW([p], beta1=0.0, beta2=0.0, seed=9)
    opt.step([x.view(-1).cuda()], lr=1.0, t=0)
    m, v, cm, cv, k = Q.read(opt.state, n // 256)
    assert bool((k[:, 0] == 112).all()) and bool((k[:, 1] == 96).all())
    rows = n // 256 * 31
    for i, s in enumerate(steps):
        c, w = cm[:, 1 + i * 31: 32 + i * 31], cv[:, 1 + i * 31: 32 + i * 31]
        if s < 2.0 ** -15 * 1.01:
            assert not c.any()                                              # zero, every time
        elif s == 2.0 ** -15 * 1.125:
            assert bool((c == 1).all())                                     # a code's own value stays
        else:                                                               # half way: to either side (6 standard deviations of a fair coin)
            low = 0 if s < 2.0 ** -15 * 1.1 else 1
            assert bool(((c == low) | (c == low + 1)).all()) and abs((c > low).sum().item() - rows / 2) <= 6 * (rows / 4) ** 0.5
        if s * s < 2.0 ** -31:
            assert not w.any()                                              # raised to code 0, which is not zero
            assert bool((v[:, 1 + i * 31: 32 + i * 31] == 2.0 ** -31).all())

"""Roots and quotients of the list step with moments of 32 bits are rounded correctly."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gdt", [torch.float32, torch.bfloat16])
def test_steps_that_are_exact(gdt):
    """With beta 0, no eps and lr 1 a step is -g / sqrt(g g): gradients of up to 12 bits have exact squares, so their steps are -1 or 1."""
    g = torch.Generator().manual_seed(41)
    bits = 8 if gdt == torch.bfloat16 else 12
    n = 1 << 16
    x = (torch.randint(2 ** (bits - 1), 2 ** bits, (n,), generator=g) * torch.where(torch.rand(n, generator=g) < 0.5, -1, 1)).float()
    x = (x * torch.exp2(torch.randint(-30, 30, (n,), generator=g).float())).to(gdt).cuda()
    p = torch.zeros(n, device="cuda")
    opt = B.AdamW([p], bits=32, beta1=0.0, beta2=0.0, eps=0.0, bias_correction=False)
    opt.step([x], lr=1.0, t=0)
    assert torch.equal(p, -x.sign().float())


def test_the_step_of_an_elementwise_program():
    """Moments that are equal bit for bit, then a root, a sum, a quotient and a product, each rounded once; with no decay and weights of zero nothing else
    is rounded but the product of the learning rate and the corrections, and eps: 6 half steps of the result."""
    U, n = 2.0 ** -24, 1 << 20
    g = torch.Generator(device="cuda").manual_seed(42)
    p = torch.zeros(n, device="cuda")
    opt = B.AdamW([p], bits=32)
    for t in range(3):
        p.zero_()
        opt.step([torch.randn(n, generator=g, device="cuda") * torch.exp2(torch.randint(-20, 20, (n,), generator=g, device="cuda").float())], lr=0.01, t=t)
        m, v = (x.double() for x in opt.moments())
        want = -0.01 * (m / (1 - 0.9 ** (t + 1))) / ((v / (1 - 0.999 ** (t + 1))).sqrt() + 1e-8)
        assert bool(((p.double() - want).abs() <= 6 * U * (1 + U) * want.abs()).all())

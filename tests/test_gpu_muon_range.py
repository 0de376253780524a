"""Orthogonalised updates of very large and very small gradients, and a small eps."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
SHAPES = [(40, 64), (64, 40), (33, 77), (1, 5), (300, 1030)]


def exact(u, eps, steps=5):
    a, b, c = COEF
    x = u.double()
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    x = x / (x.norm() + float(torch.tensor(eps)))
    for _ in range(steps):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if flip else x


# size of the entries, eps: squares beyond fp32 at either end, a norm near the largest number, numbers below the normal range,
# eps far above and far below the norm
@pytest.mark.parametrize("size,eps", [(1e25, 1e-7), (1e37, 1e-7), (1e-25, 1e-30), (1e-30, 1e-37), (1e-24, 1e-7), (1e-38, 1e-38), (1.0, 1e-38)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_any_size_of_the_gradient(size, eps, dtype):
    g = torch.Generator(device="cuda").manual_seed(4)
    us = [(torch.randn(*s, generator=g, device="cuda", dtype=torch.float64) * size).to(dtype) for s in SHAPES]
    opt = B.Muon(SHAPES, B.make_muon_config(dtype=B.DT_BF16 if dtype == torch.bfloat16 else B.DT_F32, eps=eps))
    os = [torch.full_like(u, float("nan")) for u in us]
    opt.orthogonalize(us, os)
    assert opt.status() == B.OK
    for u, o in zip(us, os):
        want = exact(u, eps)
        # 11 significant bits in every stored value (2e-3 in sum, as the header states) and the result's rounding; with pairs
        # 1e-4.  Where eps is so far above the norm that X leaves the 16-bit range (2^-24 / 2^14 = 4e-12 of 1) it counts as 0.
        rel = 2e-3 + 2.0 ** -8 if dtype == torch.bfloat16 else 1e-4
        room = 4e-12 * 3.4445 ** 5 * want.numel() ** 0.5
        assert bool(o.isfinite().all())
        assert (o.double() - want).norm().item() <= rel * want.norm().item() + room, (tuple(u.shape), (o.double() - want).norm().item(), want.norm().item())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_zero_gradient_gives_zero_whatever_eps_is(dtype):
    for eps in (1e-7, 1e-30, 1e-36, 1e-38, 1e-45):
        opt = B.Muon(SHAPES, B.make_muon_config(dtype=B.DT_BF16 if dtype == torch.bfloat16 else B.DT_F32, eps=eps))
        ws = [torch.ones(s, dtype=dtype, device="cuda") for s in SHAPES]
        gs = [torch.zeros(s, dtype=dtype, device="cuda") for s in SHAPES]
        ms = [torch.zeros(s, device="cuda") for s in SHAPES]
        opt.step(ws, gs, ms, 0.5)
        assert opt.status() == B.OK
        assert all(bool((w == 1).all()) for w in ws) and not any(m.any() for m in ms)

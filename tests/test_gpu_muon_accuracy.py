"""How far orthogonalised results are off where the input's rows or columns differ in size: what the header states."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)


def exact(u, steps=5, eps=1e-7):
    a, b, c = COEF
    x = u.double()
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    x = x / (x.norm() + eps)
    for _ in range(steps):
        g = x @ x.t()
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.t() if flip else x


def gradient(shape, side, decades, seed):
    """Normal numbers, the vectors along one side scaled by 10^-decades ... 10^decades."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(*shape, generator=g, device="cuda")
    if side is not None:
        n = max(shape) if side == "long" else min(shape)
        s = 10 ** ((torch.rand(n, generator=g, device="cuda") * 2 - 1) * decades)
        x = x * (s[:, None] if n == shape[0] else s)
    return (x * 1e-3).bfloat16()


@pytest.mark.parametrize("side,decades", [(None, 0), ("long", 1), ("long", 2), ("short", 1)])
@pytest.mark.parametrize("shape", [(512, 256), (2048, 1024), (1024, 2736), (5461, 2048), (1600, 1500)])
def test_bfloat16_results_are_as_near_as_the_header_states(shape, side, decades):
    u = gradient(shape, side, decades, 1)
    opt = B.Muon([shape], B.make_muon_config(dtype=B.DT_BF16))
    o = torch.empty_like(u)
    opt.orthogonalize([u], [o])
    assert opt.status() == B.OK
    want = exact(u)
    # the rounding of the bfloat16 result, the same as that of the exact one, is independent of the error of X before it
    total, rounding = ((v.double() - want).norm().item() for v in (o, want.bfloat16()))
    error = max(total ** 2 - rounding ** 2, 0.0) ** 0.5 / want.norm().item()
    # 1.5e-3 from 11 significant bits (the worst that a 64-bit model of the stored values shows), 1.5e-4 for the sums of the
    # tensor cores, which cut where fp32 rounds (the worst seen with fp32 weights is 1.1e-4)
    assert error <= 1.65e-3, error


@pytest.mark.parametrize("side,decades", [(None, 0), ("long", 1)])
@pytest.mark.parametrize("shape", [(1, 9), (33, 77), (512, 256), (257, 1029), (1024, 2736)])
def test_bfloat16_weights_with_products_of_pairs(shape, side, decades):
    u = gradient(shape, side, decades, 2)
    opt = B.Muon([shape], B.make_muon_config(dtype=B.DT_BF16, products=B.MUON_PRODUCTS_PAIRS))
    o = torch.empty_like(u)
    opt.orthogonalize([u], [o])
    assert opt.status() == B.OK
    want = exact(u)
    # X is at most 1e-4 off (the header states less); an entry off by d rounds to a neighbour 2^-7 of it away (at most) about
    # every (2^-7 / d)-th time, which leaves the square root of d 2^-7, and d itself
    off = (o.double() - want.bfloat16().double()).norm().item() / want.norm().item()
    assert off <= (1e-4 * 2.0 ** -7) ** 0.5 + 1e-4, off


def test_a_step_with_products_of_pairs():
    shapes = [(96, 160), (300, 1029), (33, 7)]
    g = torch.Generator(device="cuda").manual_seed(5)
    ws = [(torch.randn(*s, generator=g, device="cuda") * 0.02).bfloat16() for s in shapes]
    gs = [gradient(s, None, 0, i) for i, s in enumerate(shapes)]
    ms = [torch.zeros(s, device="cuda") for s in shapes]
    opt = B.Muon(shapes, B.make_muon_config(nesterov=False, momentum=0.5, scale=B.MUON_SCALE_NONE, products=B.MUON_PRODUCTS_PAIRS))
    old = [w.double() for w in ws]
    opt.step(ws, gs, ms, 0.125)
    assert opt.status() == B.OK
    for w0, w, gr in zip(old, ws, gs):
        want = w0 - 0.125 * exact(gr.double() * 0.5)
        # (as above, of the update beside the larger weight: half a unit of the weight and 1e-4 of the update)
        assert bool(((w.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4 * 0.125).all())


def test_products_that_do_not_exist_are_refused():
    with pytest.raises(B.ApolloError) as e:
        B.Muon([(8, 8)], B.make_muon_config(products=2))
    assert e.value.code == B.ERR_INVALID_ARG

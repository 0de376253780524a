"""Orthogonalised updates (Newton-Schulz products on the tensor cores), through the C ABI, against 64 bits."""
import math

import pytest
import torch

from paper_2412_05270_b200 import binding as B
from rounding import between

pytestmark = pytest.mark.gpu

COEF = (3.4445, -4.7750, 2.0315)
# one element, one row, shorter than a box, odd, around the tile of 256 and its halves, tall and wide, long contractions
SHAPES = [(1, 1), (1, 40), (40, 1), (3, 5), (31, 64), (64, 31), (100, 257), (255, 256), (256, 512), (257, 300), (520, 513),
          (300, 1029), (1029, 300), (128, 2736), (640, 640)]


def round_bits(x, bits):
    """x with `bits` significant bits: 16-bit floats hold 11, a sum of two of them 22."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2.0 ** bits) / 2.0 ** bits, e)


def newton_schulz(u, steps=5, coef=COEF, eps=1e-7, bits=None):
    """The definition in 64 bits; with `bits`, every product's result rounded to that many (a model of what storing
    the iterates costs, step by step as the definition says)."""
    a, b, c = coef
    keep = (lambda v: round_bits(v, bits)) if bits else (lambda v: v)
    x = u.double()
    flip = x.shape[0] > x.shape[1]
    x = x.t() if flip else x
    x = keep(x / (x.norm() + eps))
    for _ in range(steps):
        g = keep(x @ x.t())
        x = keep(a * x + keep(b * g + c * (g @ g)) @ x)
    return x.t() if flip else x


def gradient(shape, kind, seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(*shape, generator=g, device="cuda")
    if kind == "rows":
        x *= torch.pow(10.0, torch.rand(shape[0], 1, generator=g, device="cuda") * 2 - 1)
    elif kind == "tails":
        x /= torch.randn(3, *shape, generator=g, device="cuda").square().sum(0).sqrt()
    return (x * 1e-3).to(dtype)


def allowed(u, dtype, steps=5, coef=COEF):
    """Relative error (2-norm) that storing the iterates costs: three times what the 64-bit model that rounds them
    shows (its roundings fall elsewhere), fp32 sums over the contraction (2^-24 sqrt(K) each product, grown by the
    slope a of the iteration per step) and the rounding of the result."""
    want = newton_schulz(u, steps, coef)
    model = newton_schulz(u, steps, coef, bits=11 if dtype == torch.bfloat16 else 22)
    rel = 3 * ((model - want).norm() / want.norm()).item()
    rel += 2.0 ** -24 * math.sqrt(max(u.shape)) * abs(coef[0]) ** min(steps, 5) / 8
    return want, rel + (2.0 ** -9 if dtype == torch.bfloat16 else 2.0 ** -24)


def config(dtype, **kw):
    return B.make_muon_config(dtype=B.DT_BF16 if dtype == torch.bfloat16 else B.DT_F32, **kw)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["normal", "rows", "tails"])
def test_orthogonalize_matches_64_bits(kind, dtype):
    opt = B.Muon(SHAPES, config(dtype))
    us = [gradient(s, kind, 10 + i, dtype) for i, s in enumerate(SHAPES)]
    os = [torch.full(s, float("nan"), dtype=dtype, device="cuda") for s in SHAPES]
    opt.orthogonalize(us, os)
    assert opt.status() == B.OK
    for s, u, o in zip(SHAPES, us, os):
        want, rel = allowed(u, dtype)
        err = o.double() - want
        assert (err.norm() / want.norm()).item() <= rel, (s, (err.norm() / want.norm()).item(), rel)
        # no single entry far off: 40 times the share of an entry in the allowed error
        assert err.abs().max().item() <= 40 * rel * max(want.abs().max().item() / 8, want.norm().item() / math.sqrt(want.numel())), s


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
@pytest.mark.parametrize("shape", [(200, 200), (256, 1300), (1300, 256)])
def test_number_of_steps_and_coefficients(shape, steps):
    for coef in (COEF, (1.5, -0.5, 0.0), (15 / 8, -10 / 8, 3 / 8)):
        opt = B.Muon([shape], config(torch.float32, steps=steps, coef=coef))
        u = gradient(shape, "normal", 3, torch.float32)
        o = torch.empty_like(u)
        opt.orthogonalize([u], [o])
        want, rel = allowed(u, torch.float32, steps, tuple(float(torch.tensor(c)) for c in coef))
        assert ((o.double() - want).norm() / want.norm()).item() <= rel, (coef, ((o.double() - want).norm() / want.norm()).item(), rel)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["normal", "columns", "few directions"])
@pytest.mark.parametrize("steps", [3, 4, 5, 6, 7, 9])
def test_steps_taken_together(steps, kind, dtype):
    shapes = [(200, 1029), (600, 300), (64, 4000), (512, 1376)]
    g = torch.Generator(device="cuda").manual_seed(5)
    us = []
    for s in shapes:
        u = torch.randn(*s, generator=g, device="cuda")
        if kind == "columns":
            u *= torch.where(torch.rand(1, s[1], generator=g, device="cuda") < 0.01, 50.0, 1.0)
        elif kind == "few directions":
            u = 0.1 * u + torch.randn(s[0], 20, generator=g, device="cuda") @ torch.randn(20, s[1], generator=g, device="cuda") / math.sqrt(20)
        us.append((u * 1e-3).to(dtype))
    opt = B.Muon(shapes, config(dtype, steps=steps))
    os = [torch.empty_like(u) for u in us]
    opt.orthogonalize(us, os)
    assert opt.status() == B.OK
    for s, u, o in zip(shapes, us, os):
        coef = tuple(float(torch.tensor(c)) for c in COEF) if dtype == torch.float32 else COEF
        want, rel = allowed(u, dtype, steps, coef)
        if dtype == torch.float32:
            # the tensor cores cut every partial sum of 16 products to 24 bits: at most 2^-23 of a sum that grows evenly,
            # K / 16 times, half of that on average; grown by the slope of the iteration as above
            rel += max(s) / 32 * 2.0 ** -23 * abs(coef[0]) ** min(steps, 5) / 8
        assert ((o.double() - want).norm() / want.norm()).item() <= rel, (s, ((o.double() - want).norm() / want.norm()).item(), rel)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shapes", [[(512, 512)] * 3, [(1400, 1290)], [(2100, 2050), (300, 3000)]])
def test_every_tile_shape(shapes, dtype):
    """Little, some and much work at a time: the products go by tiles of three shapes, each with ragged edges here."""
    opt = B.Muon(shapes, config(dtype))
    us = [gradient(s, "rows", 40 + i, dtype) for i, s in enumerate(shapes)]
    os = [torch.full(s, float("nan"), dtype=dtype, device="cuda") for s in shapes]
    opt.orthogonalize(us, os)
    assert opt.status() == B.OK
    for s, u, o in zip(shapes, us, os):
        want, rel = allowed(u, dtype)
        if dtype == torch.float32:
            rel += max(s) / 32 * 2.0 ** -23 * abs(COEF[0]) ** 5 / 8         # the tensor cores cut, as above
        assert ((o.double() - want).norm() / want.norm()).item() <= rel, (s, ((o.double() - want).norm() / want.norm()).item(), rel)


def test_result_is_nearly_orthogonal():
    # the singular values of a well conditioned matrix end in the interval that the quintic keeps: 0.67 ... 1.21
    q = torch.linalg.qr(torch.randn(600, 300, device="cuda", dtype=torch.float64))[0]
    u = (q @ torch.diag(torch.linspace(0.2, 1.0, 300, device="cuda", dtype=torch.float64)) @ torch.randn(300, 300, device="cuda", dtype=torch.float64)).float()
    opt = B.Muon([(600, 300)], config(torch.float32, steps=10))
    o = torch.empty_like(u)
    opt.orthogonalize([u], [o])
    s = torch.linalg.svdvals(o.double())
    assert s.max().item() < 1.22 and s[: 250].min().item() > 0.65


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("scale", [B.MUON_SCALE_NONE, B.MUON_SCALE_SHAPE, B.MUON_SCALE_RMS])
def test_step_matches_64_bits(scale, nesterov, dtype):
    shapes = [(96, 160), (160, 96), (300, 1029), (33, 7), (256, 256)]
    opt = B.Muon(shapes, config(dtype, nesterov=nesterov, scale=scale, momentum=0.9))
    f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))
    mu, lr, wd = f32(0.9), f32(0.02), f32(0.1)
    g = torch.Generator(device="cuda").manual_seed(5)
    ws = [(torch.randn(*s, generator=g, device="cuda") * 0.02).to(dtype) for s in shapes]
    ms = [torch.zeros(s, device="cuda") for s in shapes]
    for t in range(3):
        gs = [gradient(s, "normal", 100 * t + i, dtype) for i, s in enumerate(shapes)]
        old_w, old_m = [w.clone() for w in ws], [m.clone() for m in ms]
        opt.step(ws, gs, ms, lr, wd)
        assert opt.status() == B.OK
        for s, w0, m0, gr, w, m in zip(shapes, old_w, old_m, gs, ws, ms):
            terms = mu * m0.double(), (1 - mu) * gr.double()
            want_m = terms[0] + terms[1]
            assert bool(((m.double() - want_m).abs() <= 4 * 2.0 ** -24 * (terms[0].abs() + terms[1].abs())).all())
            u = (1 - mu) * gr.double() + mu * m.double() if nesterov else m.double()
            want, rel = allowed(u.float(), dtype)
            gain = {B.MUON_SCALE_NONE: 1.0, B.MUON_SCALE_SHAPE: math.sqrt(max(1.0, s[0] / s[1])), B.MUON_SCALE_RMS: 0.2 * math.sqrt(max(s))}[scale]
            want_w = w0.double() - lr * (gain * want + wd * w0.double())
            err = w.double() - want_w
            # the store of W: half a unit of bf16 is at most 2^-8 of the value, of fp32 2^-24 (and as much for the sum)
            unit = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23
            assert err.norm().item() <= rel * lr * gain * want.norm().item() + unit * want_w.norm().item(), (t, s)
            entry = 40 * rel * lr * gain * max(want.abs().max().item() / 8, want.norm().item() / math.sqrt(want.numel()))
            assert between(w, want_w, entry + 2.0 ** -23 * want_w.abs()), (t, s)


def test_zero_tiny_and_non_finite_gradients():
    shapes = [(64, 96)] * 5
    opt = B.Muon(shapes, config(torch.float32))
    us = [torch.zeros(64, 96, device="cuda"), torch.randn(64, 96, device="cuda") * 1e-12, torch.randn(64, 96, device="cuda"),
          torch.randn(64, 96, device="cuda") * 1e15, torch.zeros(64, 96, device="cuda")]
    us[2][3, 5] = float("nan")
    us[4][0, 0] = 5.0                                   # rank one: one singular value, the rest exactly zero
    os = [torch.empty_like(u) for u in us]
    opt.orthogonalize(us, os)
    assert not os[0].any()
    tiny = newton_schulz(us[1])                         # eps dominates: the definition still holds, X stays small
    assert ((os[1].double() - tiny).norm() / tiny.norm()).item() < 1e-3
    assert bool(os[2].isnan().any())
    big, rel = allowed(us[3], torch.float32)
    assert ((os[3].double() - big).norm() / big.norm()).item() <= rel
    assert abs(os[4][0, 0].item() - newton_schulz(us[4])[0, 0].item()) < 1e-5 and os[4].count_nonzero().item() == 1
    assert opt.status() == B.OK


def test_in_place_on_another_stream_and_again():
    shapes = [(300, 200), (200, 700)]
    opt = B.Muon(shapes, config(torch.bfloat16))
    us = [gradient(s, "rows", i, torch.bfloat16) for i, s in enumerate(shapes)]
    os = [torch.empty_like(u) for u in us]
    opt.orthogonalize(us, os)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = [u.clone() for u in us]
    side.wait_stream(torch.cuda.current_stream())
    opt.orthogonalize(again, again, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(os, again))


def test_groups_give_the_bits_of_the_whole_list():
    # a workspace of 1 MB makes groups of one or two matrices; the products do not depend on the grouping
    shapes = [(256, 300), (300, 256), (400, 400), (64, 2000), (512, 1376), (512, 1376), (10, 10)]
    us = [gradient(s, "normal", i, torch.bfloat16) for i, s in enumerate(shapes)]
    got = []
    for mb in (0, 1):
        opt = B.Muon(shapes, config(torch.bfloat16, workspace_mb=mb))
        os = [torch.empty_like(u) for u in us]
        opt.orthogonalize(us, os)
        got.append((os, opt.workspace_bytes))
    assert all(torch.equal(x, y) for x, y in zip(got[0][0], got[1][0]))
    assert got[1][1] < got[0][1]


def test_many_matrices():
    # more than one launch of the streaming passes takes
    shapes = [(24 + i % 7, 40 + i % 5) for i in range(120)]
    opt = B.Muon(shapes, config(torch.float32))
    us = [gradient(s, "normal", i, torch.float32) for i, s in enumerate(shapes)]
    os = [torch.empty_like(u) for u in us]
    opt.orthogonalize(us, os)
    for u, o in zip(us, os):
        want, rel = allowed(u, torch.float32)
        assert ((o.double() - want).norm() / want.norm()).item() <= rel


def test_bounds_checking_build():
    B.use_library(B.DEBUG_LIB_PATH)
    try:
        shapes = [(5, 7), (7, 5), (100, 257), (257, 100), (300, 1029)]
        for dtype in (torch.bfloat16, torch.float32):
            opt = B.Muon(shapes, config(dtype))
            ws = [torch.zeros(s, dtype=dtype, device="cuda") for s in shapes]
            gs = [gradient(s, "normal", i, dtype) for i, s in enumerate(shapes)]
            ms = [torch.zeros(s, device="cuda") for s in shapes]
            opt.step(ws, gs, ms, 0.1)
            assert opt.status() == B.OK
            assert all(bool(w.any()) for w in ws)
            opt.close()
    finally:
        B.use_library(None)


def test_refusals_of_tensors():
    opt = B.Muon([(16, 32)], config(torch.bfloat16))
    w = torch.zeros(16, 32, dtype=torch.bfloat16, device="cuda")
    m = torch.zeros(16, 32, device="cuda")
    for bad in (([w], [w], [w]), ([w.float()], [w], [m]), ([w], [w.t()], [m]), ([w, w], [w], [m]), ([w.cpu()], [w], [m]), ([w[:8]], [w], [m])):
        with pytest.raises(ValueError):
            opt.step(*bad, 0.1)
    odd = torch.zeros(16 * 32 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(16, 32)
    with pytest.raises(B.ApolloError) as e:
        opt.step([odd], [w], [m], 0.1)
    assert e.value.code == B.ERR_ALIGN
    with pytest.raises(B.ApolloError) as e:
        opt.step([w], [w], [m], float("nan"))
    assert e.value.code == B.ERR_INVALID_ARG

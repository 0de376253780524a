"""The list step, the norm and the adjusted logits where it is easy to go wrong: offsets past 32 bits, several streams, a tiny eps, another library."""
import math

import pytest
import torch

import adamw8 as Q
from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FAR = 2 ** 31 + 4096 + 300


def test_a_tensor_of_more_than_31_bits():
    p = torch.zeros(FAR, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(FAR, dtype=torch.bfloat16, device="cuda")
    g[-3000:] = 1.0
    g[:5] = 1.0
    norm = B.grad_norm([g])[0].item()
    assert abs(norm - math.sqrt(3005)) <= 18 * U * math.sqrt(3005)
    opt = B.AdamW([p], seed=1)
    opt.step([g], lr=0.5, t=0)
    m, v = opt.moments()
    # the first step moves a weight by lr; m = 0.1 and v = 0.001 within a step of their codes
    assert bool((p[-3000:] == -0.5).all()) and bool((p[:5] == -0.5).all()) and not p[5:-3000].any()
    for x, want in ((m, 0.1), (v, 0.001)):
        near = x[FAR - 3000: FAR].double()
        assert bool(((near - want).abs() <= want / 8).all()) and abs(near.mean().item() - want) <= want / 8 * 8 / math.sqrt(3000)
    assert not m[5: FAR - 3300].any()
    del opt, m, v
    opt = B.AdamW([p], bits=32)
    opt.step([g], lr=0.5, t=0)
    m, v = opt.moments()
    assert bool(((m[FAR - 3000: FAR] - 0.1).abs() <= 0.1 * 4 * U).all()) and not m[5: FAR - 3000].any() and bool((p[-3000:] == -1.0).all())


def test_logits_of_more_than_31_bits():
    n, vocab = 36000, 60001
    z = torch.ones(n, vocab, dtype=torch.bfloat16, device="cuda")
    history = torch.arange(5, dtype=torch.int32, device="cuda").expand(n, 5)
    mask = torch.full((1, (vocab + 31) // 32), -1, dtype=torch.int32, device="cuda")
    mask[0, -1] = 0
    y = B.adjust_logits(z, history=history, repetition=2.0, mask=mask)
    keep = vocab // 32 * 32
    for row in (0, n // 2, n - 1):
        assert bool((y[row, :5] == 0.5).all()) and bool((y[row, 5:keep] == 1).all()) and bool((y[row, keep:] == -math.inf).all())
    d = B.adjust_logits_grad(z, z, history=history, repetition=2.0, mask=mask, bias="shared", out=y)
    assert bool((d.logits[n - 1, :5] == 0.5).all()) and bool((d.logits[n - 1, 5:keep] == 1).all()) and not d.logits[n - 1, keep:].any()
    assert bool((d.bias[:keep].float() == n).all()) is (torch.tensor(float(n)).bfloat16().item() == n) and not d.bias[keep:].any()
    B.adjust_logits(z, history=history, repetition=2.0, mask=mask, out=z)
    assert bool((z[n - 1, :5] == 0.5).all()) and bool((z[n - 1, 5:keep] == 1).all()) and bool((z[n - 1, keep:] == -math.inf).all())


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-20, 1e-13, 1e-12])
@pytest.mark.parametrize("bits", [8, 32])
def test_a_tiny_eps(bits, eps):
    """Gradients whose squares are near the end of fp32: with an eps below 1e-12 the root has to see what is below its normal range."""
    g = torch.tensor([1e-18, 3e-18, -1e-17, 1e-15, 1e-10, 1.0], device="cuda")
    p = torch.zeros(6, device="cuda")
    opt = B.AdamW([p], bits=bits, eps=eps)
    opt.step([g], lr=1.0, t=0)
    x = g.double()
    v = (x * x * 0.001).float().double()               # as fp32 holds it: multiples of 2^-149
    v = torch.where(v == 0, (x * x).float().double() * 0.001, v)
    want = -x / ((v / 0.001).sqrt() + eps)
    # v: two roundings of 2^-149 beside 1e-39, 2^-19 of it, halved by the root; root, inverse, products a few steps
    assert bool(((p.double() - want).abs() <= want.abs() * 2.0 ** -17).all())


def test_lists_and_logits_on_several_streams_at_once():
    g = torch.Generator(device="cuda").manual_seed(1)
    streams = [torch.cuda.Stream() for _ in range(3)]
    made = []
    for k in range(3):
        ps = [torch.randn(n, generator=g, device="cuda") for n in (70_000, 300, 5_000_000)]
        gs = [torch.randn(p.numel(), generator=g, device="cuda") for p in ps]
        z = torch.randn(300, 5001, generator=g, device="cuda")
        h = torch.randint(0, 5001, (300, 700), generator=g, device="cuda")
        made.append((ps, gs, z, h))

    def run(ps, gs, z, h, stream):
        opt = B.AdamW([p.clone() for p in ps], seed=3)
        torch.cuda.synchronize()
        out = []
        for t in range(3):
            factor = B.grad_norm(gs, 1.0, stream=stream)
            opt.step(gs, lr=0.1, t=t, factor=factor[1:], stream=stream)
            y = B.adjust_logits(z, history=h, repetition=1.5, presence=0.5, stream=stream)
            d = B.adjust_logits_grad(z, y, history=h, repetition=1.5, bias="shared", stream=stream)
            out += [factor, y, d.logits, d.bias]
        return out + opt.params + [opt.state]
    alone = [run(*x, None) for x in made]
    torch.cuda.synchronize()
    together = [run(*x, s) for x, s in zip(made, streams)]
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_the_current_stream_of_a_with_block():
    z = torch.randn(64, 30_001, device="cuda")
    h = torch.randint(0, 30_001, (64, 100), device="cuda")
    want = B.adjust_logits(z, history=h, repetition=1.5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        zz = z.clone()
        got = B.adjust_logits(zz, history=h, repetition=1.5)
        doubled = got * 2                              # what comes next in the stream sees both kernels' results
        norm = B.grad_norm([got])[0] * 1
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want) and torch.equal(doubled, want * 2) and torch.equal(norm, B.grad_norm([want])[0])


def test_parameters_whose_data_change():
    """The step goes by the parameters as they are, and refuses one that has become another shape."""
    p = torch.nn.Parameter(torch.zeros(300, device="cuda"))
    opt = B.AdamW([p], bits=32)
    p.data = torch.ones(300, dtype=torch.bfloat16, device="cuda")
    opt.step([torch.ones(300, device="cuda")], lr=0.5, t=0)
    assert bool((p == 0.5).all())
    p.data = torch.ones(301, device="cuda")
    with pytest.raises(ValueError, match="shapes"):
        opt.step([torch.ones(301, device="cuda")], lr=0.5, t=1)


def test_a_padded_tail_stays_what_zeros_become():
    p = torch.zeros(300, device="cuda")
    opt = B.AdamW([p], seed=5)
    for t in range(4):
        opt.step([torch.full((300,), 1.0, device="cuda")], lr=0.1, t=t)
    m, v, cm, cv, _ = Q.read(opt.state, 2)
    assert not m.view(-1)[300:].any() and not cv.view(-1)[300:].any()

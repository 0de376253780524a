"""The list step with its learning rate and step count on the device: against the definition in 64 bits, and against numbers."""
import pytest
import torch

import adamw8 as Q
from paper_2412_05270_b200 import binding as B
from test_gpu_adamw_list import B1, B2, DTYPES, EPS, SEED, SIZES, U, Reference, gradients, tensors

pytestmark = pytest.mark.gpu


def on_device(x, dtype):
    return torch.full((1,), x, dtype=dtype, device="cuda")


def from_state(params, opt, bits, **kw):
    """Copies of the parameters and an optimizer that goes on from the same state."""
    copies = [p.clone() for p in params]
    return copies, B.AdamW(copies, bits=bits, beta1=B1, beta2=B2, eps=EPS, seed=SEED, state=opt.state.clone(), **kw)


@pytest.mark.parametrize("correction", [True, False])
@pytest.mark.parametrize("t", [0, 1, 10, 5_000_000_000])
@pytest.mark.parametrize("bits", [8, 32])
def test_scalars_on_the_device(bits, t, correction):
    """Each of lr and t, and both, as tensors.  (Without corrections the definition is that of a step after which nothing is left of them.)"""
    g = torch.Generator().manual_seed(15)
    params = tensors(SIZES, DTYPES, 0.02, g)
    opt = B.AdamW(params, bits=bits, beta1=B1, beta2=B2, eps=EPS, seed=SEED, bias_correction=correction)
    opt.step(gradients(SIZES, DTYPES, g), lr=0.01, t=0)                     # moments that are not zero
    grads = gradients(SIZES, DTYPES, g)
    rate = float(torch.tensor(0.03))
    ends = []
    for lr_at, t_at in ((False, False), (True, False), (False, True), (True, True)):
        copies, one = from_state(params, opt, bits, bias_correction=correction)
        ref = Reference(one, copies, grads, rate, t if correction else 10 ** 12, 0.1, bits=bits)
        one.step(grads, lr=on_device(rate, torch.float32) if lr_at else rate, t=on_device(t, torch.int64) if t_at else t, wd=0.1)
        ref.check(one, copies, bits, t)
        ends.append((copies, one.state))
    first = Q.blocks_of(ref.numels)
    for copies, state in ends[1:]:
        assert torch.equal(state, ends[0][1])                               # the moments know of neither
        for a, b, before, k in zip(copies, ends[0][0], params, first):
            # rate, decay and eps may each differ by a step of fp32 (the doubles behind them by their last bits), 2 U of the movement each,
            # and the product and sum behind them round otherwise, 2 U each; a rounding of the result that goes the other way: a step of the type
            at = slice(k * Q.BLOCK, k * Q.BLOCK + a.numel())
            x, y, old = (z.cpu().double().view(-1) for z in (a, b, before))
            moved = (ref.p.view(-1)[at] - old).abs() + 2 * rate * 0.1 * old.abs()
            assert bool(((x - y).abs() <= 10 * U * moved + torch.finfo(a.dtype).eps * torch.maximum(x.abs(), y.abs())).all())

"""The operators together: the example trains, and the autograd functions give PyTorch's gradients."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

from paper_2412_05270_b200 import autograd as A

pytestmark = pytest.mark.gpu

ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_tiny_lm", ROOT / "examples" / "train_tiny_lm.py")
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("rule", ["muon", "apollo"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_example_learns(example, rule, dtype):
    _, losses = example.train(rule, steps=60, dtype=dtype)
    assert abs(losses[0] - math.log(509)) < 1.5                 # starts near uniform
    assert sum(losses[-5:]) / 5 < 0.75 * losses[0] and all(math.isfinite(x) for x in losses)
    again = example.train(rule, steps=5, dtype=dtype)[1]
    assert again == losses[:5]                                   # bit for bit


def test_a_whole_backward_pass_matches_pytorch(example):
    model = example.TinyLM(dtype=torch.float32)
    g = torch.Generator(device="cuda").manual_seed(3)
    last, before, target = example.batch(509, 16, 20, g)
    logprob, entropy = A.token_logprobs(model.logits(last, before), target, 0.8)
    loss = -(logprob.sum() + 0.1 * entropy.sum())
    loss.backward()
    got = [w.grad.double() for w in model.matrices + model.ends]

    # the same in PyTorch operations and 64 bits
    ws = [w.detach().double().requires_grad_() for w in model.matrices + model.ends]
    mix, up, down, table, head = ws

    def lookup(i):
        return torch.where((i >= 0)[:, None], table[i.clamp(min=0)], 0.0) * model.scale
    h = torch.cat([lookup(last), lookup(before)], -1) @ mix
    h = h + torch.nn.functional.silu(h @ up) @ down
    logp = torch.log_softmax(h @ head * 0.8, -1)
    chosen = torch.where(target >= 0, logp.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    want_loss = -(chosen.sum() + 0.1 * -(logp.exp() * logp).sum())
    want_loss.backward()
    # fp32 products of depth <= 344 and sums over 320 positions, a few of them in a row: 2^-24 * a few thousand
    assert abs(loss.item() - want_loss.item()) <= 1e-4 * abs(want_loss.item())
    for a, w in zip(got, ws):
        assert ((a - w.grad).norm() / w.grad.norm()).item() < 1e-3


def test_entropy_alone_has_a_gradient():
    z = torch.randn(5, 40, device="cuda", requires_grad=True)
    t = torch.zeros(5, dtype=torch.int64, device="cuda")
    A.token_logprobs(z, t)[1].sum().backward()
    zz = z.detach().double().requires_grad_()
    lp = torch.log_softmax(zz, -1)
    (-(lp.exp() * lp).sum()).backward()
    assert ((z.grad.double() - zz.grad).norm() / zz.grad.norm()).item() < 1e-5


def test_continuation_lists_alternatives_in_order(example):
    model, _ = example.train("muon", steps=40)
    for best in example.continue_sequence(model, 10, 12, 3, top=4):
        lps = [lp for _, lp in best]
        assert len(best) == 4 and lps == sorted(lps, reverse=True) and len({i for i, _ in best}) == 4

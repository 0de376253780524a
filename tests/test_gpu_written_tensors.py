"""A tensor that autograd has saved and a call then writes to: its gradient raises, as after PyTorch's own operations in place."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu


def saved(n, m):
    """(a tensor that its own gradient is formed from, a function that asks for that gradient)"""
    y = torch.randn(n, m, device="cuda", requires_grad=True).exp()
    return y, lambda: y.sum().backward()


def history(n):
    return torch.zeros(n, 3, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("call", [
    lambda y: B.adjust_logits(y, history=history(4), repetition=2.0, out=y),
    lambda y: B.adjust_logits(y, bias=torch.ones(50, device="cuda"), out=y),
    lambda y: B.adjust_logits(torch.zeros_like(y), out=y),
    lambda y: B.adjust_logits(y, out=y[:, :]),                             # a view of it
    lambda y: B.adjust_logits_grad(torch.ones_like(y), y, history=history(4), repetition=2.0, out=y),
    lambda y: B.adjust_logits_grad(torch.ones_like(y), torch.ones_like(y), out=y),
])
def test_logits_that_are_written(call):
    y, backward = saved(4, 50)
    call(y)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        backward()


@pytest.mark.parametrize("bits", [8, 32])
def test_parameters_that_a_step_writes(bits):
    p, q = (torch.nn.Parameter(torch.randn(300, device="cuda")) for _ in range(2))
    opt = B.AdamW([p, q], bits=bits)
    x = torch.ones(300, device="cuda", requires_grad=True)
    first, second = (p * x).sum(), (q * x).sum()                           # each saves its parameter
    opt.step((g for g in (torch.ones(300, device="cuda"), None)), lr=0.1, t=0)
    assert p._version > 0 and q._version == 0
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        first.backward()
    second.backward()                                                      # had no gradient and stayed
    assert torch.equal(x.grad, q.detach())


def test_a_norm_that_is_written_and_tensors_without_versions():
    out, backward = saved(1, 2)
    B.grad_norm([torch.ones(5, device="cuda")], out=out.view(2))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        backward()
    with torch.inference_mode():
        z, p = torch.randn(4, 50, device="cuda"), torch.zeros(30, device="cuda")
        B.adjust_logits(z, history=history(4), repetition=2.0, out=z)
        B.AdamW([p]).step([torch.ones(30, device="cuda")], lr=0.1, t=0)
        assert bool((p < 0).all())


def test_what_a_call_reads_stays_as_it_is():
    y, backward = saved(4, 50)
    version = y._version
    B.adjust_logits(y, history=history(4), repetition=2.0)
    B.adjust_logits_grad(y, y, history=history(4), repetition=2.0)
    B.grad_norm([y])
    assert y._version == version
    backward()

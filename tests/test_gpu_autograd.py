"""The autograd functions: gradients of every layout that autograd hands back, empty indices, second order, unused outputs."""
import pytest
import torch

from paper_2412_05270_b200 import autograd as A
from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu


def lookup(table, index, scale):
    """The definition in 64 bits."""
    live = ((index >= 0) & (index < table.shape[0]))[..., None]
    return torch.where(live, table[index.clamp(0, table.shape[0] - 1)], 0.0) * scale


CONSUMERS = {
    "sum": lambda y, w: y.sum(),                                                    # strides (0, 0)
    "sum over the columns": lambda y, w: (y.sum(-1) * w[..., 0]).sum(),             # strides (1, 0)
    "sum over the positions": lambda y, w: (y.sum(-2) * w[..., 0, :]).sum(),        # strides (0, 1)
    "transposed": lambda y, w: (y.transpose(-1, -2).contiguous() * w.transpose(-1, -2).contiguous()).sum(),
    "sliced": lambda y, w: (y[..., 1:3] * w[..., 1:3]).sum(),
    "as it is": lambda y, w: (y * w).sum(),
}


@pytest.mark.parametrize("how", list(CONSUMERS))
@pytest.mark.parametrize("shape", [(7,), (1, 6), (3, 5), (1, 1)])
def test_table_gradient_of_any_layout(shape, how):
    g = torch.Generator(device="cuda").manual_seed(3)
    index = torch.randint(-1, 9, shape, generator=g, device="cuda")
    table = torch.randn(8, 5, generator=g, device="cuda").requires_grad_()
    w = torch.randn(*shape, 5, generator=g, device="cuda")
    CONSUMERS[how](A.embedding(table, index, 1.5), w).backward()
    t = table.detach().double().requires_grad_()
    CONSUMERS[how](lookup(t, index, 1.5), w.double()).backward()
    # at most 15 terms of one row summed in fp32, each up to 4 x 1.5 and rounded once before
    assert bool(((table.grad.double() - t.grad).abs() <= 2 * 15 * 16 * 6 * 2.0 ** -24).all())


@pytest.mark.parametrize("shape", [(0,), (0, 4), (3, 0)])
def test_an_empty_index_has_a_zero_gradient(shape):
    table = torch.randn(8, 5, device="cuda", requires_grad=True)
    out = A.embedding(table, torch.empty(shape, dtype=torch.int64, device="cuda"))
    assert out.shape == (*shape, 5)
    (out.sum() + table[0, 0]).backward()
    want = torch.zeros(8, 5, device="cuda")
    want[0, 0] = 1
    assert torch.equal(table.grad, want)


def test_a_second_derivative_is_refused():
    index = torch.tensor([1, 2, 2], device="cuda")
    target = torch.tensor([0, 3, 1], device="cuda")
    table = torch.randn(6, 4, device="cuda", requires_grad=True)
    logits = torch.randn(3, 7, device="cuda", requires_grad=True)
    cases = [(table, A.embedding(table, index).square().sum()),
             (logits, A.token_logprobs(logits, target)[0].square().sum()),
             (logits, A.token_logprobs(logits, target)[0].sum()),          # its first derivative depends on the logits all the same
             (logits, A.token_logprobs(logits, target)[1].sum())]
    for x, loss in cases:
        once, = torch.autograd.grad(loss, x, create_graph=True)
        with pytest.raises(RuntimeError, match="first derivative"):
            # beside a term that has a gradient a penalty must not drop out without a word
            (once.square().sum() + x.sum()).backward()


def test_create_graph_gives_the_same_first_derivative():
    target = torch.tensor([0, 3, -1], device="cuda")
    logits = torch.randn(3, 7, device="cuda", requires_grad=True)
    grads = [torch.autograd.grad(A.token_logprobs(logits, target)[0].sum(), logits, create_graph=c)[0] for c in (False, True)]
    assert torch.equal(grads[0], grads[1].detach())


def test_outputs_can_be_changed_in_place():
    z = torch.randn(4, 9, device="cuda", requires_grad=True)
    t = torch.tensor([1, 8, -1, 0], device="cuda")
    weight = torch.tensor([0.5, 2.0, 1.0, 0.0], device="cuda")
    want, = torch.autograd.grad((A.token_logprobs(z, t)[0] * weight).sum(), z)
    logprob, entropy = A.token_logprobs(z, t)
    logprob.mul_(weight)
    logprob[3] = 0
    assert torch.equal(torch.autograd.grad(logprob.sum(), z)[0], want)
    logprob, entropy = A.token_logprobs(z, t)
    entropy.add_(1.0)                                  # the gradient needs the entropy as it was computed
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        entropy.sum().backward()


def test_outputs_that_no_loss_uses(monkeypatch):
    seen = []
    plain = B.token_logprobs_grad

    def watched(logits, targets, lse, entropy, d_logprob, d_entropy=None, **kw):
        seen.append((d_logprob, d_entropy))
        return plain(logits, targets, lse, entropy, d_logprob, d_entropy, **kw)
    monkeypatch.setattr(A.B, "token_logprobs_grad", watched)
    z = torch.randn(5, 40, device="cuda", requires_grad=True)
    t = torch.tensor([0, 3, 39, -1, 7], device="cuda")
    A.token_logprobs(z, t)[0].sum().backward()
    assert seen[0][1] is None                          # no entropy term is computed, no zeros are made for it
    zz = z.detach().double().requires_grad_()
    lp = torch.log_softmax(zz, -1)
    torch.where(t >= 0, lp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0).sum().backward()
    assert ((z.grad.double() - zz.grad).norm() / zz.grad.norm()).item() < 1e-5
    z.grad = None
    A.token_logprobs(z, t)[1].sum().backward()         # the entropy alone
    zz.grad = None
    lp = torch.log_softmax(zz, -1)
    (-(lp.exp() * lp).sum()).backward()
    assert ((z.grad.double() - zz.grad).norm() / zz.grad.norm()).item() < 1e-5
    assert not seen[1][0].any()

"""The operators in one run: adjusted logits, log probabilities under them, their gradients, clipping, a step with 8-bit moments."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

import adamw8 as Q
from paper_2412_05270_b200 import autograd as A
from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu

ROOT = Path(__file__).resolve().parent.parent
U = 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_tiny_lm", ROOT / "examples" / "train_tiny_lm.py")
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def adjusted(z, seen, count, rho, phi, pi, bias, index, value, allowed):
    """The definition in PyTorch operations, differentiable."""
    x = torch.where(seen, torch.where(z > 0, z / rho, z * rho), z) - torch.where(count > 0, phi * count + pi, 0.0)
    x = x + bias
    named = (index >= 0).to(x.dtype) * value
    x = x.scatter_add(1, index.clamp(min=0), named)
    return torch.where(allowed, x, -math.inf)


@pytest.mark.parametrize("shape", ["shared", "row", "broadcast"])
def test_a_loss_through_adjusted_logits(shape):
    """Logits -> adjusted -> log probabilities -> loss: gradients of logits, bias and named values against 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(1)
    n, vocab, k = 24, 70, 4
    z = torch.randn(n, vocab, generator=g, device="cuda").requires_grad_()
    bias = torch.randn(*((n, vocab) if shape == "row" else (1, vocab) if shape == "broadcast" else (vocab,)), generator=g, device="cuda").requires_grad_()
    index = torch.randint(-1, vocab, (n, k), generator=g, device="cuda")
    index[:, 2] = index[:, 0]
    value = torch.randn(n, k, generator=g, device="cuda").requires_grad_()
    history = torch.randint(-1, vocab, (n // 4, 20), generator=g, device="cuda")
    lengths = torch.randint(0, 21, (n,), generator=g, device="cuda", dtype=torch.int32)
    rho = torch.rand(n, generator=g, device="cuda") + 0.5
    bits = torch.rand(n, 96, generator=g, device="cuda") < 0.8
    bits[:, vocab:] = False
    bits[5] = False                                    # a row with nothing left
    mask = (bits.view(n, 3, 32).long() << torch.arange(32, device="cuda")).sum(-1).to(torch.int32)
    target = torch.randint(-1, vocab, (n,), generator=g, device="cuda")
    target = torch.where((target >= 0) & bits.gather(1, target.clamp(min=0)[:, None])[:, 0], target, -1)
    given = bias.expand(n, vocab) if shape == "broadcast" else bias
    y = A.adjust_logits(z, history, lengths, None, rho, 0.3, 0.2, given, index, value, mask)
    logprob, entropy = A.token_logprobs(y, target, 0.9)
    (-(logprob * 0.5).sum() + 0.1 * entropy.sum()).backward()

    zz, bb, vv = (x.detach().double().requires_grad_() for x in (z, bias, value))
    count = torch.zeros(n, vocab, dtype=torch.float64, device="cuda")
    for i in range(n):
        for w in history[i // 4][:int(lengths[i])].tolist():
            if w >= 0:
                count[i, w] += 1
    yy = adjusted(zz, count > 0, count, rho.double()[:, None], float(torch.tensor(0.3)), float(torch.tensor(0.2)), bb, index, vv, bits[:, :vocab])
    alive = bits[:, :vocab].any(1)
    logp = torch.log_softmax(torch.where(alive[:, None], yy, 0.0) * float(torch.tensor(0.9)), -1)
    p = torch.where(bits[:, :vocab], logp.exp(), 0.0)
    chosen = torch.where(target >= 0, logp.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    ent = torch.where(alive, -(p * torch.where(p > 0, logp, 0.0)).sum(1), 0.0)
    (-(chosen * 0.5).sum() + 0.1 * ent.sum()).backward()
    # every probability is within 2^-22 of its size (exponential, sums of 70 terms, the row's rounded lse of at most 8: 2^-21), times the largest
    # upstream gradient, through a factor of rho or 1 / rho (up to 2); sums over 24 rows
    for a, b, rows in ((z, zz, 1), (bias, bb, 1 if shape == "row" else n), (value, vv, 1)):
        assert bool(((a.grad.double() - b.grad).abs() <= 64 * U * 2 * rows * (b.grad.abs().max() + 1)).all())
        assert a.grad.abs().sum() > 0
    assert not z.grad[5].any() and not z.grad[~bits[:, :vocab]].any()


def test_gradients_of_any_layout_and_outputs_that_no_loss_uses():
    z = torch.randn(6, 40, device="cuda", requires_grad=True)
    mask = torch.tensor([[-2, 255]], dtype=torch.int32, device="cuda")
    for consumer in (lambda y: y[:, 1:].sum(), lambda y: y.t()[1:].contiguous().square().sum(), lambda y: y[:, 3:5].sum()):
        z.grad = None
        consumer(A.adjust_logits(z, mask=mask)).backward()
        zz = z.detach().requires_grad_()
        x = zz.masked_fill(torch.arange(40, device="cuda") == 0, -math.inf)
        consumer(x).backward()
        assert torch.equal(z.grad, zz.grad)
    bias = torch.zeros(40, device="cuda", requires_grad=True)
    A.adjust_logits(z.detach(), bias=bias).sum().backward()            # the bias alone
    assert bias.grad.tolist() == [6.0] * 40
    once, = torch.autograd.grad(A.adjust_logits(z, history=torch.zeros(6, 1, dtype=torch.int64, device="cuda"), repetition=2.0).square().sum(), z, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivative"):
        (once.square().sum() + z.sum()).backward()
    history = torch.zeros(6, 2, dtype=torch.int64, device="cuda")
    y = A.adjust_logits(z, history=history, repetition=2.0)
    history.add_(1)                                    # the gradient needs the history as it was
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


@pytest.mark.parametrize("rule", ["muon", "apollo"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("states", [8, 32])
def test_the_example_runs_with_lists_of_states(example, rule, dtype, states):
    model, losses = example.train(rule, steps=8, dtype=dtype, states=states, clip=1.0, bias=True, words=500)
    assert len(losses) == 8 and all(math.isfinite(x) for x in losses)
    again = example.train(rule, steps=8, dtype=dtype, states=states, clip=1.0, bias=True, words=500)[1]
    assert again == losses                             # bit for bit
    assert not model.bias[500:].any() and bool(model.bias[:500].any())         # masked words have no gradient
    seen = {10, 12}
    for best in example.continue_sequence(model, 10, 12, 4, top=4, repetition=1e4):
        assert all(i < 500 for i, _ in best)
        seen.add(best[0][0])
    assert len(seen) >= 5


def test_what_the_example_did_before_it_still_does(example):
    """The list with 32-bit states and no clipping is the step that the example always had, but for the order of a few roundings."""
    a, _ = example.train("muon", steps=1, dtype=torch.float32)
    b, _ = example.train("muon", steps=1, dtype=torch.float32, states=32)
    for x, y in zip(a.ends, b.ends):
        # after one step the update is lr g / (|g| + eps'), between 0 and lr: a few steps of fp32 of it and a rounding of the weight
        assert bool(((x - y).abs() <= 32 * U * 0.01 + U * x.abs()).all())


def test_a_whole_backward_pass_of_the_example(example):
    model = example.TinyLM(dtype=torch.float32, bias=True, words=450)
    with torch.no_grad():
        model.bias += torch.linspace(-1, 1, 509, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    last, before, target = example.batch(509, 16, 20, g)
    target = torch.where(target < 450, target, -1)
    logprob, entropy = A.token_logprobs(model.logits(last, before), target)
    loss = -(logprob.sum() + 0.1 * entropy.sum())
    loss.backward()
    ws = [w.detach().double().requires_grad_() for w in model.matrices + model.ends]
    mix, up, down, table, head, bias = ws

    def lookup(i):
        return torch.where((i >= 0)[:, None], table[i.clamp(min=0)], 0.0) * model.scale
    h = torch.cat([lookup(last), lookup(before)], -1) @ mix
    h = h + torch.nn.functional.silu(h @ up) @ down
    logp = torch.log_softmax((h @ head + bias)[:, :450], -1)
    chosen = torch.where(target >= 0, logp.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    want = -(chosen.sum() + 0.1 * -(logp.exp() * logp).sum())
    want.backward()
    # fp32 products of depth <= 344 and sums over 320 positions, a few of them in a row: 2^-24 * a few thousand
    assert abs(loss.item() - want.item()) <= 1e-4 * abs(want.item())
    for a, w in zip(model.matrices + model.ends, ws):
        assert ((a.grad.double() - w.grad).norm() / w.grad.norm()).item() < 1e-3


def test_codes_are_those_of_an_elementwise_program():
    """m and v are rounded as separate fp32 products and sums round them (a fused one makes about one code in two million another one), so the
    moments are the same, bit for bit: of 32 bits directly, of 8 bits their codes."""
    g = torch.Generator(device="cuda").manual_seed(4)
    n, seed = 300 * 256, 99
    p = torch.randn(n, generator=g, device="cuda")
    opt = B.AdamW([p], seed=seed)
    for t in range(3):
        grad = torch.randn(n, generator=g, device="cuda") * torch.exp2(torch.randint(-8, 8, (n,), generator=g, device="cuda").float())
        factor = torch.full((1,), 0.37, device="cuda")
        m, v, *_ = Q.read(opt.state, 300)
        gg = grad * factor
        m, v = (x.float().cuda().view(-1) for x in (m, v))
        m = m * 0.9 + gg * (1 - 0.9)
        v = v * 0.999 + gg.square() * (1 - 0.999)
        opt.step([grad], lr=0.01, t=t, factor=factor)
        _, _, cm, cv, k = Q.read(opt.state, 300)
        chance = Q.chances(300, seed, t)
        for x, c, e, binades in ((m.abs(), cm, k[:, 0], 16), (v, cv, k[:, 1], 32)):
            x = x.cpu().double().view(300, 256)
            assert torch.equal(Q.exponent(x.amax(1), binades).int(), e.int())
            assert torch.equal(Q.code(x, e, chance, binades).int(), c.int())
    n = 1 << 20
    p = torch.randn(n, generator=g, device="cuda")
    opt = B.AdamW([p], bits=32)
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    for t in range(4):
        grad = torch.randn(n, generator=g, device="cuda")
        opt.step([grad], lr=0.01, t=t)
        m = m * 0.9 + grad * (1 - 0.9)
        v = v * 0.999 + grad.square() * (1 - 0.999)
        assert torch.equal(opt.moments()[0], m) and torch.equal(opt.moments()[1], v)


def test_a_captured_training_step_is_that_of_single_calls():
    """Lookup, adjusted logits, log probabilities, their backward pass, clipping and the list step in one graph, replayed for several steps."""
    g = torch.Generator(device="cuda").manual_seed(21)
    table, bias = torch.randn(301, 1000, generator=g, device="cuda"), torch.randn(1000, generator=g, device="cuda")
    index = torch.randint(0, 301, (6, 64), generator=g, device="cuda")
    history = torch.randint(0, 1000, (6, 64, 30), generator=g, device="cuda", dtype=torch.int32)
    target = torch.randint(0, 1000, (6, 64), generator=g, device="cuda")

    def step(params, opt, index, history, target, lr, t):
        for p in params:
            p.grad = None
        logits = A.adjust_logits(A.embedding(params[0], index), history, repetition=1.3, presence=0.2, bias=params[1])
        logprob, entropy = A.token_logprobs(logits, target)
        (-(logprob.sum() + 0.1 * entropy.sum())).backward()
        grads = [p.grad for p in params]
        opt.step(grads, lr=lr, t=t, wd=0.1, factor=B.grad_norm(grads, 1.0)[1:])

    def made():
        params = [x.clone().requires_grad_() for x in (table, bias)]
        return params, B.AdamW(params, seed=5)
    params, opt = made()
    lr = torch.full((1,), 0.01, device="cuda")
    for i in range(6):
        step(params, opt, index[i], history[i], target[i], lr, torch.tensor([i], device="cuda"))
    again, opt2 = made()
    held = [x[0].clone() for x in (index, history, target)]
    t = torch.zeros(1, dtype=torch.int64, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(again, opt2, *held, lr, t)
    for i in range(6):
        for x, new in zip(held, (index, history, target)):
            x.copy_(new[i])
        t.fill_(i)
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(params + [opt.state], again + [opt2.state]))

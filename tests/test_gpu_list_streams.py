"""The state of the list step on streams other than the one it was made on, without a wait of the caller's."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu

N = 4_000_000


def busy():
    """About a tenth of a second of work on the current stream."""
    torch.cuda._sleep(200_000_000)


@pytest.mark.parametrize("bits", [8, 32])
def test_the_first_step_finds_zeros_on_any_stream(bits):
    """The state is filled behind queued work on one stream; the step follows at once on another, captured or not."""
    g = torch.Generator(device="cuda").manual_seed(1)
    start = torch.randn(N, generator=g, device="cuda")
    grad = torch.randn(N, generator=g, device="cuda")
    p = start.clone()
    plain = B.AdamW([p], bits=bits, seed=2)
    plain.step([grad], lr=0.1, t=0)
    nbytes = B.adamw_state_bytes([N], bits)
    for how in ("stream", "captured"):
        q = start.clone()
        used = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        del used                                          # (memory that the allocator will hand out again)
        other = torch.cuda.Stream()
        busy()
        opt = B.AdamW([q], bits=bits, seed=2)
        if how == "stream":
            opt.step([grad], lr=0.1, t=0, stream=other)
        else:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(other):
                graph.capture_begin()
                opt.step([grad], lr=0.1, t=0)
                graph.capture_end()
                graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p, q) and torch.equal(plain.state, opt.state)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_state_of_the_callers_is_not_handed_out_while_a_step_uses_it(bits):
    """Made on one stream, used on the one that was current for the constructor: freed, its memory waits for the step."""
    nbytes = B.adamw_state_bytes([N], bits)
    made, used = torch.cuda.Stream(), torch.cuda.Stream()
    p, grad = torch.zeros(N, device="cuda"), torch.ones(N, device="cuda")
    with torch.cuda.stream(made):
        state = torch.zeros(nbytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    at = state.data_ptr()
    with torch.cuda.stream(used):
        opt = B.AdamW([p], bits=bits, state=state)
        busy()
        opt.step([grad], lr=0.1, t=0)
    del opt, state
    with torch.cuda.stream(made):
        assert torch.empty(nbytes, dtype=torch.uint8, device="cuda").data_ptr() != at
    torch.cuda.synchronize()
    assert bool((p < 0).all())


def test_lists_on_several_streams_that_are_under_way_together():
    """Steps, norms and logits of three streams queued in turn with no wait between them are those of single calls."""
    g = torch.Generator(device="cuda").manual_seed(3)
    made = []
    for _ in range(3):
        ps = [torch.randn(n, generator=g, device="cuda") for n in (70_000, 300, 5_000_000)]
        gs = [torch.randn(p.numel(), generator=g, device="cuda") for p in ps]
        made.append((ps, gs, torch.randn(300, 5001, generator=g, device="cuda"), torch.randint(0, 5001, (300, 700), generator=g, device="cuda")))

    def queue(opt, gs, z, h, t, stream):
        factor = B.grad_norm(gs, 1.0, stream=stream)
        opt.step(gs, lr=0.1, t=t, factor=factor[1:], stream=stream)
        y = B.adjust_logits(z, history=h, repetition=1.5, presence=0.5, stream=stream)
        d = B.adjust_logits_grad(z, y, history=h, repetition=1.5, bias="shared", stream=stream)
        return [factor, y, d.logits, d.bias]
    ends = []
    for streams in ([None] * 3, [torch.cuda.Stream() for _ in range(3)]):
        opts = [B.AdamW([p.clone() for p in ps], seed=3) for ps, *_ in made]
        torch.cuda.synchronize()
        for s in streams:
            with torch.cuda.stream(s):
                busy()                                    # all three streams have their work queued before any of it runs
        out = [queue(opt, gs, z, h, t, s) for t in range(3) for opt, (_, gs, z, h), s in zip(opts, made, streams)]
        torch.cuda.synchronize()
        ends.append([x for o in out for x in o] + [x for o in opts for x in o.params + [o.state]])
    assert all(torch.equal(a, b) for a, b in zip(*ends))

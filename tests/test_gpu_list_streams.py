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

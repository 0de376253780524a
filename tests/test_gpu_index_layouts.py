"""Indices and targets that are views: columns of a batch, every other entry, transposed."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu

VIEWS = {"all but the last": lambda t: t[:, :-1], "all but the first": lambda t: t[:, 1:], "every other": lambda t: t[:, ::2],
         "transposed": lambda t: t.t(), "one repeated": lambda t: t[:, :1].expand(6, 5)}


@pytest.mark.parametrize("itype", [torch.int32, torch.int64])
@pytest.mark.parametrize("view", list(VIEWS))
def test_views_count_as_their_values(view, itype):
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.randint(-1, 12, (6, 10), generator=g, device="cuda").to(itype)
    index = VIEWS[view](tokens)
    assert not index.is_contiguous()
    table = torch.randn(12, 16, generator=g, device="cuda")
    same = index.contiguous()
    for stream in (None, torch.cuda.Stream()):
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        out = B.embedding(table, index, 2.0, stream=stream)
        d = torch.randn(index.numel(), 16, generator=g, device="cuda")
        z = torch.randn(index.numel(), 30, generator=g, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        grad = B.embedding_grad(d, index, 12, stream=stream)
        r = B.token_logprobs(z, index, top=2, stream=stream)
        dz = B.token_logprobs_grad(z, index, r.lse, r.entropy, r.lse, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(out, B.embedding(table, same, 2.0)) and out.shape == (*index.shape, 16)
        assert torch.equal(grad, B.embedding_grad(d, same, 12))
        assert all(torch.equal(a, b) for a, b in zip(r, B.token_logprobs(z, same, top=2)))
        assert torch.equal(dz, B.token_logprobs_grad(z, same, r.lse, r.entropy, r.lse))

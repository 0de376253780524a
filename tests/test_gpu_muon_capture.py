"""Orthogonalised updates and stream capture: the first call uploads what the kernels read, so it may not be recorded only."""
import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu

SHAPES = [(96, 160), (300, 200), (256, 700)]


def tensors(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    us = [torch.randn(*s, generator=g, device="cuda").bfloat16() for s in SHAPES]
    return us, [torch.zeros_like(u) for u in us]


def test_the_first_call_is_refused_while_the_stream_is_captured():
    opt = B.Muon(SHAPES, B.make_muon_config())
    us, os = tensors(1)
    ms = [torch.zeros(s, device="cuda") for s in SHAPES]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in (lambda: opt.orthogonalize(us, os), lambda: opt.step(os, us, ms, 0.1)):
            with pytest.raises(B.ApolloError) as e:
                call()
            assert e.value.code == B.ERR_INVALID_ARG
    del graph                                          # nothing was recorded, nothing is launched
    assert opt.status() == B.OK
    assert not any(o.any() for o in os)
    opt.orthogonalize(us, os)
    assert opt.status() == B.OK
    other, again = B.Muon(SHAPES, B.make_muon_config()), tensors(1)[1]
    other.orthogonalize(us, again)
    assert all(torch.equal(a, b) for a, b in zip(os, again))


def test_later_calls_can_be_captured():
    opt = B.Muon(SHAPES, B.make_muon_config())
    us, os = tensors(2)
    opt.orthogonalize(us, os)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.orthogonalize(us, os)
    for seed in (3, 4):
        new, want = tensors(seed)
        for u, v in zip(us, new):
            u.copy_(v)
        graph.replay()
        got = [o.clone() for o in os]
        assert opt.status() == B.OK
        opt.orthogonalize(new, want)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    del graph

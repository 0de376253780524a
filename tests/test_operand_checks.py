"""What the binding refuses before a pointer reaches a kernel, with stand-ins for tensors of other devices (no GPU needed)."""
import math

import pytest
import torch

from paper_2412_05270_b200 import binding as B


class Operand:
    """As much of a CUDA tensor as the checks look at; whoever asks for its address fails the test."""

    def __init__(self, *shape, dtype=torch.float32, device="cuda:0", strides=None):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device(device)
        self.is_cuda = self.device.type == "cuda"
        self.strides = strides or [math.prod(shape[i + 1:]) for i in range(len(shape))]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def element_size(self):
        return self.dtype.itemsize

    def stride(self, i):
        return self.strides[i]

    def is_contiguous(self):
        return self.strides == [math.prod(self.shape[i + 1:]) for i in range(len(self.shape))]

    def contiguous(self):
        return self

    def data_ptr(self):
        raise AssertionError("an address was taken before the checks were over")


@pytest.fixture(autouse=True)
def _device_zero(monkeypatch):
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 0)


def index(n, **kw):
    return Operand(n, dtype=torch.int64, **kw)


@pytest.mark.parametrize("workspace", [Operand(4096, dtype=torch.uint8, device="cpu"), Operand(4096, dtype=torch.uint8, strides=[2])])
def test_a_workspace_that_kernels_cannot_use(workspace):
    with pytest.raises(ValueError, match="workspace"):
        B.embedding_grad(Operand(4, 8), index(4), 10, out=Operand(10, 8), workspace=workspace)


class Stream:
    def __init__(self, device):
        self.device, self.cuda_stream = torch.device(device), 0


ELSEWHERE = dict(device="cuda:1")


def rows(n, **kw):
    return Operand(n, **kw)


@pytest.mark.parametrize("call", [
    lambda: B.embedding(Operand(10, 8), index(4, **ELSEWHERE)),
    lambda: B.embedding(Operand(10, 8), index(4), out=Operand(4, 8, **ELSEWHERE)),
    lambda: B.embedding_grad(Operand(4, 8), index(4, **ELSEWHERE), 10),
    lambda: B.embedding_grad(Operand(4, 8), index(4), 10, out=Operand(10, 8, **ELSEWHERE)),
    lambda: B.embedding_grad(Operand(4, 8), index(4), 10, out=Operand(10, 8), workspace=Operand(4096, dtype=torch.uint8, **ELSEWHERE)),
    lambda: B.token_logprobs(Operand(4, 30), index(4, **ELSEWHERE)),
    lambda: B.token_logprobs_grad(Operand(4, 30), index(4, **ELSEWHERE), rows(4), rows(4), rows(4)),
    lambda: B.token_logprobs_grad(Operand(4, 30), index(4), rows(4, **ELSEWHERE), rows(4), rows(4)),
    lambda: B.token_logprobs_grad(Operand(4, 30), index(4), rows(4), rows(4, **ELSEWHERE), rows(4), rows(4)),
    lambda: B.token_logprobs_grad(Operand(4, 30), index(4), rows(4), rows(4), rows(4, **ELSEWHERE)),
    lambda: B.token_logprobs_grad(Operand(4, 30), index(4), rows(4), rows(4), rows(4), rows(4, **ELSEWHERE)),
    lambda: B.token_logprobs_grad(Operand(4, 30), index(4), rows(4), rows(4), rows(4), out=Operand(4, 30, **ELSEWHERE)),
])
def test_tensors_of_two_devices(call):
    with pytest.raises(ValueError, match="one device"):
        call()


@pytest.mark.parametrize("call", [
    lambda s: B.embedding(Operand(10, 8), index(4), stream=s),
    lambda s: B.embedding_grad(Operand(4, 8), index(4), 10, stream=s),
    lambda s: B.token_logprobs(Operand(4, 30), index(4), stream=s),
    lambda s: B.token_logprobs_grad(Operand(4, 30), index(4), rows(4), rows(4), rows(4), stream=s),
])
def test_a_stream_of_another_device(call):
    with pytest.raises(ValueError, match="stream"):
        call(Stream("cuda:1"))


class Library:
    """Records the device and the stream that a call of the library would run on."""

    def __init__(self, on):
        self.on, self.calls = on, []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.on["device"], args[-1]))
            return 0
        return call


class Tensors(Operand):
    def data_ptr(self):
        return 4096

    def record_stream(self, stream):
        self.used_on = getattr(self, "used_on", []) + [stream]


@pytest.fixture
def context(monkeypatch):
    """A context of the second of two devices while the first is the current one."""
    on = {"device": 0}

    class Device:
        def __init__(self, device):
            index = torch.device(device).index
            self.index = on["device"] if index is None else index

        def __enter__(self):
            self.before, on["device"] = on["device"], self.index

        def __exit__(self, *_):
            on["device"] = self.before

    class OnStream(Device):
        def __init__(self, stream):
            super().__init__(stream.device)
    monkeypatch.setattr(B, "_current_device", lambda: on["device"])
    monkeypatch.setattr(B, "_raw_stream", lambda device: 1000 + device)
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch.cuda, "stream", OnStream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: "the current stream")
    library = Library(on)
    monkeypatch.setattr(B, "load", lambda: library)
    monkeypatch.setattr(B, "muon_workspace_bytes", lambda shapes, cfg: 4096)
    monkeypatch.setattr(torch, "empty", lambda n, dtype, device: Tensors(n, dtype=dtype, device=f"cuda:{on['device']}"))
    opt = B.Muon([(4, 8)], B.make_muon_config(dtype=B.DT_F32), device="cuda:1")
    library.calls.clear()
    return opt, library


def tensor_lists(device):
    return [[Tensors(4, 8, device=device)] for _ in range(3)]


def test_a_context_works_on_its_own_device(context):
    opt, library = context
    ws, gs, ms = tensor_lists("cuda:1")
    opt.step(ws, gs, ms, 0.1)
    opt.orthogonalize(gs, ws)
    opt.status()
    opt.step(ws, gs, ms, 0.1, stream=Stream("cuda:1"))
    assert [c[1] for c in library.calls] == [1, 1, 1, 1]
    assert [c[2] for c in library.calls] == [1001, 1001, 1001, 0]
    assert B._current_device() == 0


def test_a_context_refuses_other_devices(context):
    opt, library = context
    for k in range(3):
        lists = tensor_lists("cuda:1")
        lists[k] = tensor_lists("cuda:0")[0]
        with pytest.raises(ValueError, match="device"):
            opt.step(*lists, 0.1)
    with pytest.raises(ValueError, match="stream"):
        opt.step(*tensor_lists("cuda:1"), 0.1, stream=Stream("cuda:0"))
    assert not library.calls


def test_a_context_without_an_index_takes_the_current_device(context):
    opt = B.Muon([(4, 8)], B.make_muon_config(dtype=B.DT_F32))
    opt.step(*tensor_lists("cuda:0"), 0.1)
    with pytest.raises(ValueError, match="device"):
        opt.step(*tensor_lists("cuda:1"), 0.1)


def test_the_allocator_hears_of_another_stream(context):
    opt, _ = context
    opt.step(*tensor_lists("cuda:1"), 0.1)
    assert not hasattr(opt.workspace, "used_on")
    opt.step(*tensor_lists("cuda:1"), 0.1, stream=Stream("cuda:1"))
    opt.orthogonalize(*tensor_lists("cuda:1")[:2], stream=Stream("cuda:1"))
    assert opt.workspace.used_on == ["the current stream"] * 2

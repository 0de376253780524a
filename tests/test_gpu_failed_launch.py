"""A call whose launch the runtime refuses says so, and the next call knows nothing of it."""
import ctypes

import pytest
import torch

from paper_2412_05270_b200 import binding as B

pytestmark = pytest.mark.gpu

RELAXED = 2                                  # CU_STREAM_CAPTURE_MODE_RELAXED


class Refusing:
    """A stream whose capture has become invalid (it was waited for): the host refuses every launch on it."""

    def __enter__(self):
        self.driver, self.stream = ctypes.CDLL("libcuda.so.1"), torch.cuda.Stream()
        self.at = ctypes.c_void_p(self.stream.cuda_stream)
        assert self.driver.cuStreamBeginCapture_v2(self.at, RELAXED) == 0
        assert self.driver.cuStreamSynchronize(self.at) != 0
        return self.stream.cuda_stream

    def __exit__(self, *_):
        graph = ctypes.c_void_p()
        assert self.driver.cuStreamEndCapture(self.at, ctypes.byref(graph)) != 0 and not graph.value
        assert self.driver.cuStreamSynchronize(self.at) == 0


@pytest.mark.parametrize("rules", ["bias", "history", "both"])
@pytest.mark.parametrize("place", [False, True])
@pytest.mark.parametrize("gradient", [False, True])
def test_the_call_after_a_refused_launch(gradient, place, rules):
    n, vocab = 4, 100
    z, dout, out = (torch.full((n, vocab), x, device="cuda") for x in (1.0, 3.0, 5.0))
    if place:
        out = dout if gradient else z
    before = out.clone()
    bias, history = torch.ones(vocab, device="cuda"), torch.zeros(n, 3, dtype=torch.int32, device="cuda")
    shared = rules != "history" and gradient
    work = torch.empty(B.adjust_logits_grad_workspace_bytes(n, vocab), dtype=torch.uint8, device="cuda")
    r = B.LogitRules(repetition=2.0)
    if rules != "history":
        r.bias = bias.data_ptr()
    if rules != "bias":
        r.history, r.history_type, r.history_rows, r.history_len, r.history_stride = history.data_ptr(), B.INDEX_I32, n, 3, 3
    torch.cuda.synchronize()
    with Refusing() as stream:
        args = (z.data_ptr(), vocab, n, vocab, B.DT_F32, ctypes.byref(r))
        if gradient:
            code = B.load().apollo_adjust_logits_grad(*args, dout.data_ptr(), vocab, out.data_ptr(), vocab, bias.data_ptr() if shared else None, 0, None,
                                                      work.data_ptr() if shared else None, work.numel() if shared else 0, stream)
        else:
            code = B.load().apollo_adjust_logits(*args, out.data_ptr(), vocab, stream)
    assert code == B.ERR_CUDA
    assert B.grad_norm([torch.ones(4, device="cuda")])[0].item() == 2.0
    torch.cuda.synchronize()
    assert torch.equal(out, before) and bool((bias == 1).all())

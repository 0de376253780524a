"""Host-side checks of the list step, the norm and the adjusted logits: sizes, refusals before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2412_05270_b200 import binding as B
from paper_2412_05270_b200.build import build_library


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def test_state_sizes():
    # blocks of 256: codes of m and v and two exponents, or two floats an element
    assert B.adamw_state_bytes([1]) == 514 and B.adamw_state_bytes([256, 257, 0]) == 3 * 514
    assert B.adamw_state_bytes([1], 32) == 2048 and B.adamw_state_bytes([256, 257, 0], 32) == 3 * 2048
    assert B.adamw_state_bytes([0]) == 0
    assert B.adamw_state_bytes([2 ** 31]) == 2 ** 23 * 514
    for numels, bits, code in (([], 8, B.ERR_INVALID_ARG), ([4], 16, B.ERR_INVALID_ARG), ([-1], 8, B.ERR_INVALID_ARG),
                               ([2 ** 39], 8, B.ERR_SHAPE), ([2 ** 38, 2 ** 38, 2 ** 38], 32, B.ERR_SHAPE)):
        with pytest.raises(B.ApolloError) as e:
            B.adamw_state_bytes(numels, bits)
        assert e.value.code == code
    assert B.grad_norm_workspace_bytes(1) == B.grad_norm_workspace_bytes(960) < B.grad_norm_workspace_bytes(961)
    assert B.adjust_logits_grad_workspace_bytes(3, 100) == 1200
    assert B.adjust_logits_grad_workspace_bytes(10 ** 6, 1000) <= 256 * 4000          # a bounded number of partial rows


def arrays(p, g, numel, dp=0, dg=0):
    return (ctypes.c_uint64 * 1)(p), (ctypes.c_uint64 * 1)(g), (ctypes.c_int64 * 1)(numel), (ctypes.c_int32 * 1)(dp), (ctypes.c_int32 * 1)(dg)


def list_step(p=4096, g=8192, numel=10, dp=0, dg=0, state=16384, state_bytes=514, lr=0.1, wd=0.0, t=0, factor=None, lr_at=None, t_at=None, n=1, **cfg):
    c = B.AdamWListConfig(8, 1, 0.9, 0.999, 1e-8, 0)
    for k, v in cfg.items():
        setattr(c, k, v)
    a = arrays(p, g, numel, dp, dg)
    return B.load().apollo_adamw_list_step(ctypes.byref(c), a[0], a[1], a[2], a[3], a[4], n, state, state_bytes, lr, wd, t, factor, lr_at, t_at, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), B.ERR_INVALID_ARG), (dict(numel=-1), B.ERR_INVALID_ARG), (dict(dp=2), B.ERR_INVALID_ARG), (dict(dg=-1), B.ERR_INVALID_ARG),
    (dict(p=0), B.ERR_INVALID_ARG), (dict(state=0), B.ERR_INVALID_ARG), (dict(lr=float("nan")), B.ERR_INVALID_ARG), (dict(wd=float("inf")), B.ERR_INVALID_ARG),
    (dict(t=-1), B.ERR_INVALID_ARG), (dict(state_bits=4), B.ERR_INVALID_ARG), (dict(bias_correction=2), B.ERR_INVALID_ARG),
    (dict(beta1=1.0), B.ERR_INVALID_ARG), (dict(beta2=float("nan")), B.ERR_INVALID_ARG), (dict(eps=-1e-8), B.ERR_INVALID_ARG), (dict(eps=float("inf")), B.ERR_INVALID_ARG),
    (dict(p=4100), B.ERR_ALIGN), (dict(g=8194), B.ERR_ALIGN), (dict(state=16392), B.ERR_ALIGN), (dict(factor=4098), B.ERR_ALIGN), (dict(lr_at=4097), B.ERR_ALIGN),
    (dict(t_at=4100), B.ERR_ALIGN), (dict(state_bytes=513), B.ERR_WORKSPACE), (dict(numel=257), B.ERR_WORKSPACE), (dict(numel=2 ** 40), B.ERR_SHAPE),
])
def test_list_steps_that_are_refused(kw, code):
    assert list_step(**kw) == code


def norm(g=4096, numel=10, dtype=0, n=1, max_norm=1.0, out=8192, ws=16384, ws_bytes=1 << 20):
    a = arrays(0, g, numel, 0, dtype)
    return B.load().apollo_grad_norm(a[1], a[2], a[4], n, max_norm, out, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=0), B.ERR_INVALID_ARG), (dict(max_norm=0.0), B.ERR_INVALID_ARG), (dict(max_norm=float("nan")), B.ERR_INVALID_ARG), (dict(out=None), B.ERR_INVALID_ARG),
    (dict(ws=None), B.ERR_INVALID_ARG), (dict(dtype=5), B.ERR_INVALID_ARG), (dict(numel=-3), B.ERR_INVALID_ARG), (dict(g=4104), B.ERR_ALIGN),
    (dict(out=8193), B.ERR_ALIGN), (dict(ws=16388), B.ERR_ALIGN), (dict(ws_bytes=64), B.ERR_WORKSPACE),
])
def test_norms_that_are_refused(kw, code):
    assert norm(**kw) == code


def test_moments_that_are_refused():
    f = B.load().apollo_adamw_list_moments
    assert f(16, 514, -1, 16, 16, None) == B.ERR_INVALID_ARG and f(None, 514, 1, 16, 16, None) == B.ERR_INVALID_ARG
    assert f(16, 513, 1, 16, 16, None) == B.ERR_WORKSPACE and f(8, 514, 1, 16, 16, None) == B.ERR_ALIGN and f(16, 514, 1, 16, 24, None) == B.ERR_ALIGN
    assert f(None, 0, 0, None, None, None) == B.OK and f(16, 514, 2 ** 31, 16, 16, None) == B.ERR_SHAPE


def adjust(gradient=False, rows=4, vocab=100, stride=100, out_stride=100, dtype=0, logits=4096, out=8192, bias_grad=None, bias_grad_stride=0, ws=None, ws_bytes=0,
           rules=True, **kw):
    r = B.LogitRules(repetition=1.0)
    for k, v in kw.items():
        setattr(r, k, v)
    at = ctypes.byref(r) if rules else None
    if gradient:
        return B.load().apollo_adjust_logits_grad(logits, stride, rows, vocab, dtype, at, 16384, 100, out, out_stride, bias_grad, bias_grad_stride, None, ws, ws_bytes, None)
    return B.load().apollo_adjust_logits(logits, stride, rows, vocab, dtype, at, out, out_stride, None)


HISTORY = dict(history=4096, history_type=B.INDEX_I32, history_rows=4, history_len=10, history_stride=10)


@pytest.mark.parametrize("gradient", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(rules=False), B.ERR_INVALID_ARG), (dict(dtype=3), B.ERR_INVALID_ARG), (dict(rows=-1), B.ERR_SHAPE), (dict(vocab=0), B.ERR_SHAPE),
    (dict(vocab=2 ** 26 + 1, stride=2 ** 27), B.ERR_SHAPE), (dict(stride=99), B.ERR_SHAPE), (dict(out_stride=99), B.ERR_SHAPE), (dict(out=None), B.ERR_INVALID_ARG),
    (dict(logits=4098, **HISTORY), B.ERR_ALIGN), (dict(out=8193), B.ERR_ALIGN),
    (dict(HISTORY, history_type=7), B.ERR_INVALID_ARG), (dict(HISTORY, history_rows=0), B.ERR_INVALID_ARG), (dict(HISTORY, history_rows=3), B.ERR_SHAPE),
    (dict(HISTORY, history_len=-1), B.ERR_INVALID_ARG), (dict(HISTORY, history_len=1 << 20, history_stride=1 << 20), B.ERR_SHAPE),
    (dict(HISTORY, history_stride=9), B.ERR_SHAPE), (dict(HISTORY, history=4098), B.ERR_ALIGN), (dict(HISTORY, length=4098), B.ERR_ALIGN),
    (dict(HISTORY, repetition=0.0), B.ERR_INVALID_ARG), (dict(HISTORY, repetition=float("nan")), B.ERR_INVALID_ARG), (dict(HISTORY, repetition_at=4097), B.ERR_ALIGN),
    (dict(n_bias=-1), B.ERR_INVALID_ARG), (dict(n_bias=3), B.ERR_INVALID_ARG), (dict(n_bias=1025, bias_word=4096, bias_value=4096), B.ERR_SHAPE),
    (dict(n_bias=3, bias_word=4098, bias_value=4096), B.ERR_ALIGN), (dict(n_bias=3, bias_word=4096, bias_value=4096, bias_word_type=9), B.ERR_INVALID_ARG),
    (dict(mask=4096, mask_stride=3), B.ERR_SHAPE), (dict(mask=4097, mask_stride=4), B.ERR_ALIGN),
])
def test_rules_that_are_refused(gradient, kw, code):
    assert adjust(gradient, **kw) == code


def test_rules_that_one_direction_refuses():
    assert adjust(frequency=float("inf"), **HISTORY) == B.ERR_INVALID_ARG and adjust(presence=float("nan"), **HISTORY) == B.ERR_INVALID_ARG
    assert adjust(bias=4096, bias_stride=99) == B.ERR_SHAPE and adjust(bias=4098) == B.ERR_ALIGN
    assert adjust(logits=4096, out=4096, out_stride=104) == B.ERR_INVALID_ARG                          # in place with another stride
    assert adjust(True, out=16384, out_stride=104) == B.ERR_INVALID_ARG
    assert adjust(True, bias_grad=4096, bias_grad_stride=99) == B.ERR_SHAPE
    assert adjust(True, bias_grad=4096) == B.ERR_INVALID_ARG                                           # a shared bias without a workspace
    assert adjust(True, bias_grad=4096, ws=4096, ws_bytes=1599) == B.ERR_WORKSPACE
    assert adjust(True, bias_grad=4096, ws=4100, ws_bytes=1 << 20) == B.ERR_ALIGN
    assert adjust(True, logits=None, **HISTORY) == B.ERR_INVALID_ARG
    assert adjust(rows=0, logits=None, out=None) == B.OK and adjust(True, rows=0, logits=None, out=None) == B.OK


def test_tensors_that_the_binding_refuses():
    z, f32 = torch.zeros(4, 100), torch.float32
    for call in (lambda: B.adjust_logits(z), lambda: B.adjust_logits_grad(z, z), lambda: B.grad_norm([z]), lambda: B.AdamW([z]), lambda: B.AdamW([]),
                 lambda: B.AdamW([None]), lambda: B.grad_norm([]), lambda: B.grad_norm([None]), lambda: B.adjust_logits(z.half()), lambda: B.adjust_logits(z.to_sparse())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.adjust_logits([[1.0]]), lambda: B.grad_norm(3)):
        with pytest.raises((TypeError, ValueError)):
            call()
    d = B._marshal().describe
    assert d(z)[1:] == (-1, 0, 2, 4, 100, 100, 1, 1) and d(z)[0] == z.data_ptr()
    assert d(z.t())[2:] == (0, 2, 100, 4, 1, 100, 0) and d(torch.zeros(3, dtype=torch.int64))[2:] == (3, 1, 3, 1, 1, 1, 1)
    assert d(torch.zeros((), dtype=f32))[3:] == (0, 1, 1, 1, 1, 1) and d(torch.zeros(2, dtype=torch.bool))[2] == -1
    pointers, lengths, types, device, live = B._marshal().pack("grads", [None, None], None, -1)
    assert pointers == b"\0" * 16 and lengths == b"\0" * 16 and types == b"\0" * 8 and device == -1 and live == 0


def test_a_gradient_over_the_logits_whose_signs_it_asks_for():
    assert adjust(True, logits=8192, out=8192, **HISTORY) == B.ERR_INVALID_ARG

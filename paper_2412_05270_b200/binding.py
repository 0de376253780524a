"""ctypes binding of libapollo.so: argument marshalling only.

Every step of the optimizer runs inside the library's CUDA kernels; PyTorch supplies device
memory and the stream.  There is no CPU fallback: if the shared library is missing the
import of this module's symbols raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import importlib.util
import math
from pathlib import Path
from typing import NamedTuple

import torch

from .build import marshal_path

_PKG = Path(__file__).resolve().parent
LIB_PATH = _PKG / "libapollo.so"
DEBUG_LIB_PATH = _PKG / "libapollo_debug.so"     # built with -DAPOLLO_DEBUG: index checks inside the kernels of contexts

OK = 0
ERR_INVALID_ARG, ERR_SHAPE, ERR_RANK, ERR_ALIGN, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT, ERR_UNSUPPORTED = (
    -1, -2, -3, -4, -5, -6, -7, -8)
ERR_TOO_LARGE = -9
ERR_INTERNAL = -10
STATIC_SCRATCH_BYTES = 8 << 20
SCALE_CHANNEL, SCALE_TENSOR = 0, 1
DT_F32, DT_BF16 = 0, 1
FLAG_NO_TENSOR_CORES = 1
FLAG_BF16_STATES = 2
FLAG_KEEP_P = 4
TC_KERNEL_PAIR, TC_KERNEL_RING = 0, 1
P_SCRATCH, P_SHARED = 0, 1
PATH_STREAM, PATH_SIMT, PATH_TENSOR = 0, 1, 2
MUON_SCALE_NONE, MUON_SCALE_SHAPE, MUON_SCALE_RMS = 0, 1, 2
MUON_MAX_STEPS = 32
MUON_PRODUCTS_DEFAULT, MUON_PRODUCTS_PAIRS = 0, 1
INDEX_I32, INDEX_I64 = 0, 1
MAX_TOP = 32
ADAMW_BLOCK = 256
MAX_HISTORY = (1 << 20) - 1
MAX_BIAS_WORDS = 1024

EXPORTS = [
    "apollo_workspace_bytes", "apollo_create", "apollo_step", "apollo_destroy", "apollo_step_count",
    "apollo_get_scales", "apollo_get_limiter", "apollo_get_state", "apollo_set_delta_out", "apollo_status",
    "apollo_philox_draws", "apollo_projection", "apollo_get_path", "apollo_last_launches", "apollo_strerror",
    "apollo_set_timing", "apollo_get_timing", "apollo_mini_step_static", "apollo_cuda_error_string", "apollo_adamw_step",
    "apollo_state_bytes", "apollo_state_export", "apollo_state_import", "apollo_step_range", "apollo_set_projection",
    "apollo_selftest_bounded_wait", "apollo_workspace_bytes_tuned", "apollo_create_tuned",
    "apollo_muon_workspace_bytes", "apollo_muon_create", "apollo_muon_destroy", "apollo_muon_step", "apollo_muon_orthogonalize",
    "apollo_muon_status", "apollo_muon_last_launches", "apollo_embedding", "apollo_embedding_grad_workspace_bytes",
    "apollo_embedding_grad", "apollo_token_logprobs", "apollo_token_logprobs_grad",
    "apollo_grad_norm_workspace_bytes", "apollo_grad_norm", "apollo_adamw_list_state_bytes", "apollo_adamw_list_step",
    "apollo_adamw_list_moments", "apollo_adjust_logits", "apollo_adjust_logits_grad_workspace_bytes", "apollo_adjust_logits_grad",
]


class ApolloError(RuntimeError):
    def __init__(self, code: int, what: str):
        detail = f" [{load().apollo_cuda_error_string().decode()}]" if code == ERR_CUDA else ""
        super().__init__(f"{what}: {strerror(code)} ({code}){detail}")
        self.code = code


class Shape(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class Config(ctypes.Structure):
    _fields_ = [
        ("rank", ctypes.c_int32), ("mode", ctypes.c_int32), ("dtype", ctypes.c_int32), ("T", ctypes.c_int32),
        ("seed", ctypes.c_uint64),
        ("alpha", ctypes.c_float), ("gamma", ctypes.c_float),
        ("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("eps", ctypes.c_float),
        ("bias_correction", ctypes.c_int32), ("flags", ctypes.c_uint32),
    ]


class MuonConfig(ctypes.Structure):
    """apollo_muon_config."""
    _fields_ = [("dtype", ctypes.c_int32), ("ns_steps", ctypes.c_int32), ("coef", ctypes.c_float * 3),
                ("momentum", ctypes.c_float), ("nesterov", ctypes.c_int32), ("scale", ctypes.c_int32),
                ("eps", ctypes.c_float), ("workspace_mb", ctypes.c_int32), ("products", ctypes.c_int32)]


class AdamWListConfig(ctypes.Structure):
    """apollo_adamw_list_config."""
    _fields_ = [("state_bits", ctypes.c_int32), ("bias_correction", ctypes.c_int32), ("beta1", ctypes.c_double),
                ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("seed", ctypes.c_uint64)]


class LogitRules(ctypes.Structure):
    """apollo_logit_rules."""
    _fields_ = [("history", ctypes.c_void_p), ("history_type", ctypes.c_int32), ("bias_word_type", ctypes.c_int32),
                ("history_rows", ctypes.c_int64), ("history_len", ctypes.c_int64), ("history_stride", ctypes.c_int64),
                ("length", ctypes.c_void_p), ("start", ctypes.c_void_p),
                ("repetition_at", ctypes.c_void_p), ("frequency_at", ctypes.c_void_p), ("presence_at", ctypes.c_void_p),
                ("repetition", ctypes.c_float), ("frequency", ctypes.c_float), ("presence", ctypes.c_float),
                ("bias", ctypes.c_void_p), ("bias_stride", ctypes.c_int64),
                ("bias_word", ctypes.c_void_p), ("bias_value", ctypes.c_void_p), ("n_bias", ctypes.c_int64),
                ("mask", ctypes.c_void_p), ("mask_stride", ctypes.c_int64)]


class Tuning(ctypes.Structure):
    """apollo_tuning: zero fields select the defaults."""
    _fields_ = [("kernel", ctypes.c_int32), ("p_source", ctypes.c_int32), ("p_generator", ctypes.c_int32),
                ("scratch_mb", ctypes.c_int32), ("r_slice", ctypes.c_int32), ("nblk", ctypes.c_int32),
                ("epi_prefetch", ctypes.c_int32), ("realign", ctypes.c_int32), ("repitch_mb", ctypes.c_int32)]


def make_tuning(kernel=TC_KERNEL_PAIR, p_source=P_SCRATCH, p_generator=0, scratch_mb=0, r_slice=0, nblk=0,
                epi_prefetch=None, realign=0, repitch_mb=0) -> Tuning:
    """epi_prefetch: distance in chunks (0 = no prefetch), None = the default."""
    return Tuning(int(kernel), int(p_source), int(p_generator), int(scratch_mb), int(r_slice), int(nblk),
                  0 if epi_prefetch is None else int(epi_prefetch) + 1, int(realign), int(repitch_mb))


_lib = None


_libs = {}


def use_library(path=None):
    """Route all later calls of this module through the library at `path` (None: libapollo.so); the test of
    the bounds-checking build switches to libapollo_debug.so and back.  Contexts keep the library they were
    created with."""
    global _lib
    _lib = None if path is None else _load_from(Path(path))


def load():
    """Load libapollo.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        _lib = _load_from(LIB_PATH)
    return _lib


def _load_from(path: Path):
    if path in _libs:
        return _libs[path]
    if not path.exists():
        raise ImportError(f"{path} is missing: run `python -m paper_2412_05270_b200.build` (nvcc, sm_100a)")
    lib = ctypes.CDLL(str(path))
    vp, i32, u32, u64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_float
    lib.apollo_workspace_bytes.argtypes = [ctypes.POINTER(Shape), i32, ctypes.POINTER(Config),
                                           ctypes.POINTER(ctypes.c_size_t)]
    lib.apollo_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Shape), i32, ctypes.POINTER(Config), vp,
                                  ctypes.c_size_t]
    lib.apollo_workspace_bytes_tuned.argtypes = [ctypes.POINTER(Shape), i32, ctypes.POINTER(Config),
                                                 ctypes.POINTER(Tuning), ctypes.POINTER(ctypes.c_size_t)]
    lib.apollo_create_tuned.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Shape), i32, ctypes.POINTER(Config),
                                        ctypes.POINTER(Tuning), vp, ctypes.c_size_t]
    lib.apollo_step.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), f32, f32, vp]
    lib.apollo_step_range.argtypes = [vp, i32, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), f32, f32, i32, vp]
    lib.apollo_set_projection.argtypes = [vp, i32, vp]
    lib.apollo_destroy.argtypes = [vp]
    lib.apollo_step_count.argtypes = [vp, ctypes.POINTER(ctypes.c_int64)]
    lib.apollo_get_scales.argtypes = [vp, i32, vp, vp]
    lib.apollo_get_limiter.argtypes = [vp, i32, vp, vp]
    lib.apollo_get_state.argtypes = [vp, i32, vp, vp, vp]
    lib.apollo_set_delta_out.argtypes = [vp, ctypes.POINTER(vp)]
    lib.apollo_status.argtypes = [vp, vp]
    lib.apollo_selftest_bounded_wait.argtypes = [vp, vp]
    lib.apollo_philox_draws.argtypes = [u64, u32, u32, i32, i32, vp, vp]
    lib.apollo_projection.argtypes = [u64, u32, u32, i32, i32, vp, vp]
    lib.apollo_get_path.argtypes = [vp, i32, ctypes.POINTER(i32)]
    lib.apollo_last_launches.argtypes = [vp, ctypes.POINTER(i32)]
    lib.apollo_set_timing.argtypes = [vp, i32]
    lib.apollo_get_timing.argtypes = [vp, i32, ctypes.POINTER(f32)]
    lib.apollo_mini_step_static.argtypes = [vp, vp, ctypes.c_int64, ctypes.c_int64, vp, vp, vp,
                                            ctypes.POINTER(Config), u32, ctypes.c_int64, f32, f32, vp]
    lib.apollo_strerror.argtypes = [ctypes.c_int]
    lib.apollo_strerror.restype = ctypes.c_char_p
    lib.apollo_adamw_step.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                      ctypes.POINTER(ctypes.c_int64), i32, i32, f32, f32, f32, f32, f32,
                                      ctypes.c_int64, i32, ctypes.POINTER(vp), vp]
    lib.apollo_state_bytes.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
    lib.apollo_state_export.argtypes = [vp, vp, vp]
    lib.apollo_state_import.argtypes = [vp, vp, ctypes.c_int64, vp]
    lib.apollo_muon_workspace_bytes.argtypes = [ctypes.POINTER(Shape), i32, ctypes.POINTER(MuonConfig),
                                                ctypes.POINTER(ctypes.c_size_t)]
    lib.apollo_muon_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(Shape), i32, ctypes.POINTER(MuonConfig), vp,
                                       ctypes.c_size_t]
    lib.apollo_muon_destroy.argtypes = [vp]
    lib.apollo_muon_step.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), f32, f32, vp]
    lib.apollo_muon_orthogonalize.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), vp]
    lib.apollo_muon_status.argtypes = [vp, vp]
    lib.apollo_muon_last_launches.argtypes = [vp, ctypes.POINTER(i32)]
    i64 = ctypes.c_int64
    lib.apollo_embedding.argtypes = [vp, i64, i64, i32, vp, i32, i64, f32, vp, i64, vp]
    lib.apollo_embedding_grad_workspace_bytes.argtypes = [i64, i64, i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.apollo_embedding_grad.argtypes = [vp, i64, vp, i32, i64, i64, i64, i32, f32, i32, vp, vp, ctypes.c_size_t, vp]
    lib.apollo_token_logprobs.argtypes = [vp, i64, i64, i64, i32, vp, i32, f32, i32, vp, vp, vp, vp, vp, vp]
    lib.apollo_token_logprobs_grad.argtypes = [vp, i64, i64, i64, i32, vp, i32, f32, vp, vp, vp, vp, vp, i64, vp]
    f64, size_p = ctypes.c_double, ctypes.POINTER(ctypes.c_size_t)
    lib.apollo_grad_norm_workspace_bytes.argtypes = [i32, size_p]
    lib.apollo_grad_norm.argtypes = [vp, vp, vp, i32, f64, vp, vp, ctypes.c_size_t, vp]
    lib.apollo_adamw_list_state_bytes.argtypes = [vp, i32, i32, size_p]
    lib.apollo_adamw_list_step.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, ctypes.c_size_t, f64, f64, i64, vp, vp, vp, vp]
    lib.apollo_adamw_list_moments.argtypes = [vp, ctypes.c_size_t, i64, vp, vp, vp]
    lib.apollo_adjust_logits.argtypes = [vp, i64, i64, i64, i32, vp, vp, i64, vp]
    lib.apollo_adjust_logits_grad_workspace_bytes.argtypes = [i64, i64, size_p]
    lib.apollo_adjust_logits_grad.argtypes = [vp, i64, i64, i64, i32, vp, vp, i64, vp, i64, vp, i64, vp, vp, ctypes.c_size_t, vp]
    lib.apollo_cuda_error_string.argtypes = []
    lib.apollo_cuda_error_string.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name not in ("apollo_strerror", "apollo_cuda_error_string"):
            getattr(lib, name).restype = ctypes.c_int
    _libs[path] = lib
    return lib


def strerror(code: int) -> str:
    return load().apollo_strerror(code).decode()


def _check(code: int, what: str):
    if code != OK:
        raise ApolloError(code, what)


# The current stream's handle without a Stream object around it (3 us less per call), where this torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream_ptr(stream) -> int:
    if stream is None:
        if _raw_stream is not None:
            return _raw_stream(_current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _shape_array(shapes):
    arr = (Shape * len(shapes))()
    for i, (r, c) in enumerate(shapes):
        arr[i].rows, arr[i].cols = int(r), int(c)
    return arr


def make_config(rank, mode=SCALE_CHANNEL, dtype=DT_BF16, T=200, seed=0, alpha=1.0, gamma=1.01,
                beta1=0.9, beta2=0.999, eps=1e-8, bias_correction=False, flags=0) -> Config:
    return Config(int(rank), int(mode), int(dtype), int(T), int(seed), float(alpha), float(gamma),
                  float(beta1), float(beta2), float(eps), int(bool(bias_correction)), int(flags))


def config_for(wl, flags=0, bias_correction=False) -> Config:
    """The library configuration of a named workload (see workloads.py)."""
    return make_config(rank=wl.rank, mode=SCALE_TENSOR if wl.mode == "tensor" else SCALE_CHANNEL,
                       dtype=DT_BF16 if wl.dtype == "bf16" else DT_F32, T=wl.T, seed=wl.seed,
                       alpha=wl.alpha, gamma=wl.gamma, beta1=wl.beta1, beta2=wl.beta2, eps=wl.eps,
                       bias_correction=bias_correction, flags=flags)


def workspace_bytes(shapes, cfg: Config, tuning: Tuning | None = None) -> int:
    out = ctypes.c_size_t(0)
    if tuning is None:
        _check(load().apollo_workspace_bytes(_shape_array(shapes), len(shapes), ctypes.byref(cfg), ctypes.byref(out)),
               "apollo_workspace_bytes")
    else:
        _check(load().apollo_workspace_bytes_tuned(_shape_array(shapes), len(shapes), ctypes.byref(cfg),
                                                   ctypes.byref(tuning), ctypes.byref(out)),
               "apollo_workspace_bytes_tuned")
    return out.value


def philox_draws(seed: int, matrix: int, epoch: int, r: int, m: int, stream=None) -> torch.Tensor:
    out = torch.empty((r, (m + 3) // 4, 4), dtype=torch.int32, device="cuda")
    _check(load().apollo_philox_draws(seed, matrix, epoch, r, m, out.data_ptr(), _stream_ptr(stream)),
           "apollo_philox_draws")
    return out


def projection(seed: int, matrix: int, epoch: int, r: int, m: int, stream=None) -> torch.Tensor:
    out = torch.empty((r, m), dtype=torch.float32, device="cuda")
    _check(load().apollo_projection(seed, matrix, epoch, r, m, out.data_ptr(), _stream_ptr(stream)),
           "apollo_projection")
    return out


def mini_step_static(W, G, M, V, prev_norm, cfg: Config, matrix: int, t: int, lr: float, wd: float = 0.0,
                     stream=None):
    """apollo_mini_step_static: a rank-1 step for one matrix that allocates nothing.

    For callers that cannot get device memory when the optimizer has to run (see the
    header): W, G are the weight and gradient, M, V (n floats) and prev_norm (1 float) the
    state the caller keeps between steps; the temporaries live in a fixed array inside the
    library, shared by all calls on the device, so calls must not overlap on the GPU.
    """
    rows, cols = W.shape
    _check(load().apollo_mini_step_static(W.data_ptr(), G.data_ptr(), rows, cols, M.data_ptr(), V.data_ptr(),
                                          prev_norm.data_ptr(), ctypes.byref(cfg), matrix, t, lr, wd,
                                          _stream_ptr(stream)), "apollo_mini_step_static")


def adamw_step(params, grads, ms, vs, t, lr, beta1=0.9, beta2=0.999, eps=1e-8, wd=0.0, bias_correction=True,
               deltas=None, stream=None):
    """apollo_adamw_step over lists of CUDA tensors (params/grads of one dtype; ms/vs fp32, same numel)."""
    n = len(params)
    dtype = DT_BF16 if params[0].dtype == torch.bfloat16 else DT_F32

    def arr(ts):
        a = (ctypes.c_void_p * n)()
        for i, x in enumerate(ts):
            a[i] = None if x is None else x.data_ptr()
        return a
    numel = (ctypes.c_int64 * n)(*[p.numel() for p in params])
    _check(load().apollo_adamw_step(arr(params), arr(grads), arr(ms), arr(vs), numel, n, dtype, lr, beta1, beta2, eps,
                                    wd, t, int(bool(bias_correction)), arr(deltas) if deltas is not None else None,
                                    _stream_ptr(stream)), "apollo_adamw_step")


def _dtype_of(x: torch.Tensor, what: str) -> int:
    if x.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"{what} must be bfloat16 or float32, got {x.dtype}")
    return DT_BF16 if x.dtype == torch.bfloat16 else DT_F32


def _index_of(x: torch.Tensor, what: str) -> int:
    dtype = x.dtype
    if dtype is torch.int64:
        return INDEX_I64
    if dtype is not torch.int32:
        raise ValueError(f"{what} must be of int32 or int64")
    return INDEX_I32


def _rows_of(x: torch.Tensor, what: str) -> int:
    """The row stride of a 2-D CUDA tensor whose rows are contiguous."""
    shape = x.shape
    if not x.is_cuda or len(shape) != 2 or (shape[0] > 0 and shape[1] > 1 and x.stride(1) != 1):
        raise ValueError(f"{what} must be a 2-D CUDA tensor with contiguous rows")
    if shape[0] <= 1:
        return max(shape[1], 1)
    stride = x.stride(0)
    if stride < shape[1]:
        raise ValueError(f"{what} must not have overlapping rows")
    return stride


def _two_devices():
    return ValueError("the tensors of a call, out and workspace among them, must be on one device")


_here = contextlib.nullcontext()


def _on(stream, device):
    """The tensors' device; what the call allocates belongs to the stream that it runs on."""
    if stream is not None:
        if stream.device != device:
            raise ValueError(f"a stream of {stream.device} cannot work on tensors of {device}")
        return torch.cuda.stream(stream)
    return _here if device.index == _current_device() else torch.cuda.device(device)


def embedding(table, index, scale: float = 1.0, out=None, stream=None) -> torch.Tensor:
    """apollo_embedding: scale * table[index], a zero row where the index is outside the table.

    table: (rows, dim), contiguous; index: any shape and strides, int32 or int64; out: (index.numel(), dim) rows, made if None
    (then of the index's shape with dim appended)."""
    dtype, itype = _dtype_of(table, "table"), _index_of(index, "index")
    if table.dim() != 2 or not table.is_contiguous() or not table.is_cuda:
        raise ValueError("table must be a 2-D contiguous CUDA tensor")
    device = table.device
    if index.device != device or (out is not None and out.device != device):
        raise _two_devices()
    rows, dim = table.shape
    n = index.numel()
    with _on(stream, device):
        index = index.contiguous()
        res = flat = out
        if out is None:
            res = torch.empty((*index.shape, dim), dtype=table.dtype, device=device)
            flat = res.view(n, dim)
        elif out.dtype != table.dtype or tuple(out.shape) != (n, dim):
            raise ValueError("out must have the table's dtype and one row per index")
        _check(load().apollo_embedding(table.data_ptr(), rows, dim, dtype, index.data_ptr(), itype, n, scale,
                                       flat.data_ptr(), _rows_of(flat, "out"), _stream_ptr(stream)), "apollo_embedding")
    return res


def embedding_grad_workspace_bytes(n_tokens: int, rows: int, dim: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().apollo_embedding_grad_workspace_bytes(n_tokens, rows, dim, ctypes.byref(out)),
           "apollo_embedding_grad_workspace_bytes")
    return out.value


def embedding_grad(d_out, index, rows: int, scale: float = 1.0, out=None, accumulate: bool = False, workspace=None,
                   stream=None) -> torch.Tensor:
    """apollo_embedding_grad: the gradient of `embedding` for its table, (rows, dim) in d_out's dtype.

    d_out: (index.numel(), dim) rows; out: made if None, else overwritten (accumulate: added to); workspace: a uint8
    CUDA tensor of embedding_grad_workspace_bytes(), made if None."""
    dtype, itype = _dtype_of(d_out, "d_out"), _index_of(index, "index")
    stride = _rows_of(d_out, "d_out")
    n, dim = d_out.shape
    if n != index.numel():
        raise ValueError("d_out must have one row per index")
    device = d_out.device
    if index.device != device or (out is not None and out.device != device) or (workspace is not None and workspace.device != device):
        raise _two_devices()
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    with _on(stream, device):
        index = index.contiguous()
        if out is None:
            if accumulate:
                raise ValueError("accumulate needs the gradient to add to")
            out = torch.empty((rows, dim), dtype=d_out.dtype, device=device)
        elif out.dtype != d_out.dtype or tuple(out.shape) != (rows, dim) or not out.is_contiguous():
            raise ValueError("out must be a contiguous CUDA tensor (rows, dim) of d_out's dtype")
        if workspace is None:
            workspace = torch.empty(embedding_grad_workspace_bytes(n, rows, dim), dtype=torch.uint8, device=device)
        _check(load().apollo_embedding_grad(d_out.data_ptr(), stride, index.data_ptr(), itype, n, rows, dim, dtype, scale,
                                            int(bool(accumulate)), out.data_ptr(), workspace.data_ptr(),
                                            workspace.numel() * workspace.element_size(), _stream_ptr(stream)),
               "apollo_embedding_grad")
    return out


class TokenLogprobs(NamedTuple):
    logprob: torch.Tensor
    entropy: torch.Tensor
    lse: torch.Tensor
    top_logprob: torch.Tensor | None
    top_index: torch.Tensor | None


def token_logprobs(logits, targets, scale: float = 1.0, top: int = 0, stream=None) -> TokenLogprobs:
    """apollo_token_logprobs over the rows of `logits` (n, vocab); targets: n of int32 or int64 in any shape, outside [0, vocab) =
    ignored; top: how many of the best alternatives (<= MAX_TOP) come back as (n, top) log probabilities and indices."""
    dtype, itype = _dtype_of(logits, "logits"), _index_of(targets, "targets")
    stride = _rows_of(logits, "logits")
    n, vocab = logits.shape
    if targets.numel() != n:
        raise ValueError("targets must have one entry per row of logits")
    device = logits.device
    if targets.device != device:
        raise _two_devices()
    with _on(stream, device):
        targets = targets.contiguous()
        # (empty_strided: 0.8 us less a call than empty, and for few rows the call is what takes the time; tensors of their own,
        # not views of one, 0.2 us more: autograd allows no view among several outputs to be changed in place)
        logprob = torch.empty_strided((n,), (1,), dtype=torch.float32, device=device)
        entropy, lse = torch.empty_like(logprob), torch.empty_like(logprob)
        best = best_at = None
        if top > 0:
            best = torch.empty_strided((n, top), (top, 1), dtype=torch.float32, device=device)
            best_at = torch.empty_strided((n, top), (top, 1), dtype=torch.int32, device=device)
        _check(load().apollo_token_logprobs(logits.data_ptr(), stride, n, vocab, dtype, targets.data_ptr(), itype, scale, top,
                                            logprob.data_ptr(), entropy.data_ptr(), lse.data_ptr(), None if best is None else best.data_ptr(),
                                            None if best_at is None else best_at.data_ptr(), _stream_ptr(stream)),
               "apollo_token_logprobs")
    return TokenLogprobs(logprob, entropy, lse, best, best_at)


def token_logprobs_grad(logits, targets, lse, entropy, d_logprob, d_entropy=None, scale: float = 1.0, out=None,
                        stream=None) -> torch.Tensor:
    """apollo_token_logprobs_grad: the gradient of the logits for upstream gradients of logprob and (or None) entropy,
    with lse and entropy as `token_logprobs` returned them; out may be the logits themselves."""
    dtype, itype = _dtype_of(logits, "logits"), _index_of(targets, "targets")
    stride = _rows_of(logits, "logits")
    n, vocab = logits.shape
    device = logits.device
    for x, what in ((lse, "lse"), (entropy, "entropy"), (d_logprob, "d_logprob"), (d_entropy, "d_entropy")):
        if x is None:
            continue
        if x.dtype != torch.float32 or x.numel() != n or not x.is_contiguous():
            raise ValueError(f"{what} must be a contiguous float32 CUDA tensor with one entry per row")
        if x.device != device:
            raise _two_devices()
    if targets.numel() != n:
        raise ValueError("targets must have one entry per row of logits")
    if targets.device != device or (out is not None and out.device != device):
        raise _two_devices()
    with _on(stream, device):
        targets = targets.contiguous()
        if out is None:
            out = torch.empty((n, vocab), dtype=logits.dtype, device=device)
        elif out.dtype != logits.dtype or tuple(out.shape) != (n, vocab):
            raise ValueError("out must have the logits' dtype and shape")
        _check(load().apollo_token_logprobs_grad(
            logits.data_ptr(), stride, n, vocab, dtype, targets.data_ptr(), itype, scale, lse.data_ptr(),
            None if entropy is None else entropy.data_ptr(), d_logprob.data_ptr(),
            None if d_entropy is None else d_entropy.data_ptr(), out.data_ptr(), _rows_of(out, "out"), _stream_ptr(stream)),
            "apollo_token_logprobs_grad")
    return out


_marshal_module = None


def _marshal():
    """The extension that reads tensors (csrc/marshal.cpp); raises if it has not been built (there is no fallback)."""
    global _marshal_module
    if _marshal_module is None:
        path = marshal_path()
        if not path.exists():
            raise ImportError(f"{path} is missing (it is built for one Python and one torch): run `python -m paper_2412_05270_b200.build`")
        spec = importlib.util.spec_from_file_location("_marshal", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        _marshal_module = module
    return _marshal_module


def _on_index(stream, index: int):
    """As _on, for the device with that index."""
    if stream is None and index == _current_device():
        return _here
    return _on(stream, torch.device("cuda", index))


def grad_norm(grads, max_norm: float = math.inf, out=None, workspace=None, stream=None) -> torch.Tensor:
    """apollo_grad_norm: two floats on the device, the global norm of the list and min(1, max_norm / norm).

    grads: contiguous CUDA tensors, bfloat16 or float32 in any mixture, None for one that is left out; workspace: a uint8 CUDA
    tensor of grad_norm_workspace_bytes(), made if None."""
    grads = list(grads)
    pointers, lengths, types, device, live = _marshal().pack("grads", grads, None, -1)
    if live == 0:
        raise ValueError("grad_norm needs a gradient")
    n = len(grads)
    for x, what in ((out, "out"), (workspace, "workspace")):
        if x is not None:
            if x.get_device() != device:
                raise _two_devices()
            if not x.is_contiguous():
                raise ValueError(f"{what} must be contiguous")
    if out is not None and (out.dtype != torch.float32 or out.numel() != 2):
        raise ValueError("out must hold two float32 values")
    given = out
    with _on_index(stream, device):
        if out is None:
            out = torch.empty_strided((2,), (1,), dtype=torch.float32, device="cuda")
        if workspace is None:
            workspace = torch.empty_strided((grad_norm_workspace_bytes(n),), (1,), dtype=torch.uint8, device="cuda")
        _check(load().apollo_grad_norm(pointers, lengths, types, n, max_norm, out.data_ptr(), workspace.data_ptr(),
                                       workspace.numel() * workspace.element_size(), _stream_ptr(stream)), "apollo_grad_norm")
    if given is not None:
        _marshal().changed((given,), None)
    return out


def grad_norm_workspace_bytes(n_tensors: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().apollo_grad_norm_workspace_bytes(n_tensors, ctypes.byref(out)), "apollo_grad_norm_workspace_bytes")
    return out.value


def adamw_state_bytes(numels, bits: int = 8) -> int:
    out = ctypes.c_size_t(0)
    _check(load().apollo_adamw_list_state_bytes((ctypes.c_int64 * len(numels))(*numels), len(numels), bits, ctypes.byref(out)),
           "apollo_adamw_list_state_bytes")
    return out.value


class AdamW:
    """apollo_adamw_list_step over a list of parameters (contiguous CUDA tensors on one device, bfloat16 or float32 in any
    mixture, none of them twice), with the moments of all of them in one buffer, `state`: of 8 or 32 bits, zero before the first step.

    state: a uint8 CUDA tensor of adamw_state_bytes() to go on with (a checkpoint is a copy of it, with the step count and the
    seed), made if None (the constructor waits for the current stream then).  Calls run on `stream` or the device's current one,
    whichever device is current; steps on different streams are the caller's to order."""

    def __init__(self, params, bits: int = 8, beta1=0.9, beta2=0.999, eps=1e-8, seed: int = 0, bias_correction: bool = True,
                 state=None):
        self.lib = load()
        self._pack, self._changed = _marshal().pack, _marshal().changed
        self.params = list(params)
        if not self.params or any(p is None for p in self.params):
            raise ValueError("AdamW needs a list of parameters")
        _, _, _, index, _ = self._pack("params", self.params, None, -1)
        used = [p.data_ptr() for p in self.params if p.numel()]
        if len(set(used)) < len(used):
            raise ValueError("a parameter is in the list twice")
        self.device, self._index, self.bits = torch.device("cuda", index), index, bits
        self._shapes = [tuple(p.shape) for p in self.params]               # what a step must find again, whatever becomes of the parameters' data
        numels = [p.numel() for p in self.params]
        self.cfg = AdamWListConfig(int(bits), int(bool(bias_correction)), float(beta1), float(beta2), float(eps), int(seed))
        self._cfg_at = ctypes.addressof(self.cfg)
        nbytes = adamw_state_bytes(numels, bits)
        self.n_blocks = nbytes // (2 * ADAMW_BLOCK + 2 if bits == 8 else 8 * ADAMW_BLOCK)
        self._streams = set()                                # what the allocator knows of the state's use
        with _on(None, self.device):
            if state is None:
                state = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
                self._streams.add(_stream_ptr(None))         # the state belongs to this one
                if not torch.cuda.is_current_stream_capturing():
                    # whichever stream the first step runs on (or is captured on), the zeros are there
                    torch.cuda.current_stream().synchronize()
            elif state.dtype != torch.uint8 or state.numel() != nbytes or not state.is_contiguous():
                raise ValueError(f"state must be a contiguous uint8 CUDA tensor of {nbytes} bytes")
            elif state.device != self.device:
                raise _two_devices()
        self.state = state

    def _run(self, stream) -> int:
        ptr = _stream_ptr(stream)
        if ptr not in self._streams:
            # freed, the state must not be handed out again before this stream is done with it (which stream a state of the caller's belongs to
            # is not known here)
            self.state.record_stream(torch.cuda.current_stream())
            self._streams.add(ptr)
        return ptr

    def _scalar(self, x, dtype, what):
        if x.dtype != dtype or x.numel() != 1:
            raise ValueError(f"{what} must be one value of {dtype}")
        if x.device != self.device:
            raise _two_devices()
        return x.data_ptr()

    def step(self, grads, lr, t, wd: float = 0.0, factor=None, stream=None):
        """One step from the gradients (None: that parameter and its moments stay as they are), after t earlier ones.

        lr: a number, or a float32 CUDA tensor of one value; t: a number, or an int64 CUDA tensor of one value (read when the step
        runs: a captured step can be replayed with other values); factor: a float32 CUDA tensor of one value that the gradients are multiplied by
        (grad_norm(...)[1:]); where it is not finite the step changes nothing."""
        index = self._index
        if not isinstance(grads, (list, tuple)):
            grads = list(grads)                              # read twice
        pointers, lengths, types, _, _ = self._pack("params", self.params, self._shapes, index)
        g_pointers, _, g_types, _, _ = self._pack("grads", grads, self.params, index)
        lr_at = t_at = factor_at = None
        if isinstance(lr, torch.Tensor):
            lr, lr_at = 0.0, self._scalar(lr, torch.float32, "lr")
        if isinstance(t, torch.Tensor):
            t, t_at = 0, self._scalar(t, torch.int64, "t")
        if factor is not None:
            factor_at = self._scalar(factor, torch.float32, "factor")
        with _on_index(stream, index):
            _check(self.lib.apollo_adamw_list_step(self._cfg_at, pointers, g_pointers, lengths, types, g_types, len(self.params),
                                                   self.state.data_ptr(), self.state.numel(), lr, wd, t, factor_at, lr_at, t_at,
                                                   self._run(stream)), "apollo_adamw_list_step")
        self._changed(self.params, grads)

    def moments(self, stream=None):
        """(m, v) of all blocks in list order, ADAMW_BLOCK n_blocks values each: what 8-bit codes stand for, exactly, in bfloat16; of
        32 bits the state itself, not a copy."""
        if self.bits == 32:
            return self.state.view(torch.float32).chunk(2)
        with _on(stream, self.device):
            m, v = (torch.empty(self.n_blocks * ADAMW_BLOCK, dtype=torch.bfloat16, device=self.device) for _ in range(2))
            _check(self.lib.apollo_adamw_list_moments(self.state.data_ptr(), self.state.numel(), self.n_blocks, m.data_ptr(),
                                                      v.data_ptr(), self._run(stream)), "apollo_adamw_list_moments")
        return m, v


# What _marshal().describe() gives of a tensor, by place.
_AT, _DEVICE, _TYPE, _DIM, _ROWS, _COLS, _STEP, _NEXT, _WHOLE = range(9)
_F32, _BF16, _I32, _I64 = range(4)


def _described_rows(x, what: str, like=None):
    """describe() of a 2-D CUDA tensor, bfloat16 or float32, whose rows are contiguous and do not overlap, and the stride between them;
    like: describe() of one with the same type, shape and device."""
    d = _marshal().describe(x)
    if like is not None and (d[_TYPE] != like[_TYPE] or d[_DIM] != 2 or d[_ROWS:_COLS + 1] != like[_ROWS:_COLS + 1]):
        raise ValueError(f"{what} must have the logits' dtype and shape")
    if d[_TYPE] not in (_F32, _BF16):
        raise ValueError(f"{what} must be bfloat16 or float32, got {x.dtype}")
    if like is not None and d[_DEVICE] != like[_DEVICE]:
        raise _two_devices()
    rows, cols = d[_ROWS], d[_COLS]
    if d[_DEVICE] < 0 or d[_DIM] != 2 or (rows > 0 and cols > 1 and d[_NEXT] != 1):
        raise ValueError(f"{what} must be a 2-D CUDA tensor with contiguous rows")
    if rows <= 1:
        return d, max(cols, 1)
    if d[_STEP] < cols:
        raise ValueError(f"{what} must not have overlapping rows")
    return d, d[_STEP]


def _rules_of(of, history, lengths, start, repetition, frequency, presence, bias, bias_index, bias_value, mask):
    """The rules for logits described by `of` as the library takes them, and copies that they point into."""
    describe = _marshal().describe
    n, vocab, device, logits_type = of[_ROWS], of[_COLS], of[_DEVICE], of[_TYPE]
    r = LogitRules(repetition=1.0)
    kept = []

    def whole(x, d):
        if d[_DEVICE] != device:
            raise _two_devices()
        if not d[_WHOLE]:
            x = x.contiguous()
            kept.append(x)
            return x.data_ptr()
        return d[_AT]

    def per_row(x, kind, what):
        d = describe(x)
        if d[_TYPE] != kind or d[_DIM] != 1 or d[_ROWS] != n:
            raise ValueError(f"{what} must be {'int32' if kind == _I32 else 'float32'} with one entry per row of logits")
        return whole(x, d)
    if history is not None:
        d = describe(history)
        if d[_TYPE] not in (_I32, _I64):
            raise ValueError("history must be of int32 or int64")
        rows, length, stride = d[_ROWS], d[_COLS], d[_STEP]
        if d[_DIM] != 2 or (n and (rows < 1 or n % rows)):
            raise ValueError("history must have a row for each row of logits, or for the same number of them each")
        if (length > 1 and d[_NEXT] != 1) or (rows > 1 and 0 < stride < length):
            history = history.contiguous()
            kept.append(history)
            d, stride = describe(history), length
        if d[_DEVICE] != device:
            raise _two_devices()
        if rows and length:
            r.history, r.history_rows, r.history_len, r.history_stride = d[_AT], rows, length, stride if rows > 1 else 0
            r.history_type = INDEX_I64 if d[_TYPE] == _I64 else INDEX_I32
        if lengths is not None:
            r.length = per_row(lengths, _I32, "lengths")
        if start is not None:
            r.start = per_row(start, _I32, "start")
        if isinstance(repetition, torch.Tensor):
            r.repetition_at = per_row(repetition, _F32, "repetition")
        else:
            r.repetition = repetition
        if isinstance(frequency, torch.Tensor):
            r.frequency_at = per_row(frequency, _F32, "frequency")
        else:
            r.frequency = frequency
        if isinstance(presence, torch.Tensor):
            r.presence_at = per_row(presence, _F32, "presence")
        else:
            r.presence = presence
    if bias is not None:
        d = describe(bias)
        if d[_TYPE] != logits_type or not ((d[_DIM] == 1 and d[_ROWS] == vocab) or (d[_DIM] == 2 and d[_ROWS] == n and d[_COLS] == vocab)):
            raise ValueError("bias must have the logits' dtype and be a row of the vocabulary, or one for each row of logits")
        if d[_DIM] == 2 and n > 1 and d[_STEP] >= vocab and (vocab == 1 or d[_NEXT] == 1):
            if d[_DEVICE] != device:
                raise _two_devices()
            r.bias, r.bias_stride = d[_AT], d[_STEP]
        else:
            r.bias, r.bias_stride = whole(bias, d), vocab if d[_DIM] == 2 else 0
    if bias_index is not None:
        d = describe(bias_index)
        if d[_TYPE] not in (_I32, _I64):
            raise ValueError("bias_index must be of int32 or int64")
        if d[_DIM] != 2 or d[_ROWS] != n:
            raise ValueError("bias_index must have a row for each row of logits")
        r.bias_word, r.n_bias, r.bias_word_type = whole(bias_index, d), d[_COLS], INDEX_I64 if d[_TYPE] == _I64 else INDEX_I32
        if bias_value is not None:
            v = describe(bias_value)
            if v[_TYPE] != _F32 or v[_DIM] != 2 or v[_ROWS] != n or v[_COLS] != d[_COLS]:
                raise ValueError("bias_value must be float32 of bias_index's shape")
            r.bias_value = whole(bias_value, v)
    elif bias_value is not None:
        raise ValueError("bias_value needs bias_index")
    if mask is not None:
        d = describe(mask)
        words = (vocab + 31) // 32
        if d[_TYPE] != _I32 or not ((d[_DIM] == 1 and d[_ROWS] == words) or (d[_DIM] == 2 and d[_ROWS] in (1, n) and d[_COLS] == words)):
            raise ValueError(f"mask must be int32 with {words} words of 32 bits a row, one row or one for each row of logits")
        r.mask, r.mask_stride = whole(mask, d), words if d[_DIM] == 2 and d[_ROWS] > 1 else 0
    return r, kept


def adjust_logits(logits, history=None, lengths=None, start=None, repetition=1.0, frequency=0.0, presence=0.0, bias=None,
                  bias_index=None, bias_value=None, mask=None, out=None, stream=None) -> torch.Tensor:
    """apollo_adjust_logits over the rows of `logits` (n, vocab); out: made if None, may be the logits.

    history: (h, length) tokens, int32 or int64 (outside [0, vocab): none), h a divisor of n: row r of the logits has history row
    r // (n / h), of which the first lengths[r] (int32) count, for frequency and presence those from start[r] (int32) on; repetition,
    frequency, presence: numbers, or float32 (n,);  bias: (vocab,) or (n, vocab) of the logits' dtype;  bias_index, bias_value: (n, k)
    words and float32 values;  mask: int32 words of 32 bits, (1 or n, ceil(vocab / 32)), bit set = word allowed."""
    of, stride = _described_rows(logits, "logits")
    n, vocab = of[_ROWS], of[_COLS]
    if out is not None and out is not logits:
        to, out_stride = _described_rows(out, "out", of)
    else:
        to, out_stride = of, stride
    if bias_index is not None and bias_value is None:
        raise ValueError("bias_index needs bias_value")
    given = out
    with _on_index(stream, of[_DEVICE]):
        rules, kept = _rules_of(of, history, lengths, start, repetition, frequency, presence, bias, bias_index, bias_value, mask)
        out_at = to[_AT]
        if out is None:
            out = torch.empty_strided((n, vocab), (vocab, 1), dtype=logits.dtype, device="cuda")
            out_at, out_stride = out.data_ptr(), vocab
        _check(load().apollo_adjust_logits(of[_AT], stride, n, vocab, of[_TYPE], ctypes.byref(rules), out_at, out_stride, _stream_ptr(stream)),
               "apollo_adjust_logits")
    if given is not None:
        _marshal().changed((given,), None)
    return out


def adjust_logits_grad_workspace_bytes(n_rows: int, vocab: int) -> int:
    out = ctypes.c_size_t(0)
    _check(load().apollo_adjust_logits_grad_workspace_bytes(n_rows, vocab, ctypes.byref(out)), "apollo_adjust_logits_grad_workspace_bytes")
    return out.value


class AdjustLogitsGrad(NamedTuple):
    logits: torch.Tensor
    bias: torch.Tensor | None
    value: torch.Tensor | None


def adjust_logits_grad(logits, d_out, history=None, lengths=None, repetition=1.0, mask=None, bias: str = "none", bias_index=None,
                       out=None, workspace=None, stream=None) -> AdjustLogitsGrad:
    """apollo_adjust_logits_grad: the gradients of `adjust_logits` for its logits, a bias ("shared": (vocab,), "row": (n, vocab), "none")
    and, where bias_index is given, the values; rules as there.  out: of the logits' gradient, made if None, may be d_out;
    workspace ("shared"): a uint8 CUDA tensor of adjust_logits_grad_workspace_bytes(), made if None."""
    of, stride = _described_rows(logits, "logits")
    d, d_stride = _described_rows(d_out, "d_out", of)
    n, vocab = of[_ROWS], of[_COLS]
    if bias not in ("none", "shared", "row"):
        raise ValueError('bias must be "none", "shared" or "row"')
    to, out_stride = (d, d_stride) if out is d_out else (None, vocab) if out is None else _described_rows(out, "out", of)
    if workspace is not None:
        if workspace.get_device() != of[_DEVICE]:
            raise _two_devices()
        if not workspace.is_contiguous():
            raise ValueError("workspace must be contiguous")
    with _on_index(stream, of[_DEVICE]):
        rules, kept = _rules_of(of, history, lengths, None, repetition, 0.0, 0.0, None, bias_index, None, mask)
        if out is None:
            out = torch.empty_strided((n, vocab), (vocab, 1), dtype=logits.dtype, device="cuda")
        d_bias = d_value = None
        workspace_at, workspace_bytes = None, 0
        if bias == "shared":
            d_bias = torch.empty_strided((vocab,), (1,), dtype=logits.dtype, device="cuda")
            if workspace is None:
                workspace = torch.empty_strided((adjust_logits_grad_workspace_bytes(n, vocab),), (1,), dtype=torch.uint8, device="cuda")
            workspace_at, workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        elif bias == "row":
            d_bias = torch.empty_strided((n, vocab), (vocab, 1), dtype=logits.dtype, device="cuda")
        if bias_index is not None:
            k = rules.n_bias
            d_value = torch.empty_strided((n, k), (k, 1), dtype=torch.float32, device="cuda")
        _check(load().apollo_adjust_logits_grad(
            of[_AT], stride, n, vocab, of[_TYPE], ctypes.byref(rules), d[_AT], d_stride, out.data_ptr() if to is None else to[_AT], out_stride,
            None if d_bias is None else d_bias.data_ptr(), vocab if bias == "row" else 0, None if d_value is None else d_value.data_ptr(),
            workspace_at, workspace_bytes, _stream_ptr(stream)), "apollo_adjust_logits_grad")
    if to is not None:
        _marshal().changed((out,), None)
    return AdjustLogitsGrad(out, d_bias, d_value)


def make_muon_config(dtype=DT_BF16, steps=5, coef=(3.4445, -4.7750, 2.0315), momentum=0.95, nesterov=True,
                     scale=MUON_SCALE_SHAPE, eps=1e-7, workspace_mb=0, products=MUON_PRODUCTS_DEFAULT) -> MuonConfig:
    """products: MUON_PRODUCTS_PAIRS takes bfloat16 weights through products as exact as those of float32 ones."""
    return MuonConfig(int(dtype), int(steps), (ctypes.c_float * 3)(*coef), float(momentum), int(bool(nesterov)),
                      int(scale), float(eps), int(workspace_mb), int(products))


def muon_workspace_bytes(shapes, cfg: MuonConfig) -> int:
    out = ctypes.c_size_t(0)
    _check(load().apollo_muon_workspace_bytes(_shape_array(shapes), len(shapes), ctypes.byref(cfg), ctypes.byref(out)),
           "apollo_muon_workspace_bytes")
    return out.value


class Muon:
    """apollo_muon_create / apollo_muon_step: orthogonalised updates of a list of 2-D CUDA tensors (one dtype,
    contiguous, on the context's device); the fp32 momenta are the caller's.  Calls run on `stream` or the device's
    current one, whichever device is current."""

    def __init__(self, shapes, cfg: MuonConfig, device="cuda"):
        self.lib = load()
        self.shapes = [(int(r), int(c)) for r, c in shapes]
        self.cfg = cfg
        nbytes = muon_workspace_bytes(self.shapes, cfg)
        self.workspace_bytes = nbytes
        with torch.cuda.device(device):
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
            self.device = self.workspace.device              # with its index
            self._home = _stream_ptr(None)                   # the stream that the workspace belongs to
            base = (self.workspace.data_ptr() + 255) // 256 * 256
            ctx = ctypes.c_void_p()
            _check(self.lib.apollo_muon_create(ctypes.byref(ctx), _shape_array(self.shapes), len(self.shapes),
                                               ctypes.byref(cfg), base, nbytes), "apollo_muon_create")
        self.ctx = ctx
        n = len(self.shapes)
        self._arrays = [(ctypes.c_void_p * n)() for _ in range(3)]

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.apollo_muon_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _marshal(self, lists):
        want = torch.bfloat16 if self.cfg.dtype == DT_BF16 else torch.float32
        for k, (arr, xs) in enumerate(zip(self._arrays, lists)):
            if len(xs) != len(self.shapes):
                raise ValueError("parameter list length differs from the context's")
            dt = torch.float32 if k == 2 else want
            for i, (x, shp) in enumerate(zip(xs, self.shapes)):
                if x.dtype != dt or x.shape != shp or not x.is_cuda or not x.is_contiguous():
                    raise ValueError("tensors must be contiguous CUDA tensors of the context's dtype and shapes (momenta: float32)")
                if x.device != self.device:
                    raise ValueError(f"tensors must be on the context's device {self.device}, got {x.device}")
                arr[i] = x.data_ptr()

    def _call(self, name, stream, *args):
        with _on(stream, self.device):
            ptr = _stream_ptr(stream)
            if ptr != self._home:
                # freed, the workspace must not be handed out again before this stream is done with it
                self.workspace.record_stream(torch.cuda.current_stream())
            _check(getattr(self.lib, name)(self.ctx, *args, ptr), name)

    def step(self, Ws, Gs, Ms, lr: float, wd: float = 0.0, stream=None):
        """One update of the weights Ws and the momenta Ms (float32, zero before the first step) from the gradients Gs."""
        self._marshal((Ws, Gs, Ms))
        w, g, m = self._arrays
        self._call("apollo_muon_step", stream, w, g, m, lr, wd)

    def orthogonalize(self, Us, Os, stream=None):
        """Os <- the orthogonalised Us (Os may be Us)."""
        self._marshal((Os, Us))
        o, u, _ = self._arrays
        self._call("apollo_muon_orthogonalize", stream, u, o)

    def status(self, stream=None) -> int:
        with _on(stream, self.device):
            return self.lib.apollo_muon_status(self.ctx, _stream_ptr(stream))

    def last_launches(self) -> int:
        out = ctypes.c_int32(0)
        _check(self.lib.apollo_muon_last_launches(self.ctx, ctypes.byref(out)), "apollo_muon_last_launches")
        return out.value


class Apollo:
    """apollo_create / apollo_step over a list of CUDA tensors (same dtype, 2-D, contiguous)."""

    def __init__(self, shapes, cfg: Config, device="cuda", tuning: Tuning | None = None):
        self.lib = load()
        self.shapes = [(int(r), int(c)) for r, c in shapes]
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = workspace_bytes(self.shapes, cfg, tuning)
        self.workspace_bytes = nbytes
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.workspace.data_ptr()
            self._ws_ptr = (base + 255) // 256 * 256
            ctx = ctypes.c_void_p()
            if tuning is None:
                _check(self.lib.apollo_create(ctypes.byref(ctx), _shape_array(self.shapes), len(self.shapes),
                                              ctypes.byref(cfg), self._ws_ptr, nbytes), "apollo_create")
            else:
                _check(self.lib.apollo_create_tuned(ctypes.byref(ctx), _shape_array(self.shapes), len(self.shapes),
                                                    ctypes.byref(cfg), ctypes.byref(tuning), self._ws_ptr, nbytes),
                       "apollo_create_tuned")
        self.ctx = ctx
        self._delta = None
        self._w_arr = (ctypes.c_void_p * len(self.shapes))()
        self._g_arr = (ctypes.c_void_p * len(self.shapes))()

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.apollo_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check_tensors(self, Ws, Gs):
        want = torch.bfloat16 if self.cfg.dtype == DT_BF16 else torch.float32
        if len(Ws) != len(self.shapes) or len(Gs) != len(self.shapes):
            raise ValueError("parameter list length differs from the context's")
        for w, g, shp in zip(Ws, Gs, self.shapes):
            for x in (w, g):
                if not x.is_cuda or x.dtype != want or tuple(x.shape) != shp or not x.is_contiguous():
                    raise ValueError("tensors must be contiguous CUDA tensors of the context's dtype and shapes")

    def step(self, Ws, Gs, lr: float, wd: float = 0.0, stream=None, check: bool = True):
        if check:
            self._check_tensors(Ws, Gs)
        for i, (w, g) in enumerate(zip(Ws, Gs)):
            self._w_arr[i] = w.data_ptr()
            self._g_arr[i] = g.data_ptr()
        _check(self.lib.apollo_step(self.ctx, self._w_arr, self._g_arr, lr, wd, _stream_ptr(stream)), "apollo_step")

    def step_range(self, first: int, Ws, Gs, lr: float, wd: float = 0.0, close_step: bool = False, stream=None):
        """apollo_step_range: the step of matrices first .. first + len(Ws) - 1 (layer-wise updates)."""
        n = len(Ws)
        w = (ctypes.c_void_p * n)(*[x.data_ptr() for x in Ws])
        g = (ctypes.c_void_p * n)(*[x.data_ptr() for x in Gs])
        _check(self.lib.apollo_step_range(self.ctx, first, n, w, g, lr, wd, int(close_step), _stream_ptr(stream)),
               "apollo_step_range")

    def set_projection(self, mat: int, P):
        """Use the fp32 CUDA tensor P (r x m) as the projection of matrix `mat`; None restores the generator."""
        if P is not None:
            m = min(self.shapes[mat])
            assert P.is_cuda and P.dtype == torch.float32 and tuple(P.shape) == (self.cfg.rank, m) and P.is_contiguous()
            self._ext_p = getattr(self, "_ext_p", {})
            self._ext_p[mat] = P                      # keep it alive
        _check(self.lib.apollo_set_projection(self.ctx, mat, None if P is None else P.data_ptr()),
               "apollo_set_projection")

    def set_delta_out(self, deltas):
        """deltas: list of float32 CUDA tensors shaped like the weights (None entries skip a matrix), or None."""
        if deltas is None:
            _check(self.lib.apollo_set_delta_out(self.ctx, None), "apollo_set_delta_out")
            self._delta = None
            return
        arr = (ctypes.c_void_p * len(self.shapes))()
        for i, d in enumerate(deltas):
            if d is None:
                arr[i] = None
                continue
            assert d.is_cuda and d.dtype == torch.float32 and tuple(d.shape) == self.shapes[i] and d.is_contiguous()
            arr[i] = d.data_ptr()
        _check(self.lib.apollo_set_delta_out(self.ctx, arr), "apollo_set_delta_out")
        self._delta = deltas

    def scales(self, mat: int, stream=None) -> torch.Tensor:
        out = torch.empty(max(self.shapes[mat]), dtype=torch.float32, device=self.device)
        _check(self.lib.apollo_get_scales(self.ctx, mat, out.data_ptr(), _stream_ptr(stream)), "apollo_get_scales")
        return out

    def limiter(self, mat: int, stream=None) -> torch.Tensor:
        out = torch.empty(4, dtype=torch.float32, device=self.device)
        _check(self.lib.apollo_get_limiter(self.ctx, mat, out.data_ptr(), _stream_ptr(stream)), "apollo_get_limiter")
        return out

    def state(self, mat: int, stream=None):
        n = max(self.shapes[mat])
        M = torch.empty((self.cfg.rank, n), dtype=torch.float32, device=self.device)
        V = torch.empty_like(M)
        _check(self.lib.apollo_get_state(self.ctx, mat, M.data_ptr(), V.data_ptr(), _stream_ptr(stream)),
               "apollo_get_state")
        return M, V

    def status(self, stream=None) -> int:
        return self.lib.apollo_status(self.ctx, _stream_ptr(stream))

    def selftest_bounded_wait(self, stream=None):
        """Launches the kernel whose only wait runs out; the next status() then reports ERR_TIMEOUT."""
        _check(self.lib.apollo_selftest_bounded_wait(self.ctx, _stream_ptr(stream)), "apollo_selftest_bounded_wait")

    def path(self, mat: int) -> int:
        out = ctypes.c_int32(-1)
        _check(self.lib.apollo_get_path(self.ctx, mat, ctypes.byref(out)), "apollo_get_path")
        return out.value

    def step_count(self) -> int:
        out = ctypes.c_int64(0)
        _check(self.lib.apollo_step_count(self.ctx, ctypes.byref(out)), "apollo_step_count")
        return out.value

    def state_export(self, stream=None) -> torch.Tensor:
        """The optimizer state (moments and limiter norms) as one flat uint8 CUDA tensor."""
        n = ctypes.c_size_t(0)
        _check(self.lib.apollo_state_bytes(self.ctx, ctypes.byref(n)), "apollo_state_bytes")
        out = torch.empty(n.value, dtype=torch.uint8, device=self.device)
        _check(self.lib.apollo_state_export(self.ctx, out.data_ptr(), _stream_ptr(stream)), "apollo_state_export")
        return out

    def state_import(self, flat: torch.Tensor, step_count: int, stream=None):
        n = ctypes.c_size_t(0)
        _check(self.lib.apollo_state_bytes(self.ctx, ctypes.byref(n)), "apollo_state_bytes")
        assert flat.is_cuda and flat.dtype == torch.uint8 and flat.numel() == n.value and flat.is_contiguous()
        _check(self.lib.apollo_state_import(self.ctx, flat.data_ptr(), step_count, _stream_ptr(stream)),
               "apollo_state_import")

    def set_timing(self, on: bool):
        _check(self.lib.apollo_set_timing(self.ctx, int(on)), "apollo_set_timing")

    def timing(self, steps_back: int = 0):
        """{projection, finalize, update, whole step} of a recent step, in milliseconds."""
        out = (ctypes.c_float * 4)()
        _check(self.lib.apollo_get_timing(self.ctx, steps_back, out), "apollo_get_timing")
        return list(out)

    def last_launches(self) -> int:
        out = ctypes.c_int32(0)
        _check(self.lib.apollo_last_launches(self.ctx, ctypes.byref(out)), "apollo_last_launches")
        return out.value

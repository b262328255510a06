"""Thin ctypes binding of ``libbct_b200.so`` with the names of ``include/bct.h``.

Argument marshalling only: every step of the path runs in the library's CUDA kernels.
PyTorch supplies device memory (the workspace and the step tensors) and the stream.
There is no CPU fallback: ``load()`` raises when the library has not been built.
"""
from __future__ import annotations

import ctypes
import functools
import operator
import os
from typing import Optional, Tuple

import torch

BCT_OK, BCT_ERR_INVALID_ARG, BCT_ERR_UNSUPPORTED, BCT_ERR_STATE, BCT_ERR_CUDA, BCT_ERR_TIMEOUT = range(6)
BCT_F32, BCT_BF16, BCT_BF16_PAIR = 0, 1, 2
FLAG_SKIP_FIRST_WRITE, FLAG_WRITE_THEN_READ, FLAG_DENSE_WRITE, FLAG_OUT_F32, FLAG_PRECISE_READ, FLAG_CUDA_CORES = 1, 2, 4, 8, 16, 32

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libbct_b200.so")

EXPORTS = (
    "bct_version", "bct_last_error", "bct_cache_bytes", "bct_cache_create", "bct_decode_step",
    "bct_prefill_stream", "bct_decode_step_host", "bct_prefill_stream_host", "bct_cache_len",
    "bct_cache_export", "bct_cache_import", "bct_cache_status", "bct_cache_launches", "bct_cache_destroy",
    "bct_cache_tensor_path", "bct_prefill_stream_host_static", "bct_decode_step_eta", "bct_prefill_stream_eta",
    "bct_project_qkv", "bct_layer_scratch_bytes", "bct_layer_forward", "bct_update_kv",
    "bct_cache_status_clear", "bct_cache_rows_rewritten", "bct_selftest_timeout",
    "bct_update_kv_backward", "bct_stack_scratch_bytes", "bct_stack_forward",
    "bct_linear_scratch_bytes", "bct_linear_step", "bct_linear_forward", "bct_linear_backward",
    "bct_norm_rotate", "bct_norm_rotate_scratch_bytes", "bct_norm_rotate_backward",
    "bct_qcache_append", "bct_qcache_attend_scratch_bytes", "bct_qcache_attend",
    "bct_qcache_evict_scratch_bytes", "bct_qcache_evict",
)
ROTATE_INTERLEAVED = 1
QCACHE_BLOCK = 32   # slots of an 8-bit cache that share a scale
STATIC_STAGE_BYTES = 8 << 20


class BctParams(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("capacity", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("read_scale", ctypes.c_float), ("write_scale", ctypes.c_float), ("init_len", ctypes.c_int32),
        ("flags", ctypes.c_uint32), ("write_eps", ctypes.c_float), ("max_stream", ctypes.c_int32),
    ]


class BctLinearParams(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float),
    ]


class BctError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("bct status %d: %s" % (status, message))
        self.status = status


class BctQcache(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("capacity", ctypes.c_int32),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
        ("weight", ctypes.c_void_p), ("position", ctypes.c_void_p), ("state", ctypes.c_void_p),
    ]


_lib = None


def load() -> ctypes.CDLL:
    """Open the C-ABI library; raise if it is missing (build it with ``python -m paper_2411_15785_b200.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("%s not found: run `python -m paper_2411_15785_b200.build` (no CPU fallback exists)" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    pp = ctypes.POINTER(BctParams)
    lib.bct_version.restype = i32
    lib.bct_version.argtypes = []
    lib.bct_last_error.restype = ctypes.c_char_p
    lib.bct_last_error.argtypes = []
    lib.bct_cache_bytes.argtypes = [pp, ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(ctypes.c_size_t)]
    lib.bct_cache_create.argtypes = [pp, vp, ctypes.c_size_t, vp, vp, vp, ctypes.POINTER(vp)]
    lib.bct_decode_step.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.bct_prefill_stream.argtypes = [vp, vp, vp, vp, vp, i64, vp]
    lib.bct_decode_step_eta.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.bct_prefill_stream_eta.argtypes = [vp, vp, vp, vp, vp, vp, i64, vp]
    lib.bct_update_kv.argtypes = [vp, vp, vp, vp, i64, vp]
    lib.bct_project_qkv.argtypes = [i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.bct_layer_scratch_bytes.argtypes = [vp, i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.bct_layer_forward.argtypes = [vp, vp, vp, vp, vp, i32, vp, vp, ctypes.c_size_t, vp, i64, vp]
    lib.bct_decode_step_host.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.bct_prefill_stream_host.argtypes = [vp, vp, vp, vp, vp, i64, vp]
    lib.bct_cache_len.argtypes = [vp, ctypes.POINTER(i32)]
    lib.bct_cache_export.argtypes = [vp, vp, vp, i32, vp]
    lib.bct_cache_import.argtypes = [vp, vp, vp, i32, i32, vp]
    lib.bct_cache_status.argtypes = [vp, vp]
    lib.bct_cache_launches.argtypes = [vp, ctypes.POINTER(i64)]
    lib.bct_cache_destroy.argtypes = [vp]
    lib.bct_cache_tensor_path.argtypes = [vp, ctypes.POINTER(i32)]
    lib.bct_prefill_stream_host_static.argtypes = [vp, vp, vp, vp, vp, i64, vp]
    lib.bct_cache_status_clear.argtypes = [vp, vp]
    lib.bct_cache_rows_rewritten.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_uint64)]
    lib.bct_selftest_timeout.argtypes = [vp, vp]
    lib.bct_update_kv_backward.argtypes = [vp, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp]
    lib.bct_stack_scratch_bytes.argtypes = [ctypes.POINTER(vp), i32, i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.bct_stack_forward.argtypes = [ctypes.POINTER(vp), i32, vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                      ctypes.POINTER(vp), vp, ctypes.c_size_t, vp, i64, vp]
    pl, sz, f32, u32 = ctypes.POINTER(BctLinearParams), ctypes.c_size_t, ctypes.c_float, ctypes.c_uint32
    lib.bct_linear_scratch_bytes.argtypes = [pl, i64, i32, ctypes.POINTER(sz)]
    lib.bct_linear_step.argtypes = [pl, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.bct_linear_forward.argtypes = [pl, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.bct_linear_backward.argtypes = [pl, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.bct_norm_rotate.argtypes = [i64, i32, i32, i32, i32, vp, vp, vp, vp, f32, vp, vp, i32, u32, vp, vp, vp]
    lib.bct_norm_rotate_scratch_bytes.argtypes = [i64, i32, ctypes.POINTER(sz)]
    lib.bct_norm_rotate_backward.argtypes = [i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, f32, vp, vp, i32, u32,
                                             vp, vp, vp, vp, vp, sz, vp]
    pq = ctypes.POINTER(BctQcache)
    lib.bct_qcache_append.argtypes = [pq, i64, i32, vp, vp, vp, vp]
    lib.bct_qcache_attend_scratch_bytes.argtypes = [pq, i64, i32, i32, i32, ctypes.POINTER(sz)]
    lib.bct_qcache_attend.argtypes = [pq, i64, i32, i32, vp, vp, f32, f32, i32, vp, vp, sz, vp]
    lib.bct_qcache_evict_scratch_bytes.argtypes = [pq, i32, ctypes.POINTER(sz)]
    lib.bct_qcache_evict.argtypes = [pq, i32, i32, vp, sz, vp]
    for name in EXPORTS[2:]:
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


def last_error() -> str:
    return load().bct_last_error().decode()


def _check(status: int) -> None:
    if status != BCT_OK:
        raise BctError(status, last_error())


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.int32:  # checkpoint words: value-plane bits << 16 | residual-plane bits
        return BCT_BF16_PAIR
    if dt == torch.float32:
        return BCT_F32
    if dt == torch.bfloat16:
        return BCT_BF16
    raise ValueError("dtype must be torch.float32 or torch.bfloat16")


def make_params(batch, n_q_heads, n_kv_heads, head_dim, capacity, dtype, *, read_scale=0.0, write_scale=0.0,
                init_len=0, flags=0, write_eps=0.0, max_stream=1) -> BctParams:
    return BctParams(batch, n_q_heads, n_kv_heads, head_dim, capacity, _dtype_code(dtype), read_scale,
                     write_scale, init_len, flags, write_eps, max_stream)


def cache_bytes(params: BctParams) -> Tuple[int, int]:
    b, a = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(load().bct_cache_bytes(ctypes.byref(params), ctypes.byref(b), ctypes.byref(a)))
    return b.value, a.value


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


def _check_eta(eta: torch.Tensor, shape) -> None:
    if eta.dtype != torch.float32 or tuple(eta.shape) != tuple(shape) or not eta.is_contiguous() or not eta.is_cuda:
        raise ValueError("eta must be a contiguous float32 device tensor of shape %s" % (tuple(shape),))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def project_qkv(x, w_q, w_wq, w_wv, stream=None, out=None):
    """q = x W_q^T, k = x W_wq^T, v = x W_wv^T: x ``[..., d_model]`` bfloat16 on the device, weights
    ``[features, d_model]``; returns q ``[..., n_q]``, k, v ``[..., n_kv]`` (bfloat16)."""
    lib = load()
    d_model = x.shape[-1]
    n_tokens = x.numel() // d_model
    for t in (x, w_q, w_wq, w_wv):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous():
            raise ValueError("x and the weights must be contiguous bfloat16 device tensors")
    n_q, n_kv = w_q.shape[0], w_wq.shape[0]
    if out is not None:   # (q, k, v) tensors to write into
        q, k, v = out
    else:
        q = torch.empty(x.shape[:-1] + (n_q,), dtype=torch.bfloat16, device=x.device)
        k = torch.empty(x.shape[:-1] + (n_kv,), dtype=torch.bfloat16, device=x.device)
        v = torch.empty_like(k)
    _check(lib.bct_project_qkv(n_tokens, d_model, n_q, n_kv, x.data_ptr(), w_q.data_ptr(), w_wq.data_ptr(),
                               w_wv.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), _stream_ptr(stream)))
    return q, k, v


def stack_forward(caches, x, w_q, w_wq, w_wv, out=None, scratch=None, stream=None):
    """A stack of layers: layer 0 reads x ``[B, T, d_model]``, layer l > 0 the outputs of layer l - 1 as its
    tokens.  caches: list of Cache; w_q, w_wq, w_wv: lists of that layer's weights.  Returns the last layer's
    outputs ``[B, T, Hq, d]``."""
    lib = load()
    n = len(caches)
    T = x.shape[1]
    arr = lambda ptrs: (ctypes.c_void_p * n)(*ptrs)
    hs = arr([c._h.value for c in caches])
    need = ctypes.c_size_t(0)
    _check(lib.bct_stack_scratch_bytes(hs, n, T, ctypes.byref(need)))
    if scratch is None:
        scratch = torch.empty(max(need.value, 256), dtype=torch.uint8, device=x.device)
    last = caches[-1]
    if out is None:
        out = torch.empty((last.B, T, last.Hq, last.d), dtype=torch.bfloat16, device=x.device)
    _check(lib.bct_stack_forward(hs, n, x.data_ptr(), x.shape[2], arr([w.data_ptr() for w in w_q]),
                                 arr([w.data_ptr() for w in w_wq]), arr([w.data_ptr() for w in w_wv]), scratch.data_ptr(),
                                 scratch.numel(), out.data_ptr(), T, _stream_ptr(stream)))
    return out


def _operand(name, t, shape, dtype, dev) -> None:
    """The library sees pointers only: shape, type, place (device index) and layout are checked here."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or dev < 0 or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on CUDA device %s (got %s, %s, %s%s)" % (
            name, dtype, tuple(shape), dev if dev >= 0 else "0 or above", t.dtype, tuple(t.shape), t.device,
            "" if t.is_contiguous() else ", strided"))


def _result(name, t, like, shape, dtype, dev):
    """The caller's buffer, checked, or a new one on the device of `like`."""
    if t is None:
        if like.dtype is dtype and like.shape == shape:
            return torch.empty_like(like)
        return like.new_empty(shape, dtype=dtype)
    _operand(name, t, shape, dtype, dev)
    return t


def _raw_stream(dev: int) -> int:
    return torch.cuda.current_stream(dev).cuda_stream


# the same without building a Stream object (3 us of a call that takes 10), where this torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)


def _on_stream(stream, call, *args):
    """`call` with `stream` as the current one: what it allocates (results, scratch) then belongs to that stream, and
    freeing it cannot hand it to work of another stream that runs beside the call's kernels."""
    if stream.device.index != args[0].get_device():
        raise ValueError("stream is on %s, the tensors are on %s" % (stream.device, args[0].device))
    with torch.cuda.stream(stream):
        return call(*args)


def _launch(dev, call, *args) -> None:
    """The call on the tensors' device and that device's current stream."""
    raw = _raw_stream(dev)
    if dev == torch.cuda.current_device():
        st = call(*args, raw)
    else:
        with torch.cuda.device(dev):
            st = call(*args, raw)
    if st != BCT_OK:
        _check(st)


@functools.lru_cache(maxsize=256)
def _linear_params(batch, n_q_heads, n_kv_heads, head_dim, dtype, scale):
    """The parameter block of a call's sizes (never written to) and a reference to hand it over by."""
    p = BctLinearParams(batch, n_q_heads, n_kv_heads, head_dim, dtype, scale)
    return p, ctypes.byref(p)


@functools.lru_cache(maxsize=1024)
def _linear_scratch(batch, n_q_heads, n_kv_heads, head_dim, dtype, T, backward) -> int:
    n = ctypes.c_size_t(0)
    _check(load().bct_linear_scratch_bytes(_linear_params(batch, n_q_heads, n_kv_heads, head_dim, dtype, 0.0)[1], T,
                                           backward, ctypes.byref(n)))
    return n.value


def _scratch(need: int, scratch, like, dev):
    if scratch is None:
        return like.new_empty(need, dtype=torch.uint8) if need else None
    if scratch.get_device() != dev or not scratch.is_contiguous():
        raise ValueError("scratch must be a contiguous tensor on CUDA device %d" % dev)
    return scratch


def _scratch_args(scratch):
    return (None, 0) if scratch is None else (scratch.data_ptr(), scratch.numel() * scratch.element_size())


@functools.lru_cache(maxsize=1024)
def _linear_sizes(q_shape, k_shape, dtype, n_lead, scale):
    """What follows from the shapes alone: (sizes, parameters by reference, k's shape, the decays', the state's)."""
    if len(q_shape) != n_lead + 2 or len(k_shape) != n_lead + 2:
        raise ValueError("q and k must have %d dimensions" % (n_lead + 2))
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("q must be float32 or bfloat16 (got %s)" % dtype)
    Hkv, d = k_shape[-2], q_shape[-1]
    sizes = (q_shape[0], q_shape[-2], Hkv, d, BCT_BF16 if dtype is torch.bfloat16 else BCT_F32)
    return (sizes, _linear_params(*sizes, scale)[1], torch.Size((*q_shape[:-2], Hkv, d)), torch.Size((Hkv,)),
            torch.Size((q_shape[0], Hkv, d, d)))


def _linear_setup(q, k, v, log_decay, n_lead, scale):
    """Checks the operands that every linear-attention call has: q ``[*lead, Hq, d]``, k and v ``[*lead, Hkv, d]``.
    Returns the sizes, the parameters by reference, the state's shape and the device index."""
    dt, dev = q.dtype, q.get_device()
    # (float(): the sizes are kept under what they follow from, and a tensor or an array may have changed since)
    sizes, p, kv, hk, s_shape = _linear_sizes(q.shape, k.shape, dt, n_lead, float(scale))
    if not (dev >= 0 and k.shape == kv and v.shape == kv and k.dtype is dt and v.dtype is dt and log_decay.shape == hk
            and log_decay.dtype is torch.float32 and k.get_device() == dev and v.get_device() == dev
            and log_decay.get_device() == dev and q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
            and log_decay.is_contiguous()):
        _operand("q", q, q.shape, dt, dev)      # one of these says what it is
        _operand("k", k, kv, dt, dev)
        _operand("v", v, kv, dt, dev)
        _operand("log_decay", log_decay, hk, torch.float32, dev)
    return sizes, p, s_shape, dev


def linear_scratch_bytes(batch, T, n_q_heads, n_kv_heads, head_dim, dtype, *, backward=False, want_d_state=True) -> int:
    """Scratch that linear_forward (or linear_backward, with or without the state's gradient) needs for these sizes."""
    batch, T, n_q_heads, n_kv_heads, head_dim = map(operator.index, (batch, T, n_q_heads, n_kv_heads, head_dim))
    return _linear_scratch(batch, n_q_heads, n_kv_heads, head_dim, _dtype_code(dtype), T,
                           0 if not backward else (1 if want_d_state else 2))


def linear_step(q, k, v, log_decay, state, scale=0.0, out=None, state_out=None, stream=None):
    """Linear attention with a decay for each head, one token per sequence: ``S' = exp(log_decay) S + k^T v``,
    ``out = scale q S'``.  q ``[B, Hq, d]``, k, v ``[B, Hkv, d]``, state ``[B, Hkv, d, d]`` float32.  state_out: where
    S' goes; None updates `state` in place.  Returns (out, state after)."""
    if stream is not None:
        return _on_stream(stream, linear_step, q, k, v, log_decay, state, scale, out, state_out)
    lib = load()
    _, p, s_shape, dev = _linear_setup(q, k, v, log_decay, 1, scale)
    _operand("state", state, s_shape, torch.float32, dev)
    out = torch.empty_like(q) if out is None else _result("out", out, q, q.shape, q.dtype, dev)
    if state_out is None:
        state_out = state
    else:
        _operand("state_out", state_out, s_shape, torch.float32, dev)
    _launch(dev, lib.bct_linear_step, p, q.data_ptr(), k.data_ptr(), v.data_ptr(),
            log_decay.data_ptr(), state.data_ptr(), state_out.data_ptr(), out.data_ptr())
    return out, state_out


def linear_forward(q, k, v, log_decay, state=None, lens=None, scale=0.0, out=None, state_out=None, scratch=None,
                   stream=None):
    """T tokens per sequence: q ``[B, T, Hq, d]``, k, v ``[B, T, Hkv, d]``; state ``[B, Hkv, d, d]`` float32 or None
    (zeros); lens int32 ``[B]`` or None: the valid tokens of each sequence of a padded batch.  Returns (out
    ``[B, T, Hq, d]``, state after each sequence's last token); state_out may be `state`."""
    if stream is not None:
        return _on_stream(stream, linear_forward, q, k, v, log_decay, state, lens, scale, out, state_out, scratch)
    lib = load()
    sizes, p, s_shape, dev = _linear_setup(q, k, v, log_decay, 2, scale)
    T = q.shape[1]
    if state is not None:
        _operand("state", state, s_shape, torch.float32, dev)
    if lens is not None:
        _operand("lens", lens, q.shape[:1], torch.int32, dev)
    out = torch.empty_like(q) if out is None else _result("out", out, q, q.shape, q.dtype, dev)
    if state_out is None:
        state_out = q.new_empty(s_shape, dtype=torch.float32) if state is None else torch.empty_like(state)
    else:
        _operand("state_out", state_out, s_shape, torch.float32, dev)
    scratch = _scratch(_linear_scratch(*sizes, T, 0), scratch, q, dev)
    _launch(dev, lib.bct_linear_forward, p, T, q.data_ptr(), k.data_ptr(), v.data_ptr(),
            log_decay.data_ptr(), _ptr(lens), _ptr(state), state_out.data_ptr(), out.data_ptr(), *_scratch_args(scratch))
    return out, state_out


def linear_backward(d_out, q, k, v, log_decay, state=None, d_state=None, lens=None, scale=0.0, out=None, scratch=None,
                    stream=None, want_d_state=True):
    """Backward of linear_forward: d_out ``[B, T, Hq, d]`` and d_state ``[B, Hkv, d, d]`` float32 (the gradient of the
    state after the last token, or None) -> (d_q, d_k, d_v in q's dtype, d_state_in float32 or None).  out: that tuple,
    to write into."""
    if stream is not None:
        return _on_stream(stream, linear_backward, d_out, q, k, v, log_decay, state, d_state, lens, scale, out, scratch,
                          None, want_d_state)
    lib = load()
    sizes, p, s_shape, dev = _linear_setup(q, k, v, log_decay, 2, scale)
    T = q.shape[1]
    _operand("d_out", d_out, q.shape, q.dtype, dev)
    for name, t in (("state", state), ("d_state", d_state)):
        if t is not None:
            _operand(name, t, s_shape, torch.float32, dev)
    if lens is not None:
        _operand("lens", lens, q.shape[:1], torch.int32, dev)
    given = (None,) * 4 if out is None else out
    d_q = _result("d_q", given[0], q, q.shape, q.dtype, dev)
    d_k = _result("d_k", given[1], q, k.shape, q.dtype, dev)
    d_v = _result("d_v", given[2], q, v.shape, q.dtype, dev)
    d_in = _result("d_state_in", given[3], q, s_shape, torch.float32, dev) if want_d_state else None
    scratch = _scratch(_linear_scratch(*sizes, T, 1 if want_d_state else 2), scratch, q, dev)
    _launch(dev, lib.bct_linear_backward, p, T, d_out.data_ptr(), q.data_ptr(), k.data_ptr(),
            v.data_ptr(), log_decay.data_ptr(), _ptr(lens), _ptr(state), _ptr(d_state), d_q.data_ptr(), d_k.data_ptr(),
            d_v.data_ptr(), _ptr(d_in), *_scratch_args(scratch))
    return d_q, d_k, d_v, d_in


@functools.lru_cache(maxsize=1024)
def _norm_rotate_sizes(q_shape, k_shape, dtype, half):
    """What follows from the shapes alone: (tokens, Hq, Hkv, d, dtype code, rotated features), k's shape, the tokens'."""
    if len(q_shape) < 3 or len(k_shape) != len(q_shape):
        raise ValueError("q and k must be [..., heads, head_dim] with at least one token dimension")
    if dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("q must be float32 or bfloat16 (got %s)" % dtype)
    lead, d, n = q_shape[:-2], q_shape[-1], 1
    for x in lead:
        n *= x
    sizes = (n, q_shape[-2], k_shape[-2], d, BCT_BF16 if dtype is torch.bfloat16 else BCT_F32, 2 * half)
    return sizes, torch.Size((*lead, k_shape[-2], d)), torch.Size(lead), torch.Size((d,))


def _norm_rotate_setup(q, k, w_q, w_k, positions, freq):
    dt, dev = q.dtype, q.get_device()
    half = 0 if freq is None else freq.numel()
    sizes, ks, lead, wd = _norm_rotate_sizes(q.shape, k.shape, dt, half)
    if half and positions is None:
        raise ValueError("positions are needed where freq is given")
    if not (dev >= 0 and k.shape == ks and k.dtype is dt and k.get_device() == dev and q.is_contiguous() and k.is_contiguous()
            and (w_q is None or (w_q.shape == wd and w_q.dtype is dt and w_q.get_device() == dev and w_q.is_contiguous()))
            and (w_k is None or (w_k.shape == wd and w_k.dtype is dt and w_k.get_device() == dev and w_k.is_contiguous()))
            and (not half or (positions.shape == lead and positions.dtype is torch.int64 and positions.get_device() == dev
                              and positions.is_contiguous() and freq.dim() == 1 and freq.dtype is torch.float64
                              and freq.get_device() == dev and freq.is_contiguous()))):
        _operand("q", q, q.shape, dt, dev)      # one of these says what it is
        _operand("k", k, ks, dt, dev)
        for name, w in (("w_q", w_q), ("w_k", w_k)):
            if w is not None:
                _operand(name, w, wd, dt, dev)
        if half:
            _operand("freq", freq, (half,), torch.float64, dev)
            _operand("positions", positions, lead, torch.int64, dev)
    return sizes


def norm_rotate(q, k, w_q, w_k, positions, freq, eps=1e-6, interleaved=False, out=None, stream=None):
    """Norm of every head of q ``[..., Hq, d]`` and k ``[..., Hkv, d]`` with the weights w_q, w_k ``[d]`` (None: ones),
    and the rotation of their first ``2 len(freq)`` features by ``positions * freq``: positions int64 ``[...]``, freq
    float64, radians per position (None: norm only).  interleaved: neighbouring features are the pairs, instead of
    those half the rotated part away.  out: (q, k) to write into, which may be the inputs.  Returns (q, k)."""
    if stream is not None:
        return _on_stream(stream, norm_rotate, q, k, w_q, w_k, positions, freq, eps, interleaved, out)
    lib = load()
    n, Hq, Hkv, d, dt, rot = _norm_rotate_setup(q, k, w_q, w_k, positions, freq)
    dev = q.get_device()
    if out is None:
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    else:
        q_out, k_out = out
        _operand("q_out", q_out, q.shape, q.dtype, dev)
        _operand("k_out", k_out, k.shape, q.dtype, dev)
    _launch(dev, lib.bct_norm_rotate, n, Hq, Hkv, d, dt, q.data_ptr(), k.data_ptr(), _ptr(w_q), _ptr(w_k), eps,
            _ptr(positions) if rot else None, _ptr(freq) if rot else None, rot, ROTATE_INTERLEAVED if interleaved else 0,
            q_out.data_ptr(), k_out.data_ptr())
    return q_out, k_out


def norm_rotate_backward(d_q_out, d_k_out, q, k, w_q, w_k, positions, freq, eps=1e-6, interleaved=False, want_d_w=True,
                         out=None, scratch=None, stream=None):
    """Backward of norm_rotate, given the gradients of its two results and its inputs -> (d_q, d_k in q's dtype, d_w_q,
    d_w_k float32 or None).  out: that tuple, to write into (d_q may be d_q_out, d_k may be d_k_out)."""
    if stream is not None:
        return _on_stream(stream, norm_rotate_backward, d_q_out, d_k_out, q, k, w_q, w_k, positions, freq, eps, interleaved,
                          want_d_w, out, scratch)
    lib = load()
    n, Hq, Hkv, d, dt, rot = _norm_rotate_setup(q, k, w_q, w_k, positions, freq)
    dev = q.get_device()
    _operand("d_q_out", d_q_out, q.shape, q.dtype, dev)
    _operand("d_k_out", d_k_out, k.shape, q.dtype, dev)
    given = (None,) * 4 if out is None else out
    d_q = _result("d_q", given[0], q, q.shape, q.dtype, dev)
    d_k = _result("d_k", given[1], q, k.shape, q.dtype, dev)
    d_w_q = _result("d_w_q", given[2], q, (d,), torch.float32, dev) if want_d_w else None
    d_w_k = _result("d_w_k", given[3], q, (d,), torch.float32, dev) if want_d_w else None
    if want_d_w:
        need = ctypes.c_size_t(0)
        _check(lib.bct_norm_rotate_scratch_bytes(n, d, ctypes.byref(need)))
        scratch = _scratch(need.value, scratch, q, dev)
    else:
        scratch = None
    _launch(dev, lib.bct_norm_rotate_backward, n, Hq, Hkv, d, dt, d_q_out.data_ptr(), d_k_out.data_ptr(),
            q.data_ptr(), k.data_ptr(), _ptr(w_q), _ptr(w_k), eps, _ptr(positions) if rot else None,
            _ptr(freq) if rot else None, rot, ROTATE_INTERLEAVED if interleaved else 0, d_q.data_ptr(), d_k.data_ptr(),
            _ptr(d_w_q), _ptr(d_w_k), *_scratch_args(scratch))
    return d_q, d_k, d_w_q, d_w_k


class QuantCache:
    """A cache of predefined capacity in 8 bits, with a scale per block of 32 slots and head, which throws out the slots
    that attention has used least.  Its planes are ordinary tensors:

    ``k``, ``v`` int8 ``[B, Hkv, C, d]``; ``k_scale``, ``v_scale`` float32 ``[B, Hkv, ceil(C / 32)]``; ``weight`` float32 and
    ``position`` int32 ``[B, Hkv, C]``; ``state`` int32 ``[3, B]``: the slots held, the tokens seen, a word of the library's.

    planes: that tuple, in this order, to go on with a cache that exists; None makes an empty one.  Calls on one cache
    belong on one stream, or on streams that wait for one another.
    """

    def __init__(self, batch, n_kv_heads, head_dim, capacity, device="cuda", planes=None):
        self.B, self.Hkv, self.d, self.C = map(operator.index, (batch, n_kv_heads, head_dim, capacity))
        lib = self._lib = load()
        slots, blocks = (self.B, self.Hkv, self.C), (self.B, self.Hkv, -(-self.C // QCACHE_BLOCK))
        kinds = (("k", (*slots, self.d), torch.int8), ("v", (*slots, self.d), torch.int8), ("k_scale", blocks, torch.float32),
                 ("v_scale", blocks, torch.float32), ("weight", slots, torch.float32), ("position", slots, torch.int32),
                 ("state", (3, self.B), torch.int32))
        need = ctypes.c_size_t(0)     # refuses sizes that the library does not have, before memory is taken
        _check(lib.bct_qcache_evict_scratch_bytes(ctypes.byref(BctQcache(self.B, self.Hkv, self.d, self.C)), 0, ctypes.byref(need)))
        if planes is None:
            planes = [torch.zeros(shape, dtype=dt, device=device) for _, shape, dt in kinds]
            if not planes[0].is_cuda:
                raise ValueError("device must be a CUDA device (got %s)" % planes[0].device)
        elif len(planes) != len(kinds):
            raise ValueError("planes must be (%s)" % ", ".join(name for name, _, _ in kinds))
        self.dev = planes[0].get_device()
        for (name, shape, dt), t in zip(kinds, planes):
            _operand(name, t, torch.Size(shape), dt, self.dev)
        self.k, self.v, self.k_scale, self.v_scale, self.weight, self.position, self.state = planes
        self._planes = tuple(planes)   # the library has their addresses
        self._c = BctQcache(self.B, self.Hkv, self.d, self.C, *(t.data_ptr() for t in planes))
        self._p = ctypes.byref(self._c)
        self._known = {}              # sizes of the last calls, by the shapes that they follow from

    @property
    def held(self) -> torch.Tensor:
        """Slots held by each sequence, int32 ``[B]`` on the device."""
        return self.state[0]

    @property
    def seen(self) -> torch.Tensor:
        """Tokens appended to each sequence so far, int32 ``[B]`` on the device."""
        return self.state[1]

    def _know(self, key, sizes):
        if len(self._known) >= 64:
            self._known.clear()
        self._known[key] = sizes
        return sizes

    def _sizes(self, name, x, heads):
        """(T, dtype code) of x ``[B, T, heads, d]``."""
        if x.dim() != 4 or x.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("%s must be float32 or bfloat16 [B, T, heads, head_dim] (got %s, %s)" % (name, x.dtype, tuple(x.shape)))
        _operand(name, x, torch.Size((self.B, x.shape[1], heads, self.d)), x.dtype, self.dev)
        return x.shape[1], BCT_BF16 if x.dtype is torch.bfloat16 else BCT_F32

    def _lens(self, lens):
        _operand("lens", lens, torch.Size((self.B,)), torch.int32, self.dev)
        return lens.data_ptr()

    def append(self, k, v, lens=None, stream=None) -> None:
        """k, v ``[B, T, Hkv, d]`` float32 or bfloat16 go behind the slots held; lens int32 ``[B]`` or None (all T): the
        valid tokens of each sequence of a padded batch.  Tokens that find no slot free are dropped: evict first."""
        if stream is not None:
            return _on_stream(stream, lambda k_: self.append(k_, v, lens), k)
        dt, shape = k.dtype, k.shape
        sizes = self._known.get((shape, dt))     # what follows from the shape alone
        if sizes is None:
            sizes = self._know((shape, dt), self._sizes("k", k, self.Hkv))
        if not (k.get_device() == self.dev and v.get_device() == self.dev and v.shape == shape and v.dtype is dt
                and k.is_contiguous() and v.is_contiguous()):
            _operand("k", k, shape, dt, self.dev)      # one of these says what it is
            _operand("v", v, shape, dt, self.dev)
        _launch(self.dev, self._lib.bct_qcache_append, self._p, *sizes, k.data_ptr(), v.data_ptr(),
                None if lens is None else self._lens(lens))

    def attend(self, q, lens=None, scale=0.0, score_cap=0.0, accumulate=True, out=None, scratch=None, stream=None):
        """Attention of the last T tokens appended to each sequence, q ``[B, T, Hq, d]``, each over the slots up to its
        own; lens as in append.  scale <= 0: 1/sqrt(d).  score_cap > 0: scores are ``score_cap tanh(s / score_cap)``.
        accumulate: adds what each slot was given to ``weight`` (NaN, to all that a row sees, if the row's query has a NaN).
        Returns out ``[B, T, Hq, d]``."""
        if stream is not None:
            return _on_stream(stream, lambda q_: self.attend(q_, lens, scale, score_cap, accumulate, out, scratch), q)
        accumulate = 1 if accumulate else 0
        key = (q.shape, q.dtype, accumulate)
        known = self._known.get(key)
        if known is None:
            Hq = q.shape[2] if q.dim() == 4 else 0
            T, dt = self._sizes("q", q, Hq)
            n = ctypes.c_size_t(0)
            _check(self._lib.bct_qcache_attend_scratch_bytes(self._p, T, Hq, dt, accumulate, ctypes.byref(n)))
            known = self._know(key, (T, Hq, dt, n.value))
        T, Hq, dt, need = known
        if q.get_device() != self.dev or not q.is_contiguous():
            _operand("q", q, q.shape, q.dtype, self.dev)
        if out is None:
            out = torch.empty_like(q)
        else:
            _operand("out", out, q.shape, q.dtype, self.dev)
        scratch = _scratch(need, scratch, q, self.dev)
        _launch(self.dev, self._lib.bct_qcache_attend, self._p, T, Hq, dt, q.data_ptr(),
                None if lens is None else self._lens(lens), scale, score_cap, accumulate, out.data_ptr(), *_scratch_args(scratch))
        return out

    def evict(self, keep, recent=0, scratch=None, stream=None) -> None:
        """Every head of every sequence that holds more than `keep` slots gives up those of the least ``weight``, but none
        of the last `recent` tokens; slots behind the new end move into the places that have become free."""
        if stream is not None:
            return _on_stream(stream, lambda k_: self.evict(keep, recent, scratch), self.k)
        keep, recent = operator.index(keep), operator.index(recent)
        need = self._known.get(keep)
        if need is None:
            n = ctypes.c_size_t(0)
            _check(self._lib.bct_qcache_evict_scratch_bytes(self._p, keep, ctypes.byref(n)))
            need = self._know(keep, n.value)
        scratch = _scratch(need, scratch, self.k, self.dev)
        _launch(self.dev, self._lib.bct_qcache_evict, self._p, keep, recent, *_scratch_args(scratch))


class Cache:
    """A bounded cache over a torch-allocated workspace.  Methods map 1:1 to the C calls."""

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, capacity, dtype=torch.bfloat16, *,
                 read_scale=0.0, write_scale=0.0, init_len=0, flags=0, write_eps=0.0, max_stream=1,
                 mk_init: Optional[torch.Tensor] = None, mv_init: Optional[torch.Tensor] = None,
                 device="cuda", stream=None, guard_bytes: int = 0):
        self.lib = load()
        self.params = make_params(batch, n_q_heads, n_kv_heads, head_dim, capacity, dtype,
                                  read_scale=read_scale, write_scale=write_scale, init_len=init_len,
                                  flags=flags, write_eps=write_eps, max_stream=max_stream)
        self.dtype = dtype
        self.out_dtype = torch.float32 if (flags & FLAG_OUT_F32) else dtype
        self.device = torch.device(device)
        self.B, self.Hq, self.Hkv, self.d, self.C = batch, n_q_heads, n_kv_heads, head_dim, capacity
        nbytes, align = cache_bytes(self.params)
        # guard_bytes > 0 (tests): a band of 0xA5 bytes on either side of the workspace, checked by check_guards()
        self._guard = (int(guard_bytes) + align - 1) // align * align
        self.workspace = torch.empty(nbytes + align + 2 * self._guard, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + align - 1) // align * align + self._guard
        self.workspace_bytes = nbytes
        if self._guard:
            self.workspace.fill_(0xA5)
        for t, name in ((mk_init, "mk_init"), (mv_init, "mv_init")):
            if t is not None:
                assert t.is_cuda and t.is_contiguous() and t.dtype == dtype, name
                assert tuple(t.shape) == (batch, n_kv_heads, init_len, head_dim), (name, t.shape)
        self._h = ctypes.c_void_p(None)
        with torch.cuda.device(self.device):
            _check(self.lib.bct_cache_create(ctypes.byref(self.params), self._ws_ptr, nbytes, _ptr(mk_init),
                                             _ptr(mv_init), _stream_ptr(stream), ctypes.byref(self._h)))

    # ---- steps ----------------------------------------------------------------------
    def decode_step(self, q, k, v, out=None, stream=None, eta=None):
        """eta: float32 device tensor [B, Hkv], the step size of each unit's write (None = ones)."""
        if out is None:
            out = torch.empty_like(q, dtype=self.out_dtype)
        if eta is None:
            _check(self.lib.bct_decode_step(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                            _stream_ptr(stream)))
        else:
            _check_eta(eta, (self.B, self.Hkv))
            _check(self.lib.bct_decode_step_eta(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), eta.data_ptr(),
                                                out.data_ptr(), _stream_ptr(stream)))
        return out

    def prefill_stream(self, q, k, v, out=None, want_out=True, stream=None, eta=None):
        """eta: float32 device tensor [B, T, Hkv], the step size of each token's write (None = ones)."""
        T = q.shape[1]
        if out is None and want_out:
            out = torch.empty_like(q, dtype=self.out_dtype)
        if eta is None:
            _check(self.lib.bct_prefill_stream(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(out), T,
                                               _stream_ptr(stream)))
        else:
            _check_eta(eta, (self.B, T, self.Hkv))
            _check(self.lib.bct_prefill_stream_eta(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), eta.data_ptr(),
                                                   _ptr(out), T, _stream_ptr(stream)))
        return out

    def update_kv(self, wq, wv, eta=None, stream=None):
        """Algorithm 1's UpdateKV: wq, wv ``[B, T, Hkv, d]`` go into the state, nothing is read."""
        T = wq.shape[1]
        if eta is not None:
            _check_eta(eta, (self.B, T, self.Hkv))
        _check(self.lib.bct_update_kv(self._h, wq.data_ptr(), wv.data_ptr(), _ptr(eta), T, _stream_ptr(stream)))

    def update_kv_backward(self, wq, wv, d_mv, eta=None, want_d_mk=True, want_d_eta=True, out=None, stream=None):
        """Backward of update_kv: d_mv = dL/dMV_N ``[B, Hkv, C, d]`` bfloat16 -> (d_wq, d_wv ``[B, T, Hkv, d]``,
        d_mk ``[B, Hkv, C, d]`` or None, d_eta ``[B, T, Hkv]`` or None), float32.  out: that tuple, to write into."""
        T = wq.shape[1]
        if eta is not None:
            _check_eta(eta, (self.B, T, self.Hkv))
        f32 = dict(dtype=torch.float32, device=self.device)
        if out is not None:
            d_wq, d_wv, d_mk, d_eta = out
        else:
            d_wq, d_wv = torch.empty(tuple(wq.shape), **f32), torch.empty(tuple(wv.shape), **f32)
            d_mk = torch.empty((self.B, self.Hkv, self.C, self.d), **f32) if want_d_mk else None
            d_eta = torch.empty((self.B, T, self.Hkv), **f32) if want_d_eta else None
        _check(self.lib.bct_update_kv_backward(self._h, wq.data_ptr(), wv.data_ptr(), _ptr(eta), d_mv.data_ptr(), T,
                                               d_wq.data_ptr(), d_wv.data_ptr(), _ptr(d_mk), _ptr(d_eta),
                                               _stream_ptr(stream)))
        return d_wq, d_wv, d_mk, d_eta

    def layer_scratch_bytes(self, T: int) -> int:
        n = ctypes.c_size_t(0)
        _check(self.lib.bct_layer_scratch_bytes(self._h, T, ctypes.byref(n)))
        return n.value

    def layer_forward(self, x, w_q, w_wq, w_wv, out=None, want_out=True, eta=None, scratch=None, stream=None):
        """x ``[B, T, d_model]`` bfloat16: projections, then the stream call on their results."""
        T, d_model = x.shape[1], x.shape[2]
        if scratch is None:
            scratch = torch.empty(self.layer_scratch_bytes(T), dtype=torch.uint8, device=self.device)
        if out is None and want_out:
            out = torch.empty((self.B, T, self.Hq, self.d), dtype=self.out_dtype, device=self.device)
        if eta is not None:
            _check_eta(eta, (self.B, T, self.Hkv))
        _check(self.lib.bct_layer_forward(self._h, x.data_ptr(), w_q.data_ptr(), w_wq.data_ptr(), w_wv.data_ptr(),
                                          d_model, _ptr(eta), scratch.data_ptr(), scratch.numel(), _ptr(out), T,
                                          _stream_ptr(stream)))
        return out

    def decode_step_host(self, q, k, v, out, stream=None):
        """q, k, v, out: CPU tensors (pinned for asynchronous copies)."""
        _check(self.lib.bct_decode_step_host(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                             _stream_ptr(stream)))
        return out

    def prefill_stream_host(self, q, k, v, out, stream=None):
        _check(self.lib.bct_prefill_stream_host(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(out),
                                                q.shape[1], _stream_ptr(stream)))
        return out

    def prefill_stream_host_static(self, q, k, v, out, stream=None):
        """Host tensors in and out, staged in the library's built-in device array (no allocation)."""
        _check(self.lib.bct_prefill_stream_host_static(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                                       out.data_ptr(), q.shape[1], _stream_ptr(stream)))
        return out

    # ---- state ----------------------------------------------------------------------
    @property
    def len(self) -> int:
        n = ctypes.c_int32(0)
        _check(self.lib.bct_cache_len(self._h, ctypes.byref(n)))
        return n.value

    @property
    def tensor_path(self) -> bool:
        n = ctypes.c_int32(0)
        _check(self.lib.bct_cache_tensor_path(self._h, ctypes.byref(n)))
        return bool(n.value)

    @property
    def launches(self) -> int:
        n = ctypes.c_int64(0)
        _check(self.lib.bct_cache_launches(self._h, ctypes.byref(n)))
        return n.value

    def export(self, v_dtype=torch.float32, stream=None):
        shape = (self.B, self.Hkv, self.C, self.d)
        k = torch.empty(shape, dtype=self.dtype, device=self.device)
        v = torch.empty(shape, dtype=v_dtype, device=self.device)
        _check(self.lib.bct_cache_export(self._h, k.data_ptr(), v.data_ptr(), _dtype_code(v_dtype), _stream_ptr(stream)))
        return k, v

    def import_state(self, k, v, length, stream=None):
        vd = _dtype_code(v.dtype) if v is not None else _dtype_code(self.dtype)
        _check(self.lib.bct_cache_import(self._h, _ptr(k), _ptr(v), vd, length, _stream_ptr(stream)))

    def check_guards(self) -> None:
        """Raise if anything wrote outside the workspace (needs guard_bytes > 0 at construction)."""
        if not self._guard:
            return
        torch.cuda.synchronize(self.device)
        lo = self._ws_ptr - self.workspace.data_ptr()
        hi = lo + self.workspace_bytes
        for name, band in (("below", self.workspace[lo - self._guard:lo]), ("above", self.workspace[hi:hi + self._guard])):
            if not bool((band == 0xA5).all()):
                raise AssertionError("guard band %s the workspace was overwritten" % name)

    def status(self, stream=None) -> int:
        return self.lib.bct_cache_status(self._h, _stream_ptr(stream))

    def check_status(self, stream=None) -> None:
        _check(self.status(stream))

    def status_clear(self, stream=None) -> None:
        _check(self.lib.bct_cache_status_clear(self._h, _stream_ptr(stream)))

    def rows_rewritten(self, stream=None) -> int:
        """MV rows stored back by this cache's kernels so far (synchronises the stream)."""
        n = ctypes.c_uint64(0)
        _check(self.lib.bct_cache_rows_rewritten(self._h, _stream_ptr(stream), ctypes.byref(n)))
        return n.value

    def selftest_timeout(self, stream=None) -> None:
        """Launch the block whose bounded wait runs out (reports BCT_ERR_TIMEOUT, site 99)."""
        _check(self.lib.bct_selftest_timeout(self._h, _stream_ptr(stream)))

    def destroy(self) -> None:
        if self._h:
            self.lib.bct_cache_destroy(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

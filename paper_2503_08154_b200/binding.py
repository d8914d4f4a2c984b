"""Thin ctypes binding of libs2a.so: argument marshalling only.

Each function takes torch CUDA tensors (PyTorch is used for device memory and streams,
nothing else), passes their raw pointers, the element count, the row length and the
current stream to the C-ABI call of the same name, and raises on a non-zero status.
There is no CPU path: a missing or unloadable library is an error.
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libs2a.so")

F32 = 0
BF16 = 1
GELU_FWD, GELU_BWD, SOFTMAX_FWD, SOFTMAX_BWD, SILU_FWD, SILU_BWD = 0, 1, 2, 3, 4, 5

EXPORTS = (
    "s2a_codes_bytes", "s2a_meta_bytes", "s2a_status_string", "s2a_gelu_fwd", "s2a_gelu_bwd",
    "s2a_softmax_fwd", "s2a_softmax_bwd", "s2a_device_error", "s2a_describe_plan",
    "s2a_mask_bytes", "s2a_relu_fwd", "s2a_relu_bwd",
    "s2a_tensor_range_scratch_bytes", "s2a_gelu_fwd_tensor_range",
    "s2a_tensor_range_static_max_elems", "s2a_gelu_fwd_tensor_range_static",
    "s2a_silu_fwd", "s2a_silu_bwd", "s2a_cap_fwd", "s2a_cap_bwd", "s2a_lrp_fwd",
    "s2a_selftest_wait_expiry",
    "s2a_selftest_exp2_monotone",
    "s2a_codes_bytes_bits", "s2a_gelu_fwd_bits", "s2a_gelu_bwd_bits", "s2a_softmax_fwd_bits", "s2a_softmax_bwd_bits",
    "s2a_layernorm_scratch_bytes", "s2a_layernorm_fwd", "s2a_layernorm_bwd",
    "s2a_dropout_threshold", "s2a_dropout_fwd", "s2a_dropout_bwd",
    "s2a_relbias_scratch_bytes", "s2a_relbias_fwd", "s2a_relbias_bwd", "s2a_relbias_log_buckets",
    "s2a_rope_fwd", "s2a_rope_bwd", "s2a_qknorm_rope_fwd", "s2a_qknorm_rope_scratch_bytes", "s2a_qknorm_rope_bwd",
    "s2a_rope_table", "s2a_step_plan_bytes", "s2a_step_plan_fill", "s2a_adamw_step", "s2a_grad_norm_scratch_bytes",
    "s2a_grad_norm",
)

_lib = None


class S2AError(RuntimeError):
    pass


class _StepTensor(ctypes.Structure):    # s2a_step_tensor
    _fields_ = [(name, ctypes.c_void_p) for name in ("param", "grad", "exp_avg", "exp_avg_sq", "exp_avg_scale",
                                                     "exp_avg_sq_scale", "copy")]
    _fields_ += [("n", ctypes.c_size_t), ("weight_decay", ctypes.c_float), ("lr_scale", ctypes.c_float)]


class _StepPlan(ctypes.Structure):      # s2a_step_plan
    _fields_ = [(name, ctypes.c_size_t) for name in ("bytes", "n_tensors", "n_chunks", "chunk_blocks")]
    _fields_ += [(name, ctypes.c_int) for name in ("pdt", "gdt", "state_bits", "grads_only")]


def use_library(path: str) -> None:
    """Loads another build of the library (e.g. libs2a_tuning.so) instead of libs2a.so.
    Must be called before the first call into the library."""
    global LIB_PATH
    if _lib is not None:
        raise S2AError("the library is already loaded")
    LIB_PATH = os.path.abspath(path)


def lib() -> ctypes.CDLL:
    """Loads libs2a.so (built in-tree by ``build.py``); raises if it is absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise S2AError("libs2a.so is not built: run `python -m paper_2503_08154_b200.build` "
                           "(there is no fallback path)")
        L = ctypes.CDLL(LIB_PATH)
        c = ctypes
        L.s2a_codes_bytes.argtypes = [c.c_size_t]
        L.s2a_codes_bytes.restype = c.c_size_t
        L.s2a_meta_bytes.argtypes = [c.c_size_t, c.c_size_t]
        L.s2a_meta_bytes.restype = c.c_size_t
        L.s2a_status_string.argtypes = [c.c_int]
        L.s2a_status_string.restype = c.c_char_p
        L.s2a_selftest_wait_expiry.argtypes = [c.c_void_p]
        L.s2a_selftest_wait_expiry.restype = c.c_int
        L.s2a_selftest_exp2_monotone.argtypes = [c.POINTER(c.c_ulonglong), c.c_void_p]
        L.s2a_selftest_exp2_monotone.restype = c.c_int
        for name in ("s2a_gelu_fwd", "s2a_softmax_fwd", "s2a_gelu_bwd", "s2a_softmax_bwd", "s2a_silu_fwd",
                     "s2a_silu_bwd"):
            f = getattr(L, name)
            f.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_size_t, c.c_size_t,
                          c.c_int, c.c_void_p]
            f.restype = c.c_int
        L.s2a_tensor_range_scratch_bytes.argtypes = [c.c_size_t]
        L.s2a_tensor_range_scratch_bytes.restype = c.c_size_t
        L.s2a_gelu_fwd_tensor_range.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p,
                                                c.c_size_t, c.c_size_t, c.c_int, c.c_void_p]
        L.s2a_gelu_fwd_tensor_range.restype = c.c_int
        L.s2a_tensor_range_static_max_elems.argtypes = []
        L.s2a_tensor_range_static_max_elems.restype = c.c_size_t
        L.s2a_gelu_fwd_tensor_range_static.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_size_t,
                                                       c.c_size_t, c.c_int, c.c_void_p]
        L.s2a_gelu_fwd_tensor_range_static.restype = c.c_int
        for name in ("s2a_cap_fwd", "s2a_cap_bwd"):
            f = getattr(L, name)
            f.argtypes = [c.c_void_p, c.c_void_p, c.c_size_t, c.c_size_t, c.c_size_t, c.c_int, c.c_void_p]
            f.restype = c.c_int
        L.s2a_lrp_fwd.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_size_t, c.c_size_t, c.c_size_t,
                                  c.c_size_t, c.c_int, c.c_void_p]
        L.s2a_lrp_fwd.restype = c.c_int
        L.s2a_codes_bytes_bits.argtypes = [c.c_size_t, c.c_int]
        L.s2a_codes_bytes_bits.restype = c.c_size_t
        for name in ("s2a_gelu_fwd_bits", "s2a_gelu_bwd_bits", "s2a_softmax_fwd_bits", "s2a_softmax_bwd_bits"):
            f = getattr(L, name)
            f.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_void_p, c.c_size_t, c.c_size_t, c.c_int, c.c_int,
                          c.c_void_p]
            f.restype = c.c_int
        L.s2a_mask_bytes.argtypes = [c.c_size_t]
        L.s2a_mask_bytes.restype = c.c_size_t
        for name in ("s2a_relu_fwd", "s2a_relu_bwd"):
            f = getattr(L, name)
            f.argtypes = [c.c_void_p, c.c_void_p, c.c_void_p, c.c_size_t, c.c_int, c.c_void_p]
            f.restype = c.c_int
        ptr, size = c.c_void_p, c.c_size_t
        for name, res, args in (
                ("s2a_layernorm_scratch_bytes", size, [size, size]),
                ("s2a_layernorm_fwd", c.c_int, [ptr] * 5 + [size] * 4 + [c.c_float, c.c_int, c.c_int, ptr]),
                ("s2a_layernorm_bwd", c.c_int, [ptr] * 8 + [size] * 5 + [c.c_int, c.c_int, ptr]),
                ("s2a_dropout_threshold", c.c_uint32, [c.c_double]),
                ("s2a_dropout_fwd", c.c_int, [ptr, ptr, ptr, size, ptr, c.c_uint64, c.c_double, c.c_int, ptr]),
                ("s2a_dropout_bwd", c.c_int, [ptr, ptr, size, ptr, c.c_uint64, c.c_double, c.c_int, ptr]),
                ("s2a_relbias_scratch_bytes", size, [size] * 5),
                ("s2a_relbias_fwd", c.c_int, [ptr, ptr, ptr, c.c_int, ptr] + [size] * 5 + [c.c_int, c.c_int, ptr]),
                ("s2a_relbias_bwd", c.c_int, [ptr, ptr, c.c_int, ptr, ptr] + [size] * 5 + [c.c_int, c.c_int, ptr]),
                ("s2a_relbias_log_buckets", c.c_int, [ptr, c.c_int64, size, size, size, c.c_int]),
                ("s2a_rope_fwd", c.c_int, [c.c_char_p, ptr]),           # s2a_rope_args as packed bytes
                ("s2a_rope_bwd", c.c_int, [c.c_char_p, ptr]),
                ("s2a_qknorm_rope_fwd", c.c_int, [c.c_char_p, ptr]),
                ("s2a_qknorm_rope_scratch_bytes", size, [size] * 5),
                ("s2a_qknorm_rope_bwd", c.c_int, [c.c_char_p, ptr]),
                ("s2a_rope_table", c.c_int, [ptr, size, c.c_double, c.c_int] + [c.c_double] * 4 + [size]),
                ("s2a_step_plan_bytes", size, [ptr, size]),
                ("s2a_step_plan_fill", c.c_int, [ptr, size, c.c_int, c.c_int, c.c_int, ptr, ptr]),
                ("s2a_adamw_step", c.c_int, [ptr] * 5 + [c.c_uint64] + [c.c_double] * 3 + [ptr]),
                ("s2a_grad_norm_scratch_bytes", size, [ptr]),
                ("s2a_grad_norm", c.c_int, [ptr] * 3 + [c.c_double] + [ptr] * 3)):
            f = getattr(L, name)
            f.argtypes, f.restype = args, res
        L.s2a_device_error.argtypes = [c.POINTER(c.c_uint), c.c_int]
        L.s2a_device_error.restype = c.c_int
        L.s2a_describe_plan.argtypes = [c.c_int, c.c_size_t, c.c_size_t, c.c_int, c.c_char_p, c.c_size_t]
        L.s2a_describe_plan.restype = c.c_int
        _lib = L
    return _lib


def dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise S2AError("unsupported dtype %s (float32 or bfloat16)" % t.dtype)


def codes_bytes(n_elems: int) -> int:
    return int(lib().s2a_codes_bytes(n_elems))


def meta_bytes(n_elems: int, row_len: int) -> int:
    return int(lib().s2a_meta_bytes(n_elems, row_len))


def status_string(status: int) -> str:
    return lib().s2a_status_string(int(status)).decode()


def check(status: int) -> None:
    if status != 0:
        raise S2AError(status_string(status))


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_ptr(t: torch.Tensor = None) -> int:
    """The current CUDA stream of the tensor's device (of the current device without one) as
    a raw handle.  torch's raw-stream query is several times cheaper than building a Stream
    object on every call; the slower public route is the fallback."""
    if _raw_stream is not None:
        idx = t.device.index if t is not None and t.device.index is not None else torch.cuda.current_device()
        return _raw_stream(idx)
    return torch.cuda.current_stream(t.device if t is not None else None).cuda_stream


def _dev(t: torch.Tensor, what: str) -> torch.Tensor:
    if not t.is_cuda:
        raise S2AError("%s must be a CUDA tensor" % what)
    if not t.is_contiguous():
        raise S2AError("%s must be contiguous" % what)
    return t


def alloc_stash(n_elems: int, row_len: int, device) -> tuple[torch.Tensor, torch.Tensor]:
    """Device buffers for the packed codes (uint8) and the per-row (min, s) metadata."""
    codes = torch.empty(codes_bytes(n_elems), dtype=torch.uint8, device=device)
    meta = torch.empty(meta_bytes(n_elems, row_len) // 4, dtype=torch.float32, device=device)
    return codes, meta


def _fwd(fn, x, y, codes, meta, row_len):
    _dev(x, "x"), _dev(y, "y"), _dev(codes, "codes"), _dev(meta, "meta")
    n = x.numel()
    if y.numel() != n or y.dtype != x.dtype:
        raise S2AError("y must match x in size and dtype")
    if codes.dtype != torch.uint8 or meta.dtype != torch.float32:
        raise S2AError("codes must be uint8 and meta float32")
    if row_len > 0 and (codes.numel() < codes_bytes(n) or meta.numel() * 4 < meta_bytes(n, row_len)):
        raise S2AError("codes/meta buffers are too small")
    check(fn(x.data_ptr(), y.data_ptr(), codes.data_ptr(), meta.data_ptr(), n, row_len,
             dtype_code(x), _stream_ptr(x)))


def _bwd(fn, grad_out, codes, meta, grad_in, row_len):
    _dev(grad_out, "grad_out"), _dev(grad_in, "grad_in"), _dev(codes, "codes"), _dev(meta, "meta")
    n = grad_out.numel()
    if grad_in.numel() != n or grad_in.dtype != grad_out.dtype:
        raise S2AError("grad_in must match grad_out in size and dtype")
    if codes.dtype != torch.uint8 or meta.dtype != torch.float32:
        raise S2AError("codes must be uint8 and meta float32")
    if row_len > 0 and (codes.numel() < codes_bytes(n) or meta.numel() * 4 < meta_bytes(n, row_len)):
        raise S2AError("codes/meta buffers are too small")
    check(fn(grad_out.data_ptr(), codes.data_ptr(), meta.data_ptr(), grad_in.data_ptr(), n,
             row_len, dtype_code(grad_out), _stream_ptr(grad_out)))


def s2a_gelu_fwd(x, y, codes, meta, row_len: int) -> None:
    _fwd(lib().s2a_gelu_fwd, x, y, codes, meta, row_len)


def s2a_gelu_bwd(grad_out, codes, meta, grad_in, row_len: int) -> None:
    _bwd(lib().s2a_gelu_bwd, grad_out, codes, meta, grad_in, row_len)


def s2a_silu_fwd(x, y, codes, meta, row_len: int) -> None:
    _fwd(lib().s2a_silu_fwd, x, y, codes, meta, row_len)


def s2a_silu_bwd(grad_out, codes, meta, grad_in, row_len: int) -> None:
    _bwd(lib().s2a_silu_bwd, grad_out, codes, meta, grad_in, row_len)


def s2a_softmax_fwd(x, y, codes, meta, row_len: int) -> None:
    _fwd(lib().s2a_softmax_fwd, x, y, codes, meta, row_len)


def s2a_softmax_bwd(grad_out, codes, meta, grad_in, row_len: int) -> None:
    _bwd(lib().s2a_softmax_bwd, grad_out, codes, meta, grad_in, row_len)


def tensor_range_scratch_bytes(n_elems: int) -> int:
    return int(lib().s2a_tensor_range_scratch_bytes(n_elems))


def s2a_gelu_fwd_tensor_range(x, y, codes, meta, scratch, row_len: int) -> None:
    """GELU forward with one quantiser range for the whole tensor; `scratch` is a uint8 CUDA
    tensor of at least tensor_range_scratch_bytes(x.numel()) bytes."""
    _dev(x, "x"), _dev(y, "y"), _dev(codes, "codes"), _dev(meta, "meta"), _dev(scratch, "scratch")
    n = x.numel()
    if y.numel() != n or y.dtype != x.dtype:
        raise S2AError("y must match x in size and dtype")
    if codes.dtype != torch.uint8 or meta.dtype != torch.float32:
        raise S2AError("codes must be uint8 and meta float32")
    if row_len > 0 and (codes.numel() < codes_bytes(n) or meta.numel() * 4 < meta_bytes(n, row_len)):
        raise S2AError("codes/meta buffers are too small")
    if scratch.numel() * scratch.element_size() < tensor_range_scratch_bytes(n):
        raise S2AError("scratch is too small")
    check(lib().s2a_gelu_fwd_tensor_range(x.data_ptr(), y.data_ptr(), codes.data_ptr(), meta.data_ptr(),
                                          scratch.data_ptr(), n, row_len, dtype_code(x), _stream_ptr(x)))


def tensor_range_static_max_elems() -> int:
    return int(lib().s2a_tensor_range_static_max_elems())


def s2a_gelu_fwd_tensor_range_static(x, y, codes, meta, row_len: int) -> None:
    """s2a_gelu_fwd_tensor_range without a scratch argument, for callers that may not
    allocate device memory: the range partials live in a fixed array inside the library
    (shared by all calls on a GPU -- do not overlap them), and tensors beyond
    tensor_range_static_max_elems() elements are refused."""
    _dev(x, "x"), _dev(y, "y"), _dev(codes, "codes"), _dev(meta, "meta")
    n = x.numel()
    if y.numel() != n or y.dtype != x.dtype:
        raise S2AError("y must match x in size and dtype")
    if codes.dtype != torch.uint8 or meta.dtype != torch.float32:
        raise S2AError("codes must be uint8 and meta float32")
    if row_len > 0 and (codes.numel() < codes_bytes(n) or meta.numel() * 4 < meta_bytes(n, row_len)):
        raise S2AError("codes/meta buffers are too small")
    check(lib().s2a_gelu_fwd_tensor_range_static(x.data_ptr(), y.data_ptr(), codes.data_ptr(), meta.data_ptr(),
                                                 n, row_len, dtype_code(x), _stream_ptr(x)))


def s2a_cap_fwd(x, y, n_rows: int, channels: int, r: int) -> None:
    _dev(x, "x"), _dev(y, "y")
    if x.numel() != n_rows * channels or r <= 0 or y.numel() * r != x.numel() or y.dtype != x.dtype:
        raise S2AError("x must be [n_rows, channels] and y [n_rows, channels / r] of the same dtype")
    check(lib().s2a_cap_fwd(x.data_ptr(), y.data_ptr(), n_rows, channels, r, dtype_code(x), _stream_ptr(x)))


def s2a_cap_bwd(grad_out, grad_in, n_rows: int, channels: int, r: int) -> None:
    _dev(grad_out, "grad_out"), _dev(grad_in, "grad_in")
    if grad_in.numel() != n_rows * channels or r <= 0 or grad_out.numel() * r != grad_in.numel() \
            or grad_in.dtype != grad_out.dtype:
        raise S2AError("grad_out must be [n_rows, channels / r] and grad_in [n_rows, channels]")
    check(lib().s2a_cap_bwd(grad_out.data_ptr(), grad_in.data_ptr(), n_rows, channels, r, dtype_code(grad_out),
                            _stream_ptr()))


def s2a_lrp_fwd(x, A, B, y, batch: int, tokens: int, channels: int, rank: int) -> None:
    _dev(x, "x"), _dev(y, "y"), _dev(A, "A"), _dev(B, "B")
    if x.numel() != batch * tokens * channels or y.numel() != x.numel() or y.dtype != x.dtype:
        raise S2AError("x and y must be [batch, tokens, channels] of the same dtype")
    if A.dtype != torch.float32 or B.dtype != torch.float32 or A.numel() != tokens * rank or B.numel() != rank * channels:
        raise S2AError("A must be float32 [tokens, rank] and B float32 [rank, channels]")
    check(lib().s2a_lrp_fwd(x.data_ptr(), A.data_ptr(), B.data_ptr(), y.data_ptr(), batch, tokens, channels, rank,
                            dtype_code(x), _stream_ptr(x)))


def codes_bytes_bits(n_elems: int, bits: int) -> int:
    return int(lib().s2a_codes_bytes_bits(n_elems, bits))


def _call_bits(name, a, b, c_, d, n, row_len, bits, dt_code):
    check(getattr(lib(), name)(a.data_ptr(), b.data_ptr(), c_.data_ptr(), d.data_ptr(), n, row_len, bits, dt_code,
                               _stream_ptr()))


def s2a_fwd_bits(kind: str, x, y, codes, meta, row_len: int, bits: int) -> None:
    """s2a_gelu_fwd_bits / s2a_softmax_fwd_bits (kind = 'gelu' or 'softmax')."""
    _dev(x, "x"), _dev(y, "y"), _dev(codes, "codes"), _dev(meta, "meta")
    n = x.numel()
    if y.numel() != n or y.dtype != x.dtype or codes.dtype != torch.uint8 or meta.dtype != torch.float32:
        raise S2AError("y must match x; codes must be uint8 and meta float32")
    if codes.numel() < codes_bytes_bits(n, bits) or (row_len > 0 and meta.numel() * 4 < meta_bytes(n, row_len)):
        raise S2AError("codes/meta buffers are too small")
    _call_bits("s2a_%s_fwd_bits" % kind, x, y, codes, meta, n, row_len, bits, dtype_code(x))


def s2a_bwd_bits(kind: str, grad_out, codes, meta, grad_in, row_len: int, bits: int) -> None:
    _dev(grad_out, "grad_out"), _dev(grad_in, "grad_in"), _dev(codes, "codes"), _dev(meta, "meta")
    n = grad_out.numel()
    if grad_in.numel() != n or grad_in.dtype != grad_out.dtype:
        raise S2AError("grad_in must match grad_out in size and dtype")
    _call_bits("s2a_%s_bwd_bits" % kind, grad_out, codes, meta, grad_in, n, row_len, bits, dtype_code(grad_out))


def mask_bytes(n_elems: int) -> int:
    return int(lib().s2a_mask_bytes(n_elems))


def s2a_relu_fwd(x, y, mask) -> None:
    _dev(x, "x"), _dev(y, "y"), _dev(mask, "mask")
    n = x.numel()
    if y.numel() != n or y.dtype != x.dtype:
        raise S2AError("y must match x in size and dtype")
    if mask.dtype != torch.uint8 or mask.numel() < mask_bytes(n):
        raise S2AError("mask must be uint8 with at least mask_bytes(n) elements")
    check(lib().s2a_relu_fwd(x.data_ptr(), y.data_ptr(), mask.data_ptr(), n, dtype_code(x), _stream_ptr(x)))


def s2a_relu_bwd(grad_out, mask, grad_in) -> None:
    _dev(grad_out, "grad_out"), _dev(grad_in, "grad_in"), _dev(mask, "mask")
    n = grad_out.numel()
    if grad_in.numel() != n or grad_in.dtype != grad_out.dtype:
        raise S2AError("grad_in must match grad_out in size and dtype")
    if mask.dtype != torch.uint8 or mask.numel() < mask_bytes(n):
        raise S2AError("mask must be uint8 with at least mask_bytes(n) elements")
    check(lib().s2a_relu_bwd(grad_out.data_ptr(), mask.data_ptr(), grad_in.data_ptr(), n,
                             dtype_code(grad_out), _stream_ptr()))


# ------------------------------------------------- layer norm, dropout, relative position bias
_CODES = {torch.float32: F32, torch.bfloat16: BF16}
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _stream_on(dev: int) -> int:
    return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream(dev).cuda_stream


def _on_device(first: torch.Tensor, *others) -> int:
    """One device for all tensors of a call, None aside, and that device current: a launch goes to
    the current device, whatever memory its pointers name.  Returns its index."""
    try:
        dev = first.get_device()
        if dev < 0:
            raise S2AError("CUDA tensors are needed")
        for t in others:
            if t is not None and t.get_device() != dev:
                raise S2AError("all tensors of a call must be on one device")
    except AttributeError:
        raise S2AError("CUDA tensors are needed") from None
    if dev != _current_device():
        raise S2AError("the tensors' device must be the current one (torch.cuda.device)")
    return dev


def _rows(t: torch.Tensor, n_rows: int, row_len: int, what: str) -> int:
    """The stride in elements between the rows of a tensor that holds n_rows rows of row_len: a
    contiguous one of any shape, or one whose last dimension is a row and whose leading dimensions
    are evenly spaced (a slice such as x[:, 0])."""
    if t.numel() != n_rows * row_len:
        raise S2AError("%s must hold %d rows of %d elements" % (what, n_rows, row_len))
    if t.is_contiguous():
        return row_len
    shape, stride = t.shape, t.stride()
    if not shape or shape[-1] != row_len or (row_len > 1 and stride[-1] != 1):
        raise S2AError("%s: the elements of a row must be contiguous" % what)
    if len(shape) == 2:
        return stride[0] if n_rows > 1 else row_len
    dims = [(n, s) for n, s in zip(shape[:-1], stride[:-1]) if n != 1]
    for (_, outer), (n, inner) in zip(dims, dims[1:]):
        if outer != n * inner:
            raise S2AError("%s: its rows must be evenly spaced" % what)
    return dims[-1][1] if dims else row_len


def _param(t, n: int, what: str):
    """The address of a learned parameter (or of its gradient) of n elements, None for none."""
    if t is None:
        return None
    if t.numel() != n or not t.is_contiguous():
        raise S2AError("%s must be contiguous with %d elements" % (what, n))
    return t.data_ptr()


def _code(t: torch.Tensor) -> int:
    code = _CODES.get(t.dtype)
    return dtype_code(t) if code is None else code


def _param_dtype(*ts) -> int:
    found = None
    for t in ts:
        if t is not None:
            code = _code(t)
            if found is not None and code != found:
                raise S2AError("learned parameters and their gradients must have one dtype")
            found = code
    return F32 if found is None else found


def _scratch(t, need: int):
    if t is None:
        raise S2AError("scratch is needed")
    if not t.is_contiguous() or t.numel() * t.element_size() < need:
        raise S2AError("scratch must be contiguous with at least %d bytes" % need)
    return t.data_ptr()


def _stats(t, n_rows: int):
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.numel() != 2 * n_rows or not t.is_contiguous():
        raise S2AError("stats must be contiguous float32 with 2 elements a row")
    return t.data_ptr()


def layernorm_scratch_bytes(n_rows: int, row_len: int) -> int:
    return int(lib().s2a_layernorm_scratch_bytes(n_rows, row_len))


def s2a_layernorm_fwd(x, gamma, beta, y, stats, row_len: int, eps: float) -> None:
    """Layer norm over rows of row_len elements.  gamma, beta and stats ([n_rows, 2] float32, what the
    backward call needs) may be None; x and y may be slices with evenly spaced rows."""
    dev = _on_device(x, gamma, beta, y, stats)
    elems = x.numel()
    if row_len <= 0 or elems % row_len:
        raise S2AError("x must hold whole rows of row_len elements")
    if y.dtype is not x.dtype:
        raise S2AError("y must match x in dtype")
    n = elems // row_len
    status = (_lib or lib()).s2a_layernorm_fwd(
        x.data_ptr(), _param(gamma, row_len, "gamma"), _param(beta, row_len, "beta"), y.data_ptr(), _stats(stats, n), n, row_len,
        row_len if x.is_contiguous() else _rows(x, n, row_len, "x"), _rows(y, n, row_len, "y"), eps, _code(x),
        _param_dtype(gamma, beta), _stream_on(dev))
    if status:
        check(status)


def s2a_layernorm_bwd(grad_out, x, gamma, stats, grad_in, grad_gamma, grad_beta, scratch, row_len: int) -> None:
    """Layer norm's backward pass.  grad_gamma and grad_beta may be None (frozen weights; without both,
    scratch may be None too); scratch holds layernorm_scratch_bytes(n_rows, row_len) bytes."""
    dev = _on_device(x, grad_out, gamma, stats, grad_in, grad_gamma, grad_beta, scratch)
    elems = x.numel()
    if row_len <= 0 or elems % row_len:
        raise S2AError("x must hold whole rows of row_len elements")
    if grad_out.dtype is not x.dtype or grad_in.dtype is not x.dtype:
        raise S2AError("grad_out and grad_in must match x in dtype")
    if stats is None:
        raise S2AError("stats of the forward call are needed")
    n = elems // row_len
    sums = grad_gamma is not None or grad_beta is not None
    status = (_lib or lib()).s2a_layernorm_bwd(
        grad_out.data_ptr(), x.data_ptr(), _param(gamma, row_len, "gamma"), _stats(stats, n), grad_in.data_ptr(),
        _param(grad_gamma, row_len, "grad_gamma"), _param(grad_beta, row_len, "grad_beta"),
        _scratch(scratch, layernorm_scratch_bytes(n, row_len)) if sums else None, n, row_len,
        _rows(grad_out, n, row_len, "grad_out"), row_len if x.is_contiguous() else _rows(x, n, row_len, "x"),
        _rows(grad_in, n, row_len, "grad_in"), _code(x), _param_dtype(gamma, grad_gamma, grad_beta), _stream_on(dev))
    if status:
        check(status)


def dropout_threshold(p: float) -> int:
    return int(lib().s2a_dropout_threshold(p))


def _dropout_args(x, y, rng, site):
    if not (x.is_contiguous() and y.is_contiguous() and rng.is_contiguous()):
        raise S2AError("the input, the output and rng must be contiguous")
    if y.numel() != x.numel() or y.dtype is not x.dtype:
        raise S2AError("the output must match the input in size and dtype")
    if rng.dtype is not torch.int64 or rng.numel() != 2:
        raise S2AError("rng must be int64 with 2 elements, (seed, offset)")
    return site & 0xFFFFFFFFFFFFFFFF


def s2a_dropout_fwd(x, residual, y, rng, site: int, p: float) -> None:
    """y = dropout(x), or residual + dropout(x).  rng is an int64 CUDA tensor (seed, offset) that the kernel
    reads; `site` tells the calls of one step apart."""
    dev = _on_device(x, residual, y, rng)
    site = _dropout_args(x, y, rng, site)
    added = None
    if residual is not None:
        if not residual.is_contiguous() or residual.numel() != x.numel() or residual.dtype is not x.dtype:
            raise S2AError("residual must be contiguous and match x in size and dtype")
        added = residual.data_ptr()
    status = (_lib or lib()).s2a_dropout_fwd(x.data_ptr(), added, y.data_ptr(), x.numel(), rng.data_ptr(), site, p, _code(x),
                                             _stream_on(dev))
    if status:
        check(status)


def s2a_dropout_bwd(grad_out, grad_in, rng, site: int, p: float) -> None:
    dev = _on_device(grad_out, grad_in, rng)
    site = _dropout_args(grad_out, grad_in, rng, site)
    status = (_lib or lib()).s2a_dropout_bwd(grad_out.data_ptr(), grad_in.data_ptr(), grad_out.numel(), rng.data_ptr(), site, p,
                                             _code(grad_out), _stream_on(dev))
    if status:
        check(status)


def _bias_args(scores, buckets, table, batch, heads, tq, tk):
    if not (scores.is_contiguous() and buckets.is_contiguous() and table.is_contiguous()):
        raise S2AError("the scores, the buckets and the table must be contiguous")
    if min(batch, heads, tq, tk) < 0 or scores.numel() != batch * heads * tq * tk:
        raise S2AError("the scores must be [batch, heads, tq, tk]")
    shape = table.shape
    if len(shape) != 2 or shape[1] != heads:
        raise S2AError("the table must be [n_buckets, heads]")
    if buckets.dtype is not torch.int32:
        raise S2AError("buckets must be int32")
    size = buckets.shape
    if len(size) == 1 and size[0] == max(tq + tk - 1, 0):
        return 1, shape[0]
    if len(size) == 2 and size[0] == tq and size[1] == tk:
        return 0, shape[0]
    raise S2AError("buckets must be a map [tq, tk] or a vector [tq + tk - 1]")


def s2a_relbias_fwd(x, table, buckets, y, batch: int, heads: int, tq: int, tk: int) -> None:
    """y = x + table[bucket(q, k)] over scores [batch, heads, tq, tk].  buckets: int32, a map [tq, tk], or a
    vector [tq + tk - 1] over the distance k - q + tq - 1."""
    dev = _on_device(x, table, buckets, y)
    by_distance, n = _bias_args(x, buckets, table, batch, heads, tq, tk)
    if not y.is_contiguous() or y.numel() != x.numel() or y.dtype is not x.dtype:
        raise S2AError("y must be contiguous and match x in size and dtype")
    status = (_lib or lib()).s2a_relbias_fwd(x.data_ptr(), table.data_ptr(), buckets.data_ptr(), by_distance, y.data_ptr(), batch,
                                             heads, tq, tk, n, _code(x), _code(table), _stream_on(dev))
    if status:
        check(status)


def relbias_scratch_bytes(batch: int, heads: int, tq: int, tk: int, n_buckets: int) -> int:
    return int(lib().s2a_relbias_scratch_bytes(batch, heads, tq, tk, n_buckets))


def s2a_relbias_bwd(grad_out, buckets, grad_table, scratch, batch: int, heads: int, tq: int, tk: int) -> None:
    """The table's gradient; scratch holds relbias_scratch_bytes(batch, heads, tq, tk, n_buckets) bytes."""
    dev = _on_device(grad_out, buckets, grad_table, scratch)
    by_distance, n = _bias_args(grad_out, buckets, grad_table, batch, heads, tq, tk)
    need = relbias_scratch_bytes(batch, heads, tq, tk, n)
    status = (_lib or lib()).s2a_relbias_bwd(grad_out.data_ptr(), buckets.data_ptr(), by_distance, grad_table.data_ptr(),
                                             _scratch(scratch, need) if need else None, batch, heads, tq, tk, n, _code(grad_out),
                                             _code(grad_table), _stream_on(dev))
    if status:
        check(status)


def log_buckets(first_distance: int, count: int, n_buckets: int, max_distance: int, bidirectional: bool) -> torch.Tensor:
    """Buckets of the distances first_distance, first_distance + 1, ... as a CPU int32 tensor (s2a_relbias_log_buckets)."""
    out = torch.empty(count, dtype=torch.int32)
    check(lib().s2a_relbias_log_buckets(out.data_ptr(), first_distance, count, n_buckets, max_distance, int(bidirectional)))
    return out


# ------------------------------------------- rotary positions, norms of queries and keys with them
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}
# s2a_rope_args in two parts: addresses and scalars of a call, and sizes and strides
_rope_call = struct.Struct("@13Pq2f3i0q").pack
_rope_sizes = struct.Struct("@27Q").pack
_rope_layouts = {}   # the second part, with what else is known of it, by the shapes, strides and dtypes of a call's tensors


def rope_table(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original_length: float = 0.0,
               slow: float = 1.0, fast: float = 32.0, axes: int = 1) -> torch.Tensor:
    """The turns of each pair as a CPU int64 tensor [rot_dim / 2, 2] (s2a_rope_table), to be moved to the GPU once.
    scaling: 'none', 'linear', 'base' or 'parts'."""
    if scaling not in _SCALINGS:
        raise S2AError("scaling must be one of %s" % ", ".join(_SCALINGS))
    out = torch.empty((max(rot_dim, 0) // 2, 2), dtype=torch.int64)
    check(lib().s2a_rope_table(out.data_ptr(), rot_dim, base, _SCALINGS[scaling], factor, original_length, slow, fast, axes))
    return out


def _heads(t, shape, dtype, what: str):
    """The strides of a tensor of heads of this shape and dtype."""
    if t.shape != shape or t.dtype is not dtype:
        raise S2AError("%s must be [batch, tokens, heads, head_dim] like what it belongs to, and of its dtype" % what)
    stride = t.stride()
    if stride[3] != 1 and shape[3] != 1:
        raise S2AError("%s: the elements of a head's row must be contiguous" % what)
    return stride[:3]


def _address(t):
    return 0 if t is None else t.data_ptr()


def _rope_layout(q, k, out_q, out_k, positions, table, grad_q, grad_k, params):
    """What the shapes, strides and dtypes of a call's tensors come to, checked: the sizes' part of the arguments, the codes of
    the dtype and of the weights', and the bytes of scratch that the weights' gradients need."""
    shape, dtype = q.shape, q.dtype
    if len(shape) != 4:
        raise S2AError("queries and keys must be [batch, tokens, heads, head_dim]")
    batch, tokens, heads_q, dim = shape
    none, heads_k, rot = (0, 0, 0), 0, 0
    strides = [_heads(q, shape, dtype, "q"), none, _heads(out_q, shape, dtype, "the queries' output"), none, none, none]
    if grad_q is not None:
        strides[4] = _heads(grad_q, shape, dtype, "grad_q")
    if k is not None:
        other = k.shape
        if len(other) != 4 or other[0] != batch or other[1] != tokens or other[3] != dim:
            raise S2AError("the keys must match the queries but for the number of heads")
        if out_k is None or (grad_q is not None and grad_k is None):
            raise S2AError("the keys' tensors are needed")
        heads_k = other[2]
        strides[1], strides[3] = _heads(k, other, dtype, "k"), _heads(out_k, other, dtype, "the keys' output")
        if grad_k is not None:
            strides[5] = _heads(grad_k, other, dtype, "grad_k")
    per_batch = per_axis = 0
    axes = 1
    if table is not None:
        size = table.shape
        if table.dtype is not torch.int64 or len(size) != 2 or size[1] != 2 or not table.is_contiguous():
            raise S2AError("the table must be contiguous int64 [rot_dim / 2, 2]")
        rot = 2 * size[0]
        if positions is not None:
            size, stride = positions.shape, positions.stride()
            n = len(size)
            if positions.dtype is not torch.int32 or n < 1 or n > 3 or size[-1] != tokens or (n > 1 and size[-2] != batch):
                raise S2AError("positions must be int32 [tokens], [batch, tokens] or [axes, batch, tokens]")
            if tokens > 1 and stride[-1] != 1:
                raise S2AError("the positions of a sequence's tokens must be contiguous")
            if n > 1:
                per_batch = stride[-2]
                if n > 2:
                    per_axis, axes = stride[0], size[0]
    for t, what in zip(params, ("gamma_q", "gamma_k", "grad_gamma_q", "grad_gamma_k")):
        _param(t, dim, what)
    need = qknorm_rope_scratch_bytes(batch, tokens, heads_q, heads_k, dim) if any(t is not None for t in params[2:]) else None
    return (_rope_sizes(per_batch, per_axis, axes, batch, tokens, heads_q, heads_k, dim, rot, *(x for s in strides for x in s)),
            _code(q), _param_dtype(*params), need)


def _rope(call, q, k, out_q, out_k, positions, table, scale, interleaved, first, dev, eps=0.0, grad_q=None, grad_k=None, params=(),
          scratch=None):
    if out_q is None:
        raise S2AError("the queries' output is needed")
    # A call's tensors are looked up by all that is checked of them but their addresses, which the library checks each time.
    key = (q.shape, q.stride(), q.dtype, out_q.shape, out_q.stride(), out_q.dtype)
    q_at, out_q_at = q.data_ptr(), out_q.data_ptr()
    k_at = out_k_at = grad_q_at = grad_k_at = gamma_q = gamma_k = sum_q = sum_k = where = pos = room = 0
    if k is None:
        key += (None,)
    elif out_k is None:
        raise S2AError("the keys' tensors are needed")
    else:
        key += (k.shape, k.stride(), k.dtype, out_k.shape, out_k.stride(), out_k.dtype)
        k_at, out_k_at = k.data_ptr(), out_k.data_ptr()
    if table is None:
        key += (None,)
    else:
        key += (table.shape, table.stride(), table.dtype)
        where = table.data_ptr()
        if positions is not None:
            key += (positions.shape, positions.stride(), positions.dtype)
            pos = positions.data_ptr()
    if params:
        for t in params:
            key += (None,) if t is None else (t.numel(), t.is_contiguous(), t.dtype)
        gamma_q, gamma_k, sum_q, sum_k = [0 if t is None else t.data_ptr() for t in params]
        if grad_q is not None:
            key += (grad_q.shape, grad_q.stride(), grad_q.dtype)
            grad_q_at = grad_q.data_ptr()
            if grad_k is not None and k is not None:
                key += (grad_k.shape, grad_k.stride(), grad_k.dtype)
                grad_k_at = grad_k.data_ptr()
    found = _rope_layouts.get(key)
    if found is None:
        found = _rope_layout(q, k, out_q, out_k, positions, table, grad_q, grad_k, params)
        if len(_rope_layouts) >= 1024:
            _rope_layouts.clear()
        _rope_layouts[key] = found
    sizes, dt, wdt, need = found
    if need is not None:
        room = _scratch(scratch, need)
    try:
        packed = _rope_call(q_at, k_at, out_q_at, out_k_at, pos, where, gamma_q, gamma_k, grad_q_at, grad_k_at, sum_q, sum_k, room, first, scale,
                            eps, interleaved, dt, wdt)
    except (struct.error, OverflowError) as error:
        raise S2AError("scale, eps, interleaved and first must be plain numbers: %s" % error)
    status = call(packed + sizes, _stream_on(dev))
    if status:
        check(status)


def s2a_rope_fwd(q, k, out_q, out_k, positions, table, scale: float = 1.0, interleaved: bool = False, first: int = 0) -> None:
    """Rotary positions of queries and keys [batch, tokens, heads, head_dim] (any strides; k and out_k may be None; an
    output may be its input).  positions: int32 [tokens], [batch, tokens] or [axes, batch, tokens], or None for first +
    token; table: rope_table(...) on the GPU, or one of the caller's own."""
    if table is None:
        raise S2AError("a table of turns is needed")
    _rope((_lib or lib()).s2a_rope_fwd, q, k, out_q, out_k, positions, table, scale, interleaved, first,
          _on_device(q, k, out_q, out_k, positions, table))


def s2a_rope_bwd(grad_q, grad_k, grad_in_q, grad_in_k, positions, table, scale: float = 1.0, interleaved: bool = False,
                 first: int = 0) -> None:
    """The gradients of s2a_rope_fwd: turned back."""
    if table is None:
        raise S2AError("a table of turns is needed")
    _rope((_lib or lib()).s2a_rope_bwd, grad_q, grad_k, grad_in_q, grad_in_k, positions, table, scale, interleaved, first,
          _on_device(grad_q, grad_k, grad_in_q, grad_in_k, positions, table))


def s2a_qknorm_rope_fwd(q, k, gamma_q, gamma_k, out_q, out_k, positions, table, eps: float, scale: float = 1.0,
                        interleaved: bool = False, first: int = 0) -> None:
    """The norm of each head's row (by its root mean square; gamma_q, gamma_k [head_dim] or None) and the rotation in one pass.
    table None: the norm alone.  The rest as for s2a_rope_fwd."""
    _rope((_lib or lib()).s2a_qknorm_rope_fwd, q, k, out_q, out_k, positions, table, scale, interleaved, first,
          _on_device(q, k, gamma_q, gamma_k, out_q, out_k, positions, table), eps, params=(gamma_q, gamma_k, None, None))


def qknorm_rope_scratch_bytes(batch: int, tokens: int, heads_q: int, heads_k: int, head_dim: int) -> int:
    return int(lib().s2a_qknorm_rope_scratch_bytes(batch, tokens, heads_q, heads_k, head_dim))


def s2a_qknorm_rope_bwd(grad_q, grad_k, q, k, gamma_q, gamma_k, grad_in_q, grad_in_k, grad_gamma_q, grad_gamma_k, scratch,
                        positions, table, eps: float, scale: float = 1.0, interleaved: bool = False, first: int = 0) -> None:
    """The backward pass of s2a_qknorm_rope_fwd from its inputs q and k.  grad_gamma_q and grad_gamma_k may be None (frozen
    weights; without both, scratch may be None too); scratch holds qknorm_rope_scratch_bytes(...) bytes.  grad_in_q may be
    grad_q or q, grad_in_k grad_k or k."""
    if grad_q is None:
        raise S2AError("grad_q is needed")
    _rope((_lib or lib()).s2a_qknorm_rope_bwd, q, k, grad_in_q, grad_in_k, positions, table, scale, interleaved, first,
          _on_device(q, grad_q, grad_k, k, gamma_q, gamma_k, grad_in_q, grad_in_k, grad_gamma_q, grad_gamma_k, scratch, positions, table),
          eps, grad_q, grad_k, (gamma_q, gamma_k, grad_gamma_q, grad_gamma_k), scratch)


# --------------------------------------------------- the AdamW step over many tensors, the gradients' norm
class AdamWPlan:
    """The tensors of a step, checked and laid out once (adamw_plan); it keeps them alive and is good as long as they stay
    where they are.  A step with gradients that have become other tensors would go on with the old ones: zero gradients in place
    (zero_grad(set_to_none=False)), or make another plan, which costs some 6 us a tensor and a wait for the stream.  Where the parameters are leaves and
    the gradients their .grad, each call looks at one pair in turn and refuses a plan whose gradient is no longer that.  It may be dropped while a stream still runs it (its tensors are the
    caller's to keep for a stream that is not their own, as with any call); a graph that has captured its calls needs it as long as it is replayed."""

    __slots__ = ("plan", "address", "image", "device", "tensors", "room", "streams", "pairs", "turn")


def _state_bits(m, v) -> int:
    if not isinstance(m, torch.Tensor) or not isinstance(v, torch.Tensor):
        raise S2AError("exp_avgs and exp_avg_sqs must be CUDA tensors of one device")
    if m.dtype is torch.float32 and v.dtype is torch.float32:
        return 32
    if m.dtype is torch.float8_e4m3fn and v.dtype is torch.float8_e4m3fn:
        return 8
    raise S2AError("exp_avg and exp_avg_sq must both be float32 or both float8_e4m3fn")


def adamw_plan(params, grads, exp_avgs, exp_avg_sqs, exp_avg_scales=None, exp_avg_sq_scales=None, copies=None,
               weight_decay=0.0, lr_scale=1.0) -> AdamWPlan:
    """A plan for s2a_adamw_step and s2a_grad_norm over lists of contiguous CUDA tensors, one entry of each list per
    parameter.  Parameters have one dtype, gradients one, states are float32, or float8_e4m3fn codes with float32 scales of (n +
    255) // 256 elements; copies: None, or bfloat16 tensors (None in the list: no copy).  weight_decay and lr_scale: a
    number, or one for each tensor.  params None (with exp_avgs and exp_avg_sqs None): gradients alone, for s2a_grad_norm."""
    count = len(grads)
    lists = {"params": params, "exp_avgs": exp_avgs, "exp_avg_sqs": exp_avg_sqs, "exp_avg_scales": exp_avg_scales,
             "exp_avg_sq_scales": exp_avg_sq_scales, "copies": copies}
    for what, ts in lists.items():
        if ts is not None and len(ts) != count:
            raise S2AError("%s must have one entry for each gradient" % what)
    if params is None and any(ts is not None for ts in lists.values()):
        raise S2AError("a plan without parameters has gradients alone")
    if params is not None and (exp_avgs is None or exp_avg_sqs is None):
        raise S2AError("exp_avgs and exp_avg_sqs are needed")
    decays = [float(w) for w in weight_decay] if isinstance(weight_decay, (list, tuple)) else [float(weight_decay)] * count
    rates = [float(w) for w in lr_scale] if isinstance(lr_scale, (list, tuple)) else [float(lr_scale)] * count
    if len(decays) != count or len(rates) != count:
        raise S2AError("weight_decay and lr_scale must have one entry for each gradient")
    records = (_StepTensor * max(count, 1))()
    pdt, gdt, bits, dev = F32, F32, 32, None

    def same(found, new, i, what):
        if i and found != new:
            raise S2AError("%s must have one dtype" % what)
        return new

    def address(t, n, what, dtype=None):
        nonlocal dev
        if not isinstance(t, torch.Tensor) or not t.is_cuda or (dev is not None and t.get_device() != dev):
            raise S2AError("%s must be CUDA tensors of one device" % what)
        if not t.is_contiguous() or t.numel() != n or (dtype is not None and t.dtype is not dtype):
            raise S2AError("%s must be contiguous, of the right size%s" % (what, "" if dtype is None else " and %s" % dtype))
        dev = t.get_device()
        return t.data_ptr()

    for i in range(count):
        if not isinstance(grads[i], torch.Tensor):
            raise S2AError("gradients must be CUDA tensors of one device")
        r, n = records[i], grads[i].numel()
        r.n, r.weight_decay, r.lr_scale = n, decays[i], rates[i]
        r.grad = address(grads[i], n, "gradients")
        gdt = same(gdt, _code(grads[i]), i, "gradients")
        if params is None:
            continue
        r.param = address(params[i], n, "parameters")
        pdt = same(pdt, _code(params[i]), i, "parameters")
        bits = same(bits, _state_bits(exp_avgs[i], exp_avg_sqs[i]), i, "states")
        r.exp_avg = address(exp_avgs[i], n, "exp_avgs")
        r.exp_avg_sq = address(exp_avg_sqs[i], n, "exp_avg_sqs")
        if bits == 8:
            if exp_avg_scales is None or exp_avg_sq_scales is None:
                raise S2AError("states in 8 bits need their scales")
            blocks = (n + 255) // 256
            r.exp_avg_scale = address(exp_avg_scales[i], blocks, "exp_avg_scales", torch.float32)
            r.exp_avg_sq_scale = address(exp_avg_sq_scales[i], blocks, "exp_avg_sq_scales", torch.float32)
        if copies is not None and copies[i] is not None:
            r.copy = address(copies[i], n, "copies", torch.bfloat16)
    self = AdamWPlan()
    need = int(lib().s2a_step_plan_bytes(records, count))
    host = torch.zeros(max(need, 16) // 8 + 2, dtype=torch.int64)
    start = -host.data_ptr() % 16 // 8      # 16-byte aligned
    self.plan = _StepPlan()
    check(lib().s2a_step_plan_fill(records, count, pdt, gdt, bits, host.data_ptr() + 8 * start, ctypes.byref(self.plan)))
    self.device = torch.cuda.current_device() if dev is None else dev
    self.image = host[start:start + max(need, 16) // 8 + 1].to(torch.device("cuda", self.device))
    self.streams = {_stream_on(self.device)}
    self.address = ctypes.addressof(self.plan)
    self.room = int(lib().s2a_grad_norm_scratch_bytes(self.address))
    self.pairs = [(p, g) for p, g in zip(params or (), grads) if p.is_leaf and p.requires_grad and p.grad is g]
    self.turn = 0
    self.tensors = (list(grads),) + tuple(None if ts is None else list(ts) for ts in lists.values())
    return self


def _float_words(t, n: int, what: str):
    if t is None or t.dtype is not torch.float32 or t.numel() < n or not t.is_contiguous():
        raise S2AError("%s must be contiguous float32 with %d elements" % (what, n))
    return t.data_ptr()


def _plan_current(plan: AdamWPlan) -> None:
    """Refuses a plan whose gradients have been replaced.  That happens to all at once, as a rule: one pair a call, in turn, tells."""
    param, grad = plan.pairs[plan.turn % len(plan.pairs)]
    plan.turn += 1
    now = param.grad
    if now is not grad and (now is None or now.data_ptr() != grad.data_ptr()):
        raise S2AError("a parameter's gradient is another tensor than when the plan was made: make another plan, or zero gradients in place")


def _plan_stream(plan: AdamWPlan, dev: int) -> int:
    """The current stream.  The plan's image is memory of the stream on which the plan was made; once another one reads it, that
    memory may be given away only after its work."""
    if plan.pairs:
        _plan_current(plan)
    stream = _stream_on(dev)
    if stream not in plan.streams:
        plan.image.record_stream(torch.cuda.current_stream(dev))
        plan.streams.add(stream)
    return stream


def s2a_adamw_step(plan: AdamWPlan, control, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, clip=None, rng=None,
                   site: int = 0) -> None:
    """One AdamW step over the plan's tensors, in place.  control: float32 (learning rate, number of the step from 1, scale of
    the gradients) on the device; clip: what s2a_grad_norm wrote, or None; rng: int64 (seed, offset) on the device for
    rounding at random, or None."""
    try:
        dev = _on_device(plan.image, control, clip, rng)
    except AttributeError:
        raise S2AError("a plan of adamw_plan is needed") from None
    if rng is not None and (rng.dtype is not torch.int64 or rng.numel() != 2 or not rng.is_contiguous()):
        raise S2AError("rng must be contiguous int64 (seed, offset)")
    status = (_lib or lib()).s2a_adamw_step(plan.address, plan.image.data_ptr(), _float_words(control, 3, "control"),
                                            None if clip is None else _float_words(clip, 2, "clip"), _address(rng) or None, site, beta1,
                                            beta2, eps, _plan_stream(plan, dev))
    if status:
        check(status)


def grad_norm_scratch_bytes(plan: AdamWPlan) -> int:
    return plan.room


def s2a_grad_norm(plan: AdamWPlan, control, max_norm: float, clip, scratch) -> None:
    """The norm of all the plan's gradients, times control[2], and the factor that limits it to max_norm: written to clip
    (float32, two elements).  scratch holds grad_norm_scratch_bytes(plan) bytes."""
    try:
        dev = _on_device(plan.image, control, clip, scratch)
    except AttributeError:
        raise S2AError("a plan of adamw_plan is needed") from None
    status = (_lib or lib()).s2a_grad_norm(plan.address, plan.image.data_ptr(), _float_words(control, 3, "control"), max_norm,
                                           _float_words(clip, 2, "clip"), _scratch(scratch, plan.room),
                                           _plan_stream(plan, dev))
    if status:
        check(status)


def s2a_device_error(clear: bool = False) -> int:
    flags = ctypes.c_uint(0)
    check(lib().s2a_device_error(ctypes.byref(flags), int(clear)))
    return int(flags.value)


def s2a_describe_plan(kernel: int, n_elems: int, row_len: int, dt: int) -> str:
    buf = ctypes.create_string_buffer(256)
    check(lib().s2a_describe_plan(kernel, n_elems, row_len, dt, buf, 256))
    return buf.value.decode()

"""Python binding of libspla.so, the SPLA decode-step C ABI (include/spla.h).

Argument marshalling only: every step of the append and decode paths runs in
the library's HIP kernels. PyTorch provides device memory and the stream
(the current torch stream of the tensors' device); nothing here computes.
The binding fails loudly when the HIP library has not been built.
"""

from __future__ import annotations

import contextlib
import ctypes
import os
from ctypes import (POINTER, c_double, c_float, c_int32, c_int64, c_size_t, c_uint32,
                    c_void_p)
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspla.so")
HOST_LIB_PATH = os.path.join(_HERE, "libspla_host.so")

F32, BF16 = 0, 1
FLAG_NO_RLA, FLAG_FIRST_ORDER, FLAG_RLA_NORMALIZE, FLAG_SEPARATE_KERNELS = 1, 2, 4, 8
DEVERR_CAPACITY, DEVERR_SYNC, DEVERR_PAGE = 1, 2, 4
MAX_GROUP, MAX_TOP_K, MAX_BLOCKS, WORKSPACE_ALIGN = 16, 256, 32768, 256
PHASES = {"append": 0, "score": 1, "select": 2, "sparse": 3, "merge": 4, "decode": 5,
          "linear": 6}
NUM_PHASES = 8
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}
ROPE_MAX_PAIRS = 64
STATUS = {0: "ok", -1: "invalid argument", -2: "unsupported shape",
          -3: "capacity or library limit exceeded", -4: "workspace missing, too small or misaligned",
          -5: "HIP runtime error"}

# every symbol include/spla.h declares
HOST_EXPORTS = ["spla_status_string", "spla_phase_name", "spla_validate", "spla_cache_bytes",
                "spla_workspace_bytes", "spla_append_workspace_bytes", "spla_decode_phase_mask",
                "spla_prefill_workspace_bytes", "spla_rope_init",
                "spla_append_rope_workspace_bytes", "spla_append_rope_workspace_bytes_ex",
                "spla_attend_workspace_bytes", "spla_cache8_bytes", "spla_attend8_workspace_bytes",
                "spla_norm_rotate_grad_workspace_bytes"]
EXPORTS = HOST_EXPORTS + ["spla_workspace_init", "spla_reset", "spla_append", "spla_decode",
                          "spla_decode_ex", "spla_step", "spla_step_ex", "spla_prefill",
                          "spla_prefill_ex", "spla_decode_noalloc", "spla_rotate",
                          "spla_append_rope", "spla_attend", "spla_norm_rotate",
                          "spla_norm_rotate_grad", "spla_reset8", "spla_append8", "spla_read8",
                          "spla_attend8"]


class SplaError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__(f"{where}: {STATUS.get(status, 'unknown status')} ({status})")
        self.status = status


class SplaConfig(ctypes.Structure):
    _fields_ = [("batch", c_int32), ("n_q_heads", c_int32), ("n_kv_heads", c_int32),
                ("head_dim", c_int32), ("block_size", c_int32), ("top_k", c_int32),
                ("n_sink_blocks", c_int32), ("n_local_blocks", c_int32),
                ("max_seq_len", c_int32), ("dtype", c_int32), ("softmax_scale", c_float),
                ("rms_eps", c_float), ("flags", c_uint32), ("sel_window", c_int32),
                ("sel_stride", c_int32), ("kv_pages", c_int32)]


class SplaCacheStruct(ctypes.Structure):
    _fields_ = [("k_cache", c_void_p), ("v_cache", c_void_p), ("blk_stats", c_void_p),
                ("lin_state", c_void_p), ("lin_norm", c_void_p), ("seq_lens", c_void_p),
                ("err_flags", c_void_p), ("block_table", c_void_p)]


class SplaEvents(ctypes.Structure):
    _fields_ = [("start", c_void_p * NUM_PHASES), ("stop", c_void_p * NUM_PHASES)]


class SplaRopeConfig(ctypes.Structure):
    _fields_ = [("head_dim", c_int32), ("rot_dim", c_int32), ("layout", c_int32),
                ("scaling", c_int32), ("base", c_double), ("factor", c_double),
                ("orig_len", c_double), ("low", c_double), ("high", c_double),
                ("gain", c_double)]


class SplaRope(ctypes.Structure):
    _fields_ = [("head_dim", c_int32), ("rot_dim", c_int32), ("layout", c_int32),
                ("reserved", c_int32), ("gain", c_double), ("turns", c_double * ROPE_MAX_PAIRS)]


class SplaAttendOpts(ctypes.Structure):
    _fields_ = [("softcap", c_float), ("reserved", c_float), ("slopes", c_void_p),
                ("first_key", c_void_p), ("prefix_len", c_void_p), ("n_new", c_void_p)]


class SplaCache8Struct(ctypes.Structure):
    _fields_ = [("k_codes", c_void_p), ("v_codes", c_void_p), ("scales", c_void_p),
                ("seq_lens", c_void_p), ("counters", c_void_p), ("err_flags", c_void_p),
                ("block_table", c_void_p)]


class SplaAttend8Opts(ctypes.Structure):
    _fields_ = [("attend", SplaAttendOpts), ("window", c_int32), ("sinks", c_int32)]


def _declare(lib, host_only=False):
    cfgp = POINTER(SplaConfig)
    cachep = POINTER(SplaCacheStruct)
    lib.spla_status_string.restype = ctypes.c_char_p
    lib.spla_status_string.argtypes = [c_int32]
    lib.spla_phase_name.restype = ctypes.c_char_p
    lib.spla_phase_name.argtypes = [c_int32]
    lib.spla_validate.restype = c_int32
    lib.spla_validate.argtypes = [cfgp]
    lib.spla_cache_bytes.restype = c_int32
    lib.spla_cache_bytes.argtypes = [cfgp, POINTER(c_size_t)]
    lib.spla_workspace_bytes.restype = c_int32
    lib.spla_workspace_bytes.argtypes = [cfgp, POINTER(c_size_t)]
    lib.spla_append_workspace_bytes.restype = c_int32
    lib.spla_append_workspace_bytes.argtypes = [cfgp, c_int32, POINTER(c_size_t)]
    lib.spla_decode_phase_mask.restype = c_int32
    lib.spla_decode_phase_mask.argtypes = [cfgp, POINTER(c_uint32)]
    lib.spla_prefill_workspace_bytes.restype = c_int32
    lib.spla_prefill_workspace_bytes.argtypes = [cfgp, c_int32, POINTER(c_size_t)]
    lib.spla_rope_init.restype = c_int32
    lib.spla_rope_init.argtypes = [POINTER(SplaRopeConfig), POINTER(SplaRope)]
    lib.spla_append_rope_workspace_bytes.restype = c_int32
    lib.spla_append_rope_workspace_bytes.argtypes = [cfgp, c_int32, POINTER(c_size_t)]
    lib.spla_append_rope_workspace_bytes_ex.restype = c_int32
    lib.spla_append_rope_workspace_bytes_ex.argtypes = [cfgp, POINTER(SplaRope), c_int32,
                                                        POINTER(c_size_t)]
    lib.spla_attend_workspace_bytes.restype = c_int32
    lib.spla_attend_workspace_bytes.argtypes = [cfgp, c_int32, POINTER(c_size_t)]
    lib.spla_cache8_bytes.restype = c_int32
    lib.spla_cache8_bytes.argtypes = [cfgp, POINTER(c_size_t)]
    lib.spla_attend8_workspace_bytes.restype = c_int32
    lib.spla_attend8_workspace_bytes.argtypes = [cfgp, c_int32, POINTER(c_size_t)]
    lib.spla_norm_rotate_grad_workspace_bytes.restype = c_int32
    lib.spla_norm_rotate_grad_workspace_bytes.argtypes = [cfgp, c_int32, POINTER(c_size_t)]
    if host_only:
        return lib
    cache8p = POINTER(SplaCache8Struct)
    rows = [c_void_p, c_int64]  # an address and the stride of its rows
    lib.spla_norm_rotate.restype = c_int32
    lib.spla_norm_rotate.argtypes = [cfgp, POINTER(SplaRope), c_int32, c_void_p, c_void_p, c_void_p,
                                     c_void_p, c_int32, c_double, *rows * 4, c_void_p]
    lib.spla_norm_rotate_grad.restype = c_int32
    lib.spla_norm_rotate_grad.argtypes = [cfgp, POINTER(SplaRope), c_int32, c_void_p, c_void_p,
                                          c_void_p, c_void_p, c_int32, c_double, *rows * 6, c_void_p,
                                          c_void_p, c_void_p, c_size_t, c_void_p]
    lib.spla_reset8.restype = c_int32
    lib.spla_reset8.argtypes = [cfgp, cache8p, c_void_p]
    lib.spla_append8.restype = c_int32
    lib.spla_append8.argtypes = [cfgp, cache8p, c_int32, *rows * 2, c_void_p, c_void_p]
    lib.spla_read8.restype = c_int32
    lib.spla_read8.argtypes = [cfgp, cache8p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p]
    lib.spla_attend8.restype = c_int32
    lib.spla_attend8.argtypes = [cfgp, cache8p, c_int32, c_void_p, POINTER(SplaAttend8Opts),
                                 c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.spla_rotate.restype = c_int32
    lib.spla_rotate.argtypes = [cfgp, POINTER(SplaRope), c_int32, c_void_p, c_void_p,
                                c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                                c_int64, c_int32, c_void_p]
    lib.spla_append_rope.restype = c_int32
    lib.spla_append_rope.argtypes = [cfgp, cachep, POINTER(SplaRope), c_void_p, c_void_p, c_int32,
                                     c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    lib.spla_attend.restype = c_int32
    lib.spla_attend.argtypes = [cfgp, cachep, c_int32, c_void_p, POINTER(SplaAttendOpts), c_void_p,
                                c_void_p, c_void_p, c_size_t, c_void_p]
    lib.spla_workspace_init.restype = c_int32
    lib.spla_workspace_init.argtypes = [cfgp, c_void_p, c_size_t, c_void_p]
    lib.spla_reset.restype = c_int32
    lib.spla_reset.argtypes = [cfgp, cachep, c_void_p]
    lib.spla_append.restype = c_int32
    lib.spla_append.argtypes = [cfgp, cachep, c_void_p, c_void_p, c_int32, c_void_p, c_void_p,
                                c_size_t, c_void_p]
    lib.spla_decode.restype = c_int32
    lib.spla_decode.argtypes = [cfgp, cachep, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                c_size_t, c_void_p]
    lib.spla_decode_ex.restype = c_int32
    lib.spla_decode_ex.argtypes = [cfgp, cachep, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_size_t, POINTER(SplaEvents), c_void_p]
    lib.spla_step.restype = c_int32
    lib.spla_step.argtypes = [cfgp, cachep, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                              c_void_p, c_void_p, c_size_t, c_void_p]
    lib.spla_step_ex.restype = c_int32
    lib.spla_step_ex.argtypes = [cfgp, cachep, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                 c_void_p, c_void_p, c_size_t, POINTER(SplaEvents), c_void_p]
    lib.spla_prefill_ex.restype = c_int32
    lib.spla_prefill_ex.argtypes = [cfgp, cachep, c_int32, c_void_p, c_void_p, c_void_p,
                                    c_void_p, c_void_p, c_void_p, c_void_p, c_size_t,
                                    POINTER(SplaEvents), c_void_p]
    lib.spla_decode_noalloc.restype = c_int32
    lib.spla_decode_noalloc.argtypes = [cfgp, cachep, c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_void_p]
    lib.spla_prefill.restype = c_int32
    lib.spla_prefill.argtypes = [cfgp, cachep, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                 c_void_p, c_void_p, c_void_p, c_size_t, c_void_p]
    return lib


_LIB = None
_HOST_LIB = None


def lib():
    """The HIP library (raises ImportError if it has not been built)."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2601_22379_amd.build`")
        _LIB = _declare(ctypes.CDLL(LIB_PATH))
    return _LIB


def host_lib():
    """The host-only validation library (loads without a GPU or HIP runtime)."""
    global _HOST_LIB
    if _HOST_LIB is None:
        if not os.path.exists(HOST_LIB_PATH):
            raise ImportError(f"{HOST_LIB_PATH} is missing: build it with "
                              "`python -m paper_2601_22379_amd.build --host-only`")
        _HOST_LIB = _declare(ctypes.CDLL(HOST_LIB_PATH), host_only=True)
    return _HOST_LIB


def _check(status: int, where: str):
    if status != 0:
        raise SplaError(status, where)


def make_config(batch, n_q_heads, n_kv_heads, head_dim, block_size, top_k, max_seq_len,
                dtype="bf16", n_sink=1, n_local=4, softmax_scale=0.0, rms_eps=1e-6,
                flags=0, sel_window=0, sel_stride=0, kv_pages=0) -> SplaConfig:
    dt = {"f32": F32, "fp32": F32, "float32": F32, "bf16": BF16, "bfloat16": BF16}.get(dtype, dtype)
    return SplaConfig(batch, n_q_heads, n_kv_heads, head_dim, block_size, top_k, n_sink, n_local,
                      max_seq_len, int(dt), float(softmax_scale), float(rms_eps), int(flags),
                      int(sel_window), int(sel_stride), int(kv_pages))


def validate(cfg: SplaConfig, library=None) -> int:
    return int((library or lib()).spla_validate(ctypes.byref(cfg)))


def cache_bytes(cfg: SplaConfig, library=None) -> list:
    out = (c_size_t * 6)()
    _check((library or lib()).spla_cache_bytes(ctypes.byref(cfg), out), "spla_cache_bytes")
    return list(out)


def workspace_bytes(cfg: SplaConfig, library=None) -> int:
    n = c_size_t(0)
    _check((library or lib()).spla_workspace_bytes(ctypes.byref(cfg), ctypes.byref(n)),
           "spla_workspace_bytes")
    return int(n.value)


def append_workspace_bytes(cfg: SplaConfig, max_new: int, library=None) -> int:
    n = c_size_t(0)
    _check((library or lib()).spla_append_workspace_bytes(ctypes.byref(cfg), int(max_new),
                                                          ctypes.byref(n)),
           "spla_append_workspace_bytes")
    return int(n.value)


def prefill_workspace_bytes(cfg: SplaConfig, n_tokens: int, library=None) -> int:
    n = c_size_t(0)
    _check((library or lib()).spla_prefill_workspace_bytes(ctypes.byref(cfg), int(n_tokens),
                                                           ctypes.byref(n)),
           "spla_prefill_workspace_bytes")
    return int(n.value)


def append_rope_workspace_bytes(cfg: SplaConfig, max_new: int, library=None, rope=None) -> int:
    """For one rotation, or (None) whatever the rotation."""
    n = c_size_t(0)
    _check((library or lib()).spla_append_rope_workspace_bytes_ex(
        ctypes.byref(cfg), None if rope is None else ctypes.byref(rope), int(max_new),
        ctypes.byref(n)), "spla_append_rope_workspace_bytes")
    return int(n.value)


def attend_workspace_bytes(cfg: SplaConfig, n_tokens: int, library=None) -> int:
    n = c_size_t(0)
    _check((library or lib()).spla_attend_workspace_bytes(ctypes.byref(cfg), int(n_tokens),
                                                          ctypes.byref(n)),
           "spla_attend_workspace_bytes")
    return int(n.value)


def cache8_bytes(cfg: SplaConfig, library=None) -> list:
    out = (c_size_t * 5)()
    _check((library or lib()).spla_cache8_bytes(ctypes.byref(cfg), out), "spla_cache8_bytes")
    return list(out)


def attend8_workspace_bytes(cfg: SplaConfig, n_tokens: int, library=None) -> int:
    n = c_size_t(0)
    _check((library or lib()).spla_attend8_workspace_bytes(ctypes.byref(cfg), int(n_tokens),
                                                           ctypes.byref(n)),
           "spla_attend8_workspace_bytes")
    return int(n.value)


def norm_rotate_grad_workspace_bytes(cfg: SplaConfig, n_tokens: int, library=None) -> int:
    n = c_size_t(0)
    _check((library or lib()).spla_norm_rotate_grad_workspace_bytes(ctypes.byref(cfg),
                                                                    int(n_tokens), ctypes.byref(n)),
           "spla_norm_rotate_grad_workspace_bytes")
    return int(n.value)


def make_rope(head_dim, rot_dim=None, layout="half", base=10000.0, scaling="none", factor=1.0,
              orig_len=0.0, low=1.0, high=32.0, gain=1.0, library=None) -> SplaRope:
    """A rotation of the leading rot_dim coordinates (default: all) for rotate and append_rope.
    layout: "half" or "interleaved"; scaling: "none", "linear", "base" or "parts"."""
    c = SplaRopeConfig(int(head_dim), int(head_dim if rot_dim is None else rot_dim),
                       ROPE_LAYOUTS.get(layout, layout), ROPE_SCALINGS.get(scaling, scaling),
                       float(base), float(factor), float(orig_len), float(low), float(high),
                       float(gain))
    r = SplaRope()
    _check((library or lib()).spla_rope_init(ctypes.byref(c), ctypes.byref(r)), "spla_rope_init")
    return r


def decode_phases(cfg: SplaConfig, library=None) -> list:
    """Names of the phases whose events spla_decode_ex records for cfg."""
    mask = c_uint32(0)
    _check((library or lib()).spla_decode_phase_mask(ctypes.byref(cfg), ctypes.byref(mask)),
           "spla_decode_phase_mask")
    return [n for n, p in PHASES.items() if mask.value >> p & 1]


def torch_dtype(cfg: SplaConfig):
    return torch.float32 if cfg.dtype == F32 else torch.bfloat16


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else c_void_p(t.data_ptr())


def _indexed(device) -> torch.device:
    """The device, by its index: "cuda" is the current one now, not whichever is later."""
    device = torch.device(device)
    if device.type == "cuda" and device.index is None:
        return torch.device("cuda", torch.cuda.current_device())
    return device


def _stream(device) -> c_void_p:
    return c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _aligned_workspace(nbytes: int, device) -> torch.Tensor:
    # torch's caching allocator returns 512-byte aligned blocks
    t = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)
    assert t.data_ptr() % WORKSPACE_ALIGN == 0
    return t


# The handle of a device's current stream by its index: torch's own short cut for launchers,
# where it has one (a Stream object costs 2 us, a third of a small call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(fn, where, device, args):
    """fn(*args, current stream of device), with that device the current one."""
    index = device.index
    if index == torch.cuda.current_device():
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status != 0:
        raise SplaError(status, where)


def _row_stride(x: torch.Tensor, row: int) -> int:
    """Elements between the rows (t, b), (t, b + 1) of x [T, batch, heads, d] or [batch, heads,
    d], whose heads and coordinates lie one after the other (row of them) and whose rows are
    evenly spaced."""
    if x.is_contiguous():
        return row
    b, h, d = x.shape[-3:]
    T = x.shape[0] if x.dim() == 4 else 1
    row = x.stride(-3) if b > 1 else x.stride(0) if T > 1 else row
    ok = x.stride(-1) == 1 and (h == 1 or x.stride(-2) == d)
    if not ok or (b > 1 and T > 1 and x.stride(0) != b * row):
        raise ValueError("rows of heads one after the other, evenly spaced, are needed")
    return row


def _rows(name, x, y, shape, dtype, device):
    """y, or a new output of the rows x, with the addresses and row strides of both: (y, x's
    address, x's stride, y's address, y's stride)."""
    if x.shape != shape or x.dtype is not dtype or x.device != device:
        raise ValueError(f"{name}: a {dtype} tensor {list(shape)} is needed, T and the device the "
                         "same for q and k")
    if (x.requires_grad or y is not None and y.requires_grad) and torch.is_grad_enabled():
        raise ValueError(f"{name}: no gradient is recorded here (detach it, or torch.no_grad(); "
                         "transpose=True is the gradient's map)")
    row = shape[-2] * shape[-1]
    at, stride = x.data_ptr(), _row_stride(x, row)
    if y is x:
        return y, at, stride, at, stride
    if y is None:
        y = torch.empty(shape, dtype=dtype, device=device)
    elif y.shape != shape or y.dtype is not dtype or y.device != device:
        raise ValueError(f"{name}_out: a {dtype} tensor like {name} is needed")
    return y, at, stride, y.data_ptr(), _row_stride(y, row)


def _row_words(name, t, shape, device):
    """The address of the int32 values t, one per row or sequence."""
    if t.shape != shape or t.dtype is not torch.int32 or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name}: a contiguous int32 tensor {list(shape)} on the rows' device is "
                         "needed")
    return t.data_ptr()


# A write to tensors of a list, as torch.autograd.graph.increment_version counts it (which takes as
# long again to look at its argument).
_count_writes = getattr(torch._C, "_increment_version", None) or (
    torch.autograd.graph.increment_version)


def _written(a, b):
    """Counts a write to a and to b (or None), memory that the caller handed in for results:
    products that kept it, under whatever name, then refuse their backward passes."""
    if a is not None:
        _count_writes((a,) if b is None else (a, b))
    elif b is not None:
        _count_writes((b,))


def rotate(cfg: SplaConfig, rope: SplaRope, q=None, k=None, positions=None, seq_lens=None,
           q_out=None, k_out=None, transpose=False):
    """Rotates q [T, batch, Hq, d] and / or k [T, batch, Hkv, d] (or without T: one position)
    into q_out, k_out (new tensors by default; q_out=q rotates in place) and returns the two.
    Rows may be slices of wider ones (a fused projection's). positions int32 [T, batch] (rows
    without T: [batch] too); without it row (t, b) stands at seq_lens[b] + t (seq_lens int32
    [batch], or zeros). transpose: the transposed map (the gradient); nothing is recorded for
    autograd, and rows that it would record are refused."""
    x = k if q is None else q
    if x is None or (q is None and q_out is not None) or (k is None and k_out is not None):
        raise ValueError("q or k is needed, and no output without its input")
    given = q_out, k_out
    n, batch, d, device, dtype = x.dim(), cfg.batch, cfg.head_dim, x.device, torch_dtype(cfg)
    if n not in (3, 4):
        raise ValueError(f"rows of [T, {batch}] or [{batch}] positions are needed")
    T = x.shape[0] if n == 4 else 1
    lead = (T, batch) if n == 4 else (batch,)
    qp = qs = op = os_ = kp = ks = tp = ts = 0
    if q is not None:
        q_out, qp, qs, op, os_ = _rows("q", q, q_out, lead + (cfg.n_q_heads, d), dtype, device)
    if k is not None:
        k_out, kp, ks, tp, ts = _rows("k", k, k_out, lead + (cfg.n_kv_heads, d), dtype, device)
    at = None
    if positions is not None:
        at = _row_words("positions", positions, (T, batch) if positions.dim() == 2 else lead, device)
    lens = None if seq_lens is None else _row_words("seq_lens", seq_lens, (batch,), device)
    if device.type != "cuda":
        raise ValueError("tensors on a GPU are needed")
    _launch(lib().spla_rotate, "spla_rotate", device,
            (ctypes.byref(cfg), ctypes.byref(rope), T, at, lens, qp, qs, op, os_, kp, ks, tp, ts,
             1 if transpose else 0))
    _written(*given)
    return q_out, k_out


def _rotated_rows(cfg, q, k, positions, seq_lens):
    """What the calls that rotate rows have in common: (T, the rows' leading sizes, d, dtype,
    device, address of positions, of seq_lens)."""
    x = k if q is None else q
    if x is None:
        raise ValueError("q or k is needed")
    shape, batch, device = x.shape, cfg.batch, x.device
    n = len(shape)
    if n == 4:
        T = shape[0]
        lead = (T, batch)
    elif n == 3:
        T, lead = 1, (batch,)
    else:
        raise ValueError(f"rows of [T, {batch}] or [{batch}] positions are needed")
    at = lens = None
    if positions is not None:
        at = _row_words("positions", positions, (T, batch) if positions.dim() == 2 else lead, device)
    if seq_lens is not None:
        lens = _row_words("seq_lens", seq_lens, (batch,), device)
    if device.type != "cuda":
        raise ValueError("tensors on a GPU are needed")
    return T, lead, cfg.head_dim, torch_dtype(cfg), device, at, lens


def _head_weight(name, w, heads, d, device):
    """The address of a weight, and whether it is one per head; checked."""
    shape = w.shape
    per_head = len(shape) == 2
    if (w.dtype is not torch.float32 or (shape != (heads, d) if per_head else shape != (d,))
            or not w.is_contiguous() or w.device != device):
        raise ValueError(f"{name}: a contiguous fp32 tensor [{d}] or [{heads}, {d}] on the rows' "
                         "device is needed")
    if w.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{name}: no gradient is recorded here (detach it, or torch.no_grad(); "
                         "norm_rotate_grad gives it)")
    return w.data_ptr(), per_head


def _head_weights(cfg, q_weight, k_weight, d, device):
    """Whether the weights are one per head, and their addresses."""
    qw = kw = qh = kh = None
    if q_weight is not None:
        qw, qh = _head_weight("q_weight", q_weight, cfg.n_q_heads, d, device)
    if k_weight is not None:
        kw, kh = _head_weight("k_weight", k_weight, cfg.n_kv_heads, d, device)
    if qh is not None and kh is not None and qh is not kh:
        raise ValueError("q_weight and k_weight: a weight per head for both, or one for all heads")
    return 1 if qh or kh else 0, qw, kw


def _unrecorded(a, b, c=None, d=None):
    """Refuses rows, and memory for results, that autograd would record (or None)."""
    if ((a is not None and a.requires_grad or b is not None and b.requires_grad
         or c is not None and c.requires_grad or d is not None and d.requires_grad)
            and torch.is_grad_enabled()):
        raise ValueError("no gradient is recorded here (detach the rows, or torch.no_grad())")


def norm_rotate(cfg: SplaConfig, rope: SplaRope, q=None, k=None, q_weight=None, k_weight=None,
                eps=1e-6, positions=None, seq_lens=None, q_out=None, k_out=None):
    """rotate() of rows whose heads are normed first: x / sqrt(mean(x^2) + eps) times the weight
    (fp32, [d] for all heads or [Hq, d] and [Hkv, d]; None: ones). Rows, positions and outputs as
    rotate() takes them; nothing is recorded for autograd (norm_rotate_grad gives the
    gradients)."""
    if (q is None and q_out is not None) or (k is None and k_out is not None):
        raise ValueError("no output without its input")
    given = q_out, k_out
    T, lead, d, dtype, device, at, lens = _rotated_rows(cfg, q, k, positions, seq_lens)
    qp = qs = op = os_ = kp = ks = tp = ts = 0
    if q is not None:
        q_out, qp, qs, op, os_ = _rows("q", q, q_out, lead + (cfg.n_q_heads, d), dtype, device)
    if k is not None:
        k_out, kp, ks, tp, ts = _rows("k", k, k_out, lead + (cfg.n_kv_heads, d), dtype, device)
    per_head, qw, kw = _head_weights(cfg, q_weight, k_weight, d, device)
    _launch(lib().spla_norm_rotate, "spla_norm_rotate", device,
            (ctypes.byref(cfg), ctypes.byref(rope), T, at, lens, qw, kw, per_head, eps, qp, qs, op,
             os_, kp, ks, tp, ts))
    _written(*given)
    return q_out, k_out


def norm_rotate_grad(cfg: SplaConfig, rope: SplaRope, q=None, k=None, q_grad=None, k_grad=None,
                     q_weight=None, k_weight=None, eps=1e-6, positions=None, seq_lens=None,
                     q_out=None, k_out=None):
    """Gradients of norm_rotate(cfg, rope, q, k, ...) from those of its results, q_grad and k_grad
    (laid out like q and k, with row strides of their own): (with respect to q, to k, to
    q_weight, to k_weight), None for what was not given. q_out, k_out: where the first two go (new
    tensors by default; the rows' or the gradients' own are allowed); the weights' are new fp32
    tensors, sums over the rows (and the heads that share a weight)."""
    if ((q is None) != (q_grad is None) or (k is None) != (k_grad is None)
            or (q is None and (q_out is not None or q_weight is not None))
            or (k is None and (k_out is not None or k_weight is not None))):
        raise ValueError("rows and their gradients go together, outputs and weights with them")
    T, lead, d, dtype, device, at, lens = _rotated_rows(cfg, q, k, positions, seq_lens)
    per_head, qw, kw = _head_weights(cfg, q_weight, k_weight, d, device)
    args, outs = [], []
    for name, x, g, y, h in (("q", q, q_grad, q_out, cfg.n_q_heads),
                             ("k", k, k_grad, k_out, cfg.n_kv_heads)):
        if x is None:
            args += [0] * 6
            outs.append(None)
            continue
        shape = lead + (h, d)
        y, xp, xs, yp, ys = _rows(name, x, y, shape, dtype, device)
        _, gp, gs, _, _ = _rows(f"{name}_grad", g, g, shape, dtype, device)
        args += [xp, xs, gp, gs, yp, ys]
        outs.append(y)
    qwg, kwg = (None if w is None else torch.empty_like(w) for w in (q_weight, k_weight))
    ws = None
    if qwg is not None or kwg is not None:
        ws = _aligned_workspace(norm_rotate_grad_workspace_bytes(cfg, T), device)
    _launch(lib().spla_norm_rotate_grad, "spla_norm_rotate_grad", device,
            (ctypes.byref(cfg), ctypes.byref(rope), T, at, lens, qw, kw, per_head, eps, *args,
             None if qwg is None else qwg.data_ptr(), None if kwg is None else kwg.data_ptr(),
             None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel()))
    _written(q_out, k_out)
    return outs[0], outs[1], qwg, kwg


class _DeviceCache:
    """What the caches have in common: the error word, workspaces, checks."""

    _outgrown: list  # workspaces that captured graphs name
    _ws_sizes: dict

    def device_errors(self) -> int:
        """The SPLA_DEVERR_* bits the device has set in this cache's error
        word (waits for the work queued on the current stream)."""
        return int(self.err.item())

    def clear_device_errors(self):
        self.err.zero_()

    def check_device_errors(self, allowed: int = 0):
        """Raises SplaError when a bit outside `allowed` is set: after a
        SPLA_DEVERR_SYNC the outputs of the call that set it are undefined."""
        e = self.device_errors()
        if e & ~allowed:
            names = [n for n, v in (("CAPACITY", DEVERR_CAPACITY), ("SYNC", DEVERR_SYNC),
                                    ("PAGE", DEVERR_PAGE)) if e & v]
            raise SplaError(-5, "device error word: " + "|".join(names))

    def _workspace(self, kind, n, sizes, ws):
        """The workspace ws, or a larger one in its place (zeros: its counters), for a call of
        n tokens; the sizes of earlier calls are remembered. It grows by half at least, so that
        calls that get longer one by one seldom make a new one, and one that a capture has used
        is kept."""
        need = self._ws_sizes.get((kind, n))
        if need is None:
            need = self._ws_sizes[kind, n] = sizes(self.cfg, n)
        capturing = torch.cuda.is_current_stream_capturing()
        if ws is None or ws.numel() < need:
            if capturing:  # its zeros would come with a replay only
                raise RuntimeError("a capture needs a call of its sizes ahead of it, which makes "
                                   "the workspace")
            if ws is not None:
                need = max(need, ws.numel() * 3 // 2)
                if ws.is_cuda:  # calls on this stream, not its own, may still use it
                    ws.record_stream(torch.cuda.current_stream(ws.device))
            ws = _aligned_workspace(need, self.device).zero_()
        elif capturing and not any(ws is kept for kept in self._outgrown):
            self._outgrown.append(ws)
        return ws

    def _given(self, name, t, shape, dtype):
        """The address of t, checked."""
        if (t.shape != shape or t.dtype is not dtype or not t.is_contiguous()
                or t.device != self.device):
            raise ValueError(f"{name}: a contiguous {dtype} tensor {list(shape)} on the cache's "
                             "device is needed")
        return t.data_ptr()

    def _attend_args(self, opts, q, out, lse, softcap, slopes, first_key, prefix_len, n_new):
        """Checked arguments of attend(): (T, address of q, out, its address, lse, its address);
        fills opts, a zero-filled SplaAttendOpts."""
        c, shape, dtype = self.cfg, q.shape, torch_dtype(self.cfg)
        if len(shape) not in (3, 4):
            raise ValueError("q: [T, batch, Hq, d] is needed")
        T = shape[0] if len(shape) == 4 else 1
        lead = (T, c.batch) if len(shape) == 4 else (c.batch,)
        qp = self._given("q", q, lead + (c.n_q_heads, c.head_dim), dtype)
        new = torch.empty if n_new is None else torch.zeros
        if out is None:
            out = new(shape, dtype=dtype, device=q.device)
        if lse is None:
            lse = new(shape[:-1], dtype=torch.float32, device=q.device)
        op = self._given("out", out, shape, dtype)
        lp = self._given("lse", lse, shape[:-1], torch.float32)
        opts.softcap = softcap
        if slopes is not None:
            opts.slopes = self._given("slopes", slopes, (c.n_q_heads,), torch.float32)
        if first_key is not None:
            opts.first_key = self._given("first_key", first_key, lead, torch.int32)
        if prefix_len is not None:
            opts.prefix_len = self._given("prefix_len", prefix_len, (c.batch,), torch.int32)
        if n_new is not None:
            opts.n_new = self._given("n_new", n_new, (c.batch,), torch.int32)
        return T, qp, out, op, lse, lp


class SplaCache(_DeviceCache):
    """Device buffers of one SPLA cache, allocated with torch, plus the
    workspaces the calls need. Thin wrapper over the C ABI."""

    def __init__(self, cfg: SplaConfig, device="cuda", block_table: Optional[torch.Tensor] = None):
        """block_table: int32 [batch, max_seq_len / block_size] on the device,
        page of each block, required when cfg.kv_pages > 0 (paged pool)."""
        self.cfg = cfg
        self.device = _indexed(device)
        if (cfg.kv_pages > 0) != (block_table is not None):
            raise ValueError("a block table goes with kv_pages > 0, and only then")
        if block_table is not None:
            assert block_table.dtype == torch.int32 and block_table.is_contiguous()
            assert block_table.shape == (cfg.batch, cfg.max_seq_len // cfg.block_size)
            assert block_table.device == self.device
        self.block_table = block_table
        sz = cache_bytes(cfg)
        dt = torch_dtype(cfg)
        e = 4 if cfg.dtype == F32 else 2
        self.k = torch.zeros(sz[0] // e, dtype=dt, device=self.device)
        self.v = torch.zeros(sz[1] // e, dtype=dt, device=self.device)
        self.stats = torch.zeros(sz[2] // 4, dtype=torch.float32, device=self.device)
        self.state = torch.zeros(sz[3] // 4, dtype=torch.float32, device=self.device)
        self.norm = torch.zeros(sz[4] // 4, dtype=torch.float32, device=self.device)
        self.seq_lens = torch.zeros(cfg.batch, dtype=torch.int32, device=self.device)
        self.err = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.workspace = _aligned_workspace(workspace_bytes(cfg), self.device)
        _check(lib().spla_workspace_init(ctypes.byref(cfg), _ptr(self.workspace),
                                         self.workspace.numel(), _stream(self.device)),
               "spla_workspace_init")
        self._append_ws = None
        self._prefill_ws = None
        self._rope_ws = None
        self._attend_ws = None
        self._outgrown = []  # workspaces that captured graphs name
        self._ws_sizes = {}
        self._struct = SplaCacheStruct(self.k.data_ptr(), self.v.data_ptr(),
                                       self.stats.data_ptr(), self.state.data_ptr(),
                                       self.norm.data_ptr(), self.seq_lens.data_ptr(),
                                       self.err.data_ptr(),
                                       None if block_table is None else block_table.data_ptr())

    @property
    def struct(self) -> SplaCacheStruct:
        return self._struct

    def reset(self):
        _check(lib().spla_reset(ctypes.byref(self.cfg), ctypes.byref(self._struct),
                                _stream(self.device)), "spla_reset")

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor,
               n_new: Optional[torch.Tensor] = None):
        """k_new, v_new: [batch, Hkv, max_new, d] in the cache dtype."""
        c = self.cfg
        assert k_new.shape == v_new.shape and k_new.dim() == 4
        assert k_new.shape[0] == c.batch and k_new.shape[1] == c.n_kv_heads
        assert k_new.shape[3] == c.head_dim
        assert k_new.dtype == torch_dtype(c) and v_new.dtype == torch_dtype(c)
        assert k_new.is_contiguous() and v_new.is_contiguous()
        max_new = int(k_new.shape[2])
        need = append_workspace_bytes(c, max_new)
        if self._append_ws is None or self._append_ws.numel() < need:
            self._append_ws = _aligned_workspace(need, self.device)
        if n_new is not None:
            assert n_new.dtype == torch.int32 and n_new.numel() == c.batch and n_new.is_contiguous()
        _check(lib().spla_append(ctypes.byref(c), ctypes.byref(self._struct), _ptr(k_new),
                                 _ptr(v_new), max_new, _ptr(n_new), _ptr(self._append_ws),
                                 self._append_ws.numel(), _stream(self.device)), "spla_append")

    def _decode_args(self, q, gamma, out, sel):
        c = self.cfg
        assert q.shape == (c.batch, c.n_q_heads, c.head_dim) and q.dtype == torch_dtype(c)
        assert q.is_contiguous()
        assert gamma.shape == (c.n_q_heads, c.head_dim) and gamma.dtype == torch.float32
        assert gamma.is_contiguous()
        if out is None:
            out = torch.empty_like(q)
        if sel is None:
            sel = torch.empty((c.batch, c.n_kv_heads, c.top_k), dtype=torch.int32,
                              device=self.device)
        return out, sel

    def decode(self, q: torch.Tensor, gamma: torch.Tensor, out=None, sel=None, events=None):
        """q [batch, Hq, d] (cache dtype), gamma [Hq, d] fp32 -> (out, sel)."""
        out, sel = self._decode_args(q, gamma, out, sel)
        ev = None if events is None else ctypes.byref(events)
        _check(lib().spla_decode_ex(ctypes.byref(self.cfg), ctypes.byref(self._struct), _ptr(q),
                                    _ptr(gamma), _ptr(out), _ptr(sel), _ptr(self.workspace),
                                    self.workspace.numel(), ev, _stream(self.device)),
               "spla_decode")
        return out, sel

    def decode_noalloc(self, q: torch.Tensor, gamma: torch.Tensor, out, sel=None):
        """spla_decode_noalloc: the decode on the library's own device scratch
        (no workspace); out must be given (nothing is allocated here either)."""
        c = self.cfg
        assert q.shape == (c.batch, c.n_q_heads, c.head_dim) and q.dtype == torch_dtype(c)
        assert gamma.shape == (c.n_q_heads, c.head_dim) and gamma.dtype == torch.float32
        assert out is not None and out.shape == q.shape and out.dtype == q.dtype
        assert q.is_contiguous() and gamma.is_contiguous() and out.is_contiguous()
        if sel is not None:
            assert sel.shape == (c.batch, c.n_kv_heads, c.top_k) and sel.dtype == torch.int32
            assert sel.is_contiguous()
        _check(lib().spla_decode_noalloc(ctypes.byref(c), ctypes.byref(self._struct), _ptr(q),
                                         _ptr(gamma), _ptr(out), _ptr(sel),
                                         _stream(self.device)), "spla_decode_noalloc")
        return out, sel

    def step(self, k_new, v_new, q, gamma, out=None, sel=None, events=None):
        """Append one token per (sequence, KV head) ([batch, Hkv, d]), then decode."""
        c = self.cfg
        assert k_new.shape == (c.batch, c.n_kv_heads, c.head_dim) and k_new.is_contiguous()
        assert v_new.shape == k_new.shape and v_new.is_contiguous()
        assert k_new.dtype == torch_dtype(c) and v_new.dtype == torch_dtype(c)
        out, sel = self._decode_args(q, gamma, out, sel)
        ev = None if events is None else ctypes.byref(events)
        _check(lib().spla_step_ex(ctypes.byref(c), ctypes.byref(self._struct), _ptr(k_new),
                                  _ptr(v_new), _ptr(q), _ptr(gamma), _ptr(out), _ptr(sel),
                                  _ptr(self.workspace), self.workspace.numel(), ev,
                                  _stream(self.device)), "spla_step")
        return out, sel

    def prefill(self, k_new, v_new, q, gamma, out=None, sel=None, events=None):
        """Causal prefill of T tokens per sequence: k_new, v_new [T, batch,
        Hkv, d], q [T, batch, Hq, d] (cache dtype) -> out [T, batch, Hq, d],
        sel [T, batch, Hkv, top_k]; position t is appended, then decoded."""
        c = self.cfg
        T = k_new.shape[0]
        assert k_new.shape == (T, c.batch, c.n_kv_heads, c.head_dim) and k_new.is_contiguous()
        assert v_new.shape == k_new.shape and v_new.is_contiguous()
        assert k_new.dtype == torch_dtype(c) and v_new.dtype == torch_dtype(c)
        assert q.shape == (T, c.batch, c.n_q_heads, c.head_dim) and q.dtype == torch_dtype(c)
        assert q.is_contiguous()
        assert gamma.shape == (c.n_q_heads, c.head_dim) and gamma.dtype == torch.float32
        if out is None:
            out = torch.empty_like(q)
        if sel is None:
            sel = torch.empty((T, c.batch, c.n_kv_heads, c.top_k), dtype=torch.int32,
                              device=self.device)
        need = prefill_workspace_bytes(c, T)
        if self._prefill_ws is None or self._prefill_ws.numel() < need:
            self._prefill_ws = _aligned_workspace(need, self.device)
        ws = self._prefill_ws
        ev = None if events is None else ctypes.byref(events)
        _check(lib().spla_prefill_ex(ctypes.byref(c), ctypes.byref(self._struct), int(T),
                                     _ptr(k_new), _ptr(v_new), _ptr(q), _ptr(gamma), _ptr(out),
                                     _ptr(sel), _ptr(ws), ws.numel(), ev,
                                     _stream(self.device)), "spla_prefill")
        return out, sel

    def rotate(self, rope: SplaRope, q=None, k=None, positions=None, q_out=None, k_out=None,
               transpose=False):
        """rotate() of rows that stand at the positions after the tokens the cache holds (the
        queries and keys that the next append, step or prefill brings), or at `positions`."""
        return rotate(self.cfg, rope, q, k, positions, None if positions is not None
                      else self.seq_lens, q_out, k_out, transpose)

    def append_rope(self, rope: SplaRope, k_new: torch.Tensor, v_new: torch.Tensor,
                    n_new: Optional[torch.Tensor] = None,
                    pos_shift: Optional[torch.Tensor] = None):
        """append() with the keys rotated on the way, the token that lands at position p of the
        cache by the angles of p (+ pos_shift[b], int32 [batch]). Ahead of a graph capture a
        call of the same max_new makes the workspace."""
        c = self.cfg
        if k_new.dim() != 4:
            raise ValueError("k_new: [batch, Hkv, max_new, d] is needed")
        max_new = k_new.shape[2]
        shape, dtype = (c.batch, c.n_kv_heads, max_new, c.head_dim), torch_dtype(c)
        kp = self._given("k_new", k_new, shape, dtype)
        vp = self._given("v_new", v_new, shape, dtype)
        np_ = None if n_new is None else self._given("n_new", n_new, (c.batch,), torch.int32)
        sp = (None if pos_shift is None
              else self._given("pos_shift", pos_shift, (c.batch,), torch.int32))
        ws = self._rope_ws = self._workspace(
            ("rope", rope.head_dim, rope.rot_dim), max_new,
            lambda cfg, n: append_rope_workspace_bytes(cfg, n, rope=rope), self._rope_ws)
        _launch(lib().spla_append_rope, "spla_append_rope", self.device,
                (ctypes.byref(c), ctypes.byref(self._struct), ctypes.byref(rope), kp, vp, max_new,
                 np_, sp, ws.data_ptr(), ws.numel()))

    def attend(self, q: torch.Tensor, out=None, lse=None, softcap=0.0, slopes=None,
               first_key=None, prefix_len=None, n_new=None):
        """Exact attention of the last T tokens of every sequence over the cache, which holds
        them already: q [T, batch, Hq, d] (or [batch, Hq, d]: one token) -> (out, lse), lse
        fp32 [T, batch, Hq] (natural logarithm). softcap: scores x become softcap
        tanh(x / softcap). slopes fp32 [Hq]: slopes[m] |p - j| is subtracted. first_key int32
        [T, batch]: the first position each query sees. prefix_len int32 [batch]: positions
        every query sees. n_new int32 [batch]: the queries each sequence really has; the
        rows of out and lse past them are left as they are (zeros in tensors made here). Ahead
        of a graph capture a call of the same T makes the workspace."""
        opts = SplaAttendOpts()
        T, qp, out, op, lse, lp = self._attend_args(opts, q, out, lse, softcap, slopes, first_key,
                                                    prefix_len, n_new)
        ws = self._attend_ws = self._workspace("attend", T, attend_workspace_bytes,
                                               self._attend_ws)
        _launch(lib().spla_attend, "spla_attend", self.device,
                (ctypes.byref(self.cfg), ctypes.byref(self._struct), T, qp, ctypes.byref(opts), op,
                 lp, ws.data_ptr(), ws.numel()))
        _count_writes((out, lse))
        return out, lse

    def norm_rotate(self, rope: SplaRope, q=None, k=None, q_weight=None, k_weight=None, eps=1e-6,
                    positions=None, q_out=None, k_out=None):
        """norm_rotate() of rows that stand at the positions after the tokens the cache holds, or
        at `positions`."""
        return norm_rotate(self.cfg, rope, q, k, q_weight, k_weight, eps, positions,
                           None if positions is not None else self.seq_lens, q_out, k_out)

    # ---- layout views (for checks; pure indexing) ----
    def stats_logical(self):
        """(mean, M2) as [batch, Hkv, n_units, d] fp32 tensors: one unit per
        block, or per selection window with strided selection."""
        c = self.cfg
        nb = c.max_seq_len // (c.sel_stride if c.sel_stride else c.block_size)
        nt = -(-nb // 64)
        s = self.stats.view(c.batch, c.n_kv_heads, nt, 2, c.head_dim // 4, 64, 4)
        s = s.permute(0, 1, 3, 2, 5, 4, 6).reshape(c.batch, c.n_kv_heads, 2, nt * 64, c.head_dim)
        return s[:, :, 0, :nb], s[:, :, 1, :nb]

    def _per_sequence(self, pool):
        """A K or V buffer in the per-sequence layout ([batch][Hkv][nb][B d]):
        the buffer itself, or the pages of a paged pool gathered through the
        block table (entries outside the pool give zeros)."""
        c = self.cfg
        if c.kv_pages == 0:
            return pool
        bd = c.block_size * c.head_dim
        pages = pool.view(c.kv_pages, c.n_kv_heads, bd)
        tab = self.block_table.long()
        ok = (tab >= 0) & (tab < c.kv_pages)
        g = pages[tab.clamp(0, c.kv_pages - 1)] * ok[..., None, None].to(pool.dtype)
        return g.permute(0, 2, 1, 3).contiguous().view(-1)

    def k_logical(self):
        """Keys as [batch][Hkv][max_seq_len][d] (undoing the bf16 step order)."""
        c = self.cfg
        B, H, T, d = c.batch, c.n_kv_heads, c.max_seq_len, c.head_dim
        kbuf = self._per_sequence(self.k)
        if c.dtype == F32:
            return kbuf.view(B, H, T, d)
        # step chunk (mt, ks, g, a, b) holds token 8a + 4mt + b, coordinates 32ks + 8g ..
        k = kbuf.view(B, H, T // 32, 2, d // 32, 4, 4, 4, 8)
        return k.permute(0, 1, 2, 6, 3, 7, 4, 5, 8).reshape(B, H, T, d)

    def v_logical(self):
        """Values as [batch][Hkv][max_seq_len][d] (undoing the block transpose
        of fp32 caches and the step order of bf16 ones)."""
        c = self.cfg
        B, H, T, d = c.batch, c.n_kv_heads, c.max_seq_len, c.head_dim
        vbuf = self._per_sequence(self.v)
        if c.dtype == F32:
            v = vbuf.view(B, H, T // c.block_size, d, c.block_size)
            return v.permute(0, 1, 2, 4, 3).reshape(B, H, T, d)
        # step chunk (t, g, i) holds coordinate 16t + i, tokens 8g .. 8g + 7
        v = vbuf.view(B, H, T // 32, d // 16, 4, 16, 8)
        return v.permute(0, 1, 2, 4, 6, 3, 5).reshape(B, H, T, d)

    def state_logical(self):
        c = self.cfg
        return (self.state.view(c.batch, c.n_kv_heads, c.head_dim, c.head_dim),
                self.norm.view(c.batch, c.n_kv_heads, c.head_dim))


class SplaCache8(_DeviceCache):
    """Device buffers of one 8-bit cache for exact attention (codes, a power of two per block and
    KV head, lengths), allocated with torch. Thin wrapper over the C ABI."""

    def __init__(self, cfg: SplaConfig, device="cuda", block_table: Optional[torch.Tensor] = None):
        """block_table: int32 [batch, max_seq_len / block_size] on the device, page of each block,
        required when cfg.kv_pages > 0 (paged pool)."""
        self.cfg = cfg
        self.device = _indexed(device)
        if (cfg.kv_pages > 0) != (block_table is not None):
            raise ValueError("a block table goes with kv_pages > 0, and only then")
        sz = cache8_bytes(cfg)
        self.seq_lens = torch.zeros(cfg.batch, dtype=torch.int32, device=self.device)
        if block_table is not None:
            self._given("block_table", block_table,
                        (cfg.batch, cfg.max_seq_len // cfg.block_size), torch.int32)
        self.block_table = block_table
        self.k = torch.zeros(sz[0], dtype=torch.uint8, device=self.device)
        self.v = torch.zeros(sz[1], dtype=torch.uint8, device=self.device)
        self.scales = torch.zeros(sz[2] // 4, dtype=torch.float32, device=self.device)
        self.counters = torch.zeros(sz[4] // 4, dtype=torch.int32, device=self.device)
        self.err = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._attend_ws = None
        self._outgrown = []
        self._ws_sizes = {}
        self._struct = SplaCache8Struct(self.k.data_ptr(), self.v.data_ptr(),
                                        self.scales.data_ptr(), self.seq_lens.data_ptr(),
                                        self.counters.data_ptr(), self.err.data_ptr(),
                                        None if block_table is None else block_table.data_ptr())
        self._refs = (ctypes.byref(self.cfg), ctypes.byref(self._struct))
        self._dtype = torch_dtype(cfg)
        self._heads = (cfg.batch, cfg.n_kv_heads, cfg.head_dim)  # of a position's rows
        self._batch = (cfg.batch,)
        self._row = cfg.n_kv_heads * cfg.head_dim

    @property
    def struct(self) -> SplaCache8Struct:
        return self._struct

    def reset(self):
        _launch(lib().spla_reset8, "spla_reset8", self.device, self._refs)

    def _new_rows(self, name, x, shape):
        """Address and row stride of new rows, checked."""
        if x.shape != shape or x.dtype is not self._dtype or x.device != self.device:
            raise ValueError(f"{name}: a {self._dtype} tensor {list(shape)} on the cache's device "
                             "is needed")
        return x.data_ptr(), _row_stride(x, self._row)

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor,
               n_new: Optional[torch.Tensor] = None):
        """k_new, v_new: [T, batch, Hkv, d] (or [batch, Hkv, d]: one token) in the cfg's dtype, as
        norm_rotate() and rotate() give them; rows may be slices of wider ones (a fused
        projection's). n_new int32 [batch]: the tokens each sequence really has. Nothing here is
        recorded for autograd, and tensors that it would record are refused by all calls."""
        n = k_new.dim()
        if n not in (3, 4):
            raise ValueError("k_new: [T, batch, Hkv, d] is needed")
        if k_new.requires_grad or v_new.requires_grad:
            _unrecorded(k_new, v_new)
        T = k_new.shape[0] if n == 4 else 1
        shape = (T,) + self._heads if n == 4 else self._heads
        kp, ks = self._new_rows("k_new", k_new, shape)
        vp, vs = self._new_rows("v_new", v_new, shape)
        np_ = None if n_new is None else self._given("n_new", n_new, self._batch, torch.int32)
        _launch(lib().spla_append8, "spla_append8", self.device,
                self._refs + (T, kp, ks, vp, vs, np_))

    def read(self, n_tokens: int, first: Optional[torch.Tensor] = None, k_out=None, v_out=None):
        """Keys and values [n_tokens, batch, Hkv, d], the numbers the cache holds of the tokens at
        positions first[b] + t (first int32 [batch], or 0); zeros where a sequence holds none."""
        if n_tokens < 0:
            raise ValueError("n_tokens: a count is needed")
        shape, dtype = (int(n_tokens),) + self._heads, self._dtype
        if k_out is None:
            k_out = torch.empty(shape, dtype=dtype, device=self.device)
        if v_out is None:
            v_out = torch.empty(shape, dtype=dtype, device=self.device)
        if k_out.requires_grad or v_out.requires_grad:
            _unrecorded(k_out, v_out)
        kp = self._given("k_out", k_out, shape, dtype)
        vp = self._given("v_out", v_out, shape, dtype)
        fp = None if first is None else self._given("first", first, self._batch, torch.int32)
        _launch(lib().spla_read8, "spla_read8", self.device, self._refs + (shape[0], fp, kp, vp))
        _count_writes((k_out, v_out))
        return k_out, v_out

    def rotate(self, rope: SplaRope, q=None, k=None, positions=None, q_out=None, k_out=None,
               transpose=False):
        """rotate() of rows that stand at the positions after the tokens the cache holds, or at
        `positions`."""
        return rotate(self.cfg, rope, q, k, positions, None if positions is not None
                      else self.seq_lens, q_out, k_out, transpose)

    def norm_rotate(self, rope: SplaRope, q=None, k=None, q_weight=None, k_weight=None, eps=1e-6,
                    positions=None, q_out=None, k_out=None):
        """norm_rotate() of rows that stand at the positions after the tokens the cache holds, or
        at `positions`."""
        return norm_rotate(self.cfg, rope, q, k, q_weight, k_weight, eps, positions,
                           None if positions is not None else self.seq_lens, q_out, k_out)

    def attend(self, q: torch.Tensor, out=None, lse=None, softcap=0.0, slopes=None,
               first_key=None, prefix_len=None, n_new=None, window=0, sinks=0):
        """Exact attention of the last T tokens of every sequence over the cache, as
        SplaCache.attend; window > 0: the query at position p sees the keys after p - window, and
        beside them the first `sinks` of the sequence (from first_key on where it is given)."""
        _unrecorded(q, out, lse, slopes)
        opts = SplaAttend8Opts()
        T, qp, out, op, lse, lp = self._attend_args(opts.attend, q, out, lse, softcap, slopes,
                                                    first_key, prefix_len, n_new)
        if not (0 <= window < 1 << 31 and 0 <= sinks < 1 << 31):
            raise ValueError("window and sinks: counts of tokens are needed")
        opts.window, opts.sinks = window, sinks
        ws = self._attend_ws = self._workspace("attend8", T, attend8_workspace_bytes,
                                               self._attend_ws)
        _launch(lib().spla_attend8, "spla_attend8", self.device,
                self._refs + (T, qp, ctypes.byref(opts), op, lp, ws.data_ptr(), ws.numel()))
        _count_writes((out, lse))
        return out, lse


def make_events(phases: Sequence[str] = ("score", "select", "sparse", "merge", "decode",
                                        "append")):
    """torch.cuda.Event pairs for the given phases, and the SplaEvents that
    points at their HIP events. Returns (events_struct, {phase: (start, stop)})."""
    ev = SplaEvents()
    pairs = {}
    for name in phases:
        p = PHASES[name]
        a = torch.cuda.Event(enable_timing=True)
        b = torch.cuda.Event(enable_timing=True)
        a.record()
        b.record()   # materialise the underlying events
        ev.start[p] = c_void_p(a.cuda_event)
        ev.stop[p] = c_void_p(b.cuda_event)
        pairs[name] = (a, b)
    return ev, pairs

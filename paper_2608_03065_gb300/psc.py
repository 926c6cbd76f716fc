"""Thin Python binding of the PSC C ABI (include/psc.h, psc_ops.h, psc_mx4.h, psc_norm.h): argument marshalling only.

Every function here converts its arguments (torch tensors -> device pointers,
torch streams -> cudaStream_t) and calls the library function of the same
name; all work runs in the library's CUDA kernels.  There is no fallback: if
``libpsc_gb300.so`` is missing or fails to load, every call raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpsc_gb300.so")

PSC_F32, PSC_BF16 = 0, 1
ROW_OK, ROW_DONE, ROW_REJECTED, ROW_OVERFLOW, ROW_LIMIT = 0, 1, 2, 3, 4
STATUS_NAMES = {0: "PSC_OK", 1: "PSC_ERR_ARG", 2: "PSC_ERR_GRAMMAR", 3: "PSC_ERR_CONFLICT",
                4: "PSC_ERR_LEXER_AMBIGUOUS", 5: "PSC_ERR_LIMIT", 6: "PSC_ERR_OOM", 7: "PSC_ERR_CUDA",
                8: "PSC_ERR_IO"}

EXPORTED = ["psc_compile", "psc_destroy", "psc_last_error", "psc_info", "psc_state_init", "psc_state_reset",
            "psc_state_destroy", "psc_advance", "psc_fill_mask", "psc_apply_mask", "psc_fill_apply",
            "psc_argmax_masked", "psc_states_download", "psc_host_classify", "psc_host_mask_row",
            "psc_host_advance", "psc_fill_apply_noalloc", "psc_fill_apply_argmax", "psc_save", "psc_load",
            "psc_decode_step", "psc_decode_step_mask", "psc_decode_step_advance", "psc_state_copy",
            "psc_host_classify_bottom_up", "psc_state_faults", "psc_check_wait"]
# include/psc_ops.h: the operators around the mask
EXPORTED_OPS = ["psc_quantize_rows", "psc_head_work_bytes", "psc_head_logits", "psc_process_logits",
                "psc_sample_work_bytes", "psc_sample"]
# include/psc_mx4.h: the vocabulary projection in microscaled 4-bit floating point
EXPORTED_MX4 = ["psc_mx4_block_bytes", "psc_quantize_mx4", "psc_dequantize_mx4", "psc_head_logits_mx4",
                "psc_mx4_faults", "psc_mx4_check_wait"]
# include/psc_norm.h: the norm in front of either projection
EXPORTED_NORM = ["psc_norm_quantize_rows", "psc_norm_quantize_mx4"]
NOALLOC_MAX_ROWS = 16384


class PscError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {message}")
        self.code = code


class Options(ctypes.Structure):
    _fields_ = [("max_states", ctypes.c_int64), ("max_mask_bytes", ctypes.c_int64),
                ("threads", ctypes.c_int32), ("host_only", ctypes.c_int32),
                ("global_tables", ctypes.c_int32), ("max_bottom_up_bytes", ctypes.c_int64),
                ("max_dense_classifier_bytes", ctypes.c_int64)]


class InfoT(ctypes.Structure):
    _fields_ = [("V", ctypes.c_int32), ("W", ctypes.c_int32), ("n_lexer_states", ctypes.c_int32),
                ("n_parser_states", ctypes.c_int32), ("n_terminals", ctypes.c_int32),
                ("n_classifier_states", ctypes.c_int32), ("n_masks", ctypes.c_int32), ("eos_id", ctypes.c_int32),
                ("classifier_bytes", ctypes.c_int64), ("mask_bytes", ctypes.c_int64),
                ("states_built", ctypes.c_int64), ("compile_seconds", ctypes.c_double),
                ("advance_table_bytes", ctypes.c_int64), ("device_timeouts", ctypes.c_int64),
                ("bottom_up_states", ctypes.c_int64), ("bottom_up_bytes", ctypes.c_int64),
                ("classifier_sparse", ctypes.c_int64), ("advance_tables_packed", ctypes.c_int64)]


_lib = None
_marshal = None          # csrc/marshal.cpp, where it is built: the small calls' tensors taken apart in C


def _load_marshal(lib, device=None):
    global _marshal
    import sysconfig
    # by this interpreter's tag: a module that another one's headers have gone into is not looked at
    path = os.path.join(_HERE, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))
    if not os.path.exists(path):
        return
    try:
        import importlib.util
        import torch
        spec = importlib.util.spec_from_file_location("_marshal", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    except ImportError:                     # no torch, or a file that is no module
        return
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731
    module.setup((torch.bfloat16, torch.float32, torch.int8, torch.uint8, torch.int32),
                 tuple(address(f) for f in (lib.psc_norm_quantize_rows, lib.psc_norm_quantize_mx4, lib.psc_quantize_mx4,
                                            lib.psc_dequantize_mx4, lib.psc_head_logits_mx4)), _stream,
                 device or getattr(torch._C, "_cuda_getDevice", _device))
    _marshal = module


def load(path: str = LIB_PATH):
    """Load the library (raises if it is missing: there is no other backend)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2608_03065_gb300.build.build()")
    lib = ctypes.CDLL(path)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    f32 = ctypes.c_float
    sig = {
        "psc_compile": (i32, [ctypes.c_char_p, sz, vp, vp, i32, i32, vp, vp]),
        "psc_destroy": (None, [vp]),
        "psc_last_error": (ctypes.c_char_p, []),
        "psc_info": (i32, [vp, vp]),
        "psc_state_init": (i32, [vp, i32, i32, vp, vp]),
        "psc_state_reset": (i32, [vp, vp, i32, vp]),
        "psc_state_destroy": (None, [vp]),
        "psc_advance": (i32, [vp, vp, vp, i32, vp, vp]),
        "psc_fill_mask": (i32, [vp, vp, i32, vp, vp]),
        "psc_apply_mask": (i32, [vp, i32, i64, vp, i32, i32, vp]),
        "psc_fill_apply": (i32, [vp, vp, i32, vp, i32, i64, i32, vp, vp]),
        "psc_argmax_masked": (i32, [vp, vp, i32, vp, i32, i64, i32, vp, vp]),
        "psc_states_download": (i32, [vp, vp, vp, vp, vp, vp]),
        "psc_host_classify": (i32, [vp, i32, vp, i32, i32]),
        "psc_host_classify_bottom_up": (i32, [vp, i32, vp, i32, i32]),
        "psc_host_mask_row": (i32, [vp, i32, vp]),
        "psc_host_advance": (i32, [vp, vp, vp, vp, i32, vp, i32]),
        "psc_fill_apply_noalloc": (i32, [vp, vp, vp, vp, vp, i32, i32, vp, i32, i64, i32, vp, vp]),
        "psc_fill_apply_argmax": (i32, [vp, vp, i32, vp, i32, i64, i32, vp, vp, vp]),
        "psc_save": (i32, [vp, ctypes.c_char_p]),
        "psc_decode_step": (i32, [vp, vp, i32, vp, i32, i64, i32, vp, vp, vp, vp]),
        "psc_decode_step_mask": (i32, [vp, vp, i32, vp, i32, i64, i32, vp, vp]),
        "psc_state_copy": (i32, [vp, vp, vp]),
        "psc_decode_step_advance": (i32, [vp, vp, i32, vp, vp, vp]),
        "psc_load": (i32, [ctypes.c_char_p, vp, vp]),
        "psc_state_faults": (i32, [vp, vp, i32, vp]),
        "psc_check_wait": (i32, [vp, i32, vp]),
        "psc_quantize_rows": (i32, [vp, i32, i64, i32, i32, vp, i64, vp, vp]),
        "psc_head_work_bytes": (i64, [i32, i32, i32, i32]),
        "psc_head_logits": (i32, [vp, i64, vp, i32, vp, i64, vp, i32, i32, vp, vp, i32, i64, vp, i64, vp]),
        "psc_process_logits": (i32, [vp, i32, i64, vp, i64, i32, i32, vp, i64, i32, vp, vp, vp, vp, vp, vp, vp, i32,
                                     vp, vp]),
        "psc_norm_quantize_rows": (i32, [vp, i32, i64, vp, i64, vp, i64, vp, f32, i32, i32, vp, i64, vp, vp]),
        "psc_mx4_block_bytes": (i64, [i32, i32]),
        "psc_quantize_mx4": (i32, [vp, i32, i64, i32, i32, vp, i64, vp, vp]),
        "psc_dequantize_mx4": (i32, [vp, i64, vp, vp, i32, i32, vp, i32, i64, vp]),
        "psc_norm_quantize_mx4": (i32, [vp, i32, i64, vp, i64, vp, i64, vp, f32, i32, i32, vp, i64, vp, vp, vp]),
        "psc_head_logits_mx4": (i32, [vp, i64, vp, vp, i32, vp, i64, vp, vp, i32, i32, vp, vp, i32, i64, vp]),
        "psc_mx4_faults": (i32, [vp, i32, vp]),
        "psc_mx4_check_wait": (i32, [vp, i64, vp, vp, i32, vp, i64, vp, vp, i32, i32, vp, vp, i32, i64, i32, vp]),
        "psc_sample_work_bytes": (i64, [i32]),
        "psc_sample": (i32, [vp, i32, i64, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp]),
    }
    for name, (res, args) in sig.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    _load_marshal(lib)
    return lib


def _check(code: int):
    if code != 0:
        raise PscError(code, (load().psc_last_error() or b"").decode(errors="replace"))


def _device() -> int:
    """The current device."""
    import torch
    return torch.cuda.current_device()


def _here(**tensors):
    """Kernels run on the current device: a tensor of another one is refused."""
    for name, t in tensors.items():
        if t is not None and t.is_cuda and t.get_device() != _device():
            raise ValueError(f"{name} is on cuda:{t.get_device()}, and the current device is cuda:{_device()}")


_current = None         # of the current device, the current stream's handle


def _stream(stream) -> int | None:
    global _current
    if stream is None:
        if _current is None:
            import torch
            try:                            # without a Stream object around it
                raw, device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice
                _current = lambda: raw(device())  # noqa: E731
            except AttributeError:
                _current = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
        return _current() or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _ptr(t, dtype=None, name="tensor", n=None):
    """Device address of a tensor argument; n = the elements the call reads or
    writes (a smaller or non-contiguous tensor is refused before any launch)."""
    if t is None:
        return None
    if t.is_cuda and (dtype is None or t.dtype is dtype) and (n is None or (t.numel() >= n and t.is_contiguous())):
        return t.data_ptr()
    if n is not None and (t.numel() < n or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous tensor of at least {n} elements")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    raise ValueError(f"{name} must have dtype {dtype}, got {t.dtype}")


def _dtype_code(t):
    import torch
    if t.dtype == torch.bfloat16:
        return PSC_BF16
    if t.dtype == torch.float32:
        return PSC_F32
    raise ValueError(f"logits must be bf16 or f32, got {t.dtype}")


def _row_stride(t):
    if t.dim() != 2 or t.stride(1) != 1:
        raise ValueError("logits must be a 2-D tensor with unit column stride")
    return t.stride(0)


@dataclass
class Info:
    V: int
    W: int
    n_lexer_states: int
    n_parser_states: int
    n_terminals: int
    n_classifier_states: int
    n_masks: int
    eos_id: int
    classifier_bytes: int
    mask_bytes: int
    states_built: int
    compile_seconds: float
    advance_table_bytes: int
    device_timeouts: int
    bottom_up_states: int
    bottom_up_bytes: int
    classifier_sparse: int
    advance_tables_packed: int


class Handle:
    """A compiled grammar x vocabulary (owns the device tables)."""

    def __init__(self, ptr: int, V: int):
        self.ptr = ptr
        self.V = V
        self.W = (V + 31) // 32

    def __del__(self):
        if getattr(self, "ptr", None) and _lib is not None:
            _lib.psc_destroy(self.ptr)
            self.ptr = None

    def info(self) -> Info:
        out = InfoT()
        _check(load().psc_info(self.ptr, ctypes.byref(out)))
        return Info(*[getattr(out, f) for f, _ in InfoT._fields_])

    # --- host-side inspection of the compiled tables
    def host_classify(self, q: int, stack, status: int = ROW_OK) -> int:
        st = np.ascontiguousarray(np.asarray(stack, dtype=np.uint16))
        return load().psc_host_classify(self.ptr, q, st.ctypes.data if len(st) else None, len(st), status)

    def host_classify_bottom_up(self, q: int, stack, status: int = ROW_OK) -> int:
        """The same mask id through the bottom-up classifier (-2: not built, or
        the stack is not a path of the LR automaton)."""
        st = np.ascontiguousarray(np.asarray(stack, dtype=np.uint16))
        return load().psc_host_classify_bottom_up(self.ptr, q, st.ctypes.data if len(st) else None, len(st),
                                                  status)

    def host_mask_row(self, mask_id: int) -> np.ndarray:
        row = np.zeros(self.W, dtype=np.uint32)
        _check(load().psc_host_mask_row(self.ptr, mask_id, row.ctypes.data))
        return row

    def host_advance(self, cfg: dict, token: int, cap: int = 256) -> dict:
        """cfg = {"q", "stack" (list), "status"}; returns the next configuration."""
        stack = np.zeros(cap, dtype=np.uint16)
        stack[:len(cfg["stack"])] = cfg["stack"]
        q = ctypes.c_int32(cfg["q"])
        depth = ctypes.c_int32(len(cfg["stack"]))
        status = ctypes.c_int32(cfg["status"])
        _check(load().psc_host_advance(self.ptr, ctypes.byref(q), stack.ctypes.data, ctypes.byref(depth), cap,
                                       ctypes.byref(status), int(token)))
        return {"q": q.value, "stack": stack[:depth.value].tolist(), "status": status.value}

    def host_initial(self) -> dict:
        return {"q": 0, "stack": [0], "status": ROW_OK}


class States:
    """A batch of device-resident parser configurations (owns its device arrays)."""

    def __init__(self, ptr: int, handle: Handle, B: int, cap: int):
        self.ptr = ptr
        self.handle = handle
        self.B = B
        self.cap = cap

    def __del__(self):
        if getattr(self, "ptr", None) and _lib is not None:
            _lib.psc_state_destroy(self.ptr)
            self.ptr = None


# ------------------------------------------------------------------- the ABI
def _tables(global_tables: bool, packed_tables: bool) -> int:
    if global_tables and packed_tables:
        raise ValueError("global_tables and packed_tables exclude each other")
    return 1 if global_tables else 2 if packed_tables else 0


def psc_compile(grammar: str, vocab: list[bytes] | tuple, eos_id: int, host_only: bool = False,
                threads: int = 0, max_states: int = 0, max_mask_bytes: int = 0,
                global_tables: bool = False, bottom_up: bool = True, max_bottom_up_bytes: int = 0,
                max_dense_classifier_bytes: int = 0, packed_tables: bool = False) -> Handle:
    """vocab: list of token byte strings, or (blob uint8 array, offsets int64[V+1]).
    bottom_up=False builds no bottom-up classifier (every stack is walked from the top);
    max_dense_classifier_bytes < 0 holds the classifier in the sparse layout;
    global_tables=True has the advance read its parser tables from global memory,
    packed_tables=True stages them in the packed layout even when the dense one fits."""
    if isinstance(vocab, tuple):
        blob, offs = vocab
        blob = np.ascontiguousarray(blob, dtype=np.uint8)
        offs = np.ascontiguousarray(offs, dtype=np.int64)
    else:
        offs = np.zeros(len(vocab) + 1, dtype=np.int64)
        offs[1:] = np.cumsum([len(t) for t in vocab])
        blob = np.frombuffer(b"".join(vocab), dtype=np.uint8).copy()
    if blob.size == 0:
        blob = np.zeros(1, dtype=np.uint8)
    V = len(offs) - 1
    opts = Options(max_states, max_mask_bytes, threads, 1 if host_only else 0, _tables(global_tables, packed_tables),
                   max_bottom_up_bytes if bottom_up else -1, max_dense_classifier_bytes)
    g = grammar.encode("utf-8")
    out = ctypes.c_void_p()
    _check(load().psc_compile(g, len(g), blob.ctypes.data, offs.ctypes.data, V, eos_id, ctypes.byref(opts),
                              ctypes.byref(out)))
    return Handle(out.value, V)


def psc_save(h: Handle, path: str):
    _check(load().psc_save(h.ptr, os.fsencode(path)))


def psc_load(path: str, host_only: bool = False, global_tables: bool = False, bottom_up: bool = True,
             packed_tables: bool = False) -> Handle:
    opts = Options(0, 0, 0, 1 if host_only else 0, _tables(global_tables, packed_tables), 0 if bottom_up else -1, 0)
    out = ctypes.c_void_p()
    _check(load().psc_load(os.fsencode(path), ctypes.byref(opts), ctypes.byref(out)))
    h = Handle(out.value, 0)
    h.V = h.info().V
    h.W = (h.V + 31) // 32
    return h


def psc_state_init(h: Handle, B: int, cap: int = 256, stream=None) -> States:
    out = ctypes.c_void_p()
    _check(load().psc_state_init(h.ptr, B, cap, _stream(stream), ctypes.byref(out)))
    return States(out.value, h, B, cap)


def psc_state_reset(st: States, rows=None, stream=None):
    import torch
    n = st.B if rows is None else rows.numel()
    _check(load().psc_state_reset(st.ptr, _ptr(rows, torch.int32, "rows", n), n, _stream(stream)))


def psc_state_copy(dst: States, src: States, stream=None):
    """dst's rows := src's rows (same handle, B and cap), on the device."""
    _check(load().psc_state_copy(dst.ptr, src.ptr, _stream(stream)))


def psc_advance(h: Handle, st: States, tokens, row_status=None, stream=None):
    import torch
    _check(load().psc_advance(h.ptr, st.ptr, _ptr(tokens, torch.int32, "tokens", st.B), st.B,
                              _ptr(row_status, torch.int32, "row_status", st.B), _stream(stream)))


def psc_fill_mask(h: Handle, st: States, bitmask, stream=None):
    import torch
    if bitmask.shape != (st.B, h.W) or not bitmask.is_contiguous():
        raise ValueError(f"bitmask must be a contiguous [{st.B}, {h.W}] tensor")
    _check(load().psc_fill_mask(h.ptr, st.ptr, st.B, _ptr(bitmask, torch.int32, "bitmask"), _stream(stream)))


def psc_apply_mask(logits, bitmask, B: int, V: int, stream=None):
    import torch
    W = (V + 31) // 32
    if bitmask.shape[0] < B or bitmask.shape[1] != W or not bitmask.is_contiguous():
        raise ValueError(f"bitmask must be a contiguous [B, {W}] tensor")
    if logits.shape[0] < B or logits.shape[1] < V:
        raise ValueError("logits are smaller than [B, V]")
    _check(load().psc_apply_mask(_ptr(logits, None, "logits"), _dtype_code(logits), _row_stride(logits),
                                 _ptr(bitmask, torch.int32, "bitmask"), B, V, _stream(stream)))


def psc_fill_apply(h: Handle, st: States, logits, bitmask_out=None, V: int | None = None, stream=None):
    import torch
    V = h.V if V is None else V
    if logits.shape[0] != st.B or logits.shape[1] < V:
        raise ValueError("logits must be [B, >=V]")
    if bitmask_out is not None and (bitmask_out.shape != (st.B, h.W) or not bitmask_out.is_contiguous()):
        raise ValueError("bitmask_out must be a contiguous [B, W] tensor")
    _check(load().psc_fill_apply(h.ptr, st.ptr, st.B, _ptr(logits, None, "logits"), _dtype_code(logits),
                                 _row_stride(logits), V, _ptr(bitmask_out, torch.int32, "bitmask_out"),
                                 _stream(stream)))


def psc_argmax_masked(h: Handle, st: States, logits, tokens, stream=None):
    import torch
    if tokens.numel() != st.B:
        raise ValueError("tokens must hold B int32 values")
    _check(load().psc_argmax_masked(h.ptr, st.ptr, st.B, _ptr(logits, None, "logits"), _dtype_code(logits),
                                    _row_stride(logits), h.V, _ptr(tokens, torch.int32, "tokens", st.B),
                                    _stream(stream)))


def psc_fill_apply_argmax(h: Handle, st: States, logits, tokens, bitmask_out=None, stream=None):
    import torch
    if logits.shape[0] != st.B or logits.shape[1] < h.V:
        raise ValueError("logits must be [B, >=V]")
    if tokens.numel() != st.B:
        raise ValueError("tokens must hold B int32 values")
    if bitmask_out is not None and (bitmask_out.shape != (st.B, h.W) or not bitmask_out.is_contiguous()):
        raise ValueError("bitmask_out must be a contiguous [B, W] tensor")
    _check(load().psc_fill_apply_argmax(h.ptr, st.ptr, st.B, _ptr(logits, None, "logits"), _dtype_code(logits),
                                        _row_stride(logits), h.V, _ptr(bitmask_out, torch.int32, "bitmask_out"),
                                        _ptr(tokens, torch.int32, "tokens", st.B), _stream(stream)))


def psc_decode_step(h: Handle, st: States, logits, tokens, bitmask_out=None, row_status=None, stream=None):
    import torch
    if logits.shape[0] != st.B or logits.shape[1] < h.V:
        raise ValueError("logits must be [B, >=V]")
    if tokens.numel() != st.B:
        raise ValueError("tokens must hold B int32 values")
    if bitmask_out is not None and (bitmask_out.shape != (st.B, h.W) or not bitmask_out.is_contiguous()):
        raise ValueError("bitmask_out must be a contiguous [B, W] tensor")
    _check(load().psc_decode_step(h.ptr, st.ptr, st.B, _ptr(logits, None, "logits"), _dtype_code(logits),
                                  _row_stride(logits), h.V, _ptr(bitmask_out, torch.int32, "bitmask_out"),
                                  _ptr(tokens, torch.int32, "tokens", st.B),
                                  _ptr(row_status, torch.int32, "row_status", st.B), _stream(stream)))


def psc_decode_step_mask(h: Handle, st: States, logits, bitmask_out=None, stream=None):
    """First half of psc_decode_step: masking pass, greedy choices kept in the states."""
    import torch
    if logits.shape[0] != st.B or logits.shape[1] < h.V:
        raise ValueError("logits must be [B, >=V]")
    if bitmask_out is not None and (bitmask_out.shape != (st.B, h.W) or not bitmask_out.is_contiguous()):
        raise ValueError("bitmask_out must be a contiguous [B, W] tensor")
    _check(load().psc_decode_step_mask(h.ptr, st.ptr, st.B, _ptr(logits, None, "logits"), _dtype_code(logits),
                                       _row_stride(logits), h.V, _ptr(bitmask_out, torch.int32, "bitmask_out"),
                                       _stream(stream)))


def psc_decode_step_advance(h: Handle, st: States, tokens, row_status=None, stream=None):
    """Second half of psc_decode_step: tokens out, rows advanced and classified."""
    import torch
    if tokens.numel() != st.B:
        raise ValueError("tokens must hold B int32 values")
    _check(load().psc_decode_step_advance(h.ptr, st.ptr, st.B, _ptr(tokens, torch.int32, "tokens", st.B),
                                          _ptr(row_status, torch.int32, "row_status", st.B), _stream(stream)))


def psc_state_faults(st: States, reset: bool = False, stream=None) -> int:
    """Bounded in-kernel waits on these states that gave up (synchronises the stream)."""
    out = ctypes.c_int32(0)
    _check(load().psc_state_faults(st.ptr, ctypes.byref(out), 1 if reset else 0, _stream(stream)))
    return out.value


def psc_check_wait(st: States, limit: int = 4096, stream=None):
    """Self-test of fault reporting: a bounded wait that nothing completes gives up
    after `limit` polls and is counted on the states object."""
    _check(load().psc_check_wait(st.ptr, limit, _stream(stream)))


def psc_states_download(st: States, stream=None) -> dict:
    q = np.zeros(st.B, dtype=np.int32)
    depth = np.zeros(st.B, dtype=np.int32)
    stack = np.zeros((st.B, st.cap), dtype=np.uint16)
    status = np.zeros(st.B, dtype=np.int32)
    _check(load().psc_states_download(st.ptr, q.ctypes.data, depth.ctypes.data, stack.ctypes.data,
                                      status.ctypes.data, _stream(stream)))
    return {"q": q, "depth": depth, "stack": stack, "status": status}


def psc_fill_apply_noalloc(h: Handle, q, depth, status, stack, logits, bitmask_out=None, V: int | None = None,
                           stream=None):
    """psc_fill_apply on caller-owned state arrays (q, depth, status int32 [B];
    stack uint16 [B][cap] as a torch int16/uint16 tensor); allocates nothing."""
    import torch
    B = q.numel()
    V = h.V if V is None else V
    if stack.dim() != 2 or stack.shape[0] != B or not stack.is_contiguous() or stack.element_size() != 2:
        raise ValueError("stack must be a contiguous [B, cap] 16-bit tensor")
    if logits.dim() != 2 or logits.shape[0] != B or logits.shape[1] < V:
        raise ValueError("logits must be [B, >=V]")
    if bitmask_out is not None and (bitmask_out.shape != (B, h.W) or not bitmask_out.is_contiguous()):
        raise ValueError(f"bitmask_out must be a contiguous [{B}, {h.W}] tensor")
    _check(load().psc_fill_apply_noalloc(h.ptr, _ptr(q, torch.int32, "q", B), _ptr(depth, torch.int32, "depth", B),
                                         _ptr(status, torch.int32, "status", B), _ptr(stack, None, "stack"),
                                         stack.shape[1], B, _ptr(logits, None, "logits"), _dtype_code(logits),
                                         _row_stride(logits), V, _ptr(bitmask_out, torch.int32, "bitmask_out"),
                                         _stream(stream)))


# ------------------------------------------------- the operators around the mask
def _rows(t, dtype, name, rows=None, cols=None):
    """(device address, row stride) of a 2-D tensor with unit column stride, at
    least `rows` x `cols` elements."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor with unit column stride")
    (r, c), (stride, unit) = t.shape, t.stride()
    if c > 1 and unit != 1:
        raise ValueError(f"{name} must be a 2-D tensor with unit column stride")
    if (rows is not None and r != rows) or (cols is not None and c < cols):
        raise ValueError(f"{name} must be [{rows}, >={cols}], got {list(t.shape)}")
    # a row of its own may carry any stride
    return _ptr(t, dtype, name), stride if r > 1 else max(c, stride)


def _at(t, dtype, name, rows, cols):
    """What _rows gives, without its questions one by one for a tensor that is as it should be
    (of the time of a small call the questions are a large part)."""
    shape = t.shape
    if t.dtype is dtype and t.is_cuda and len(shape) == 2 and shape[0] == rows and shape[1] >= cols:
        stride, unit = t.stride()
        if unit == 1:
            return t.data_ptr(), stride if rows > 1 else max(shape[1], stride)
    return _rows(t, dtype, name, rows, cols)


def _mask_ptr(bitmask, B, V):
    import torch
    if bitmask is None:
        return None
    W = (V + 31) // 32
    if bitmask.shape != (B, W) or not bitmask.is_contiguous():
        raise ValueError(f"bitmask must be a contiguous [{B}, {W}] tensor")
    return _ptr(bitmask, torch.int32, "bitmask")


def _workspace(n: int, device, stream):
    """n bytes of torch's allocator, from the pool of the stream that the kernels run on."""
    import torch
    if stream is None:
        return torch.empty(n, dtype=torch.uint8, device=device)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
        return torch.empty(n, dtype=torch.uint8, device=device)


def psc_quantize_rows(x, q, scale, stream=None):
    """q, scale := the rows of x (bf16 or f32 [T, K]) in 8-bit integers (int8 [T, K])
    with a scale each (f32 [T]): activations by token, or weights by output channel."""
    import torch
    if x.dim() != 2:
        raise ValueError("x must be a 2-D tensor")
    T, K = x.shape
    code = _dtype_code(x)
    px, sx = _rows(x, None, "x", T, K)
    pq, sq = _rows(q, torch.int8, "q", T, K)
    _check(load().psc_quantize_rows(px, code, sx, T, K, pq, sq, _ptr(scale, torch.float32, "scale", T),
                                    _stream(stream)))


def _norm_inputs(x, residual, sum_out, gain, **outputs):
    """What the two norms share: x's sizes, and the inputs' addresses and strides."""
    import torch
    shape, dtype = x.shape, x.dtype
    if len(shape) != 2:
        raise ValueError("x must be a 2-D tensor")
    T, K = shape
    code = _dtype_code(x)
    _here(x=x, residual=residual, sum_out=sum_out, gain=gain, **outputs)
    px, sx = _at(x, dtype, "x", T, K)
    pr, sr = (None, 0) if residual is None else _at(residual, dtype, "residual", T, K)
    ps, ss = (None, 0) if sum_out is None else _at(sum_out, dtype, "sum_out", T, K)
    return T, K, (px, code, sx, pr, sr, ps, ss, _ptr(gain, torch.float32, "gain", K))


def psc_norm_quantize_rows(x, q, scale, gain=None, eps: float = 1e-6, residual=None, sum_out=None, stream=None):
    """q, scale := the rows of the root-mean-square norm of h = x + residual, times gain, in
    8-bit integers (int8 [T, K]) with a scale each (f32 [T]), as psc_quantize_rows makes
    them of activations; sum_out := h.  x, residual, sum_out bf16 or f32 [T, K], gain f32 [K];
    gain, residual and sum_out may be None, and sum_out may be x or residual."""
    if _marshal is not None:
        code = _marshal.norm_rows(x, q, scale, gain, eps, residual, sum_out, stream)
        if code is not None:
            return _check(code) if code else None
    import torch
    T, K, inputs = _norm_inputs(x, residual, sum_out, gain, q=q, scale=scale)
    pq, sq = _at(q, torch.int8, "q", T, K)
    _check((_lib or load()).psc_norm_quantize_rows(*inputs, eps, T, K, pq, sq, _ptr(scale, torch.float32, "scale", T),
                                                   _stream(stream)))


def psc_head_work_bytes(T: int, V: int, K: int, aligned: bool = True) -> int:
    """Bytes of workspace for psc_head_logits; aligned: the weights' rows are at addresses
    that are multiples of 16."""
    return load().psc_head_work_bytes(T, V, K, 1 if aligned else 0)


def psc_head_logits(q, scale, w, w_scale, logits, bitmask=None, work=None, stream=None):
    """logits[:, :V] := (q @ w.T) * scale[:, None] * w_scale, -inf where bitmask forbids.
    q int8 [T, K], w int8 [V, K] (rows at 16-byte-aligned addresses are read where they
    are, others packed first), scale f32 [T], w_scale f32 [V], logits bf16 or f32 [T, >=V].  work: a
    uint8 tensor of at least psc_head_work_bytes(T, V, K) bytes to reuse (one is
    taken from torch's allocator for the call otherwise).  Returns the workspace, for
    psc_head_faults."""
    import torch
    if q.dim() != 2 or w.dim() != 2 or q.shape[1] != w.shape[1]:
        raise ValueError("q and w must be [T, K] and [V, K]")
    (T, K), V = q.shape, w.shape[0]
    code = _dtype_code(logits)
    pq, sq = _rows(q, torch.int8, "q")
    pw, sw = _rows(w, torch.int8, "w")
    pl, sl = _rows(logits, None, "logits", T, V)
    n = load().psc_head_work_bytes(T, V, K, 0 if (pw or 0) % 16 or sw % 16 else 1)
    pm = _mask_ptr(bitmask, T, V)
    if work is None:
        work = _workspace(n, logits.device, stream)
    _check(load().psc_head_logits(pq, sq, _ptr(scale, torch.float32, "scale", T), T, pw, sw,
                                  _ptr(w_scale, torch.float32, "w_scale", V), V, K, pm, pl, code, sl,
                                  _ptr(work, torch.uint8, "work", n), work.numel(), _stream(stream)))
    return work


def psc_head_faults(work, stream=None) -> int:
    """Blocks of the last psc_head_logits call with this workspace in which a bounded wait
    gave up (synchronises the stream); not 0: some of its logits were not written."""
    import torch
    _ptr(work, torch.uint8, "work", 4)
    if stream is None:
        return work.view(-1)[:4].view(torch.int32).item()
    with torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
        return work.view(-1)[:4].view(torch.int32).item()


def psc_process_logits(logits, out=None, history=None, history_len=None, prompt_len=None, repetition=None,
                       frequency=None, presence=None, bias_ids=None, bias=None, bitmask=None, V: int | None = None,
                       stream=None):
    """out[:, :V] := logits[:, :V] with penalties for the tokens of the history, biases
    and the mask applied (in place when out is None).  history int32 [B, H] of
    token ids, its first history_len[b] used, the first prompt_len[b] of those the
    prompt; repetition, frequency, presence f32 [B]; bias_ids int32 and bias f32
    [B, n].  Each may be None."""
    import torch
    if logits.dim() != 2:
        raise ValueError("logits must be a 2-D tensor")
    B = logits.shape[0]
    V = logits.shape[1] if V is None else V
    code = _dtype_code(logits)
    pl, sl = _rows(logits, None, "logits", B, V)
    po, so = (pl, sl) if out is None else _rows(out, logits.dtype, "out", B, V)
    ph, sh, H = None, 0, 0
    if history is not None and history.numel():
        ph, sh = _rows(history, torch.int32, "history", B, 0)
        H = history.shape[1]
    n_bias = 0
    if (bias_ids is None) != (bias is None):
        raise ValueError("bias_ids and bias come together")
    if bias_ids is not None:
        if bias_ids.dim() != 2 or bias_ids.shape[0] != B or bias.shape != bias_ids.shape:
            raise ValueError("bias_ids and bias must be [B, n] tensors")
        n_bias = bias_ids.shape[1]
    _check(load().psc_process_logits(
        pl, code, sl, po, so, B, V, ph, sh, H, _ptr(history_len, torch.int32, "history_len", B),
        _ptr(prompt_len, torch.int32, "prompt_len", B), _ptr(repetition, torch.float32, "repetition", B),
        _ptr(frequency, torch.float32, "frequency", B), _ptr(presence, torch.float32, "presence", B),
        _ptr(bias_ids, torch.int32, "bias_ids", B * n_bias) if n_bias else None,
        _ptr(bias, torch.float32, "bias", B * n_bias) if n_bias else None, n_bias, _mask_ptr(bitmask, B, V),
        _stream(stream)))


def psc_sample(logits, uniform, tokens, logprobs=None, bitmask=None, temperature=None, top_k=None, top_p=None,
               min_p=None, V: int | None = None, work=None, stream=None):
    """tokens[b] := a token drawn among the allowed ones with uniform[b] (f32 in [0, 1)),
    logprobs[b] := ln of the probability it was drawn with.  temperature, top_p,
    min_p f32 [B], top_k int32 [B]; None leaves a filter off (temperature 1).  work: a
    uint8 tensor of at least psc_sample_work_bytes(B) bytes to reuse (0 for small batches)."""
    import torch
    if logits.dim() != 2:
        raise ValueError("logits must be a 2-D tensor")
    B = logits.shape[0]
    V = logits.shape[1] if V is None else V
    code = _dtype_code(logits)
    pl, sl = _rows(logits, None, "logits", B, V)
    n = load().psc_sample_work_bytes(B)
    if work is None and n:
        work = _workspace(n, logits.device, stream)
    _check(load().psc_sample(
        pl, code, sl, B, V, _mask_ptr(bitmask, B, V), _ptr(uniform, torch.float32, "uniform", B),
        _ptr(temperature, torch.float32, "temperature", B), _ptr(top_k, torch.int32, "top_k", B),
        _ptr(top_p, torch.float32, "top_p", B), _ptr(min_p, torch.float32, "min_p", B),
        _ptr(tokens, torch.int32, "tokens", B), _ptr(logprobs, torch.float32, "logprobs", B),
        _ptr(work, torch.uint8, "work", n), n, _stream(stream)))


# ------------------------------------ the projection in microscaled 4-bit floating point
def psc_mx4_row_bytes(K: int) -> int:
    """Bytes of a row's codes: whole blocks of 32 columns."""
    return (K + 31) // 32 * 16


def psc_mx4_block_bytes(rows: int, K: int) -> int:
    """Bytes of the blocks' exponents of a matrix, in tiles as include/psc_mx4.h lays them out."""
    return load().psc_mx4_block_bytes(rows, K)


def _mx4(q, blocks, rows, K, name):
    """(address of the codes, their stride, address of the exponents)."""
    import torch
    pq, sq = _at(q, torch.uint8, name, rows, (K + 31) // 32 * 16)
    return pq, sq, _ptr(blocks, torch.uint8, f"{name}'s blocks", (rows + 127) // 128 * ((K + 127) // 128) * 512)


def psc_quantize_mx4(x, q, blocks, stream=None):
    """q, blocks := the rows of x (bf16 or f32 [T, K]) in microscaled 4-bit floating point:
    uint8 [T, >= psc_mx4_row_bytes(K)] codes, two a byte, and uint8 [psc_mx4_block_bytes(T, K)]
    exponents of blocks of 32 columns.  Activations by token, or weights by output channel."""
    if _marshal is not None:
        code = _marshal.quantize_mx4(x, q, blocks, stream)
        if code is not None:
            return _check(code) if code else None
    shape = x.shape
    if len(shape) != 2:
        raise ValueError("x must be a 2-D tensor")
    T, K = shape
    code = _dtype_code(x)
    _here(x=x, q=q, blocks=blocks)
    px, sx = _at(x, x.dtype, "x", T, K)
    pq, sq, pb = _mx4(q, blocks, T, K, "q")
    _check((_lib or load()).psc_quantize_mx4(px, code, sx, T, K, pq, sq, pb, _stream(stream)))


def psc_dequantize_mx4(q, blocks, y, scale=None, stream=None):
    """y := the values that q and blocks hold (bf16 or f32 [T, K]), times scale (f32 [T])."""
    if _marshal is not None:
        code = _marshal.dequantize_mx4(q, blocks, y, scale, stream)
        if code is not None:
            return _check(code) if code else None
    import torch
    shape = y.shape
    if len(shape) != 2:
        raise ValueError("y must be a 2-D tensor")
    T, K = shape
    code = _dtype_code(y)
    _here(y=y, q=q, blocks=blocks, scale=scale)
    py, sy = _at(y, y.dtype, "y", T, K)
    pq, sq, pb = _mx4(q, blocks, T, K, "q")
    _check((_lib or load()).psc_dequantize_mx4(pq, sq, pb, _ptr(scale, torch.float32, "scale", T), T, K, py, code, sy,
                                               _stream(stream)))


def psc_norm_quantize_mx4(x, q, blocks, scale, gain=None, eps: float = 1e-6, residual=None, sum_out=None, stream=None):
    """psc_norm_quantize_rows with an output in 4 bits: q and blocks as psc_quantize_mx4 makes
    them of h * gain, scale (f32 [T]) := 1 / sqrt(mean h^2 + eps)."""
    if _marshal is not None:
        code = _marshal.norm_mx4(x, q, blocks, scale, gain, eps, residual, sum_out, stream)
        if code is not None:
            return _check(code) if code else None
    import torch
    T, K, inputs = _norm_inputs(x, residual, sum_out, gain, q=q, blocks=blocks, scale=scale)
    pq, sq, pb = _mx4(q, blocks, T, K, "q")
    _check((_lib or load()).psc_norm_quantize_mx4(*inputs, eps, T, K, pq, sq, pb, _ptr(scale, torch.float32, "scale", T),
                                                  _stream(stream)))


def psc_head_logits_mx4(q, q_blocks, w, w_blocks, logits, K: int, scale=None, w_scale=None, bitmask=None, stream=None):
    """logits[:, :V] := (x @ w.T) * scale[:, None] * w_scale over the values of matrices in 4 bits,
    x [T, K] (q, q_blocks) and w [V, K] (w, w_blocks), -inf where bitmask forbids.  scale f32 [T]
    and w_scale f32 [V] may be None; logits bf16 or f32 [T, >=V]."""
    if _marshal is not None:
        code = _marshal.head_logits_mx4(q, q_blocks, w, w_blocks, logits, K, scale, w_scale, bitmask, stream)
        if code is not None:
            return _check(code) if code else None
    _check((_lib or load()).psc_head_logits_mx4(*_head_mx4(q, q_blocks, w, w_blocks, logits, K, scale, w_scale, bitmask),
                                                _stream(stream)))


def _head_mx4(q, q_blocks, w, w_blocks, logits, K, scale, w_scale, bitmask):
    """The library's arguments of the projection, up to the stream."""
    import torch
    qs, ws = q.shape, w.shape
    if len(qs) != 2 or len(ws) != 2:
        raise ValueError("q and w must be 2-D tensors")
    T, V = qs[0], ws[0]
    code = _dtype_code(logits)
    _here(q=q, q_blocks=q_blocks, w=w, w_blocks=w_blocks, logits=logits, scale=scale, w_scale=w_scale, bitmask=bitmask)
    pq, sq, pqb = _mx4(q, q_blocks, T, K, "q")
    pw, sw, pwb = _mx4(w, w_blocks, V, K, "w")
    pl, sl = _at(logits, logits.dtype, "logits", T, V)
    return (pq, sq, pqb, _ptr(scale, torch.float32, "scale", T), T, pw, sw, pwb, _ptr(w_scale, torch.float32, "w_scale", V),
            V, K, _mask_ptr(bitmask, T, V), pl, code, sl)


def psc_mx4_faults(reset: bool = False, stream=None) -> int:
    """Blocks of psc_head_logits_mx4 on the current device in which a bounded wait gave up, since
    the library was loaded or the last reset (synchronises the stream); not 0: logits are missing."""
    out = ctypes.c_int32(0)
    _check(load().psc_mx4_faults(ctypes.byref(out), 1 if reset else 0, _stream(stream)))
    return out.value


def psc_mx4_check_wait(q, q_blocks, w, w_blocks, logits, K: int, limit: int, scale=None, w_scale=None, bitmask=None,
                       stream=None):
    """Self-test of the fault path: psc_head_logits_mx4 into f32 logits, with waits that give up after `limit`
    looks at a barrier (some logits are not written; psc_mx4_faults counts the blocks)."""
    _check(load().psc_mx4_check_wait(*_head_mx4(q, q_blocks, w, w_blocks, logits, K, scale, w_scale, bitmask), limit,
                                     _stream(stream)))


def psc_sample_work_bytes(B: int) -> int:
    return load().psc_sample_work_bytes(B)

"""ctypes binding of the C ABI in include/ (argument marshalling only)."""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import torch

SWARM_F32, SWARM_BF16 = 0, 1
SWARM_BLOCK_GELU, SWARM_BLOCK_ROTARY_GEGLU = 0, 1
PARAM_FIELDS = ("ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o",
                "ln2_g", "ln2_b", "w_1", "b_1", "w_2", "b_2")
EXPORTED_SYMBOLS = ("swarm_stage_workspace_bytes", "swarm_stage_forward", "swarm_stage_backward",
                    "swarm_codec_encode", "swarm_codec_decode", "swarm_status_string",
                    "swarm_stage_coded_workspace_bytes", "swarm_stage_forward_coded", "swarm_stage_backward_coded",
                    "swarm_boundary_workspace_bytes", "swarm_compress_forward", "swarm_compress_backward",
                    "swarm_decompress_forward", "swarm_decompress_backward",
                    "swarm_embedding_forward", "swarm_embedding_backward", "swarm_head_workspace_bytes",
                    "swarm_head_loss", "swarm_head_loss_backward",
                    "swarm_lamb_workspace_bytes", "swarm_lamb_step", "swarm_lamb_step_static",
                    "swarm_codec_encode_s16", "swarm_codec_decode_s16",
                    "swarm_stage_forward_coded_s16", "swarm_stage_backward_coded_s16",
                    "swarm_cache_append", "swarm_cache_read", "swarm_cache_keep",
                    "swarm_cache_attention_workspace_bytes", "swarm_cache_attention",
                    "swarm_stage_extend_workspace_bytes", "swarm_stage_extend",
                    "swarm_head_logits", "swarm_logits_adjust")
SWARM_COMPRESS_BOTTLENECK, SWARM_COMPRESS_MAXOUT = 0, 1

_PKG = os.path.dirname(os.path.abspath(__file__))


class SwarmError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, swarm_status_string(status), status))


class _Config(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("n_heads", C.c_int32), ("d_ffn", C.c_int32),
                ("n_layers", C.c_int32), ("n_repeat", C.c_int32), ("batch", C.c_int32),
                ("seq", C.c_int32), ("dtype", C.c_int32), ("ln_eps", C.c_float), ("block_kind", C.c_int32)]


class _BlockPtrs(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in PARAM_FIELDS]


class _BoundaryConfig(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("d_comp", C.c_int32), ("kind", C.c_int32), ("tokens", C.c_int32),
                ("dtype", C.c_int32), ("ln_eps", C.c_float)]


class _Ptrs3(C.Structure):       # swarm_compress_params / _grads and swarm_decompress_params / _grads
    _fields_ = [("ln_g", C.c_void_p), ("ln_b", C.c_void_p), ("w", C.c_void_p)]


class BoundaryConfig:
    """Host-side description of a compressed stage boundary (mirrors swarm_boundary_config)."""

    def __init__(self, d_model, d_comp, kind, tokens, dtype, ln_eps=1e-5):
        if isinstance(kind, str):
            kind = {"bottleneck": SWARM_COMPRESS_BOTTLENECK, "maxout": SWARM_COMPRESS_MAXOUT}[kind]
        if isinstance(dtype, str):
            dtype = {"f32": SWARM_F32, "bf16": SWARM_BF16}[dtype]
        elif isinstance(dtype, torch.dtype):
            dtype = {torch.float32: SWARM_F32, torch.bfloat16: SWARM_BF16}[dtype]
        self.c = _BoundaryConfig(d_model, d_comp, kind, tokens, dtype, ln_eps)


class _HeadConfig(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("vocab", C.c_int32), ("vocab_rows", C.c_int32), ("tokens", C.c_int32),
                ("dtype", C.c_int32), ("ln_eps", C.c_float)]


class HeadConfig:
    """Host-side description of the language-modelling head (mirrors swarm_head_config)."""

    def __init__(self, d_model, vocab, vocab_rows, tokens, dtype, ln_eps=1e-5):
        if isinstance(dtype, str):
            dtype = {"f32": SWARM_F32, "bf16": SWARM_BF16}[dtype]
        elif isinstance(dtype, torch.dtype):
            dtype = {torch.float32: SWARM_F32, torch.bfloat16: SWARM_BF16}[dtype]
        self.c = _HeadConfig(d_model, vocab, vocab_rows, tokens, dtype, ln_eps)


class _LambConfig(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("weight_decay", C.c_float), ("grad_scale", C.c_float), ("step", C.c_int32)]


class _CacheConfig(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("d_head", C.c_int32), ("page_tokens", C.c_int32),
                ("n_pages", C.c_int32), ("batch", C.c_int32), ("table_pages", C.c_int32), ("dtype", C.c_int32),
                ("scale_bits", C.c_int32)]


class _Cache(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p)]


class CacheConfig:
    """Host-side description of a paged int8 key / value cache and the sequences in it (mirrors swarm_cache_config)."""

    def __init__(self, n_heads, n_kv_heads, d_head, page_tokens, n_pages, batch, table_pages, dtype, scale_bits=32):
        if isinstance(dtype, str):
            dtype = {"f32": SWARM_F32, "bf16": SWARM_BF16}[dtype]
        elif isinstance(dtype, torch.dtype):
            dtype = {torch.float32: SWARM_F32, torch.bfloat16: SWARM_BF16}[dtype]
        self.c = _CacheConfig(n_heads, n_kv_heads, d_head, page_tokens, n_pages, batch, table_pages, dtype, scale_bits)
        self._ref = C.byref(self.c)
        self.torch_dtype = torch.float32 if dtype == SWARM_F32 else torch.bfloat16
        self._pool = (n_kv_heads, d_head, page_tokens, n_pages, scale_bits)        # what a Cache of it has to be made for
        self._sizes = (batch, batch * table_pages, n_heads * d_head, n_kv_heads * d_head, self.torch_dtype)

    def shapes(self):
        """Shape and dtype of the four tensors of a Cache (16-bit scales are bf16 values; their bit patterns as 16-bit integers do too)."""
        c = self.c
        scale = torch.float32 if c.scale_bits == 32 else torch.bfloat16
        return {"k_codes": ((c.n_pages, c.n_kv_heads, c.page_tokens, c.d_head), torch.int8),
                "v_codes": ((c.n_pages, c.n_kv_heads, c.d_head, c.page_tokens), torch.int8),
                "k_scales": ((c.n_pages, c.n_kv_heads, c.d_head // 64, c.page_tokens), scale),
                "v_scales": ((c.n_pages, c.n_kv_heads, c.d_head // 64, c.page_tokens), scale)}


_PATTERNS = tuple(getattr(torch, n) for n in ("int16", "uint16") if hasattr(torch, n))     # of bf16 values


class Cache:
    """The pool of one block application: four tensors as CacheConfig.shapes() says, checked once here."""

    def __init__(self, cfg: CacheConfig, k_codes, v_codes, k_scales, v_scales):
        self.tensors = {"k_codes": k_codes, "v_codes": v_codes, "k_scales": k_scales, "v_scales": v_scales}
        for name, (shape, dtype) in cfg.shapes().items():
            t = self.tensors[name]
            if tuple(t.shape) != shape:
                raise ValueError("%s has shape %s, the cache has %s" % (name, tuple(t.shape), shape))
            if t.dtype != dtype and not (dtype == torch.bfloat16 and t.dtype in _PATTERNS):
                raise TypeError("%s must be %s" % (name, dtype))
            if not t.is_contiguous():
                raise ValueError("%s must be contiguous" % name)
        devices = {t.get_device() for t in self.tensors.values()}
        if len(devices) != 1:
            raise ValueError("the tensors of a cache must be on one device")
        self._device = devices.pop()
        self._pool = cfg._pool
        self.c = _Cache(*(t.data_ptr() for t in self.tensors.values()))
        self._ref = C.byref(self.c)


class _LogitsRules(C.Structure):
    _fields_ = [("rows", C.c_int32), ("vocab", C.c_int32), ("history_max", C.c_int32), ("bias_max", C.c_int32)] + \
               [(k, C.c_void_p) for k in ("history", "history_len", "repetition", "frequency", "presence", "bias_ids", "bias",
                                          "bias_len", "allowed")]


class LogitsRules:
    """The rules of swarm_logits_adjust (mirrors swarm_logits_rules); the tensors are kept alive and read at every call.
    history, bias_ids [rows, n] int32; history_len, bias_len [rows] int32; bias [rows, n] and repetition, frequency, presence [rows]
    fp32; allowed [rows, ceil(vocab / 32)] int32 (bit patterns)."""

    def __init__(self, rows, vocab, history=None, history_len=None, repetition=None, frequency=None, presence=None, bias_ids=None,
                 bias=None, bias_len=None, allowed=None):
        given = dict(history=history, history_len=history_len, repetition=repetition, frequency=frequency, presence=presence,
                     bias_ids=bias_ids, bias=bias, bias_len=bias_len, allowed=allowed)
        n_history = history.shape[1] if history is not None else 0
        n_bias = bias_ids.shape[1] if bias_ids is not None else 0
        whole = {"history": (rows, n_history), "history_len": (rows,), "bias_ids": (rows, n_bias), "bias_len": (rows,),
                 "allowed": (rows, (vocab + 31) // 32)}
        real = {"repetition": (rows,), "frequency": (rows,), "presence": (rows,), "bias": (rows, n_bias)}
        for name, t in given.items():
            if t is None:
                continue
            if name in whole and (t.dtype not in (torch.int32, getattr(torch, "uint32", torch.int32))):
                raise TypeError("%s must be int32" % name)
            if name in real and t.dtype != torch.float32:
                raise TypeError("%s must be fp32" % name)
            if tuple(t.shape) != (whole.get(name) or real.get(name)):
                raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), whole.get(name) or real.get(name)))
            if not t.is_contiguous():
                raise ValueError("%s must be contiguous" % name)
        devices = {t.get_device() for t in given.values() if t is not None}
        if len(devices) > 1:
            raise ValueError("the tensors of the rules must be on one device")
        self.tensors = given
        self._sizes = (rows, vocab, devices.pop() if devices else None)
        self.c = _LogitsRules(rows, vocab, n_history, n_bias, *(None if t is None else t.data_ptr() for t in given.values()))
        self._ref = C.byref(self.c)


class StageConfig:
    """Host-side description of a stage (mirrors swarm_stage_config)."""

    def __init__(self, d_model, n_heads, d_ffn, n_layers, n_repeat, batch, seq, dtype, ln_eps=1e-5,
                 block_kind=SWARM_BLOCK_GELU):
        if isinstance(block_kind, str):
            block_kind = {"gelu": SWARM_BLOCK_GELU, "rotary_geglu": SWARM_BLOCK_ROTARY_GEGLU}[block_kind]
        if isinstance(dtype, str):
            dtype = {"f32": SWARM_F32, "bf16": SWARM_BF16}[dtype]
        elif isinstance(dtype, torch.dtype):
            dtype = {torch.float32: SWARM_F32, torch.bfloat16: SWARM_BF16}[dtype]
        self.c = _Config(d_model, n_heads, d_ffn, n_layers, n_repeat, batch, seq, dtype, ln_eps, block_kind)

    @property
    def torch_dtype(self):
        return torch.float32 if self.c.dtype == SWARM_F32 else torch.bfloat16


def lib_path() -> str:
    return os.environ.get("SWARM_STAGE_LIB", os.path.join(_PKG, "libswarm_stage.so"))


def hooks_lib_path() -> str:
    return os.environ.get("SWARM_HOOKS_LIB", os.path.join(_PKG, "libswarm_hooks.so"))


_lib = None
_hooks_lib = None


def load_library():
    """Load libswarm_stage.so; raises if it has not been built (there is no fallback).  Inside a
    `with using_hooks_library():` block the instrumented build is returned instead."""
    global _lib
    if _lib is not None:
        return _lib
    _lib = _open(lib_path())
    return _lib


def load_hooks_library():
    """Load libswarm_hooks.so: the same sources plus the single-kernel entry points (swarm_kernel_*), the per-launch
    GEMM timer and the micro-benchmarks.  For tests and measurements only; the product is libswarm_stage.so."""
    global _hooks_lib
    if _hooks_lib is None:
        _hooks_lib = _open(hooks_lib_path())
    return _hooks_lib


@contextlib.contextmanager
def using_hooks_library():
    """Route every binding call inside the block to libswarm_hooks.so (bench.py times GEMM launches this way)."""
    global _lib
    product = load_library()
    _lib = load_hooks_library()
    try:
        yield _lib
    finally:
        _lib = product


def _open(path):
    if not os.path.exists(path):
        raise FileNotFoundError(
            "%s not found: build it with `python -m paper_2301_11913_amd.build` "
            "(the library has no CPU fallback)" % path)
    lib = C.CDLL(path)
    lib.swarm_stage_workspace_bytes.restype = C.c_size_t
    lib.swarm_stage_workspace_bytes.argtypes = [C.POINTER(_Config), C.c_int]
    lib.swarm_stage_forward.restype = C.c_int
    lib.swarm_stage_forward.argtypes = [C.POINTER(_Config), C.POINTER(_BlockPtrs), C.c_void_p, C.c_void_p,
                                        C.c_void_p, C.c_size_t, C.c_void_p]
    lib.swarm_stage_backward.restype = C.c_int
    lib.swarm_stage_backward.argtypes = [C.POINTER(_Config), C.POINTER(_BlockPtrs), C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.POINTER(_BlockPtrs), C.c_void_p, C.c_size_t, C.c_void_p]
    lib.swarm_codec_encode.restype = C.c_int
    lib.swarm_codec_encode.argtypes = [C.c_void_p, C.c_int32, C.c_size_t, C.c_int32, C.c_void_p, C.c_void_p,
                                       C.c_void_p]
    lib.swarm_codec_decode.restype = C.c_int
    lib.swarm_codec_decode.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.c_int32,
                                       C.c_void_p]
    lib.swarm_codec_encode_s16.restype = C.c_int
    lib.swarm_codec_encode_s16.argtypes = lib.swarm_codec_encode.argtypes
    lib.swarm_codec_decode_s16.restype = C.c_int
    lib.swarm_codec_decode_s16.argtypes = lib.swarm_codec_decode.argtypes
    lib.swarm_stage_coded_workspace_bytes.restype = C.c_size_t
    lib.swarm_stage_coded_workspace_bytes.argtypes = [C.POINTER(_Config), C.c_int]
    lib.swarm_stage_forward_coded.restype = C.c_int
    lib.swarm_stage_forward_coded.argtypes = [C.POINTER(_Config), C.POINTER(_BlockPtrs)] + [C.c_void_p] * 6 + \
                                             [C.c_size_t, C.c_void_p]
    lib.swarm_stage_backward_coded.restype = C.c_int
    lib.swarm_stage_backward_coded.argtypes = [C.POINTER(_Config), C.POINTER(_BlockPtrs)] + [C.c_void_p] * 5 + \
                                              [C.POINTER(_BlockPtrs), C.c_void_p, C.c_size_t, C.c_void_p]
    for suffix in ("", "_s16"):
        getattr(lib, "swarm_stage_forward_coded" + suffix).restype = C.c_int
        getattr(lib, "swarm_stage_forward_coded" + suffix).argtypes = lib.swarm_stage_forward_coded.argtypes
        getattr(lib, "swarm_stage_backward_coded" + suffix).restype = C.c_int
        getattr(lib, "swarm_stage_backward_coded" + suffix).argtypes = lib.swarm_stage_backward_coded.argtypes
    lib.swarm_boundary_workspace_bytes.restype = C.c_size_t
    lib.swarm_boundary_workspace_bytes.argtypes = [C.POINTER(_BoundaryConfig), C.c_int, C.c_int]
    for name in ("swarm_compress_forward", "swarm_decompress_forward"):
        fn = getattr(lib, name)
        fn.restype = C.c_int
        fn.argtypes = [C.POINTER(_BoundaryConfig), C.POINTER(_Ptrs3), C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t,
                       C.c_void_p]
    for name in ("swarm_compress_backward", "swarm_decompress_backward"):
        fn = getattr(lib, name)
        fn.restype = C.c_int
        fn.argtypes = [C.POINTER(_BoundaryConfig), C.POINTER(_Ptrs3), C.c_void_p, C.c_void_p, C.c_void_p,
                       C.POINTER(_Ptrs3), C.c_void_p, C.c_size_t, C.c_void_p]
    lib.swarm_embedding_forward.restype = C.c_int
    lib.swarm_embedding_forward.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                            C.c_void_p, C.c_void_p]
    lib.swarm_embedding_backward.restype = C.c_int
    lib.swarm_embedding_backward.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                             C.c_void_p, C.c_void_p]
    lib.swarm_head_workspace_bytes.restype = C.c_size_t
    lib.swarm_head_workspace_bytes.argtypes = [C.POINTER(_HeadConfig), C.c_int]
    lib.swarm_head_loss.restype = C.c_int
    lib.swarm_head_loss.argtypes = [C.POINTER(_HeadConfig), C.POINTER(_Ptrs3), C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.swarm_head_loss_backward.restype = C.c_int
    lib.swarm_head_loss_backward.argtypes = [C.POINTER(_HeadConfig), C.POINTER(_Ptrs3), C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(_Ptrs3), C.c_void_p,
                                             C.c_size_t, C.c_void_p]
    lib.swarm_lamb_workspace_bytes.restype = C.c_size_t
    lib.swarm_lamb_workspace_bytes.argtypes = [C.c_size_t]
    lib.swarm_lamb_step.restype = C.c_int
    lib.swarm_lamb_step.argtypes = [C.POINTER(_LambConfig), C.c_size_t, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    lib.swarm_lamb_step_static.restype = C.c_int
    lib.swarm_lamb_step_static.argtypes = [C.POINTER(_LambConfig), C.c_size_t, C.c_void_p, C.c_void_p, C.c_int32,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    P, I32, SZ = C.c_void_p, C.c_int32, C.c_size_t
    lib.swarm_cache_append.restype = C.c_int
    lib.swarm_cache_append.argtypes = [P] * 5 + [I32, P, P, P, SZ, P, I32, P, SZ, P]
    lib.swarm_cache_read.restype = C.c_int
    lib.swarm_cache_read.argtypes = [P] * 5 + [I32, P, P, P]
    lib.swarm_cache_keep.restype = C.c_int
    lib.swarm_cache_keep.argtypes = [P] * 6 + [I32, P]
    lib.swarm_cache_attention_workspace_bytes.restype = SZ
    lib.swarm_cache_attention_workspace_bytes.argtypes = [P, I32, I32]
    lib.swarm_cache_attention.restype = C.c_int
    lib.swarm_cache_attention.argtypes = [P] * 5 + [I32, I32, P, SZ, P, P, SZ, P, SZ, P]
    lib.swarm_stage_extend_workspace_bytes.restype = SZ
    lib.swarm_stage_extend_workspace_bytes.argtypes = [P, P, I32]
    lib.swarm_stage_extend.restype = C.c_int
    lib.swarm_stage_extend.argtypes = [P] * 9 + [I32, P, P, P, SZ, P]
    lib.swarm_head_logits.restype = C.c_int
    lib.swarm_head_logits.argtypes = [P] * 5 + [SZ, P]
    lib.swarm_logits_adjust.restype = C.c_int
    lib.swarm_logits_adjust.argtypes = [P, P, I32, SZ, P, SZ, P]
    lib.swarm_status_string.restype = C.c_char_p
    lib.swarm_status_string.argtypes = [C.c_int]
    return lib


def swarm_status_string(status: int) -> str:
    return load_library().swarm_status_string(int(status)).decode()


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to the stage library must be contiguous")
    return t.data_ptr()


# The current stream's handle without the torch.cuda.Stream object around it, which takes longer to make than a launch (a call
# of a small kernel 7.5 -> 5.0 us); where torch has no such functions, or CUDA is not initialised yet, the object is made.
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_current_device()) or None
        stream = torch.cuda.current_stream()
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


# The calls of token-by-token generation are as short as a launch, so their checks ask each tensor as little as they can: type, size,
# contiguity and device in one condition, and what is wrong only once something is.
_I32, _F32 = torch.int32, torch.float32
_WORDS = tuple(getattr(torch, n) for n in ("int64", "uint64") if hasattr(torch, n))


def _device() -> Optional[int]:
    """The current GPU; None where there is none, or none has been used yet (so no tensor can lie on it)."""
    return _current_device() if _current_device is not None and torch.cuda.is_initialized() else None


def _on(stream, device: Optional[int]) -> Optional[int]:
    """_stream where the current GPU is known already."""
    if stream is None and device is not None and _raw_stream is not None:
        return _raw_stream(device) or None
    return _stream(stream)


def _refuse(t: torch.Tensor, name: str, dtypes, n: Optional[int], device: Optional[int]):
    if t.dtype not in dtypes:
        raise TypeError("%s must be %s" % (name, " or ".join(str(d) for d in dtypes)))
    if n is not None and t.numel() != n:
        raise ValueError("%s has %d elements, expected %d" % (name, t.numel(), n))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    raise ValueError("%s is on %s, not on the current GPU (%s)" % (name, t.device, device))


def _ints(t: Optional[torch.Tensor], n: int, name: str, device: Optional[int]):
    """Pointer of n int32 values."""
    if t is None:
        return None
    if t.dtype is not _I32 or t.numel() != n or not t.is_contiguous() or t.get_device() != device:
        _refuse(t, name, (_I32,), n, device)
    return t.data_ptr()


def _buffer(t: torch.Tensor, n: Optional[int], dtype: torch.dtype, name: str, device: Optional[int]):
    """Pointer of n (None: any number of) values of a type."""
    if t.dtype is not dtype or (n is not None and t.numel() != n) or not t.is_contiguous() or t.get_device() != device:
        _refuse(t, name, (dtype,), n, device)
    return t.data_ptr()


def _rows(t: torch.Tensor, rows: int, width: int, dtype: torch.dtype, name: str, device: Optional[int]):
    """(pointer, pitch in elements) of a [rows, width] tensor whose rows may lie further apart; a single row has the pitch `width`."""
    if t.dtype is not dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    if t.shape != (rows, width):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), (rows, width)))
    pitch, step = t.stride()
    if step != 1 and width > 1:
        raise ValueError("the elements of a row of %s must be contiguous" % name)
    if t.get_device() != device:
        _refuse(t, name, (dtype,), None, device)
    return t.data_ptr(), (pitch if rows > 1 else width)


def _tree(tree: Optional[torch.Tensor], rows: int, device: Optional[int]):
    if tree is None:
        return None
    if tree.dtype not in _WORDS or tree.numel() != rows or not tree.is_contiguous() or tree.get_device() != device:
        _refuse(tree, "tree", _WORDS, rows, device)
    return tree.data_ptr()


def _workspace(t: Optional[torch.Tensor], device: Optional[int]):
    """(pointer, bytes); an empty workspace is none."""
    if t is None:
        return None, 0
    n = t.numel() * t.element_size()
    if n == 0:
        return None, 0
    if not t.is_contiguous() or t.get_device() != device:
        _refuse(t, "workspace", (t.dtype,), None, device)
    return t.data_ptr(), n


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return SWARM_F32
    if t.dtype == torch.bfloat16:
        return SWARM_BF16
    raise TypeError("unsupported dtype %s" % t.dtype)


def _block_array(blocks: Sequence[Dict[str, torch.Tensor]]):
    return (_BlockPtrs * len(blocks))(*(_BlockPtrs(*(_ptr(b[k]) for k in PARAM_FIELDS)) for b in blocks))


def swarm_stage_workspace_bytes(cfg: StageConfig, for_backward: bool) -> int:
    return int(load_library().swarm_stage_workspace_bytes(C.byref(cfg.c), 1 if for_backward else 0))


def swarm_stage_forward(cfg: StageConfig, params: List[Dict[str, torch.Tensor]], x_in: torch.Tensor,
                        x_out: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    st = load_library().swarm_stage_forward(C.byref(cfg.c), _block_array(params), _ptr(x_in), _ptr(x_out),
                                            _ptr(workspace), workspace.numel() * workspace.element_size(),
                                            _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_stage_forward")


def swarm_stage_backward(cfg: StageConfig, params: List[Dict[str, torch.Tensor]], x_in: torch.Tensor,
                         grad_out: torch.Tensor, grad_in: torch.Tensor,
                         grad_params: List[Dict[str, torch.Tensor]], workspace: torch.Tensor,
                         stream=None) -> None:
    for g in grad_params:
        for k in PARAM_FIELDS:
            if g[k].dtype != torch.float32:
                raise TypeError("grad_params must be fp32")
    st = load_library().swarm_stage_backward(C.byref(cfg.c), _block_array(params), _ptr(x_in), _ptr(grad_out),
                                             _ptr(grad_in), _block_array(grad_params), _ptr(workspace),
                                             workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_stage_backward")


def swarm_codec_encode(tensor: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, block: int = 64,
                       stream=None) -> None:
    if codes.dtype != torch.int8 or scales.dtype != torch.float32:
        raise TypeError("codes must be int8 and scales fp32")
    st = load_library().swarm_codec_encode(_ptr(tensor), _dtype_code(tensor), tensor.numel(), block, _ptr(codes),
                                           _ptr(scales), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_codec_encode")


def swarm_codec_decode(codes: torch.Tensor, scales: torch.Tensor, tensor: torch.Tensor, block: int = 64,
                       stream=None) -> None:
    if codes.dtype != torch.int8 or scales.dtype != torch.float32:
        raise TypeError("codes must be int8 and scales fp32")
    st = load_library().swarm_codec_decode(_ptr(codes), _ptr(scales), tensor.numel(), block, _ptr(tensor),
                                           _dtype_code(tensor), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_codec_decode")


def swarm_codec_encode_s16(tensor: torch.Tensor, codes: torch.Tensor, scales: torch.Tensor, block: int = 64,
                           stream=None) -> None:
    """scales: int16 / uint16 tensor receiving bf16 bit patterns (or a bf16 tensor, which is the same memory)."""
    if codes.dtype != torch.int8 or scales.element_size() != 2:
        raise TypeError("codes must be int8 and scales a 16-bit tensor")
    st = load_library().swarm_codec_encode_s16(_ptr(tensor), _dtype_code(tensor), tensor.numel(), block, _ptr(codes),
                                               _ptr(scales), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_codec_encode_s16")


def swarm_codec_decode_s16(codes: torch.Tensor, scales: torch.Tensor, tensor: torch.Tensor, block: int = 64,
                           stream=None) -> None:
    if codes.dtype != torch.int8 or scales.element_size() != 2:
        raise TypeError("codes must be int8 and scales a 16-bit tensor")
    st = load_library().swarm_codec_decode_s16(_ptr(codes), _ptr(scales), tensor.numel(), block, _ptr(tensor),
                                               _dtype_code(tensor), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_codec_decode_s16")


def swarm_stage_coded_workspace_bytes(cfg: StageConfig, for_backward: bool) -> int:
    return int(load_library().swarm_stage_coded_workspace_bytes(C.byref(cfg.c), 1 if for_backward else 0))


def _scale_suffix(*scales: torch.Tensor) -> str:
    """"" for fp32 block scales, "_s16" for 16-bit ones (all scale tensors of a call must agree)."""
    sizes = {t.element_size() for t in scales}
    if sizes == {4} and all(t.dtype == torch.float32 for t in scales):
        return ""
    if sizes == {2}:
        return "_s16"
    raise TypeError("block scales must be all fp32 or all 16-bit tensors")


def swarm_stage_forward_coded(cfg: StageConfig, params: List[Dict[str, torch.Tensor]], x_codes: torch.Tensor,
                              x_scales: torch.Tensor, x_dec: torch.Tensor, y_codes: torch.Tensor,
                              y_scales: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """fp32 scale tensors call swarm_stage_forward_coded, 16-bit ones swarm_stage_forward_coded_s16."""
    name = "swarm_stage_forward_coded" + _scale_suffix(x_scales, y_scales)
    st = getattr(load_library(), name)(C.byref(cfg.c), _block_array(params), _ptr(x_codes), _ptr(x_scales),
                                       _ptr(x_dec), _ptr(y_codes), _ptr(y_scales), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SwarmError(st, name)


def swarm_stage_backward_coded(cfg: StageConfig, params: List[Dict[str, torch.Tensor]], x_in: torch.Tensor,
                               g_codes: torch.Tensor, g_scales: torch.Tensor, gin_codes: torch.Tensor,
                               gin_scales: torch.Tensor, grad_params: List[Dict[str, torch.Tensor]],
                               workspace: torch.Tensor, stream=None) -> None:
    name = "swarm_stage_backward_coded" + _scale_suffix(g_scales, gin_scales)
    st = getattr(load_library(), name)(C.byref(cfg.c), _block_array(params), _ptr(x_in), _ptr(g_codes),
                                       _ptr(g_scales), _ptr(gin_codes), _ptr(gin_scales),
                                       _block_array(grad_params), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SwarmError(st, name)


def _ptrs3(d: Dict[str, torch.Tensor], wkey: str):
    return _Ptrs3(_ptr(d["ln_g"]), _ptr(d["ln_b"]), _ptr(d.get(wkey)))


def _check_f32(grads: Dict[str, torch.Tensor]):
    for g in grads.values():
        if g is not None and g.dtype != torch.float32:
            raise TypeError("parameter gradients must be fp32")


def swarm_boundary_workspace_bytes(cfg: BoundaryConfig, decompress: bool, for_backward: bool) -> int:
    return int(load_library().swarm_boundary_workspace_bytes(C.byref(cfg.c), int(decompress), int(for_backward)))


def swarm_compress_forward(cfg: BoundaryConfig, params: Dict[str, torch.Tensor], y: torch.Tensor, z: torch.Tensor,
                           workspace: torch.Tensor, stream=None) -> None:
    st = load_library().swarm_compress_forward(C.byref(cfg.c), C.byref(_ptrs3(params, "w_c")), _ptr(y), _ptr(z),
                                               _ptr(workspace), workspace.numel() * workspace.element_size(),
                                               _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_compress_forward")


def swarm_compress_backward(cfg: BoundaryConfig, params: Dict[str, torch.Tensor], y: torch.Tensor, dz: torch.Tensor,
                            dy: torch.Tensor, grads: Dict[str, torch.Tensor], workspace: torch.Tensor,
                            stream=None) -> None:
    _check_f32(grads)
    st = load_library().swarm_compress_backward(C.byref(cfg.c), C.byref(_ptrs3(params, "w_c")), _ptr(y), _ptr(dz),
                                                _ptr(dy), C.byref(_ptrs3(grads, "w_c")), _ptr(workspace),
                                                workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_compress_backward")


def swarm_decompress_forward(cfg: BoundaryConfig, params: Dict[str, torch.Tensor], z: torch.Tensor, x: torch.Tensor,
                             workspace: torch.Tensor, stream=None) -> None:
    st = load_library().swarm_decompress_forward(C.byref(cfg.c), C.byref(_ptrs3(params, "w_d")), _ptr(z), _ptr(x),
                                                 _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                 _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_decompress_forward")


def swarm_decompress_backward(cfg: BoundaryConfig, params: Dict[str, torch.Tensor], z: torch.Tensor, dx: torch.Tensor,
                              dz: torch.Tensor, grads: Dict[str, torch.Tensor], workspace: torch.Tensor,
                              stream=None) -> None:
    _check_f32(grads)
    st = load_library().swarm_decompress_backward(C.byref(cfg.c), C.byref(_ptrs3(params, "w_d")), _ptr(z), _ptr(dx),
                                                  _ptr(dz), C.byref(_ptrs3(grads, "w_d")), _ptr(workspace),
                                                  workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_decompress_backward")


def swarm_embedding_forward(tokens: torch.Tensor, table: torch.Tensor, vocab: int, x: torch.Tensor,
                            stream=None) -> None:
    if tokens.dtype != torch.int32:
        raise TypeError("token ids must be int32")
    st = load_library().swarm_embedding_forward(_ptr(tokens), _ptr(table), _dtype_code(table), tokens.numel(), vocab,
                                                table.shape[1], _ptr(x), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_embedding_forward")


def swarm_embedding_backward(tokens: torch.Tensor, dx: torch.Tensor, vocab: int, grad_table: torch.Tensor,
                             stream=None) -> None:
    if tokens.dtype != torch.int32 or grad_table.dtype != torch.float32:
        raise TypeError("token ids must be int32 and grad_table fp32")
    st = load_library().swarm_embedding_backward(_ptr(tokens), _ptr(dx), _dtype_code(dx), tokens.numel(), vocab,
                                                 dx.shape[1], _ptr(grad_table), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_embedding_backward")


def swarm_head_workspace_bytes(cfg: HeadConfig, for_backward: bool) -> int:
    return int(load_library().swarm_head_workspace_bytes(C.byref(cfg.c), int(for_backward)))


def swarm_head_loss(cfg: HeadConfig, params: Dict[str, torch.Tensor], x: torch.Tensor, targets: torch.Tensor,
                    loss: torch.Tensor, token_loss: Optional[torch.Tensor], workspace: torch.Tensor,
                    stream=None) -> None:
    if targets.dtype != torch.int32 or loss.dtype != torch.float32:
        raise TypeError("targets must be int32 and loss fp32")
    st = load_library().swarm_head_loss(C.byref(cfg.c), C.byref(_ptrs3(params, "w_vocab")), _ptr(x), _ptr(targets),
                                        _ptr(loss), _ptr(token_loss), _ptr(workspace),
                                        workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_head_loss")


def swarm_head_loss_backward(cfg: HeadConfig, params: Dict[str, torch.Tensor], x: torch.Tensor, targets: torch.Tensor,
                             loss: torch.Tensor, token_loss: Optional[torch.Tensor], dx: torch.Tensor,
                             grads: Dict[str, torch.Tensor], workspace: torch.Tensor, stream=None) -> None:
    if targets.dtype != torch.int32 or loss.dtype != torch.float32:
        raise TypeError("targets must be int32 and loss fp32")
    _check_f32(grads)
    st = load_library().swarm_head_loss_backward(C.byref(cfg.c), C.byref(_ptrs3(params, "w_vocab")), _ptr(x),
                                                 _ptr(targets), _ptr(loss), _ptr(token_loss), _ptr(dx),
                                                 C.byref(_ptrs3(grads, "w_vocab")), _ptr(workspace),
                                                 workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_head_loss_backward")


def swarm_lamb_workspace_bytes(n_elems: int) -> int:
    return int(load_library().swarm_lamb_workspace_bytes(n_elems))


def swarm_lamb_step(master: torch.Tensor, param: Optional[torch.Tensor], grad: torch.Tensor, m: torch.Tensor,
                    v: torch.Tensor, step: int, workspace: torch.Tensor, lr: float = 1e-3, beta1: float = 0.9,
                    beta2: float = 0.95, eps: float = 1e-6, weight_decay: float = 0.01, grad_scale: float = 1.0,
                    trust_ratio: Optional[torch.Tensor] = None, stream=None) -> None:
    for t in (master, grad, m, v):
        if t.dtype != torch.float32:
            raise TypeError("master weights, gradient and moments must be fp32")
    cfg = _LambConfig(lr, beta1, beta2, eps, weight_decay, grad_scale, step)
    st = load_library().swarm_lamb_step(C.byref(cfg), master.numel(), _ptr(master), _ptr(param),
                                        _dtype_code(param) if param is not None else SWARM_F32, _ptr(grad), _ptr(m),
                                        _ptr(v), _ptr(trust_ratio), _ptr(workspace),
                                        workspace.numel() * workspace.element_size(), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_lamb_step")


SWARM_LAMB_STATIC_MAX_ELEMS = 1 << 24


def swarm_lamb_step_static(master: torch.Tensor, param: Optional[torch.Tensor], grad: torch.Tensor, m: torch.Tensor,
                           v: torch.Tensor, step: int, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.95,
                           eps: float = 1e-6, weight_decay: float = 0.01, grad_scale: float = 1.0,
                           trust_ratio: Optional[torch.Tensor] = None, stream=None) -> None:
    for t in (master, grad, m, v):
        if t.dtype != torch.float32:
            raise TypeError("master weights, gradient and moments must be fp32")
    cfg = _LambConfig(lr, beta1, beta2, eps, weight_decay, grad_scale, step)
    st = load_library().swarm_lamb_step_static(C.byref(cfg), master.numel(), _ptr(master), _ptr(param),
                                               _dtype_code(param) if param is not None else SWARM_F32, _ptr(grad),
                                               _ptr(m), _ptr(v), _ptr(trust_ratio), _stream(stream))
    if st != 0:
        raise SwarmError(st, "swarm_lamb_step_static")


def _pool(cfg: CacheConfig, cache: Cache, device: Optional[int]):
    if cache._pool != cfg._pool:
        raise ValueError("the cache was made for another configuration")
    if cache._device != device:
        raise ValueError("the cache is on GPU %d, the current GPU is %s" % (cache._device, device))
    return cache._ref


def swarm_cache_append(cfg: CacheConfig, cache: Cache, page_table: torch.Tensor, past: torch.Tensor,
                       fresh: Optional[torch.Tensor], tokens: int, k: torch.Tensor, v: torch.Tensor,
                       q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                       positions: Optional[torch.Tensor] = None, rotary: bool = False, stream=None) -> None:
    """q, k, v: [batch * tokens, heads * d_head] views of one row pitch (the columns of a fused product)."""
    batch, pages, q_width, kv_width, dt = cfg._sizes
    rows, dev = batch * tokens, _device()
    kp, pitch = _rows(k, rows, kv_width, dt, "k", dev)
    vp, v_pitch = _rows(v, rows, kv_width, dt, "v", dev)
    qp, q_pitch, op, out_pitch = None, pitch, None, 0
    if q is not None:
        qp, q_pitch = _rows(q, rows, q_width, dt, "q", dev)
        if rows == 1:                   # a single row has no pitch
            pitch = v_pitch = q_pitch
    if q_out is not None:
        op, out_pitch = _rows(q_out, rows, q_width, dt, "q_out", dev)
    if v_pitch != pitch or q_pitch != pitch:
        raise ValueError("q, k and v must have the same row pitch")
    st = load_library().swarm_cache_append(cfg._ref, _pool(cfg, cache, dev), _ints(page_table, pages, "page_table", dev),
                                           _ints(past, batch, "past", dev), _ints(fresh, batch, "fresh", dev), tokens, qp, kp, vp,
                                           pitch, _ints(positions, rows, "positions", dev), 1 if rotary else 0, op, out_pitch,
                                           _on(stream, dev))
    if st != 0:
        raise SwarmError(st, "swarm_cache_append")


def swarm_cache_read(cfg: CacheConfig, cache: Cache, page_table: torch.Tensor, first: torch.Tensor,
                     count: Optional[torch.Tensor], tokens: int, k_out: torch.Tensor, v_out: torch.Tensor, stream=None) -> None:
    batch, pages, _, kv_width, dt = cfg._sizes
    n, dev = batch * tokens * kv_width, _device()
    st = load_library().swarm_cache_read(cfg._ref, _pool(cfg, cache, dev), _ints(page_table, pages, "page_table", dev),
                                         _ints(first, batch, "first", dev), _ints(count, batch, "count", dev), tokens,
                                         _buffer(k_out, n, dt, "k_out", dev), _buffer(v_out, n, dt, "v_out", dev), _on(stream, dev))
    if st != 0:
        raise SwarmError(st, "swarm_cache_read")


def swarm_cache_keep(cfg: CacheConfig, cache: Cache, page_table: torch.Tensor, past: torch.Tensor, kept: torch.Tensor,
                     n_kept: torch.Tensor, tokens: int, stream=None) -> None:
    batch, pages = cfg._sizes[:2]
    dev = _device()
    st = load_library().swarm_cache_keep(cfg._ref, _pool(cfg, cache, dev), _ints(page_table, pages, "page_table", dev),
                                         _ints(past, batch, "past", dev), _ints(kept, batch * tokens, "kept", dev),
                                         _ints(n_kept, batch, "n_kept", dev), tokens, _on(stream, dev))
    if st != 0:
        raise SwarmError(st, "swarm_cache_keep")


def swarm_cache_attention_workspace_bytes(cfg: CacheConfig, tokens: int, max_len: int = 0) -> int:
    return int(load_library().swarm_cache_attention_workspace_bytes(cfg._ref, tokens, max_len))


def swarm_cache_attention(cfg: CacheConfig, cache: Cache, page_table: torch.Tensor, past: torch.Tensor,
                          fresh: Optional[torch.Tensor], tokens: int, q: torch.Tensor, out: torch.Tensor,
                          workspace: Optional[torch.Tensor], tree: Optional[torch.Tensor] = None, max_len: int = 0,
                          stream=None) -> None:
    """q, out: [batch * tokens, n_heads * d_head]; their rows may lie further apart."""
    batch, pages, width, _, dt = cfg._sizes
    rows, dev = batch * tokens, _device()
    qp, q_pitch = _rows(q, rows, width, dt, "q", dev)
    op, out_pitch = _rows(out, rows, width, dt, "out", dev)
    wp, n = _workspace(workspace, dev)
    st = load_library().swarm_cache_attention(cfg._ref, _pool(cfg, cache, dev), _ints(page_table, pages, "page_table", dev),
                                              _ints(past, batch, "past", dev), _ints(fresh, batch, "fresh", dev), tokens, max_len,
                                              qp, q_pitch, _tree(tree, rows, dev), op, out_pitch, wp, n, _on(stream, dev))
    if st != 0:
        raise SwarmError(st, "swarm_cache_attention")


def swarm_stage_extend_workspace_bytes(cfg: StageConfig, cache_cfg: CacheConfig, max_len: int = 0) -> int:
    return int(load_library().swarm_stage_extend_workspace_bytes(C.byref(cfg.c), cache_cfg._ref, max_len))


def swarm_stage_extend(cfg: StageConfig, params: List[Dict[str, torch.Tensor]], cache_cfg: CacheConfig, caches: Sequence[Cache],
                       page_table: torch.Tensor, past: torch.Tensor, fresh: Optional[torch.Tensor], x_in: torch.Tensor,
                       x_out: torch.Tensor, workspace: torch.Tensor, positions: Optional[torch.Tensor] = None,
                       tree: Optional[torch.Tensor] = None, max_len: int = 0, stream=None) -> None:
    """caches: one for each of the n_layers * n_repeat applications, in their order."""
    c, dev = cfg.c, _device()
    batch, pages = cache_cfg._sizes[:2]
    rows = c.batch * c.seq
    if len(params) != c.n_layers or len(caches) != c.n_layers * c.n_repeat:
        raise ValueError("the stage has %d parameter sets and %d applications" % (c.n_layers, c.n_layers * c.n_repeat))
    for pool in caches:
        _pool(cache_cfg, pool, dev)
    pools = (_Cache * len(caches))(*(pool.c for pool in caches))
    wp, n = _workspace(workspace, dev)
    st = load_library().swarm_stage_extend(C.byref(c), _block_array(params), cache_cfg._ref, pools,
                                           _ints(page_table, pages, "page_table", dev), _ints(past, batch, "past", dev),
                                           _ints(fresh, batch, "fresh", dev), _ints(positions, rows, "positions", dev),
                                           _tree(tree, rows, dev), max_len, _buffer(x_in, rows * c.d_model, cfg.torch_dtype, "x_in", dev),
                                           _buffer(x_out, rows * c.d_model, cfg.torch_dtype, "x_out", dev), wp, n, _on(stream, dev))
    if st != 0:
        raise SwarmError(st, "swarm_stage_extend")


def swarm_head_logits(cfg: HeadConfig, params: Dict[str, torch.Tensor], x: torch.Tensor, logits: torch.Tensor,
                      workspace: torch.Tensor, stream=None) -> None:
    c, dev = cfg.c, _device()
    dt = torch.float32 if c.dtype == SWARM_F32 else torch.bfloat16
    wp, n = _workspace(workspace, dev)
    st = load_library().swarm_head_logits(C.byref(c), C.byref(_ptrs3(params, "w_vocab")), _buffer(x, c.tokens * c.d_model, dt, "x", dev),
                                          _buffer(logits, c.tokens * c.vocab_rows, dt, "logits", dev), wp, n, _on(stream, dev))
    if st != 0:
        raise SwarmError(st, "swarm_head_logits")


def swarm_logits_adjust(rules: LogitsRules, logits: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """logits [rows, >= vocab] fp32 or bf16, out [rows, >= vocab] fp32; rows may lie further apart."""
    rows, vocab, rules_dev = rules._sizes
    dev = _device()
    if logits.dim() != 2 or logits.shape[1] < vocab or out.dim() != 2 or out.shape[1] < vocab:
        raise ValueError("logits and out must be [rows, vocab or more]")
    lp, pitch = _rows(logits, rows, logits.shape[1], logits.dtype, "logits", dev)
    op, out_pitch = _rows(out, rows, out.shape[1], _F32, "out", dev)
    if rules_dev is not None and rules_dev != dev:
        raise ValueError("the rules are on GPU %d, the current GPU is %s" % (rules_dev, dev))
    st = load_library().swarm_logits_adjust(rules._ref, lp, _dtype_code(logits), pitch, op, out_pitch, _on(stream, dev))
    if st != 0:
        raise SwarmError(st, "swarm_logits_adjust")

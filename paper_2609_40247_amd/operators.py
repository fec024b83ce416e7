"""Reference operators: the attention layer of a served model on MI355X, and what a decoder layer has around it.

The C ABI is ``include/herschel_ops.h``; this module checks tensors, fills its
structures and calls the HIP library:

``PagedCache``       a paged cache of keys and values, 16-bit or 8-bit
``rotary_table``     cos and sin of the rotary positions, scaled for long contexts
``rope_write``       rotary positions, and the quantising write into the cache
``cache_read``       rows of the cache back in 16 bits
``attn_prompt``      attention over packed prompts
``DecodeAttention``  attention of new tokens over the cache (keeps the workspace)
``norm_rows``        root-mean-square norm with the residual's addition, to 16 bits or 8 (``Rows8``)
``Weights4``         a matrix of 4-bit weights with a scale for each group of a row
``product4``         rows, 16-bit or 8-bit, times such a matrix, gated where asked for
``verify_drafts``    drafted tokens against the target's probabilities

Every call is enqueued on torch's current stream and returns at once.  What
only the device can see to be wrong (a page id, a length, a position, a slot)
is reported by ``PagedCache.check`` or, without a cache, through ``status``.
There is no backward pass: rows that require gradients are refused in grad
mode.  There is no CPU fallback: without the built library or a GPU the calls raise.
"""
from __future__ import annotations

import ctypes
import functools
import math
import struct
from typing import NamedTuple

import torch

from . import herschel as H

BF16, F16, FP8, INT8, F32 = 0, 1, 2, 3, 4
TYPES = {torch.bfloat16: BF16, torch.float16: F16}
KINDS = {**TYPES, torch.float8_e4m3fn: FP8, torch.int8: INT8}
LAYOUTS = {"half": 0, "interleaved": 1}
CODES = {torch.float8_e4m3fn: FP8, torch.int8: INT8}
BAD_PAGE, BAD_LENGTH, BAD_POSITION, BAD_SLOT, BAD_TOKEN, BAD_ROW = 1, 2, 4, 8, 16, 32
MAX_DECODE_SEQS, MAX_NORM_DIM, MAX_PRODUCT_ROWS, MAX_WEIGHT_ROWS, MAX_DRAFTS = 4096, 32768, 4_194_240, 715_827_840, 1024
_FAULTS = {BAD_PAGE: "a block table entry outside the cache", BAD_LENGTH: "lengths that do not fit the buffers",
           BAD_POSITION: "a position outside the rotary table", BAD_SLOT: "a slot beyond the cache's end",
           BAD_TOKEN: "a drafted token outside the vocabulary", BAD_ROW: "probabilities of which none is above 0"}

_P = ctypes.c_void_p
_I64, _I32 = ctypes.c_int64, ctypes.c_int32


class _Strides(ctypes.Structure):
    _fields_ = [("row", _I64), ("head", _I64)]


class HerschelCache(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("k_scale", _P), ("v_scale", _P), ("n_pages", _I64), ("n_heads", _I32),
                ("page_size", _I32), ("head_dim", _I32), ("kind", _I32)]


class HerschelRopeArgs(ctypes.Structure):
    _fields_ = [("q", _P), ("k", _P), ("v", _P), ("q_strides", _Strides), ("k_strides", _Strides),
                ("v_strides", _Strides), ("q_out", _P), ("k_out", _P), ("q_out_strides", _Strides),
                ("k_out_strides", _Strides), ("positions", _P), ("table", _P), ("n_positions", _I64), ("slots", _P),
                ("n_tokens", _I64), ("q_heads", _I32), ("kv_heads", _I32), ("head_dim", _I32), ("rotary_dim", _I32),
                ("layout", _I32), ("type", _I32), ("status", _P), ("hip_stream", _P)]


class HerschelReadArgs(ctypes.Structure):
    _fields_ = [("block_table", _P), ("table_stride", _I64), ("cu", _P), ("n_seqs", _I32), ("n_rows", _I64),
                ("k_out", _P), ("v_out", _P), ("type", _I32), ("status", _P), ("hip_stream", _P)]


class HerschelPromptArgs(ctypes.Structure):
    _fields_ = [("q", _P), ("k", _P), ("v", _P), ("q_strides", _Strides), ("k_strides", _Strides),
                ("v_strides", _Strides), ("out", _P), ("lse", _P), ("cu_q", _P), ("cu_k", _P), ("n_seqs", _I32),
                ("n_q", _I64), ("n_k", _I64), ("max_q", _I32), ("q_heads", _I32), ("kv_heads", _I32),
                ("head_dim", _I32), ("type", _I32), ("causal", _I32), ("window", _I32), ("scale", ctypes.c_float),
                ("workspace", _P), ("workspace_bytes", ctypes.c_size_t), ("status", _P), ("hip_stream", _P)]


class HerschelDecodeArgs(ctypes.Structure):
    _fields_ = [("q", _P), ("q_seq_stride", _I64), ("q_strides", _Strides), ("out", _P), ("lse", _P),
                ("block_table", _P), ("table_stride", _I64), ("seq_lens", _P), ("n_seqs", _I32), ("new_tokens", _I32),
                ("q_heads", _I32), ("type", _I32), ("window", _I32), ("scale", ctypes.c_float), ("workspace", _P),
                ("workspace_bytes", ctypes.c_size_t), ("status", _P), ("hip_stream", _P)]


class HerschelNormArgs(ctypes.Structure):
    _fields_ = [("x", _P), ("x_row", _I64), ("residual", _P), ("residual_row", _I64), ("residual_out", _P),
                ("residual_out_row", _I64), ("weight", _P), ("out", _P), ("scale", _P), ("n_rows", _I64), ("dim", _I32),
                ("group", _I32), ("type", _I32), ("residual_type", _I32), ("weight_type", _I32), ("out_kind", _I32),
                ("eps", ctypes.c_float), ("hip_stream", _P)]


class HerschelWeights4(ctypes.Structure):
    _fields_ = [("codes", _P), ("scales", _P), ("n", _I32), ("k", _I32), ("group", _I32)]


class HerschelProductArgs(ctypes.Structure):
    _fields_ = [("x", _P), ("x_row", _I64), ("x_scale", _P), ("out", _P), ("n_rows", _I64), ("kind", _I32),
                ("x_group", _I32), ("type", _I32), ("gated", _I32), ("workspace", _P), ("workspace_bytes", ctypes.c_size_t),
                ("hip_stream", _P)]


class HerschelVerifyArgs(ctypes.Structure):
    _fields_ = [("target", _P), ("target_seq", _I64), ("target_row", _I64), ("draft", _P), ("draft_seq", _I64),
                ("draft_row", _I64), ("tokens", _P), ("counts", _P), ("accept_u", _P), ("final_u", _P), ("out", _P),
                ("accepted", _P), ("n_seqs", _I32), ("n_drafts", _I32), ("vocab", _I32), ("type", _I32),
                ("workspace", _P), ("workspace_bytes", ctypes.c_size_t), ("status", _P), ("hip_stream", _P)]


# The same structures as struct formats: filling one this way takes 0.2 us
# instead of 1 to 2, and a decode step's calls are as short as their host time.
_ROPE = struct.Struct("@3P6q2P4q2PqPq6i2P")
_READ = struct.Struct("@PqPiq2Pi2P")
_PROMPT = struct.Struct("@3P6q4Pi2q7ifPN2P")
_DECODE = struct.Struct("@P3q3PqP5ifPN2P")
_NORM = struct.Struct("@PqPqPq3Pq6ifP")
_PRODUCT = struct.Struct("@Pq2Pq4iPNP")
_VERIFY = struct.Struct("@P2qP2q6P4iPN2P")

_ready = {}


def load(variant: str | None = None) -> ctypes.CDLL:
    """The library of ``herschel.load`` with the operators' signatures."""
    lib = _ready.get(variant) if variant else None
    if lib is None:
        lib = H.load(variant)
        for name, n in (("herschel_rope_write", 2), ("herschel_cache_read", 2), ("herschel_attn_prompt", 1),
                        ("herschel_attn_decode", 2), ("herschel_norm_rows", 1), ("herschel_product4", 2),
                        ("herschel_verify_drafts", 1)):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = ctypes.c_int, [_P] * n
        lib.herschel_attn_prompt_workspace.restype = ctypes.c_int
        lib.herschel_attn_prompt_workspace.argtypes = [_I32, _I64, _I64, _I32, _I32, _I32, _I32,
                                                       ctypes.POINTER(ctypes.c_size_t)]
        lib.herschel_attn_decode_workspace.restype = ctypes.c_int
        lib.herschel_attn_decode_workspace.argtypes = [_I32, _I32, _I32, _P, ctypes.POINTER(ctypes.c_size_t)]
        lib.herschel_product4_workspace.restype = ctypes.c_int
        lib.herschel_product4_workspace.argtypes = [_I64, _I32, _I32, _I32, _I32, ctypes.POINTER(ctypes.c_size_t)]
        lib.herschel_verify_workspace.restype = ctypes.c_int
        lib.herschel_verify_workspace.argtypes = [_I32, _I32, ctypes.POINTER(ctypes.c_size_t)]
        if variant:
            _ready[variant] = lib
    return lib


def _lib() -> ctypes.CDLL:
    """The library that $HERSCHEL_LIB named at the first call."""
    lib = _ready.get(None)
    if lib is None:
        lib = _ready[None] = load()
    return lib


# ------------------------------------------------------------ checks
def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _rows(t: torch.Tensor, name: str, dims: int = 3) -> tuple:
    """The strides of a tensor of rows of heads on a GPU whose heads' elements are contiguous."""
    st = t.stride()
    if not (t.is_cuda and len(st) == dims and t.dtype in TYPES and (st[-1] == 1 or t.shape[-1] < 2)):
        _need(t.is_cuda, f"{name} must be on a GPU")
        _need(t.dim() == dims, f"{name} must have {dims} dimensions")
        _need(t.dtype in TYPES, f"{name} must be bfloat16 or float16")
        _need(False, f"{name}'s last dimension must be contiguous")
    return st


def _ints(t: torch.Tensor, name: str, dtype, shape: tuple, device: int) -> int:
    """The address of a contiguous tensor of this type and shape on a GPU."""
    if t.dtype is not dtype or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        _need(t.dtype == dtype, f"{name} must be {dtype}")
        _need(t.get_device() == device, f"{name} must be on GPU {device}")
        _need(tuple(t.shape) == tuple(shape), f"{name} must have shape {tuple(shape)}")
        _need(False, f"{name} must be contiguous")
    return t.data_ptr()


def _like(t: torch.Tensor, first: torch.Tensor, name: str) -> None:
    if t.dtype is not first.dtype or t.get_device() != first.get_device():
        _need(False, f"{name} must have the type and device of the other rows")


def _table(t: torch.Tensor, n_seqs: int, device: int) -> int:
    if not (t.dtype == torch.int32 and t.dim() == 2 and t.shape[0] == n_seqs and t.get_device() == device and
            t.is_contiguous()):
        _need(False, f"block_table must be int32 [{n_seqs}, entries], contiguous, on GPU {device}")
    return t.data_ptr()


def _no_gradients(name: str) -> None:
    """For a call with tensors that require gradients: its results would be cut off from them without a word."""
    if torch.is_grad_enabled():
        raise ValueError(f"{name} has no backward pass: call it under torch.no_grad() or with detached tensors")


# Tells autograd that tensors were written, so that a backward pass that needs their old values raises.
_written = getattr(torch._C, "_increment_version", None) or torch.autograd.graph.increment_version


def _call(fn, device: int, name: str, args: bytes, cache: int | None = None) -> None:
    """Calls an entry point with the tensors' device current."""
    if _device() == device:
        code = fn(args) if cache is None else fn(args, cache or None)
    else:
        with torch.cuda.device(device):
            code = fn(args) if cache is None else fn(args, cache or None)
    if code != H.OK:
        raise (ValueError if code == H.EINVAL else RuntimeError)(f"{name}: {H.herschel_strerror(code)}")


# The current stream's handle by itself: 0.1 us, the Stream object around it 2.
# The device likewise: the tensors have initialised torch's GPU state by then.
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", None) or torch.cuda.is_current_stream_capturing


def _captured(device: int) -> bool:
    """Whether the device's current stream is being captured into a graph."""
    if _device() == device:
        return _capturing()
    with torch.cuda.device(device):
        return _capturing()


def _status(status: torch.Tensor | None, device: int) -> int:
    if status is None:
        return 0
    _need(status.dtype == torch.int32 and status.numel() == 1 and status.get_device() == device,
          "status must be one int32 on the tensors' device")
    return status.data_ptr()


def raise_faults(status: torch.Tensor) -> None:
    """Waits for the device, all its streams, takes what calls reported out of ``status`` and raises it.  What calls
    report meanwhile, enqueued by another thread, stays for the next time."""
    torch.cuda.synchronize(status.device)
    bits = int(status.item())
    if bits:
        # bits are only ever set, so an addition clears them; it is atomic, like the kernels' setting of others
        status.view(1).index_add_(0, torch.zeros(1, dtype=torch.int32, device=status.device), torch.full_like(status.view(1), -bits))
        raise ValueError("; ".join(text for bit, text in _FAULTS.items() if bits & bit))


# ------------------------------------------------------------ the cache
class PagedCache:
    """Keys and values [pages, heads, page size, head dim], contiguous, of
    bfloat16, float16, float8_e4m3fn or int8; 8-bit ones with a float32 scale
    [pages, heads, page size] for each row.  The tensors are the caller's."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None,
                 v_scale: torch.Tensor | None = None):
        _need(k.is_cuda and k.dim() == 4 and k.dtype in KINDS, "k must be [pages, heads, page size, head dim] on a GPU, "
              "bfloat16, float16, float8_e4m3fn or int8")
        _need(v.shape == k.shape and v.dtype == k.dtype and v.device == k.device, "v must be like k")
        _need(k.is_contiguous() and v.is_contiguous(), "k and v must be contiguous")
        _need(k.shape[2] in (16, 32, 64, 128, 256), "the page size must be 16, 32, 64, 128 or 256")
        _need(2 <= k.shape[3] <= 256 and k.shape[3] % 2 == 0, "the head dimension must be even, at most 256")
        _need(k.shape[0] >= 1 and k.shape[1] >= 1, "the cache must have a page and a head")
        _need(not (k.requires_grad or v.requires_grad), "k and v must not require gradients")
        self.quantised = KINDS[k.dtype] in (FP8, INT8)
        for s, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _need((s is not None) == self.quantised, f"{name} goes with an 8-bit cache, and with no other")
            if s is not None:
                _ints(s, name, torch.float32, k.shape[:3], k.get_device())
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.n_heads, self.page_size, self.head_dim = k.shape
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.struct = HerschelCache(k.data_ptr(), v.data_ptr(), None if k_scale is None else k_scale.data_ptr(),
                                    None if v_scale is None else v_scale.data_ptr(), *k.shape, KINDS[k.dtype])
        self._tensors = tuple(t for t in (k, v, k_scale, v_scale) if t is not None)
        self._at, self._status, self._device = ctypes.addressof(self.struct), self.status.data_ptr(), k.get_device()

    @classmethod
    def allocate(cls, n_pages: int, n_heads: int, page_size: int, head_dim: int, dtype=torch.bfloat16, device="cuda"):
        """A cache of zeros."""
        shape = (n_pages, n_heads, page_size, head_dim)
        k, v = (torch.zeros(shape, dtype=torch.uint8 if dtype == torch.float8_e4m3fn else dtype, device=device)
                for _ in range(2))
        if dtype not in (torch.float8_e4m3fn, torch.int8):
            return cls(k, v)
        return cls(k.view(dtype), v.view(dtype), *(torch.zeros(shape[:3], device=device) for _ in range(2)))

    def check(self) -> None:
        """Waits for the device, all its streams, and raises what calls with this cache reported since the last check."""
        raise_faults(self.status)

    def _fits(self, t: torch.Tensor) -> None:
        if t.get_device() != self._device or not (self.quantised or t.dtype == self.k.dtype):
            _need(t.get_device() == self._device, "the cache is on another device")
            _need(False, "a 16-bit cache has the type of the rows")


def rotary_table(n_positions: int, rotary_dim: int, base: float = 10_000.0, stretch: float = 1.0,
                 blend: tuple | None = None, device="cuda") -> torch.Tensor:
    """cos and sin of position * base^(-2 i / rotary_dim), [n_positions, rotary_dim / 2, 2] in float32, from
    angles in 64 bits (a position of 131,072 in 32-bit angles would be 0.004 off in its fastest pair).

    ``stretch`` > 1 compresses positions for contexts longer than the trained ones.  ``blend`` = (trained
    length, slow, fast) leaves pairs that turn more than ``fast`` times over the trained length as they are,
    compresses those that turn fewer than ``slow`` times, and goes linearly from one to the other between."""
    _need(rotary_dim >= 0 and rotary_dim % 2 == 0, "rotary_dim must be even")
    _need(n_positions >= 1 and base > 0 and stretch > 0, "n_positions, base and stretch must be positive")
    freq = float(base) ** (-torch.arange(0, rotary_dim, 2, device=device, dtype=torch.float64) / max(rotary_dim, 1))
    if blend is None:
        freq = freq / stretch
    else:
        length, slow, fast = blend
        _need(length > 0 and 0 <= slow < fast, "blend is (trained length, slow, fast) with slow < fast")
        keep = ((freq * length / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        freq = freq * keep + freq / stretch * (1 - keep)
    angle = torch.arange(n_positions, device=device, dtype=torch.float64)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


# ------------------------------------------------------------ the operators
_NO_ROWS = (0, 0, 0, 0)


def rope_write(q: torch.Tensor | None, k: torch.Tensor | None, v: torch.Tensor | None, positions: torch.Tensor,
               table: torch.Tensor, cache: PagedCache | None = None, slots: torch.Tensor | None = None, *,
               layout: str = "half", keep_keys: bool = False, q_out: torch.Tensor | None = None,
               k_out: torch.Tensor | None = None, status: torch.Tensor | None = None, lib=None):
    """Rotates q [tokens, heads, dim] and k [tokens, kv heads, dim] by ``table[positions]`` and, with a cache,
    writes k's rotated rows and v's rows to ``slots`` (page * page size + row; negative: not cached).

    Returns (q rotated, k rotated): new tensors, ``q_out`` and ``k_out`` where given (they may be q and k
    themselves); k's is None unless ``keep_keys`` or ``k_out`` asks for it or there is no cache."""
    first = q if q is not None else k
    if first is None:
        raise ValueError("q or k must be given")
    dev, dtype, shape = first.get_device(), first.dtype, first.shape
    if dev < 0 or dtype not in TYPES or len(shape) != 3:
        _rows(first, "q" if q is not None else "k")
    T, _, D = shape

    def rows(t, name, like=None):
        """(address, row stride, head stride, heads) of rows that go with the first ones."""
        shape, stride = t.shape, t.stride()
        if len(shape) != 3:
            _rows(t, name)
        (n, heads, d), (row, head, step) = shape, stride
        if (t.dtype is not dtype or t.get_device() != dev or n != T or d != D or step != 1 and D > 1 or
                like is not None and heads != like):
            _rows(t, name)
            _like(t, first, name)
            _need(False, f"{name} must have the tokens, heads and head size of the rows it goes with")
        if t.requires_grad:
            _no_gradients("rope_write")
        return t.data_ptr(), row, head, heads

    qa = rows(q, "q") if q is not None else _NO_ROWS
    ka = rows(k, "k") if k is not None else _NO_ROWS
    va = rows(v, "v", None if k is None else ka[3]) if v is not None else _NO_ROWS
    if layout not in LAYOUTS:
        raise ValueError("layout must be 'half' or 'interleaved'")
    pairs = table.shape
    if not (table.dtype is torch.float32 and len(pairs) == 3 and pairs[2] == 2 and table.is_contiguous() and
            table.get_device() == dev):
        raise ValueError("table must be float32 [positions, pairs, 2], contiguous, on the rows' device")
    pos, slot = _ints(positions, "positions", torch.int64, (T,), dev), 0
    if cache is not None:
        if k is None or v is None or slots is None:
            raise ValueError("a cache needs k, v and slots")
        if ka[3] != cache.n_heads or D != cache.head_dim:
            raise ValueError("the cache has another number of heads or head size")
        cache._fits(k)
        slot = _ints(slots, "slots", torch.int64, (T,), dev)
    given = ()
    if q_out is not None:
        _need(q is not None, "q_out needs q")
        qo, given = rows(q_out, "q_out", qa[3]), (q_out,)
    elif q is not None:
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
        qo = q_out.data_ptr(), qa[3] * D, D
    else:
        qo = _NO_ROWS
    if k_out is not None:
        _need(k is not None, "k_out needs k")
        ko, given = rows(k_out, "k_out", ka[3]), given + (k_out,)
    elif k is not None and (keep_keys or cache is None):
        k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
        ko = k_out.data_ptr(), ka[3] * D, D
    else:
        ko = _NO_ROWS
    reported = _status(status, dev) if status is not None else cache._status if cache is not None else 0
    args = _ROPE.pack(qa[0], ka[0], va[0], qa[1], qa[2], ka[1], ka[2], va[1], va[2], qo[0], ko[0], qo[1], qo[2], ko[1],
                      ko[2], pos, table.data_ptr(), pairs[0], slot, T, qa[3], ka[3], D, 2 * pairs[1],
                      LAYOUTS[layout], TYPES[dtype], reported, _stream(dev))
    _call((lib or _lib()).herschel_rope_write, dev, "rope_write", args, 0 if cache is None else cache._at)
    if cache is not None:
        given += cache._tensors
    if given:
        _written(given)
    return q_out, k_out


def cache_read(cache: PagedCache, block_table: torch.Tensor, cu: torch.Tensor, *, total: int, dtype=None,
               k_out: torch.Tensor | None = None, v_out: torch.Tensor | None = None, lib=None):
    """The first cu[b + 1] - cu[b] cached tokens of every sequence b as rows cu[b] ... of dense keys and
    values [total, heads, dim] of ``dtype`` (the cache's for a 16-bit one, else bfloat16 if not given)."""
    if dtype is None:
        dtype = torch.bfloat16 if cache.quantised else cache.k.dtype
    _need(dtype in TYPES, "dtype must be bfloat16 or float16")
    _need(cache.head_dim % 16 == 0, "cache_read needs a head size that is a multiple of 16")
    _need(cu.dim() == 1 and cu.shape[0] >= 2, "cu must hold a sequence's start and end")
    dev, n = cache._device, cu.shape[0] - 1
    starts, table = _ints(cu, "cu", torch.int32, cu.shape, dev), _table(block_table, n, dev)
    _need(total >= 0, "total must not be negative")
    shape = (total, cache.n_heads, cache.head_dim)
    if not (cache.quantised or dtype is cache.k.dtype):
        raise ValueError("a 16-bit cache has the type of the rows")
    given = ()
    if k_out is None:
        k_out = cache.k.new_empty(shape, dtype=dtype)
        to_k = k_out.data_ptr()
    else:
        to_k, given = _ints(k_out, "k_out", dtype, shape, dev), (k_out,)
    if v_out is None:
        v_out = torch.empty_like(k_out)
        to_v = v_out.data_ptr()
    else:
        to_v, given = _ints(v_out, "v_out", dtype, shape, dev), given + (v_out,)
    for t in given:
        if t.requires_grad:
            _no_gradients("cache_read")
    args = _READ.pack(table, block_table.shape[1], starts, n, total, to_k, to_v, TYPES[dtype], cache._status,
                      _stream(dev))
    _call((lib or _lib()).herschel_cache_read, dev, "cache_read", args, cache._at)
    if given:
        _written(given)
    return k_out, v_out


@functools.lru_cache(maxsize=1024)
def _prompt_workspace(lib, *sizes) -> int:
    """Bytes of workspace for a call of these sizes (0: none)."""
    size = ctypes.c_size_t(0)
    lib.herschel_attn_prompt_workspace(*sizes, ctypes.byref(size))
    return int(size.value)


def attn_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: torch.Tensor | None = None,
                *, max_q: int, scale: float | None = None, causal: bool = True, window: int = 0,
                return_lse: bool = False, out: torch.Tensor | None = None, status: torch.Tensor | None = None, lib=None):
    """Attention of q [queries, heads, dim] over k and v [keys, kv heads, dim], sequence b being rows
    cu_q[b] ... cu_q[b + 1] - 1 of q and cu_k[b] ... of k and v (``cu_k`` None: the same as ``cu_q``).

    Query i of nq sees key j of nk iff, causal, j <= i + nk - nq and, with a window, j > i + nk - nq - window.
    ``max_q`` is the longest sequence's number of queries, ``scale`` the scores' (dim ** -0.5 if not given).
    Rows of q from cu_q[-1] on are padding: their outputs are 0.  So are those of queries beyond ``max_q``, which
    ``status`` reports, like every other fault of the lengths; without it nothing tells of them.
    Returns the outputs, with ``return_lse`` also the log of each row's sum of exponentials [queries, heads]."""
    sq, sk, sv = _rows(q, "q"), _rows(k, "k"), _rows(v, "v")
    _like(k, q, "k")
    _like(v, q, "v")
    if q.requires_grad or k.requires_grad or v.requires_grad or out is not None and out.requires_grad:
        _no_gradients("attn_prompt")
    dev, (n_q, heads, D), (n_k, kv_heads, _) = q.get_device(), q.shape, k.shape
    starts = cu_q.shape
    if not ((D == 64 or D == 128) and k.shape == v.shape == (n_k, kv_heads, D) and kv_heads >= 1 and heads >= 1 and
            heads % kv_heads == 0 and len(starts) == 1 and starts[0] >= 2 and 0 <= max_q <= n_q and 0 <= window < 2 ** 31):
        _need(D == 64 or D == 128, "attention needs heads of 64 or 128")
        _need(k.shape == v.shape and k.shape[2] == D, "k and v must have one shape, and q's head size")
        _need(kv_heads >= 1 and heads >= 1 and heads % kv_heads == 0, "q's heads must be a multiple of k's")
        _need(cu_q.dim() == 1 and cu_q.shape[0] >= 2, "cu_q must hold a sequence's start and end")
        _need(0 <= max_q <= n_q, "max_q must be a number of q's rows")
        _need(False, "window must be 0 or a number of keys below 2^31")
    from_q = _ints(cu_q, "cu_q", torch.int32, starts, dev)
    from_k = from_q if cu_k is None else _ints(cu_k, "cu_k", torch.int32, starts, dev)
    given = out
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        to = out.data_ptr()
    else:
        to = _ints(out, "out", q.dtype, q.shape, dev)
    lse = q.new_empty((n_q, heads), dtype=torch.float32) if return_lse else None
    lib, n_seqs = lib or _lib(), starts[0] - 1
    size = _prompt_workspace(lib, n_seqs, n_q, n_k, max_q, heads, kv_heads, D)
    workspace = q.new_empty(size, dtype=torch.uint8) if size else None
    args = _PROMPT.pack(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), sq[0], sq[1], sk[0], sk[1], sv[0], sv[1],
        to, lse.data_ptr() if return_lse else 0, from_q, from_k,
        n_seqs, n_q, n_k, max_q, heads, kv_heads, D, TYPES[q.dtype], bool(causal), window,
        D ** -0.5 if scale is None else scale, workspace.data_ptr() if size else 0, size,
        0 if status is None else _status(status, dev), _stream(dev))
    _call(lib.herschel_attn_prompt, dev, "attn_prompt", args)
    if given is not None:
        _written((given,))
    return (out, lse) if return_lse else out


class DecodeAttention:
    """Causal attention of the last ``new_tokens`` tokens of up to ``batch`` sequences over a cache.

    Keeps the workspace, one for each stream it is called on; calls allocate nothing but an output that is
    not given.  A call that is captured (``torch.cuda.graph``) takes a workspace from the graph's own memory:
    graphs may be replayed beside each other and beside other calls."""

    def __init__(self, cache: PagedCache, *, batch: int, heads: int, new_tokens: int = 1, dtype=None, lib=None):
        dtype = dtype or (torch.bfloat16 if cache.quantised else cache.k.dtype)
        _need(dtype in TYPES, "dtype must be bfloat16 or float16")
        _need(cache.quantised or dtype == cache.k.dtype, "a 16-bit cache has the type of the rows")
        _need(cache.head_dim in (64, 128), "attention needs heads of 64 or 128")
        _need(1 <= batch <= MAX_DECODE_SEQS, f"batch must be 1 to {MAX_DECODE_SEQS}")
        _need(heads >= 1 and heads % cache.n_heads == 0, "heads must be a multiple of the cache's")
        _need(1 <= new_tokens <= 1024, "new_tokens must be 1 to 1024")
        self.cache, self.batch, self.heads, self.new_tokens, self.dtype = cache, batch, heads, new_tokens, dtype
        self.lib = lib or _lib()
        size = ctypes.c_size_t(0)
        code = self.lib.herschel_attn_decode_workspace(batch, new_tokens, heads, cache._at, ctypes.byref(size))
        _need(code == H.OK, "DecodeAttention: invalid sizes")
        self.workspace_bytes = int(size.value)
        self._workspaces = {}

    def __call__(self, q: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor, *,
                 scale: float | None = None, window: int = 0, out: torch.Tensor | None = None,
                 return_lse: bool = False):
        """q [sequences, new tokens, heads, dim], block_table [sequences, entries], seq_lens [sequences]: the
        cached tokens, the new ones among them.  Returns [sequences, new tokens, heads, dim], with
        ``return_lse`` also the log of each row's sum of exponentials."""
        c = self.cache
        sq, shape, dev = _rows(q, "q", 4), q.shape, q.get_device()
        B = shape[0]
        if q.requires_grad or out is not None and out.requires_grad:
            _no_gradients("DecodeAttention")
        _need(q.dtype == self.dtype, "q must have the type that DecodeAttention was made for")
        c._fits(q)
        _need(B <= self.batch and shape == (B, self.new_tokens, self.heads, c.head_dim),
              "q must have the sizes that the workspace is for")
        table, lens = _table(block_table, B, dev), _ints(seq_lens, "seq_lens", torch.int32, (B,), dev)
        _need(0 <= window < 2 ** 31, "window must be 0 or a number of keys below 2^31")
        given = out
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            to = out.data_ptr()
        else:
            to = _ints(out, "out", q.dtype, shape, dev)
        lse = q.new_empty(shape[:3], dtype=torch.float32) if return_lse else None
        if B == 0:  # a step in which no sequence takes part
            return (out, lse) if return_lse else out
        stream = _stream(dev)
        ws = self._workspaces.get(stream)
        if ws is None or (stream and _captured(dev)):  # the default stream, 0, is never captured
            ws = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=q.device)
            if not (stream and _captured(dev)):
                self._workspaces[stream] = ws
        args = _DECODE.pack(
            q.data_ptr(), sq[0], sq[1], sq[2], to,
            lse.data_ptr() if return_lse else 0, table, block_table.shape[1], lens, B, self.new_tokens, self.heads,
            TYPES[q.dtype], window, c.head_dim ** -0.5 if scale is None else scale, ws.data_ptr(),
            self.workspace_bytes, c._status, stream)
        _call(self.lib.herschel_attn_decode, dev, "DecodeAttention", args, c._at)
        if given is not None:
            _written((given,))
        return (out, lse) if return_lse else out


# ------------------------------------------------------------ around the attention
class Rows8(NamedTuple):
    """Rows of 8-bit codes [rows, columns], float8_e4m3fn or int8, each worth itself times its scale, float32
    [rows, 1] or [rows, groups of columns].  The group is the one, of 128, 64 or 32 columns, of which a row has as many
    as there are scales; the last may have fewer."""
    codes: torch.Tensor
    scale: torch.Tensor

    def values(self) -> torch.Tensor:
        """The rows in 32 bits."""
        columns, groups = self.codes.shape[1], self.scale.shape[1]
        group = columns if groups == 1 else next((g for g in (128, 64, 32) if -(-columns // g) == groups), 0)
        if not group:  # equal parts of another size
            _need(groups > 0 and columns % groups == 0, "scale must be one a row, or one for each 32, 64 or 128 columns")
            group = columns // groups
        return self.codes.float() * self.scale.repeat_interleave(group, 1)[:, :columns]


def _row(t: torch.Tensor, name: str, shape: tuple, dtype, device: int) -> int:
    """The row stride of a tensor [rows, columns] of this type on this GPU, columns contiguous."""
    if t.dtype is dtype and t.get_device() == device and t.shape == shape:
        row, step = t.stride()
        if step == 1 or shape[1] < 2:
            return row
    _need(t.dtype == dtype, f"{name} must be {dtype}")
    _need(t.get_device() == device, f"{name} must be on GPU {device}")
    _need(tuple(t.shape) == tuple(shape), f"{name} must have shape {tuple(shape)}")
    raise ValueError(f"{name}'s last dimension must be contiguous")


def norm_rows(x: torch.Tensor, weight: torch.Tensor, residual: torch.Tensor | None = None, *, eps: float = 1e-6,
              kind: torch.dtype | None = None, group: int = 0, residual_out: torch.Tensor | None = None,
              out: torch.Tensor | Rows8 | None = None, lib=None):
    """h / sqrt(mean(h^2) + eps) * weight for each row h of x [rows, columns], with a residual of h = x + residual.

    ``residual`` has x's type or is float32; the sums go to ``residual_out``, without it back into ``residual``.
    The norm is that of the sums in 32 bits, before they are rounded.  ``weight`` [columns] has x's type or is
    float32.  ``kind`` float8_e4m3fn or int8 asks for ``Rows8``, with a scale for each row, or for each ``group``
    (32, 64 or 128) of its columns; without it the result has x's type.  ``out`` is written where given.  x can be
    ``residual_out`` or a 16-bit ``out`` as well; calls in which what is written shares other memory are refused."""
    dev, dtype, shape, code = x.get_device(), x.dtype, x.shape, 0
    if dev < 0 or dtype not in TYPES or len(shape) != 2 or x.stride(1) != 1 and shape[1] > 1:
        _need(x.dim() == 2, "x must have 2 dimensions")
        _rows(x, "x", 2)
    n, dim = shape
    if not (1 <= dim <= MAX_NORM_DIM and 0 <= eps < math.inf):
        _need(1 <= dim <= MAX_NORM_DIM, f"rows must have 1 to {MAX_NORM_DIM} columns")
        _need(False, "eps must be finite and not negative")
    w_type = weight.dtype
    if w_type is not dtype and w_type is not torch.float32:
        raise ValueError("weight must have x's type or be float32")
    w = _ints(weight, "weight", w_type, (dim,), dev)
    needs, given = x.requires_grad or weight.requires_grad, ()
    rp = rs = op = os = 0
    r_type = dtype
    if residual is not None:
        r_type = residual.dtype
        if r_type is not dtype and r_type is not torch.float32:
            raise ValueError("residual must have x's type or be float32")
        rp, rs = residual.data_ptr(), _row(residual, "residual", shape, r_type, dev)
        needs = needs or residual.requires_grad
        if residual_out is None:
            residual_out, op, os = residual, rp, rs
        else:
            op, os = residual_out.data_ptr(), _row(residual_out, "residual_out", shape, r_type, dev)
            needs = needs or residual_out.requires_grad
        if os < dim:
            if n > 1:
                raise ValueError("residual_out's rows must not overlap")
            os = dim
        given = (residual_out,)
    elif residual_out is not None:
        raise ValueError("residual_out needs a residual")
    scale = 0
    if kind is None:
        if group:
            raise ValueError("group goes with rows of 8 bits")
        if out is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
            to = out.data_ptr()
        else:
            to, given = _ints(out, "out", dtype, shape, dev), given + (out,)
            needs = needs or out.requires_grad
    else:
        if kind not in CODES:
            raise ValueError("kind must be float8_e4m3fn or int8")
        if group not in (0, 32, 64, 128) or group and dim % group:
            raise ValueError("group must be 0, or 32, 64 or 128 and a divisor of the columns")
        code, groups = CODES[kind], (n, dim // group if group else 1)
        if out is None:
            out = Rows8(x.new_empty(shape, dtype=kind), x.new_empty(groups, dtype=torch.float32))
            to, scale = out.codes.data_ptr(), out.scale.data_ptr()
        else:
            to, scale = _ints(out[0], "out's codes", kind, shape, dev), _ints(out[1], "out's scale", torch.float32, groups, dev)
            given += (out[0], out[1])
            needs = needs or out[1].requires_grad
    if needs:
        _no_gradients("norm_rows")
    plain = TYPES[dtype]
    args = _NORM.pack(x.data_ptr(), x.stride(0), rp, rs, op, os, w, to, scale, n, dim, group, plain,
                      plain if r_type is dtype else F32, plain if w_type is dtype else F32,
                      plain if kind is None else code, eps, _stream(dev))
    _call((lib or _lib()).herschel_norm_rows, dev, "norm_rows", args)
    if given:
        _written(given)
    return out


class Weights4:
    """A matrix [n, k] of 4-bit weights, each (code - zero) * scale with the zero and scale of its row's group of
    32, 64 or 128 columns, laid out once in the tiles that ``product4`` reads.

    ``codes`` uint8 [n, k / 2 rounded up], the even column in the low four bits (and the last bits of an odd k of no
    effect); ``scales`` [n, groups] bfloat16 or float16; ``zeros`` uint8 [n, groups] of 0 to 15, 8 everywhere
    without them.  The group is the one of which a row of k has as many as there are scales."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, zeros: torch.Tensor | None = None, *, k: int | None = None):
        _need(codes.dtype == torch.uint8 and codes.dim() == 2 and codes.numel() > 0, "codes must be uint8 [n, k / 2]")
        n, half = codes.shape
        k = 2 * half if k is None else k
        _need(k >= 1 and (k + 1) // 2 == half, "codes must have k / 2 bytes a row, rounded up")
        _need(n <= MAX_WEIGHT_ROWS and k <= 2 ** 30, f"at most {MAX_WEIGHT_ROWS} rows and 2^30 columns")
        _need(scales.dtype in TYPES, "scales must be bfloat16 or float16")
        _need(scales.dim() == 2 and scales.shape[0] == n and scales.device == codes.device,
              "scales must be [n, groups], on the codes' device")
        group = next((g for g in (128, 64, 32) if -(-k // g) == scales.shape[1]), 0)
        _need(group > 0, "scales must be one for each 32, 64 or 128 columns")
        if scales.requires_grad:
            _no_gradients("Weights4")
        if zeros is not None:
            _need(zeros.dtype == torch.uint8 and zeros.shape == scales.shape and zeros.device == codes.device,
                  "zeros must be uint8, like scales")
            _need(int(zeros.max()) <= 15, "zeros must be 0 to 15")
        self.n, self.k, self.group, self.groups, self.device = n, k, group, scales.shape[1], codes.device
        tiles_n, tiles_k = -(-n // 16), -(-k // 128)
        self.codes = codes.new_empty((tiles_k, tiles_n, 4, 16, 4, 4))
        for at in range(0, tiles_n, 256):  # 4096 rows at a time, so that no copy of a byte a weight is made of them all
            part = codes[at * 16:(at + 256) * 16]
            wide = codes.new_zeros((-(-part.shape[0] // 16) * 16, tiles_k * 128))
            wide[:part.shape[0], 0:k:2] = part & 15
            wide[:part.shape[0], 1:k:2] = part[:, :k // 2] >> 4
            # rows of a tile, its columns as groups of 4 lanes' words, each two halves of 4 bytes
            wide = wide.view(-1, 16, tiles_k, 128 // group, 4, group // 32, 2, 4)
            packed = wide[..., 0, :] | (wide[..., 1, :] << 4)
            self.codes[:, at:at + 256] = packed.permute(2, 0, 4, 1, 3, 5, 6).reshape(tiles_k, -1, 4, 16, 4, 4)
        # a scale and its zero in a word; bfloat16 and half have no more than the 24 upper bits of a 32-bit float
        words = (scales.float().view(torch.int32) & -256) | (8 if zeros is None else zeros.to(torch.int32))
        wide = words.new_zeros((tiles_n * 16, tiles_k * (128 // group)))
        wide[:n, :self.groups] = words
        self.scales = wide.view(tiles_n, 4, 4, tiles_k, 128 // group).permute(3, 0, 1, 4, 2).contiguous()
        self.struct = HerschelWeights4(self.codes.data_ptr(), self.scales.data_ptr(), n, k, group)
        self._at, self._device = ctypes.addressof(self.struct), codes.get_device()

    @classmethod
    def quantise(cls, weights: torch.Tensor, group: int = 128, *, zeros: bool = False, scale_dtype=None):
        """To the nearest codes: -7 to 7 times a group's scale, or with ``zeros`` 16 steps from its smallest weight
        (or 0) to its largest (or 0), of the weights as they are: gradients end here.  ``scale_dtype``: that of 16-bit
        weights, else bfloat16."""
        _need(weights.dim() == 2 and weights.numel() > 0 and weights.is_floating_point(), "weights must be [n, k] of numbers")
        _need(group in (32, 64, 128), "group must be 32, 64 or 128")
        scale_dtype = scale_dtype or (weights.dtype if weights.dtype in TYPES else torch.bfloat16)
        _need(scale_dtype in TYPES, "scale_dtype must be bfloat16 or float16")
        n, k = weights.shape
        groups = -(-k // group)
        codes = torch.empty((n, (k + 1) // 2), dtype=torch.uint8, device=weights.device)
        scales = torch.empty((n, groups), dtype=scale_dtype, device=weights.device)
        zero = torch.empty((n, groups), dtype=torch.uint8, device=weights.device) if zeros else None
        for at in range(0, n, 4096):
            w = weights.detach()[at:at + 4096].float()
            w = torch.nn.functional.pad(w, (0, groups * group - k)).view(-1, groups, group)
            if zeros:
                low, high = w.amin(-1).clamp_max(0), w.amax(-1).clamp_min(0)
                s = (high / 15 - low / 15).to(scale_dtype)
            else:
                s = (w.abs().amax(-1) / 7).to(scale_dtype)
            _need(bool(torch.isfinite(s).all()), "weights must be finite, and their scales in the type's range")
            inv = torch.where(s >= 2.0 ** -126, 1 / s.float(), 0.0)  # a group of next to nothing is 0
            z = (-low * inv).round().clamp(0, 15) if zeros else torch.full_like(inv, 8.0)
            c = (w * inv[..., None] + z[..., None]).round().clamp(0 if zeros else 1, 15).to(torch.uint8).view(-1, groups * group)
            c = torch.nn.functional.pad(c[:, :k], (0, k % 2))
            codes[at:at + 4096] = c[:, ::2] | (c[:, 1::2] << 4)
            scales[at:at + 4096] = s
            if zeros:
                zero[at:at + 4096] = z.to(torch.uint8)
        return cls(codes, scales, zero, k=k)

    def dense(self) -> torch.Tensor:
        """The weights [n, k] in 32 bits."""
        tiles_k, tiles_n, per = *self.codes.shape[:2], 128 // self.group
        b = self.codes.view(tiles_k, tiles_n, 4, 16, per, self.group // 32, 4).permute(1, 3, 0, 4, 2, 5, 6)
        c = torch.stack([b & 15, b >> 4], -2).reshape(tiles_n * 16, tiles_k * per, self.group).float()
        words = self.scales.permute(1, 2, 4, 0, 3).reshape(tiles_n * 16, tiles_k * per, 1)
        c = (c - (words & 255)) * (words & -256).view(torch.float32)
        return c.view(tiles_n * 16, -1)[:self.n, :self.k].contiguous()


@functools.lru_cache(maxsize=1024)
def _product_workspace(lib, *sizes) -> int:
    """Bytes of workspace for a call of these sizes (0: none)."""
    size = ctypes.c_size_t(0)
    lib.herschel_product4_workspace(*sizes, ctypes.byref(size))
    return int(size.value)


def product4(x: torch.Tensor | Rows8, weights: Weights4, *, gated: bool = False, dtype: torch.dtype | None = None,
             out: torch.Tensor | None = None, lib=None) -> torch.Tensor:
    """Rows x [rows, k], or 8-bit ones with a scale a row or for each of the weights' groups, times ``weights``
    [n, k]: [rows, n].  Gated, the first half of the weights' rows gates the second: silu(a) * b, [rows, n / 2].

    ``dtype`` is the result's: the type of 16-bit rows, else bfloat16 or float16 (bfloat16 if not given).  A row
    that holds an infinity or a NaN comes out as NaN.  ``out`` shares no memory with x or the weights."""
    if isinstance(x, Rows8):
        t, scale = x
        if t.dtype not in CODES:
            raise ValueError("rows of 8 bits must be float8_e4m3fn or int8")
        kind, dtype = CODES[t.dtype], dtype or torch.bfloat16
        if dtype not in TYPES:
            raise ValueError("dtype must be bfloat16 or float16")
    else:
        t, scale = x, None
        if t.dtype not in TYPES or dtype is not None and dtype != t.dtype:
            _need(t.dtype in TYPES, "x must be bfloat16, float16 or Rows8")
            _need(False, "dtype must be that of rows of 16 bits")
        kind, dtype = TYPES[t.dtype], t.dtype
    dev, shape = t.get_device(), t.shape
    if dev < 0 or len(shape) != 2 or weights._device != dev:
        _need(len(shape) == 2, "x must have 2 dimensions")
        _need(dev >= 0, "x must be on a GPU")
        _need(False, "the weights are on another device")
    n, k = shape
    stride, x_group, scales = _row(t, "x", (n, weights.k), t.dtype, dev), 0, 0
    if scale is not None:
        groups = scale.shape[1] if scale.dim() == 2 else 0
        if groups != 1 and groups != weights.groups:
            raise ValueError("rows of 8 bits have a scale a row, [rows, 1], or one for each of the weights' groups")
        scales = _ints(scale, "scale", torch.float32, (n, groups), dev)
        x_group = weights.group if groups > 1 else 0
    if n > MAX_PRODUCT_ROWS:
        raise ValueError(f"at most {MAX_PRODUCT_ROWS} rows")
    if gated and weights.n % 32:
        raise ValueError("a gated product needs a multiple of 32 weight rows")
    if t.requires_grad or scale is not None and scale.requires_grad or out is not None and out.requires_grad:
        _no_gradients("product4")
    given, shape = out, (n, weights.n // 2 if gated else weights.n)
    if out is None:
        out = t.new_empty(shape, dtype=dtype)
        to = out.data_ptr()
    else:
        to = _ints(out, "out", dtype, shape, dev)
    lib = lib or _lib()
    size = _product_workspace(lib, n, kind, bool(gated), weights.n, weights.k)
    workspace = t.new_empty(size, dtype=torch.uint8) if size else None
    args = _PRODUCT.pack(t.data_ptr(), stride, scales, to, n, kind, x_group, TYPES[dtype], bool(gated),
                         workspace.data_ptr() if size else 0, size, _stream(dev))
    _call(lib.herschel_product4, dev, "product4", args, weights._at)
    if given is not None:
        _written((given,))
    return out


@functools.lru_cache(maxsize=1024)
def _verify_workspace(lib, *sizes) -> int:
    """Bytes of workspace for a call of these sizes (0: none)."""
    size = ctypes.c_size_t(0)
    lib.herschel_verify_workspace(*sizes, ctypes.byref(size))
    return int(size.value)


_PROBABILITIES = {torch.float32: F32, **TYPES}


def verify_drafts(target: torch.Tensor, tokens: torch.Tensor, accept: torch.Tensor, final: torch.Tensor, *,
                  draft: torch.Tensor | None = None, counts: torch.Tensor | None = None,
                  status: torch.Tensor | None = None, lib=None) -> tuple:
    """Drafted tokens [sequences, drafts] (int64) against the target's probabilities [sequences, drafts + 1, vocab],
    float32, bfloat16 or float16, at each draft and behind the last.

    Draft t of a sequence is accepted iff those before it are and accept[t] * draft[t, token] < target[t, token],
    with ``draft`` [sequences, drafts, vocab] the probabilities that the drafts were drawn from (None: each was the
    one choice, of probability 1).  Behind the accepted ones one token is drawn, from max(target - draft, 0) at the
    first that is not accepted or from the target behind the last (or where nothing of the difference is left): the
    lowest whose cumulative sum is above final times the whole sum.  ``accept`` [sequences, drafts] and ``final``
    [sequences] are random numbers in [0, 1), float32; ``counts`` (int32) the drafts of each sequence where some
    have fewer.  Returns the tokens [sequences, drafts + 1], -1 behind the drawn one, and the numbers of accepted
    drafts (int32)."""
    shape, dev = target.shape, target.get_device()
    if dev < 0 or len(shape) != 3 or target.dtype not in _PROBABILITIES or shape[2] < 1 or target.stride(2) != 1 and shape[2] > 1:
        _need(dev >= 0, "target must be on a GPU")
        _need(len(shape) == 3 and shape[2] >= 1, "target must be [sequences, drafts + 1, vocab]")
        _need(target.dtype in _PROBABILITIES, "target must be float32, bfloat16 or float16")
        _need(False, "target's last dimension must be contiguous")
    B, S, V = shape[0], shape[1] - 1, shape[2]
    if not (0 <= S <= MAX_DRAFTS and B <= 65535 and V <= 2 ** 30):
        raise ValueError(f"at most 65535 sequences, 0 to {MAX_DRAFTS} drafts and a vocabulary of at most 2^30")
    drafted = _ints(tokens, "tokens", torch.int64, (B, S), dev)
    u, last = _ints(accept, "accept", torch.float32, (B, S), dev), _ints(final, "final", torch.float32, (B,), dev)
    dp = ds = dr = 0
    if draft is not None:
        if draft.dtype is not target.dtype or draft.get_device() != dev or draft.shape != (B, S, V) or (
                draft.stride(2) != 1 and V > 1):
            _like(draft, target, "draft")
            _need(tuple(draft.shape) == (B, S, V), f"draft must have shape {(B, S, V)}")
            _need(False, "draft's last dimension must be contiguous")
        dp, ds, dr = draft.data_ptr(), draft.stride(0), draft.stride(1)
    if target.requires_grad or draft is not None and draft.requires_grad:
        _no_gradients("verify_drafts")
    n = 0 if counts is None else _ints(counts, "counts", torch.int32, (B,), dev)
    out, accepted = tokens.new_empty((B, S + 1)), tokens.new_empty((B,), dtype=torch.int32)
    lib = lib or _lib()
    size = _verify_workspace(lib, B, V)
    workspace = target.new_empty(size, dtype=torch.uint8) if size else None
    args = _VERIFY.pack(target.data_ptr(), target.stride(0), target.stride(1), dp, ds, dr, drafted, n, u, last,
                        out.data_ptr(), accepted.data_ptr(), B, S, V, _PROBABILITIES[target.dtype],
                        workspace.data_ptr() if size else 0, size, 0 if status is None else _status(status, dev), _stream(dev))
    _call(lib.herschel_verify_drafts, dev, "verify_drafts", args)
    return out, accepted

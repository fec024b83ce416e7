"""Reference operators: the attention layer of a served model on MI355X.

The C ABI is ``include/herschel_ops.h``; this module checks tensors, fills its
structures and calls the HIP library:

``PagedCache``       a paged cache of keys and values, 16-bit or 8-bit
``rotary_table``     cos and sin of the rotary positions, scaled for long contexts
``rope_write``       rotary positions, and the quantising write into the cache
``cache_read``       rows of the cache back in 16 bits
``attn_prompt``      attention over packed prompts
``DecodeAttention``  attention of new tokens over the cache (keeps the workspace)

Every call is enqueued on torch's current stream and returns at once.  What
only the device can see to be wrong (a page id, a length, a position, a slot)
is reported by ``PagedCache.check`` or, without a cache, through ``status``.
There is no CPU fallback: without the built library or a GPU the calls raise.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import herschel as H

BF16, F16, FP8, INT8 = 0, 1, 2, 3
TYPES = {torch.bfloat16: BF16, torch.float16: F16}
KINDS = {**TYPES, torch.float8_e4m3fn: FP8, torch.int8: INT8}
LAYOUTS = {"half": 0, "interleaved": 1}
BAD_PAGE, BAD_LENGTH, BAD_POSITION, BAD_SLOT = 1, 2, 4, 8
MAX_DECODE_SEQS = 4096
_FAULTS = {BAD_PAGE: "a block table entry outside the cache", BAD_LENGTH: "lengths that do not fit the buffers",
           BAD_POSITION: "a position outside the rotary table", BAD_SLOT: "a slot beyond the cache's end"}

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
                ("status", _P), ("hip_stream", _P)]


class HerschelDecodeArgs(ctypes.Structure):
    _fields_ = [("q", _P), ("q_seq_stride", _I64), ("q_strides", _Strides), ("out", _P), ("lse", _P),
                ("block_table", _P), ("table_stride", _I64), ("seq_lens", _P), ("n_seqs", _I32), ("new_tokens", _I32),
                ("q_heads", _I32), ("type", _I32), ("window", _I32), ("scale", ctypes.c_float), ("workspace", _P),
                ("workspace_bytes", ctypes.c_size_t), ("status", _P), ("hip_stream", _P)]


_ready = set()


def load(variant: str | None = None) -> ctypes.CDLL:
    """The library of ``herschel.load`` with the operators' signatures."""
    lib = H.load(variant)
    if id(lib) not in _ready:
        for name, args in (("herschel_rope_write", [HerschelRopeArgs, HerschelCache]),
                           ("herschel_cache_read", [HerschelReadArgs, HerschelCache]),
                           ("herschel_attn_prompt", [HerschelPromptArgs]),
                           ("herschel_attn_decode", [HerschelDecodeArgs, HerschelCache])):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = ctypes.c_int, [ctypes.POINTER(a) for a in args]
        lib.herschel_attn_decode_workspace.restype = ctypes.c_int
        lib.herschel_attn_decode_workspace.argtypes = [_I32, _I32, _I32, ctypes.POINTER(HerschelCache),
                                                       ctypes.POINTER(ctypes.c_size_t)]
        _ready.add(id(lib))
    return lib


# ------------------------------------------------------------ checks
def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _rows(t: torch.Tensor, name: str, dims: int = 3) -> None:
    """A tensor of rows of heads on a GPU whose heads' elements are contiguous."""
    _need(t.is_cuda, f"{name} must be on a GPU")
    _need(t.dim() == dims, f"{name} must have {dims} dimensions")
    _need(t.dtype in TYPES, f"{name} must be bfloat16 or float16")
    _need(t.shape[-1] < 2 or t.stride(-1) == 1, f"{name}'s last dimension must be contiguous")


def _ints(t: torch.Tensor, name: str, dtype, shape: tuple, like: torch.Tensor) -> None:
    _need(t.dtype == dtype, f"{name} must be {dtype}")
    _need(t.device == like.device, f"{name} must be on {like.device}")
    _need(tuple(t.shape) == shape, f"{name} must have shape {shape}")
    _need(t.is_contiguous(), f"{name} must be contiguous")


def _same(a: torch.Tensor, b: torch.Tensor, name: str) -> None:
    _need(a.dtype == b.dtype and a.device == b.device, f"{name} must have the type and device of the other rows")


def _table(t: torch.Tensor, n_seqs: int, like: torch.Tensor) -> None:
    _need(t.dtype == torch.int32 and t.dim() == 2 and t.shape[0] == n_seqs, "block_table must be int32 [sequences, entries]")
    _need(t.device == like.device, f"block_table must be on {like.device}")
    _need(t.shape[1] < 2 or t.stride(1) == 1, "block_table's rows must be contiguous")
    _need(t.shape[0] < 2 or t.stride(0) == t.shape[1], "block_table's rows must follow each other")


def _call(code: int, name: str) -> None:
    if code == H.EINVAL:
        raise ValueError(f"{name}: {H.herschel_strerror(code)}")
    if code != H.OK:
        raise RuntimeError(f"{name}: {H.herschel_strerror(code)}")


def _st(t: torch.Tensor) -> _Strides:
    return _Strides(t.stride(-3), t.stride(-2))


def _stream(t: torch.Tensor) -> int:
    return torch.cuda.current_stream(t.device).cuda_stream


def _status(status: torch.Tensor | None, like: torch.Tensor) -> int | None:
    if status is None:
        return None
    _need(status.dtype == torch.int32 and status.numel() == 1 and status.device == like.device,
          "status must be one int32 on the tensors' device")
    return status.data_ptr()


def raise_faults(status: torch.Tensor) -> None:
    """Waits for the device, clears ``status`` and raises what it reported."""
    bits = int(status.item())
    if bits:
        status.zero_()
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
        self.quantised = KINDS[k.dtype] in (FP8, INT8)
        for s, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _need((s is not None) == self.quantised, f"{name} goes with an 8-bit cache, and with no other")
            if s is not None:
                _ints(s, name, torch.float32, tuple(k.shape[:3]), k)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.n_heads, self.page_size, self.head_dim = k.shape
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.struct = HerschelCache(k.data_ptr(), v.data_ptr(), None if k_scale is None else k_scale.data_ptr(),
                                    None if v_scale is None else v_scale.data_ptr(), *k.shape, KINDS[k.dtype])
        self._ref = ctypes.byref(self.struct)

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
        """Waits for the device and raises what calls with this cache reported since the last check."""
        raise_faults(self.status)

    def _fits(self, t: torch.Tensor) -> None:
        _need(t.device == self.k.device, "the cache is on another device")
        _need(self.quantised or t.dtype == self.k.dtype, "a 16-bit cache has the type of the rows")


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
def rope_write(q: torch.Tensor | None, k: torch.Tensor | None, v: torch.Tensor | None, positions: torch.Tensor,
               table: torch.Tensor, cache: PagedCache | None = None, slots: torch.Tensor | None = None, *,
               layout: str = "half", keep_keys: bool = False, q_out: torch.Tensor | None = None,
               k_out: torch.Tensor | None = None, status: torch.Tensor | None = None, lib=None):
    """Rotates q [tokens, heads, dim] and k [tokens, kv heads, dim] by ``table[positions]`` and, with a cache,
    writes k's rotated rows and v's rows to ``slots`` (page * page size + row; negative: not cached).

    Returns (q rotated, k rotated): new tensors, ``q_out`` and ``k_out`` where given (they may be q and k
    themselves); k's is None unless ``keep_keys`` or ``k_out`` asks for it or there is no cache."""
    _need(q is not None or k is not None, "q or k must be given")
    first = q if q is not None else k
    T, D = first.shape[0], first.shape[-1]
    for t, name in ((q, "q"), (k, "k"), (v, "v"), (q_out, "q_out"), (k_out, "k_out")):
        if t is not None:
            _rows(t, name)
            _same(t, first, name)
            _need(t.shape[0] == T and t.shape[2] == D, f"{name} must have the tokens and head size of the other rows")
    _need(layout in LAYOUTS, "layout must be 'half' or 'interleaved'")
    _need(table.dtype == torch.float32 and table.dim() == 3 and table.shape[2] == 2 and table.is_contiguous() and
          table.device == first.device, "table must be float32 [positions, pairs, 2], contiguous, on the rows' device")
    _ints(positions, "positions", torch.int64, (T,), first)
    if cache is not None:
        _need(k is not None and v is not None and slots is not None, "a cache needs k, v and slots")
        _need(v.shape == k.shape, "v must have k's shape")
        _need(k.shape[1] == cache.n_heads and D == cache.head_dim, "the cache has another number of heads or head size")
        cache._fits(k)
        _ints(slots, "slots", torch.int64, (T,), first)
    if q is not None and q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if k is not None and k_out is None and (keep_keys or cache is None):
        k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    for o, i, name in ((q_out, q, "q_out"), (k_out, k, "k_out")):
        _need(o is None or (i is not None and o.shape == i.shape), f"{name} must have its input's shape")
    zero = _Strides(0, 0)
    args = HerschelRopeArgs(
        None if q is None else q.data_ptr(), None if k is None else k.data_ptr(), None if v is None else v.data_ptr(),
        zero if q is None else _st(q), zero if k is None else _st(k), zero if v is None else _st(v),
        None if q_out is None else q_out.data_ptr(), None if k_out is None else k_out.data_ptr(),
        zero if q_out is None else _st(q_out), zero if k_out is None else _st(k_out), positions.data_ptr(),
        table.data_ptr(), table.shape[0], None if cache is None else slots.data_ptr(), T,
        0 if q is None else q.shape[1], 0 if k is None else k.shape[1], D, 2 * table.shape[1], LAYOUTS[layout],
        TYPES[first.dtype], cache.status.data_ptr() if status is None and cache is not None else _status(status, first),
        _stream(first))
    lib = lib or load()
    with torch.cuda.device(first.device):
        _call(lib.herschel_rope_write(ctypes.byref(args), None if cache is None else cache._ref), "rope_write")
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
    _ints(cu, "cu", torch.int32, tuple(cu.shape), cache.k)
    _table(block_table, cu.shape[0] - 1, cache.k)
    _need(total >= 0, "total must not be negative")
    shape = (total, cache.n_heads, cache.head_dim)
    k_out = torch.empty(shape, dtype=dtype, device=cache.k.device) if k_out is None else k_out
    v_out = torch.empty(shape, dtype=dtype, device=cache.k.device) if v_out is None else v_out
    for o, name in ((k_out, "k_out"), (v_out, "v_out")):
        _ints(o, name, dtype, shape, cache.k)
        cache._fits(o)
    args = HerschelReadArgs(block_table.data_ptr(), block_table.shape[1], cu.data_ptr(), cu.shape[0] - 1, total,
                            k_out.data_ptr(), v_out.data_ptr(), TYPES[dtype], cache.status.data_ptr(), _stream(cache.k))
    lib = lib or load()
    with torch.cuda.device(cache.k.device):
        _call(lib.herschel_cache_read(ctypes.byref(args), cache._ref), "cache_read")
    return k_out, v_out


def attn_prompt(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, cu_k: torch.Tensor | None = None,
                *, max_q: int, scale: float | None = None, causal: bool = True, window: int = 0,
                return_lse: bool = False, out: torch.Tensor | None = None, status: torch.Tensor | None = None, lib=None):
    """Attention of q [queries, heads, dim] over k and v [keys, kv heads, dim], sequence b being rows
    cu_q[b] ... cu_q[b + 1] - 1 of q and cu_k[b] ... of k and v (``cu_k`` None: the same as ``cu_q``).

    Query i of nq sees key j of nk iff, causal, j <= i + nk - nq and, with a window, j > i + nk - nq - window.
    ``max_q`` is the longest sequence's number of queries, ``scale`` the scores' (dim ** -0.5 if not given).
    Returns the outputs, with ``return_lse`` also the log of each row's sum of exponentials [queries, heads]."""
    for t, name in ((q, "q"), (k, "k"), (v, "v")):
        _rows(t, name)
        _same(t, q, name)
    D = q.shape[2]
    _need(D in (64, 128), "attention needs heads of 64 or 128")
    _need(k.shape == v.shape and k.shape[2] == D, "k and v must have one shape, and q's head size")
    _need(k.shape[1] >= 1 and q.shape[1] >= 1 and q.shape[1] % k.shape[1] == 0, "q's heads must be a multiple of k's")
    cu_k = cu_q if cu_k is None else cu_k
    _need(cu_q.dim() == 1 and cu_q.shape[0] >= 2, "cu_q must hold a sequence's start and end")
    _ints(cu_q, "cu_q", torch.int32, tuple(cu_q.shape), q)
    _ints(cu_k, "cu_k", torch.int32, tuple(cu_q.shape), q)
    _need(0 <= max_q <= q.shape[0], "max_q must be a number of q's rows")
    _need(window >= 0, "window must not be negative")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    else:
        _ints(out, "out", q.dtype, tuple(q.shape), q)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if return_lse else None
    args = HerschelPromptArgs(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), _st(q), _st(k), _st(v), out.data_ptr(),
        None if lse is None else lse.data_ptr(), cu_q.data_ptr(), cu_k.data_ptr(), cu_q.shape[0] - 1, q.shape[0],
        k.shape[0], max_q, q.shape[1], k.shape[1], D, TYPES[q.dtype], int(causal), window,
        D ** -0.5 if scale is None else scale, _status(status, q), _stream(q))
    lib = lib or load()
    with torch.cuda.device(q.device):
        _call(lib.herschel_attn_prompt(ctypes.byref(args)), "attn_prompt")
    return (out, lse) if return_lse else out


class DecodeAttention:
    """Causal attention of the last ``new_tokens`` tokens of up to ``batch`` sequences over a cache.

    Keeps the workspace, one for each stream it is called on; calls allocate nothing but an output that is
    not given.  A graph captured from a call uses the workspace of the stream it was captured on."""

    def __init__(self, cache: PagedCache, *, batch: int, heads: int, new_tokens: int = 1, dtype=None, lib=None):
        dtype = dtype or (torch.bfloat16 if cache.quantised else cache.k.dtype)
        _need(dtype in TYPES, "dtype must be bfloat16 or float16")
        _need(cache.quantised or dtype == cache.k.dtype, "a 16-bit cache has the type of the rows")
        _need(cache.head_dim in (64, 128), "attention needs heads of 64 or 128")
        _need(1 <= batch <= MAX_DECODE_SEQS, f"batch must be 1 to {MAX_DECODE_SEQS}")
        _need(heads >= 1 and heads % cache.n_heads == 0, "heads must be a multiple of the cache's")
        _need(1 <= new_tokens <= 1024, "new_tokens must be 1 to 1024")
        self.cache, self.batch, self.heads, self.new_tokens, self.dtype = cache, batch, heads, new_tokens, dtype
        self.lib = lib or load()
        size = ctypes.c_size_t(0)
        _call(self.lib.herschel_attn_decode_workspace(batch, new_tokens, heads, cache._ref, ctypes.byref(size)),
              "DecodeAttention")
        self.workspace_bytes = int(size.value)
        self._workspaces = {}

    def __call__(self, q: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor, *,
                 scale: float | None = None, window: int = 0, out: torch.Tensor | None = None,
                 return_lse: bool = False):
        """q [sequences, new tokens, heads, dim], block_table [sequences, entries], seq_lens [sequences]: the
        cached tokens, the new ones among them.  Returns [sequences, new tokens, heads, dim], with
        ``return_lse`` also the log of each row's sum of exponentials."""
        c = self.cache
        _rows(q, "q", 4)
        B = q.shape[0]
        _need(q.dtype == self.dtype, f"q must be {self.dtype}")
        c._fits(q)
        _need(1 <= B <= self.batch and tuple(q.shape[1:]) == (self.new_tokens, self.heads, c.head_dim),
              "q must have the sizes that the workspace is for")
        _table(block_table, B, q)
        _ints(seq_lens, "seq_lens", torch.int32, (B,), q)
        _need(window >= 0, "window must not be negative")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        else:
            _ints(out, "out", q.dtype, tuple(q.shape), q)
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device) if return_lse else None
        stream = _stream(q)
        ws = self._workspaces.get(stream)
        if ws is None:
            ws = self._workspaces[stream] = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=q.device)
        args = HerschelDecodeArgs(
            q.data_ptr(), q.stride(0), _st(q), out.data_ptr(), None if lse is None else lse.data_ptr(),
            block_table.data_ptr(), block_table.shape[1], seq_lens.data_ptr(), B, self.new_tokens, self.heads,
            TYPES[q.dtype], window, c.head_dim ** -0.5 if scale is None else scale, ws.data_ptr(),
            self.workspace_bytes, c.status.data_ptr(), stream)
        with torch.cuda.device(q.device):
            _call(self.lib.herschel_attn_decode(ctypes.byref(args), c._ref), "DecodeAttention")
        return (out, lse) if return_lse else out

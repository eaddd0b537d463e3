"""The operators around the verification step, for PyTorch users and by address.

Python side of include/asymspec_serving.h, in the same library as the step: logits
under penalties, biases and grammar masks; block tables and slot maps of a paged
key-value cache; the writing of new keys and values; attention over the cache.  The
functions on tensors below extract addresses, sizes and strides, enqueue on the
current stream and raise ``AsymSpecError`` on a status other than OK; everything is
computed in the library's CUDA kernels.  Nothing is read back to the host.
"""
from __future__ import annotations

import ctypes
import math

from . import asymspec as A
from .asymspec import AsymSpecError, BF16, FP32, OK, _ptr, _stream

DATA_BAD_PENALTY = 0x40
DATA_BAD_LENGTH = 0x80
DATA_BAD_INDEX = 0x100
DATA_NO_BLOCKS = 0x200

CONSTRAIN_MAX_P = 256  # positions that constrain_logits takes
CACHE_MAX_B = 8192     # requests that cache_plan and cache_attend take
CACHE_MAX_D = 256      # head size that cache_attend takes

FLT_MAX = 3.4028234663852886e38

_P, _I, _L = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
_L2, _L3 = ctypes.c_int64 * 2, ctypes.c_int64 * 3


class Constraints(ctypes.Structure):
    _fields_ = [("history", _P), ("history_ld", _L), ("history_width", ctypes.c_int32),
                ("history_len", _P), ("prompt_len", _P), ("drafts", _P), ("drafts_ld", _L),
                ("repetition", _P), ("frequency", _P), ("presence", _P), ("bias_offsets", _P),
                ("bias_tokens", _P), ("bias_values", _P), ("bias_count", ctypes.c_int32),
                ("mask", _P), ("mask_ld", _L), ("mask_count", ctypes.c_int32), ("mask_rows", _P),
                ("mask_value", ctypes.c_float)]


class Cache(ctypes.Structure):
    _fields_ = [("keys", _P), ("values", _P), ("key_strides", _L3), ("value_strides", _L3),
                ("num_blocks", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


_lib = None


def lib():
    """The loaded library with this module's prototypes (raises if it is missing)."""
    global _lib
    if _lib is None:
        L = A.lib()
        L.asymspec_constrain_logits.argtypes = [ctypes.POINTER(Constraints), _P, _L, _P, _L, _I, _I,
                                                _I, _I, _P, _P]
        L.asymspec_constrain_logits.restype = _I
        L.asymspec_cache_plan.argtypes = [_P, _P, _P, _I, _I, _I, _I, _P, _L, _I, _P, _P, _P, _P, _P,
                                          _P, _P, _P, _P, _P, _L, _P, _P]
        L.asymspec_cache_plan.restype = _I
        L.asymspec_cache_write.argtypes = [ctypes.POINTER(Cache), _P, _P, _L2, _L2, _P, _I, _P, _P]
        L.asymspec_cache_write.restype = _I
        L.asymspec_cache_attend_workspace_bytes.argtypes = [_I, _I, _I, _I, _I]
        L.asymspec_cache_attend_workspace_bytes.restype = ctypes.c_size_t
        L.asymspec_cache_attend.argtypes = [ctypes.POINTER(Cache), _P, _L3, _I, _I, _I, _P, _L, _I,
                                            _P, ctypes.c_float, _I, _P, _L3, _P, _P,
                                            ctypes.c_size_t, _P, _P]
        L.asymspec_cache_attend.restype = _I
        _lib = L
    return _lib


def cache_attend_workspace_bytes(B: int, Q: int, heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().asymspec_cache_attend_workspace_bytes(B, Q, heads, kv_heads, head_dim))


# ----------------------------------------------------------------- PyTorch

def _dtype(torch, x) -> int:
    if x.dtype == torch.float32:
        return FP32
    if x.dtype == torch.bfloat16:
        return BF16
    raise TypeError("tensors must be float32 or bfloat16")


def _check(name, x, dtype, dev, shape=None):
    """`x` is None or a contiguous tensor of this type (and shape) on the call's device."""
    if x is None:
        return
    if x.dtype != dtype or x.device != dev or not x.is_contiguous() \
            or (shape is not None and tuple(x.shape) != shape):
        want = "x".join(map(str, shape)) + " " if shape is not None else ""
        raise ValueError(f"{name} must be a contiguous {want}{dtype} tensor on {dev}")


def _rows(name, x, dtype, dev, n):
    """`x` is None or [n, any] of this type whose rows are contiguous, any distance apart."""
    if x is None:
        return
    if x.dtype != dtype or x.device != dev or x.dim() != 2 or x.shape[0] != n \
            or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError(f"{name} must be a [{n}, ...] {dtype} tensor with contiguous rows on {dev}")


def constrain_logits(logits, *, history=None, history_len=None, prompt_len=None, drafts=None,
                     repetition=None, frequency=None, presence=None, bias=None, mask=None,
                     mask_rows=None, mask_value=None, out=None, error_word=None):
    """Logits of a round's positions under penalties, biases and grammar masks.

    logits [B, P, V] float32 or bfloat16, each row contiguous, rows any fixed distance
    apart; history [B, N] int32 with history_len, prompt_len [B] int32 (the first
    prompt_len are the prompt); drafts [B, P - 1] int32; repetition, frequency, presence
    [B] float32; bias (offsets [B + 1] int32, tokens int32, values float32); mask [M,
    words] int32, bit v % 32 of word v / 32 set where v is allowed, mask_rows [B, P]
    int32 (-1: none).  A masked logit becomes mask_value (default: the type's lowest).
    Returns `out`, which may be `logits` itself."""
    import torch
    if logits.dim() != 3 or not logits.is_cuda:
        raise ValueError("logits must be a [B, P, V] CUDA tensor")
    B, P, V = logits.shape
    dtype, dev, i32, f32 = _dtype(torch, logits), logits.device, torch.int32, torch.float32
    if out is None:
        out = torch.empty(B, P, V, dtype=logits.dtype, device=dev)
    elif out.shape != logits.shape or out.dtype != logits.dtype or out.device != dev:
        raise ValueError("out must have the shape, type and device of logits")
    lds = []
    for x in (logits, out):
        ld = x.stride(1) if P > 1 else x.stride(0) if B > 1 else V
        if x.stride(2) != 1 or (B > 1 and P > 1 and x.stride(0) != P * ld):
            raise ValueError("the rows of logits and out must be contiguous and evenly spaced")
        lds.append(max(ld, V) if B * P <= 1 else ld)
    _rows("history", history, i32, dev, B)
    _rows("drafts", drafts, i32, dev, B)
    if history is not None and history_len is None:
        raise ValueError("a history needs history_len")
    if drafts is not None and drafts.shape[1] < P - 1:
        raise ValueError("drafts must hold P - 1 tokens of each request")
    for name, x in (("history_len", history_len), ("prompt_len", prompt_len)):
        _check(name, x, i32, dev, (B,))
    for name, x in (("repetition", repetition), ("frequency", frequency), ("presence", presence)):
        _check(name, x, f32, dev, (B,))
    c = Constraints()
    if history is not None:
        c.history, c.history_ld, c.history_width = _ptr(history), history.stride(0), history.shape[1]
    c.history_len, c.prompt_len = _ptr(history_len), _ptr(prompt_len)
    if drafts is not None and P > 1:
        c.drafts, c.drafts_ld = _ptr(drafts), drafts.stride(0)
    c.repetition, c.frequency, c.presence = _ptr(repetition), _ptr(frequency), _ptr(presence)
    if bias is not None:
        offsets, tokens, values = bias
        _check("bias offsets", offsets, i32, dev, (B + 1,))
        _check("bias tokens", tokens, i32, dev)
        _check("bias values", values, f32, dev, tuple(tokens.shape))
        c.bias_offsets, c.bias_tokens, c.bias_values = _ptr(offsets), _ptr(tokens), _ptr(values)
        c.bias_count = tokens.numel()
    if mask is not None:
        if mask.dim() != 2:
            raise ValueError("mask must be [rows, words]")
        _rows("mask", mask, i32, dev, mask.shape[0])
        if mask.shape[1] * 32 < V:
            raise ValueError("a mask row must hold a bit for every token")
        c.mask, c.mask_ld, c.mask_count = _ptr(mask), mask.stride(0), mask.shape[0]
        c.mask_ld = max(c.mask_ld, mask.shape[1])
    elif mask_rows is not None:
        raise ValueError("mask_rows without a mask")
    _check("mask_rows", mask_rows, i32, dev, (B, P))
    c.mask_rows = _ptr(mask_rows)
    c.mask_value = -FLT_MAX if mask_value is None else mask_value
    _check("error_word", error_word, i32, dev, (1,))
    st = lib().asymspec_constrain_logits(ctypes.byref(c), logits.data_ptr(), lds[0], out.data_ptr(),
                                         lds[1], B, P, V, dtype, _ptr(error_word),
                                         _stream(torch, dev))
    if st != OK:
        raise AsymSpecError(st, "asymspec_constrain_logits")
    return out


def cache_plan(lens, tables, held, free_list, free_count, *, block_size, accepted=None, grow=0,
               capacity=None, out=None, error_word=None):
    """Moves B requests of a paged cache on by a round; see asymspec_cache_plan.

    lens, held, accepted [B] int32; tables [B, width] int32, rows any distance apart;
    free_list [blocks] and free_count [1] int32; grow a number, or [B] int32, which needs
    `capacity`, the entries of the slot map.  `tables` and `free_list` are updated in place.
    Returns a dict of start, len, held [B], free_count [1], offsets [B + 1] int32, slots
    [capacity] int64 and positions [capacity] int32; ``out`` may pass it to fill (with
    start = lens, held = held and free_count = free_count if those need not be kept)."""
    import torch
    if not lens.is_cuda or lens.dim() != 1:
        raise ValueError("lens must be a [B] CUDA tensor")
    B, dev, i32 = lens.shape[0], lens.device, torch.int32
    each = None if isinstance(grow, int) else grow
    for name, x in (("lens", lens), ("held", held), ("accepted", accepted), ("grow", each)):
        _check(name, x, i32, dev, (B,))
    _rows("tables", tables, i32, dev, B)
    _check("free_list", free_list, i32, dev)
    _check("free_count", free_count, i32, dev, (1,))
    if each is None:
        capacity = B * grow if capacity is None else capacity
    elif capacity is None:
        raise ValueError("grow as a tensor needs a capacity")
    r = out
    if r is None:
        ints = torch.empty(4 * B + 2, dtype=i32, device=dev)
        r = dict(start=ints[:B], len=ints[B:2 * B], held=ints[2 * B:3 * B],
                 free_count=ints[3 * B:3 * B + 1], offsets=ints[3 * B + 1:],
                 slots=torch.empty(capacity, dtype=torch.int64, device=dev),
                 positions=torch.empty(capacity, dtype=i32, device=dev))
    else:
        for name, shape in (("start", (B,)), ("len", (B,)), ("held", (B,)), ("free_count", (1,)),
                            ("offsets", (B + 1,)), ("positions", (capacity,))):
            _check(name, r[name], i32, dev, shape)
        _check("slots", r["slots"], torch.int64, dev, (capacity,))
    _check("error_word", error_word, i32, dev, (1,))
    width = tables.shape[1]
    st = lib().asymspec_cache_plan(
        lens.data_ptr(), _ptr(accepted), _ptr(each), grow if each is None else 0, B, block_size,
        free_list.numel(), tables.data_ptr(), max(tables.stride(0), width), width, held.data_ptr(),
        free_list.data_ptr(), free_count.data_ptr(), _ptr(r["start"]), _ptr(r["len"]),
        _ptr(r["held"]), _ptr(r["free_count"]), _ptr(r["offsets"]), _ptr(r["slots"]),
        _ptr(r["positions"]), capacity, _ptr(error_word), _stream(torch, dev))
    if st != OK:
        raise AsymSpecError(st, "asymspec_cache_plan")
    return r


def _cache(torch, keys, values):
    """The C view of a cache: keys and values [blocks, block_size, kv_heads, head_dim], the
    last axis contiguous, the others in any order in memory."""
    shape = keys.shape
    if len(shape) != 4 or values.shape != shape or values.dtype != keys.dtype or not keys.is_cuda \
            or values.device != keys.device:
        raise ValueError("keys and values must be CUDA tensors of one shape "
                         "[blocks, block_size, kv_heads, head_dim] and type")
    ks, vs = keys.stride(), values.stride()
    if ks[3] != 1 or vs[3] != 1:
        raise ValueError("the heads of keys and values must be contiguous")
    return Cache(keys.data_ptr(), values.data_ptr(), _L3(*ks[:3]), _L3(*vs[:3]), *shape,
                 _dtype(torch, keys))


def cache_write(k, v, key_cache, value_cache, slots, *, error_word=None):
    """Writes k, v [T, kv_heads, head_dim] into a paged cache ([blocks, block_size, kv_heads,
    head_dim], any order in memory) at slots [T] int64; negative slots are skipped."""
    import torch
    cache = _cache(torch, key_cache, value_cache)
    dev, (T, heads, dim) = key_cache.device, k.shape
    for x in (k, v):
        if x.dtype != key_cache.dtype or x.device != dev or x.shape != (T,) + key_cache.shape[2:] \
                or x.stride(2) != 1:
            raise ValueError("k and v must be [T, kv_heads, head_dim] like the cache, heads contiguous")
    _check("slots", slots, torch.int64, dev, (T,))
    _check("error_word", error_word, torch.int32, dev, (1,))
    st = lib().asymspec_cache_write(ctypes.byref(cache), k.data_ptr(), v.data_ptr(),
                                    _L2(*k.stride()[:2]), _L2(*v.stride()[:2]), slots.data_ptr(), T,
                                    _ptr(error_word), _stream(torch, dev))
    if st != OK:
        raise AsymSpecError(st, "asymspec_cache_write")


class CacheAttend:
    """Holds a workspace for the attention of up to B_max requests with Q_max queries each.

    ``__call__`` takes q [B, Q, heads, head_dim] (any strides, heads contiguous), a paged
    cache as cache_write does, tables [B, width] int32 and lens [B] int32 (the cached
    tokens of each request, the Q new ones included) and returns (out [B, Q, heads,
    head_dim], lse [B, Q, heads] float32), enqueued on the current stream.
    """

    def __init__(self, B_max: int, Q_max: int, heads: int, kv_heads: int, head_dim: int, device=None):
        import torch
        self.B_max, self.Q_max = B_max, Q_max
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.nbytes = cache_attend_workspace_bytes(B_max, Q_max, heads, kv_heads, head_dim)
        if self.nbytes == 0:
            raise ValueError("no attention of this shape")
        self.workspace = torch.empty(self.nbytes, dtype=torch.uint8,
                                     device=torch.device(device or "cuda"))

    def __call__(self, q, key_cache, value_cache, tables, lens, *, scale=None, window=0, out=None,
                 lse=None, error_word=None):
        import torch
        cache = _cache(torch, key_cache, value_cache)
        B, Q, heads, dim = q.shape
        dev = q.device
        if B > self.B_max or Q > self.Q_max or (heads, cache.kv_heads, dim) != (
                self.heads, self.kv_heads, self.head_dim):
            raise ValueError("batch does not fit this workspace")
        if out is None:
            out = torch.empty(B, Q, heads, dim, dtype=q.dtype, device=dev)
        if lse is None:
            lse = torch.empty(B, Q, heads, dtype=torch.float32, device=dev)
        for x in (q, out):
            if x.dtype != key_cache.dtype or x.device != key_cache.device or x.shape != q.shape \
                    or x.stride(3) != 1 or cache.head_dim != dim:
                raise ValueError("q and out must be [B, Q, heads, head_dim] like the cache, "
                                 "heads contiguous")
        _rows("tables", tables, torch.int32, dev, B)
        _check("lens", lens, torch.int32, dev, (B,))
        _check("lse", lse, torch.float32, dev, (B, Q, heads))
        _check("error_word", error_word, torch.int32, dev, (1,))
        width = tables.shape[1]
        st = lib().asymspec_cache_attend(
            ctypes.byref(cache), q.data_ptr(), _L3(*q.stride()[:3]), B, Q, heads, tables.data_ptr(),
            max(tables.stride(0), width), width, lens.data_ptr(),
            1.0 / math.sqrt(dim) if scale is None else scale, window, out.data_ptr(),
            _L3(*out.stride()[:3]), lse.data_ptr(), self.workspace.data_ptr(), self.nbytes,
            _ptr(error_word), _stream(torch, dev))
        if st != OK:
            raise AsymSpecError(st, "asymspec_cache_attend")
        return out, lse

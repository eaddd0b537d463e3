"""The operators around the verification step, for PyTorch users and by address.

Python side of include/asymspec_serving.h, in the same library as the step: logits
under penalties, biases and grammar masks; block tables and slot maps of a paged
key-value cache; the writing of new keys and values; attention over the cache.  The
functions on tensors below extract addresses, sizes and strides, enqueue on the
current stream and raise ``AsymSpecError`` on a status other than OK; everything is
computed in the library's CUDA kernels.  Nothing is read back to the host.  All tensors
of a call lie on the current device.
"""
from __future__ import annotations

import ctypes
import math
import struct

from . import asymspec as A
from .asymspec import AsymSpecError, BF16, FP32, OK

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
    """asymspec_constraints, for calls by address through lib()."""
    _fields_ = [("history", _P), ("history_ld", _L), ("history_width", ctypes.c_int32),
                ("history_len", _P), ("prompt_len", _P), ("drafts", _P), ("drafts_ld", _L),
                ("repetition", _P), ("frequency", _P), ("presence", _P), ("bias_offsets", _P),
                ("bias_tokens", _P), ("bias_values", _P), ("bias_count", ctypes.c_int32),
                ("mask", _P), ("mask_ld", _L), ("mask_count", ctypes.c_int32), ("mask_rows", _P),
                ("mask_value", ctypes.c_float)]


class Cache(ctypes.Structure):
    """asymspec_cache, for calls by address through lib()."""
    _fields_ = [("keys", _P), ("values", _P), ("key_strides", _L3), ("value_strides", _L3),
                ("num_blocks", ctypes.c_int32), ("block_size", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


# The same structs as bytes, filled in one step: field by field took a third of a small
# call's host time.
_CONSTRAINTS = struct.Struct("@PqixxxxPPPqPPPPPPixxxxPqixxxxPfxxxx")
_CACHE = struct.Struct("@PP6q5ixxxx")
_STRIDES2, _STRIDES3 = struct.Struct("@2q"), struct.Struct("@3q")

torch = None  # imported with the first call: the addresses' side needs no PyTorch


_lib = None


def lib():
    """The loaded library with this module's prototypes (raises if it is missing)."""
    global _lib
    if _lib is None:
        L = A.lib()
        L.asymspec_constrain_logits.argtypes = [_P, _P, _L, _P, _L, _I, _I, _I, _I, _P, _P]
        L.asymspec_constrain_logits.restype = _I
        L.asymspec_cache_plan.argtypes = [_P, _P, _P, _I, _I, _I, _I, _P, _L, _I, _P, _P, _P, _P, _P,
                                          _P, _P, _P, _P, _P, _L, _P, _P]
        L.asymspec_cache_plan.restype = _I
        L.asymspec_cache_write.argtypes = [_P, _P, _P, _P, _P, _P, _I, _P, _P]
        L.asymspec_cache_write.restype = _I
        L.asymspec_cache_attend_workspace_bytes.argtypes = [_I, _I, _I, _I, _I]
        L.asymspec_cache_attend_workspace_bytes.restype = ctypes.c_size_t
        L.asymspec_cache_attend.argtypes = [_P, _P, _P, _I, _I, _I, _P, _L, _I, _P, ctypes.c_float, _I,
                                            _P, _P, _P, _P, ctypes.c_size_t, _P, _P]
        L.asymspec_cache_attend.restype = _I
        _lib = L
    return _lib


def cache_attend_workspace_bytes(B: int, Q: int, heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().asymspec_cache_attend_workspace_bytes(B, Q, heads, kv_heads, head_dim))


# ----------------------------------------------------------------- PyTorch

_DTYPES = {}


def _begin():
    """The library and PyTorch, at the first call on tensors."""
    global torch
    import torch as t
    lib()
    _DTYPES.update({t.float32: FP32, t.bfloat16: BF16})
    torch = t


def _dtype(x) -> int:
    dtype = _DTYPES.get(x.dtype)
    if dtype is None:
        raise TypeError("tensors must be float32 or bfloat16")
    return dtype


def _int(n) -> int:
    """n for a C int, which would take the low bits of a larger number: past its range the range's
    largest, below zero -1."""
    return n if -1 <= n <= 0x7FFFFFFF else 0x7FFFFFFF if n > 0 else -1


def _flat(name, x, dtype, dev, n):
    """The address of `x`: contiguous, n entries of this type, on device `dev`."""
    if x.dtype is not dtype or x.get_device() != dev or x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} entries on cuda:{dev}")
    return x.data_ptr()


def _rows(name, x, dtype, dev, n):
    """(address, distance of rows, width) of `x`: [n, width], rows contiguous, any distance apart."""
    shape, strides = x.shape, x.stride()
    if x.dtype is not dtype or x.get_device() != dev or len(shape) != 2 or shape[0] != n \
            or (strides[1] != 1 and shape[1] > 1):
        raise ValueError(f"{name} must be a [{n}, ...] {dtype} tensor with contiguous rows on cuda:{dev}")
    return x.data_ptr(), strides[0] if n > 1 else shape[1], shape[1]


def _error_word(x, dev):
    return 0 if x is None else _flat("error_word", x, torch.int32, dev, 1)


def _row_distance(name, x, B, P, V):
    """Elements between the rows of [B, P, V]: contiguous, evenly spaced, each its own memory."""
    s0, s1, s2 = x.stride()
    ld = s1 if P > 1 else s0 if B > 1 else V
    if s2 != 1 or ld < V or (B > 1 and P > 1 and s0 != P * ld):
        raise ValueError(f"the rows of {name} must be contiguous, evenly spaced and apart")
    return ld


def constrain_logits(logits, *, history=None, history_len=None, prompt_len=None, drafts=None,
                     repetition=None, frequency=None, presence=None, bias=None, mask=None,
                     mask_rows=None, mask_value=None, out=None, error_word=None):
    """Logits of a round's positions under penalties, biases and grammar masks.

    logits [B, P, V] float32 or bfloat16, each row contiguous, rows any fixed distance
    apart; history [B, N] int32 with history_len, prompt_len [B] int32 (the first
    prompt_len are the prompt); drafts [B, P - 1] int32; repetition, frequency, presence
    [B] float32; bias (offsets [B + 1] int32, tokens int32, values float32); mask [M,
    words] int32, bit v % 32 of word v / 32 set where v is allowed, mask_rows [B, P]
    int32 (-1: none).  A masked logit becomes mask_value (default: the type's lowest, which
    the draw and the step's streaming kernels take; its staged and generic kernels answer
    about -1e30 and lower with a data error, and -1e4 serves everywhere).  Position k counts
    the drafts before it: with P = 1 none, so those belong into the history then.  Returns
    `out`, which may be `logits` itself."""
    if torch is None:
        _begin()
    dev = logits.get_device()
    if dev < 0 or logits.dim() != 3:
        raise ValueError("logits must be a [B, P, V] CUDA tensor")
    B, P, V = logits.shape
    dtype, i32, f32 = _dtype(logits), torch.int32, torch.float32
    ld = out_ld = _row_distance("logits", logits, B, P, V)
    if out is None:
        out = logits.new_empty((B, P, V))
        out_ld = V
    elif out is not logits:
        if out.shape != logits.shape or out.dtype is not logits.dtype or out.get_device() != dev:
            raise ValueError("out must have the shape, type and device of logits")
        out_ld = _row_distance("out", out, B, P, V)
    h = h_ld = h_width = h_len = p_len = d = d_ld = 0
    if history is not None:
        if history_len is None:
            raise ValueError("a history needs history_len")
        h, h_ld, h_width = _rows("history", history, i32, dev, B)
        h_len = _flat("history_len", history_len, i32, dev, B)
        # (a tensor without elements has address 0, which would be a group that is absent: any
        # other does for one that nothing is read from)
        h = h or h_len
        if prompt_len is not None:
            p_len = _flat("prompt_len", prompt_len, i32, dev, B)
    elif history_len is not None or prompt_len is not None:
        raise ValueError("lengths of no history")
    if drafts is not None:
        d, d_ld, width = _rows("drafts", drafts, i32, dev, B)
        if width < P - 1:
            raise ValueError("drafts must hold P - 1 tokens of each request")
    rep = 0 if repetition is None else _flat("repetition", repetition, f32, dev, B)
    freq = 0 if frequency is None else _flat("frequency", frequency, f32, dev, B)
    pres = 0 if presence is None else _flat("presence", presence, f32, dev, B)
    b_at = b_tok = b_val = b_n = m = m_ld = m_n = m_rows = 0
    if bias is not None:
        offsets, tokens, values = bias
        b_n = tokens.numel()
        b_at = _flat("bias offsets", offsets, i32, dev, B + 1)
        b_tok = _flat("bias tokens", tokens, i32, dev, b_n)
        b_val = _flat("bias values", values, f32, dev, b_n)
    if mask is not None:
        m_n = mask.shape[0]
        m, m_ld, width = _rows("mask", mask, i32, dev, m_n)
        if width * 32 < V:
            raise ValueError("a mask row must hold a bit for every token")
        if mask_rows is not None:
            m_rows = _flat("mask_rows", mask_rows, i32, dev, B * P)
            m = m or m_rows
        elif m_n == 0 and B * P > 0:
            raise ValueError("a mask without mask_rows must hold a row for every position")
    elif mask_rows is not None:
        raise ValueError("mask_rows without a mask")
    st = _lib.asymspec_constrain_logits(
        _CONSTRAINTS.pack(h, h_ld, h_width, h_len, p_len, d if P > 1 else 0, d_ld, rep, freq, pres, b_at,
                          b_tok, b_val, b_n, m, m_ld, m_n, m_rows,
                          -FLT_MAX if mask_value is None else mask_value),
        logits.data_ptr(), ld, out.data_ptr(), out_ld, B, P, V,
        dtype, 0 if error_word is None else _error_word(error_word, dev), _stream(dev))
    if st != OK:
        raise AsymSpecError(st, "asymspec_constrain_logits")
    return out


def _stream(dev) -> int:
    """The handle of device `dev`'s current stream.  A launch goes to the current device, whatever the
    stream (a device's default one has the same handle on all): that has to be `dev`."""
    current = torch.cuda.current_device()
    if dev != current:
        raise ValueError(f"the tensors are on cuda:{dev}, the current device is cuda:{current}: "
                         f"call under torch.cuda.device({dev})")
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(dev) if raw else torch.cuda.current_stream(dev).cuda_stream


def cache_plan(lens, tables, held, free_list, free_count, *, block_size, accepted=None, grow=0,
               capacity=None, out=None, error_word=None):
    """Moves B requests of a paged cache on by a round; see asymspec_cache_plan.

    lens, held, accepted [B] int32; tables [B, width] int32, rows any distance apart;
    free_list [blocks] and free_count [1] int32; grow a number, or [B] int32, which needs
    `capacity`, the entries of the slot map.  `tables` and `free_list` are updated in place.
    Returns a dict of start, len, held [B], free_count [1], offsets [B + 1] int32, slots
    [capacity] int64 and positions [capacity] int32; ``out`` may pass it to fill (with
    start = lens, held = held and free_count = free_count if those need not be kept)."""
    if torch is None:
        _begin()
    dev, i32 = lens.get_device(), torch.int32
    if dev < 0 or lens.dim() != 1:
        raise ValueError("lens must be a [B] CUDA tensor")
    B = lens.numel()
    each, all_ = 0, 0
    if isinstance(grow, int):
        all_ = grow
        if capacity is None:
            capacity = B * grow
    else:
        each = _flat("grow", grow, i32, dev, B)
        if capacity is None:
            raise ValueError("grow as a tensor needs a capacity")
    t, t_ld, width = _rows("tables", tables, i32, dev, B)
    blocks = free_list.numel()
    r = out
    if r is None:
        positions, start, end, kept, left, offsets = lens.new_empty(4 * B + 2 + capacity) \
            .split_with_sizes((capacity, B, B, B, 1, B + 1))
        r = {"start": start, "len": end, "held": kept, "free_count": left, "offsets": offsets,
             "slots": lens.new_empty(capacity, dtype=torch.int64), "positions": positions}
        at = (start.data_ptr(), end.data_ptr(), kept.data_ptr(), left.data_ptr(), offsets.data_ptr(),
              r["slots"].data_ptr(), positions.data_ptr())
    else:
        at = (_flat("start", r["start"], i32, dev, B), _flat("len", r["len"], i32, dev, B),
              _flat("held", r["held"], i32, dev, B), _flat("free_count", r["free_count"], i32, dev, 1),
              _flat("offsets", r["offsets"], i32, dev, B + 1),
              _flat("slots", r["slots"], torch.int64, dev, capacity),
              _flat("positions", r["positions"], i32, dev, capacity))
    st = _lib.asymspec_cache_plan(
        _flat("lens", lens, i32, dev, B), 0 if accepted is None else _flat("accepted", accepted, i32, dev, B),
        each, _int(all_), B, _int(block_size), blocks, t, t_ld, width, _flat("held", held, i32, dev, B),
        _flat("free_list", free_list, i32, dev, blocks), _flat("free_count", free_count, i32, dev, 1), *at,
        capacity, 0 if error_word is None else _error_word(error_word, dev), _stream(dev))
    if st != OK:
        raise AsymSpecError(st, "asymspec_cache_plan")
    return r


def _cache(keys, values):
    """(the C view of a cache, its device, its shape): keys and values [blocks, block_size,
    kv_heads, head_dim], the last axis contiguous, the others in any order in memory."""
    shape, dev = keys.shape, keys.get_device()
    if len(shape) != 4 or values.shape != shape or values.dtype is not keys.dtype or dev < 0 \
            or values.get_device() != dev:
        raise ValueError("keys and values must be CUDA tensors of one shape "
                         "[blocks, block_size, kv_heads, head_dim] and type")
    k0, k1, k2, k3 = keys.stride()
    v0, v1, v2, v3 = values.stride()
    if k3 != 1 or v3 != 1:
        raise ValueError("the heads of keys and values must be contiguous")
    return _CACHE.pack(keys.data_ptr(), values.data_ptr(), k0, k1, k2, v0, v1, v2, *shape,
                       _dtype(keys)), dev, shape


def cache_write(k, v, key_cache, value_cache, slots, *, error_word=None):
    """Writes k, v [T, kv_heads, head_dim] into a paged cache ([blocks, block_size, kv_heads,
    head_dim], any order in memory) at slots [T] int64; negative slots are skipped."""
    if torch is None:
        _begin()
    view, dev, (_, _, heads, dim) = _cache(key_cache, value_cache)
    kind, shape = key_cache.dtype, k.shape
    k0, k1, k2 = k.stride() if len(shape) == 3 else (0, 0, 0)
    v0, v1, v2 = v.stride() if len(shape) == 3 else (0, 0, 0)
    if k.dtype is not kind or v.dtype is not kind or k.get_device() != dev or v.get_device() != dev \
            or v.shape != shape or shape[1:] != (heads, dim) or k2 != 1 or v2 != 1:
        raise ValueError("k and v must be [T, kv_heads, head_dim] like the cache, heads contiguous")
    T = shape[0]
    st = _lib.asymspec_cache_write(view, k.data_ptr(), v.data_ptr(), _STRIDES2.pack(k0, k1),
                                   _STRIDES2.pack(v0, v1), _flat("slots", slots, torch.int64, dev, T), T,
                                   0 if error_word is None else _error_word(error_word, dev), _stream(dev))
    if st != OK:
        raise AsymSpecError(st, "asymspec_cache_write")


class CacheAttend:
    """Holds a workspace for the attention of up to B_max requests with Q_max queries each.

    ``__call__`` takes q [B, Q, heads, head_dim] (any strides, heads contiguous), a paged
    cache as cache_write does, tables [B, width] int32 and lens [B] int32 (the cached
    tokens of each request, the Q new ones included) and returns (out [B, Q, heads,
    head_dim], lse [B, Q, heads] float32), enqueued on the current stream; ``out`` may pass a
    tensor to fill, which must not overlap q or the cache.  Calls that
    share the workspace must follow one another: on one stream, or ordered by events.
    """

    def __init__(self, B_max: int, Q_max: int, heads: int, kv_heads: int, head_dim: int, device=None):
        if torch is None:
            _begin()
        self.B_max, self.Q_max = B_max, Q_max
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.nbytes = cache_attend_workspace_bytes(B_max, Q_max, heads, kv_heads, head_dim)
        if self.nbytes == 0:
            raise ValueError("no attention of this shape")
        self.workspace = torch.empty(self.nbytes, dtype=torch.uint8,
                                     device=torch.device("cuda" if device is None else device))
        self.device_index = self.workspace.get_device()
        self.scale = 1.0 / math.sqrt(head_dim)

    def __call__(self, q, key_cache, value_cache, tables, lens, *, scale=None, window=0, out=None,
                 lse=None, error_word=None):
        view, dev, (_, _, kv_heads, head_dim) = _cache(key_cache, value_cache)
        B, Q, heads, dim = shape = q.shape
        kind = key_cache.dtype
        if dev != self.device_index:
            raise ValueError("the cache must be on the workspace's device")
        if B > self.B_max or Q > self.Q_max or (heads, kv_heads, head_dim) != (
                self.heads, self.kv_heads, self.head_dim):
            raise ValueError("batch does not fit this workspace")
        q0, q1, q2, q3 = q.stride()
        if q.dtype is not kind or q.get_device() != dev or q3 != 1 or dim != head_dim:
            raise ValueError("q must be [B, Q, heads, head_dim] like the cache, heads contiguous")
        if out is None:
            out = q.new_empty(shape)
            o0, o1, o2 = Q * heads * dim, heads * dim, dim
        else:
            o0, o1, o2, o3 = out.stride()
            if out.dtype is not kind or out.get_device() != dev or out.shape != shape or o3 != 1:
                raise ValueError("out must be [B, Q, heads, head_dim] like q, heads contiguous")
        if lse is None:
            lse = q.new_empty((B, Q, heads), dtype=torch.float32)
            l = lse.data_ptr()
        else:
            l = _flat("lse", lse, torch.float32, dev, B * Q * heads)
        t, t_ld, width = _rows("tables", tables, torch.int32, dev, B)
        st = _lib.asymspec_cache_attend(
            view, q.data_ptr(), _STRIDES3.pack(q0, q1, q2), B, Q, heads, t, t_ld, width,
            _flat("lens", lens, torch.int32, dev, B), self.scale if scale is None else scale, _int(window),
            out.data_ptr(), _STRIDES3.pack(o0, o1, o2), l, self.workspace.data_ptr(), self.nbytes,
            0 if error_word is None else _error_word(error_word, dev), _stream(dev))
        if st != OK:
            raise AsymSpecError(st, "asymspec_cache_attend")
        return out, lse

"""The operators around the verification step, for PyTorch users and by address.

Python side of include/asymspec_serving.h, in the same library as the step: logits
under penalties, biases and grammar masks; block tables and slot maps of a paged
key-value cache; the writing of new keys and values; attention over the cache; rotary
positions; a cache in 4 bits with its writing, reading and attention.  The functions on tensors below extract addresses, sizes and strides, enqueue on the
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
ROTARY_MAX_D = 1024    # head size that rotary takes

ROTARY_KINDS = {"linear": 1, "base": 2, "ramp": 3, "wavelength": 4}

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


class RotaryScaling(ctypes.Structure):
    """asymspec_rotary_scaling."""
    _fields_ = [("kind", ctypes.c_int32), ("original_length", ctypes.c_int32),
                ("factor", ctypes.c_double), ("fast", ctypes.c_double), ("slow", ctypes.c_double)]


class RotaryHeads(ctypes.Structure):
    """asymspec_rotary_heads, for calls by address through lib()."""
    _fields_ = [("x", _P), ("out", _P), ("in_strides", _L2), ("out_strides", _L2),
                ("heads", ctypes.c_int32)]


class PackedCache(ctypes.Structure):
    """asymspec_cache4, for calls by address through lib()."""
    _fields_ = [("key_codes", _P), ("key_scales", _P), ("value_codes", _P), ("value_scales", _P),
                ("key_code_strides", _L3), ("key_scale_strides", _L3), ("value_code_strides", _L3),
                ("value_scale_strides", _L3), ("num_blocks", ctypes.c_int32),
                ("block_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("key_scale", ctypes.c_float),
                ("value_scale", ctypes.c_float)]


# The same structs as bytes, filled in one step: field by field took a third of a small
# call's host time.
_CONSTRAINTS = struct.Struct("@PqixxxxPPPqPPPPPPixxxxPqixxxxPfxxxx")
_CACHE = struct.Struct("@PP6q5ixxxx")
_HEADS = struct.Struct("@PP4qixxxx")
_CACHE4 = struct.Struct("@4P12q4iff")
_STRIDES2, _STRIDES3 = struct.Struct("@2q"), struct.Struct("@3q")

torch = None  # imported with the first call: the addresses' side needs no PyTorch
_Turned = None  # what autograd keeps of a Rotary call, likewise


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
        L.asymspec_rotary_steps.argtypes = [_I, ctypes.c_double, _P, _P, _P, _P]
        L.asymspec_rotary_steps.restype = _I
        L.asymspec_rotary.argtypes = [_P, _P, _I, _I, _I, _I, _I, _P, _P, ctypes.c_float, _I, _P]
        L.asymspec_rotary.restype = _I
        L.asymspec_cache4_write.argtypes = [_P, _P, _P, _I, _P, _P, _P, _I, _P, _P]
        L.asymspec_cache4_write.restype = _I
        L.asymspec_cache4_read.argtypes = [_P, _P, _I, _P, _P, _I, _P, _P, _P, _P]
        L.asymspec_cache4_read.restype = _I
        L.asymspec_cache4_attend_workspace_bytes.argtypes = [_I, _I, _I, _I, _I]
        L.asymspec_cache4_attend_workspace_bytes.restype = ctypes.c_size_t
        L.asymspec_cache4_attend.argtypes = [_P, _P, _I, _P, _I, _I, _I, _P, _L, _I, _P, ctypes.c_float, _I,
                                             _P, _P, _P, _P, ctypes.c_size_t, _P, _P]
        L.asymspec_cache4_attend.restype = _I
        _lib = L
    return _lib


def cache_attend_workspace_bytes(B: int, Q: int, heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().asymspec_cache_attend_workspace_bytes(B, Q, heads, kv_heads, head_dim))


def cache4_attend_workspace_bytes(B: int, Q: int, heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().asymspec_cache4_attend_workspace_bytes(B, Q, heads, kv_heads, head_dim))


def rotary_steps(rotary_dim: int, base: float = 10000.0, scaling=None, frequencies=None):
    """([turns of each pair a position, as 64-bit fractions], magnitude): what asymspec_rotary takes.

    scaling: None, or a dict of kind ("linear", "base", "ramp", "wavelength"), factor and, for the
    last two, original_length, fast and slow; frequencies: radians a position of each of the
    rotary_dim / 2 pairs, in the place of base and scaling."""
    pairs = max(rotary_dim // 2, 0)
    given = None
    if frequencies is not None:
        if len(frequencies) != pairs:
            raise ValueError(f"frequencies must be {pairs} numbers")
        given = (ctypes.c_double * pairs)(*frequencies)
    s = None
    if scaling is not None:
        unknown = set(scaling) - {"kind", "factor", "original_length", "fast", "slow"}
        if unknown or scaling.get("kind") not in ROTARY_KINDS:
            raise ValueError(f"scaling must be a dict of kind {tuple(ROTARY_KINDS)}, factor, original_length, "
                             "fast, slow")
        s = RotaryScaling(ROTARY_KINDS[scaling["kind"]], _int(scaling.get("original_length", 0)),
                          scaling.get("factor", 1.0), scaling.get("fast", 0.0), scaling.get("slow", 0.0))
    steps, magnitude = (ctypes.c_uint64 * max(pairs, 1))(), ctypes.c_float()
    st = lib().asymspec_rotary_steps(rotary_dim, base, None if s is None else ctypes.byref(s), given, steps,
                                     ctypes.byref(magnitude))
    if st != OK:
        raise AsymSpecError(st, "asymspec_rotary_steps")
    return list(steps), magnitude.value


# ----------------------------------------------------------------- PyTorch

_DTYPES = {}


def _begin():
    """The library and PyTorch, at the first call on tensors."""
    global torch, _Turned
    import torch as t
    lib()
    _DTYPES.update({t.float32: FP32, t.bfloat16: BF16})
    torch = t

    class Turned(t.autograd.Function):
        @staticmethod
        def forward(ctx, rotary, transpose, positions, q, k):
            ctx.rotary, ctx.transpose = rotary, transpose
            ctx.save_for_backward(positions)
            ctx.set_materialize_grads(False)
            return rotary._turn(q, positions, k, transpose, None, None)

        @staticmethod
        def backward(ctx, q_grad, k_grad):
            positions, = ctx.saved_tensors
            # (a sum's gradient is one number for all elements)
            given = [g if g is None or g.stride(-1) == 1 else g.contiguous() for g in (q_grad, k_grad)]
            turned = [None, None]
            if given[0] is not None:
                turned = ctx.rotary(given[0], positions, given[1], transpose=not ctx.transpose)
            elif given[1] is not None:
                turned[1], _ = ctx.rotary(given[1], positions, transpose=not ctx.transpose)
            return None, None, None, *turned

    _Turned = Turned


def _dtype(x) -> int:
    dtype = _DTYPES.get(x.dtype)
    if dtype is None:
        raise TypeError("tensors must be float32 or bfloat16")
    return dtype


def _int(n) -> int:
    """n for a C int, which would take the low bits of a larger number: past its range the range's
    largest, below zero -1."""
    return n if -1 <= n <= 0x7FFFFFFF else 0x7FFFFFFF if n > 0 else -1


def _tokens_of(x) -> int:
    """The length of a tensor's first axis, for a C int."""
    T = x.shape[0] if x.dim() else 0
    if T > 0x7FFFFFFF:
        raise ValueError("more than 2^31 - 1 tokens")
    return T


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


class Rotary:
    """Rotary positions: the frequencies of a head's pairs, on the device.

    head_dim, rotary_dim (the elements that are turned, from the first on; default all), base,
    scaling and frequencies as rotary_steps takes them; interleaved: pairs of neighbours, else of
    the halves; magnitude: in the place of the scaling's.

    ``__call__`` turns q [T, heads, head_dim] and k [T, kv_heads, head_dim] (or None), float32 or
    bfloat16, any strides with contiguous heads, by positions [T] int32 (negative: a token that stays
    as it is), and returns (q, k) in new tensors or in q_out, k_out, which may be q and k themselves or
    must not overlap them.  transpose: by the opposite angle (times the same magnitude): the gradient of
    q and k from the gradients of the results.  Where q or k requires a gradient, autograd takes that as its
    backward pass; such a call has no q_out or k_out.
    """

    def __init__(self, head_dim: int, *, rotary_dim=None, base: float = 10000.0, interleaved: bool = False,
                 scaling=None, frequencies=None, magnitude=None, device=None):
        if torch is None:
            _begin()
        self.head_dim, self.rotary_dim = head_dim, head_dim if rotary_dim is None else rotary_dim
        if not 2 <= self.rotary_dim <= head_dim:
            raise ValueError("rotary_dim must be 2 to head_dim")
        self.interleaved = bool(interleaved)
        steps, own = rotary_steps(self.rotary_dim, base, scaling, frequencies)
        self.magnitude = own if magnitude is None else float(magnitude)
        # (as signed numbers of the same bits)
        self.steps = torch.tensor([s - (s >> 63 << 64) for s in steps], dtype=torch.int64,
                                  device=torch.device("cuda" if device is None else device))
        self.device_index = self.steps.get_device()

    def _heads(self, name, x, out, T, kind, dev):
        shape = x.shape
        if len(shape) != 3 or shape[0] != T or shape[2] != self.head_dim or x.dtype is not kind \
                or x.get_device() != dev:
            raise ValueError(f"{name} must be a [{T}, heads, {self.head_dim}] {kind} tensor on cuda:{dev}")
        s0, s1, s2 = x.stride()
        if out is None:
            out = x.new_empty(shape)
        elif out.shape != shape or out.dtype is not kind or out.get_device() != dev:
            raise ValueError(f"{name}_out must have the shape, type and device of {name}")
        o0, o1, o2 = out.stride()
        if (s2 != 1 or o2 != 1) and self.head_dim > 1:
            raise ValueError(f"the heads of {name} must be contiguous")
        return _HEADS.pack(x.data_ptr(), out.data_ptr(), s0, s1, o0, o1, shape[1]), out

    def __call__(self, q, positions, k=None, *, transpose=False, q_out=None, k_out=None):
        if torch.is_grad_enabled() and (q.requires_grad or (k is not None and k.requires_grad)
                                        or (q_out is not None and q_out.requires_grad)
                                        or (k_out is not None and k_out.requires_grad)):
            if q_out is not None or k_out is not None:
                raise ValueError("q_out and k_out are for calls without gradients")
            return _Turned.apply(self, bool(transpose), positions, q, k)
        return self._turn(q, positions, k, transpose, q_out, k_out)

    def _turn(self, q, positions, k, transpose, q_out, k_out):
        dev, kind = q.get_device(), q.dtype
        if dev != self.device_index:
            raise ValueError("q must be on the frequencies' device")
        if k is None and k_out is not None:
            raise ValueError("k_out without k")
        T = _tokens_of(q)
        dtype = _dtype(q)
        q_heads, q_out = self._heads("q", q, q_out, T, kind, dev)
        k_heads = None
        if k is not None:
            k_heads, k_out = self._heads("k", k, k_out, T, kind, dev)
        st = _lib.asymspec_rotary(
            q_heads, k_heads, T, self.head_dim, self.rotary_dim, self.interleaved, bool(transpose),
            _flat("positions", positions, torch.int32, dev, T), self.steps.data_ptr(), self.magnitude, dtype,
            _stream(dev))
        if st != OK:
            raise AsymSpecError(st, "asymspec_rotary")
        return q_out, k_out


class Cache4:
    """A paged key-value cache in 4 bits: codes and scales of the keys and of the values.

    key_codes, value_codes [blocks, block_size, kv_heads, head_dim / 2] uint8, two codes (e2m1) a
    byte, and key_scales, value_scales [blocks, block_size, kv_heads, head_dim / 16] uint8 or
    float8_e4m3fn, a scale for each 16 elements; last axes contiguous, the others in any order in memory;
    key_scale, value_scale: numbers that all elements are times of.  Holds the tensors, no copies.
    """

    def __init__(self, key_codes, key_scales, value_codes, value_scales, *, key_scale=1.0, value_scale=1.0):
        if torch is None:
            _begin()
        tensors = (key_codes, key_scales, value_codes, value_scales)
        dev, shape = key_codes.get_device(), key_codes.shape
        if dev < 0 or len(shape) != 4 or value_codes.shape != shape or any(
                x.dtype is not torch.uint8 for x in (key_codes, value_codes)):
            raise ValueError("codes must be CUDA uint8 tensors of one shape [blocks, block_size, kv_heads, head_dim / 2]")
        of_scales = (*shape[:3], shape[3] // 8)
        if any(x.shape != of_scales or x.dtype not in (torch.uint8, torch.float8_e4m3fn)
               for x in (key_scales, value_scales)):
            raise ValueError(f"scales must be uint8 or float8_e4m3fn tensors of shape {list(of_scales)}")
        if any(x.get_device() != dev or (x.stride(3) != 1 and x.shape[3] > 1) for x in tensors):
            raise ValueError("codes and scales must be on one device, each token's of a head contiguous")
        self.key_codes, self.key_scales, self.value_codes, self.value_scales = tensors
        self.key_scale, self.value_scale = float(key_scale), float(value_scale)
        self.device_index = dev
        self.kv_heads, self.head_dim = shape[2], shape[3] * 2
        self.token_strides = _STRIDES2.pack(self.kv_heads * self.head_dim, self.head_dim)
        strides = (s if n > 1 else 0 for x in tensors for s, n in zip(x.stride()[:3], x.shape))
        self.view = _CACHE4.pack(*(x.data_ptr() for x in tensors), *strides, *shape[:3], self.head_dim,
                                 self.key_scale, self.value_scale)

    @classmethod
    def zeros(cls, blocks: int, block_size: int, kv_heads: int, head_dim: int, *, key_scale=1.0, value_scale=1.0,
              device=None):
        """A pool of zeros in which a block's tokens of one head lie next to one another."""
        if torch is None:
            _begin()

        def part(width):
            return torch.zeros(blocks, kv_heads, block_size, width, dtype=torch.uint8,
                               device=torch.device("cuda" if device is None else device)).transpose(1, 2)

        return cls(*(part(head_dim // n) for n in (2, 16, 2, 16)), key_scale=key_scale, value_scale=value_scale)


def _tokens(name, x, cache, kind, T):
    """The strides of `x`: [T, kv_heads, head_dim] like the cache's heads, which are contiguous."""
    shape = x.shape
    if x.dtype is not kind or x.get_device() != cache.device_index or shape != (T, cache.kv_heads, cache.head_dim) \
            or x.stride(2) != 1:
        raise ValueError(f"{name} must be a [{T}, {cache.kv_heads}, {cache.head_dim}] {kind} tensor like the cache, "
                         "heads contiguous")
    s0, s1, _ = x.stride()
    return _STRIDES2.pack(s0, s1)


def cache4_write(k, v, cache, slots, *, error_word=None):
    """Writes k, v [T, kv_heads, head_dim], float32 or bfloat16, into a cache in 4 bits at slots [T]
    int64; negative slots are skipped.  (include/asymspec_serving.h says how they are rounded.)"""
    dev, T, kind = cache.device_index, _tokens_of(k), k.dtype
    st = _lib.asymspec_cache4_write(
        cache.view, k.data_ptr(), v.data_ptr(), _dtype(k), _tokens("k", k, cache, kind, T),
        _tokens("v", v, cache, kind, T), _flat("slots", slots, torch.int64, dev, T), T,
        0 if error_word is None else _error_word(error_word, dev), _stream(dev))
    if st != OK:
        raise AsymSpecError(st, "asymspec_cache4_write")


def cache4_read(cache, slots, *, dtype=None, out=None, error_word=None):
    """(k, v) [T, kv_heads, head_dim] of a cache in 4 bits at slots [T] int64, of `dtype` (float32 or
    bfloat16, the default) or in the tensors `out`; negative slots give zeros."""
    dev, T = cache.device_index, _tokens_of(slots)
    if out is None:
        shape, kind, new = (T, cache.kv_heads, cache.head_dim), dtype or torch.bfloat16, cache.key_codes.new_empty
        k, v = new(shape, dtype=kind), new(shape, dtype=kind)
        code = _dtype(k)
        k_strides = v_strides = cache.token_strides
    else:
        k, v = out
        if dtype is not None and k.dtype is not dtype:
            raise ValueError(f"out must be of {dtype}")
        code = _dtype(k)
        k_strides, v_strides = _tokens("k", k, cache, k.dtype, T), _tokens("v", v, cache, k.dtype, T)
    st = _lib.asymspec_cache4_read(
        cache.view, _flat("slots", slots, torch.int64, dev, T), T, k.data_ptr(), v.data_ptr(), code, k_strides, v_strides,
        0 if error_word is None else _error_word(error_word, dev), _stream(dev))
    if st != OK:
        raise AsymSpecError(st, "asymspec_cache4_read")
    return k, v


class Cache4Attend:
    """CacheAttend over a cache in 4 bits: holds a workspace for up to B_max requests with Q_max
    queries each.

    ``__call__`` takes q [B, Q, heads, head_dim], float32 or bfloat16, a Cache4, tables [B, width]
    int32 and lens [B] int32 and returns (out like q, lse [B, Q, heads] float32); everything else as
    CacheAttend has it.
    """

    def __init__(self, B_max: int, Q_max: int, heads: int, kv_heads: int, head_dim: int, device=None):
        if torch is None:
            _begin()
        self.B_max, self.Q_max = B_max, Q_max
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.nbytes = cache4_attend_workspace_bytes(B_max, Q_max, heads, kv_heads, head_dim)
        if self.nbytes == 0:
            raise ValueError("no attention of this shape")
        self.workspace = torch.empty(self.nbytes, dtype=torch.uint8,
                                     device=torch.device("cuda" if device is None else device))
        self.device_index = self.workspace.get_device()
        self.scale = 1.0 / math.sqrt(head_dim)

    def __call__(self, q, cache, tables, lens, *, scale=None, window=0, out=None, lse=None, error_word=None):
        dev = cache.device_index
        B, Q, heads, dim = shape = q.shape
        kind = q.dtype
        if dev != self.device_index:
            raise ValueError("the cache must be on the workspace's device")
        if B > self.B_max or Q > self.Q_max or (heads, cache.kv_heads, cache.head_dim) != (
                self.heads, self.kv_heads, self.head_dim):
            raise ValueError("batch does not fit this workspace")
        q0, q1, q2, q3 = q.stride()
        if q.get_device() != dev or q3 != 1 or dim != self.head_dim:
            raise ValueError("q must be [B, Q, heads, head_dim] like the cache, heads contiguous")
        dtype = _dtype(q)
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
        st = _lib.asymspec_cache4_attend(
            cache.view, q.data_ptr(), dtype, _STRIDES3.pack(q0, q1, q2), B, Q, heads, t, t_ld, width,
            _flat("lens", lens, torch.int32, dev, B), self.scale if scale is None else scale, _int(window),
            out.data_ptr(), _STRIDES3.pack(o0, o1, o2), l, self.workspace.data_ptr(), self.nbytes,
            0 if error_word is None else _error_word(error_word, dev), _stream(dev))
        if st != OK:
            raise AsymSpecError(st, "asymspec_cache4_attend")
        return out, lse

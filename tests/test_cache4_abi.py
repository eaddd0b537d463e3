"""The checks of arguments of rotary positions and of the cache in 4 bits, before any CUDA call; and what
their binding hands over, on a library that launches nothing."""
import ctypes

import pytest

from paper_2608_26004_gb300 import asymspec as A
from paper_2608_26004_gb300 import build
from paper_2608_26004_gb300 import serving as S

FAKE = 0x10000  # never dereferenced: every call below fails validation first, or does nothing


@pytest.fixture(scope="module")
def lib():
    build.build_cuda()
    return S.lib()


# ---------------------------------------------------------------- rotary

def heads(x=FAKE, out=2 * FAKE, in_strides=(256, 64), out_strides=(256, 64), n=4):
    return S.RotaryHeads(x, out, (ctypes.c_int64 * 2)(*in_strides), (ctypes.c_int64 * 2)(*out_strides), n)


def rotary(lib, q=None, k=None, T=3, head_dim=64, rotary_dim=64, interleaved=0, positions=FAKE, steps=FAKE,
           magnitude=1.0, dtype=A.BF16):
    q = heads() if q is None else q
    return lib.asymspec_rotary(ctypes.byref(q) if q else None, ctypes.byref(k) if k else None, T, head_dim,
                               rotary_dim, interleaved, 0, positions, steps, magnitude, dtype, None)


def test_rotary_validation_codes(lib):
    f = lambda **a: rotary(lib, **a)  # noqa: E731
    assert f(dtype=7) == A.ERR_UNSUPPORTED
    assert f(head_dim=S.ROTARY_MAX_D + 2) == A.ERR_UNSUPPORTED
    for bad in (dict(q=0), dict(T=-1), dict(head_dim=0, rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=0),
                dict(rotary_dim=66), dict(magnitude=float("nan")), dict(magnitude=float("inf")),
                dict(positions=0), dict(steps=0), dict(q=heads(n=0)), dict(q=heads(x=0)), dict(q=heads(out=0)),
                dict(q=heads(in_strides=(-1, 64))), dict(q=heads(out_strides=(256, -64))),
                dict(q=heads(out_strides=(0, 64))), dict(q=heads(out_strides=(256, 0))),
                dict(q=heads(out=FAKE, out_strides=(512, 64))), dict(k=heads(n=-1)),
                dict(k=heads()),                                         # both into one output
                dict(q=heads(x=FAKE, out=2 * FAKE), k=heads(x=3 * FAKE, out=FAKE)),  # one's output the other's input
                dict(q=heads(x=FAKE, out=2 * FAKE), k=heads(x=2 * FAKE, out=3 * FAKE)),
                dict(q=heads(x=FAKE, out=2 * FAKE), k=heads(x=2 * FAKE, out=FAKE))):
        assert f(**bad) == A.ERR_INVALID_ARG, bad
    assert f(q=heads(n=65537)) == A.ERR_TOO_LARGE
    for bad in (dict(positions=FAKE + 2), dict(steps=FAKE + 4), dict(q=heads(x=FAKE + 1)), dict(q=heads(out=FAKE + 1)),
                dict(q=heads(x=FAKE + 2), dtype=A.FP32)):
        assert f(**bad) == A.ERR_MISALIGNED, bad
    assert f(T=0, positions=0, q=heads(x=0, out=0)) == A.OK
    assert f(T=0, q=heads(out_strides=(0, 64), out=4 * FAKE), positions=0) == A.OK


# ---------------------------------------------------------------- the cache

def cache(**members):
    c = S.PackedCache(FAKE, FAKE, FAKE, FAKE, *((ctypes.c_int64 * 3)(*s) for s in (
        (1024, 32, 512), (128, 4, 64), (1024, 32, 512), (128, 4, 64))), 8, 16, 2, 64, 1.0, 1.0)
    for name, v in members.items():
        setattr(c, name, (ctypes.c_int64 * 3)(*v) if isinstance(v, tuple) else v)
    return c


def write(lib, c=None, k=FAKE, v=FAKE, dtype=A.BF16, strides=(128, 64), slots=FAKE, T=2, err=0):
    c = cache() if c is None else c
    s = (ctypes.c_int64 * 2)(*strides) if strides else None
    return lib.asymspec_cache4_write(ctypes.byref(c) if c else None, k, v, dtype, s, s, slots, T, err, None)


def read(lib, c=None, k=FAKE, v=2 * FAKE, dtype=A.BF16, strides=(128, 64), slots=FAKE, T=2, err=0):
    c = cache() if c is None else c
    s = (ctypes.c_int64 * 2)(*strides) if strides else None
    return lib.asymspec_cache4_read(ctypes.byref(c) if c else None, slots, T, k, v, dtype, s, s, err, None)


def attend(lib, c=None, B=2, Q=2, heads=4, q=FAKE, dtype=A.BF16, q_strides=(512, 256, 64), tables=FAKE, table_ld=4,
           table_width=4, lens=FAKE, scale=1.0, window=0, out=2 * FAKE, out_strides=(512, 256, 64), lse=0,
           ws=FAKE, ws_bytes=1 << 40, err=0):
    c = cache() if c is None else c
    strides = [(ctypes.c_int64 * 3)(*s) if s else None for s in (q_strides, out_strides)]
    return lib.asymspec_cache4_attend(ctypes.byref(c) if c else None, q, dtype, strides[0], B, Q, heads, tables,
                                      table_ld, table_width, lens, scale, window, out, strides[1], lse, ws, ws_bytes,
                                      err, None)


@pytest.mark.parametrize("call", [write, read, attend])
def test_every_call_checks_the_cache(lib, call):
    f = lambda **m: call(lib, cache(**m))  # noqa: E731
    assert call(lib, c=0) == A.ERR_INVALID_ARG
    for bad in (dict(key_codes=0), dict(key_scales=0), dict(value_codes=0), dict(value_scales=0), dict(num_blocks=0),
                dict(block_size=0), dict(kv_heads=0), dict(head_dim=0), dict(key_code_strides=(-16, 0, 0)),
                dict(value_scale_strides=(0, 0, -2)), dict(key_scale=0.0), dict(value_scale=-1.0),
                dict(key_scale=float("nan")), dict(value_scale=2.0 ** 65), dict(key_scale=2.0 ** -65)):
        assert f(**bad) == A.ERR_INVALID_ARG, bad
    assert f(head_dim=48) == A.ERR_UNSUPPORTED and f(head_dim=288) == A.ERR_UNSUPPORTED
    for bad in (dict(key_codes=FAKE + 8), dict(value_codes=FAKE + 8), dict(key_scales=FAKE + 1),
                dict(value_scales=FAKE + 1), dict(key_code_strides=(1024, 24, 512)),
                dict(value_scale_strides=(128, 3, 64))):
        assert f(**bad) == A.ERR_MISALIGNED, bad
    assert f(num_blocks=1 << 27) == A.ERR_TOO_LARGE and f(kv_heads=65538) == A.ERR_TOO_LARGE


@pytest.mark.parametrize("call", [write, read])
def test_write_and_read_validation_codes(lib, call):
    f = lambda **a: call(lib, **a)  # noqa: E731
    assert f(dtype=5) == A.ERR_UNSUPPORTED
    for bad in (dict(T=-1), dict(strides=None), dict(strides=(-1, 64)), dict(k=0), dict(v=0), dict(slots=0)):
        assert f(**bad) == A.ERR_INVALID_ARG, bad
    for bad in (dict(k=FAKE + 1), dict(v=3 * FAKE + 2, dtype=A.FP32), dict(slots=FAKE + 4), dict(err=FAKE + 2)):
        assert f(**bad) == A.ERR_MISALIGNED, bad
    assert f(T=0, k=0, v=0, slots=0) == A.OK
    if call is read:
        assert f(v=FAKE) == A.ERR_INVALID_ARG                            # one output for both
        assert f(strides=(0, 64)) == A.ERR_INVALID_ARG and f(strides=(128, 0)) == A.ERR_INVALID_ARG


def test_attend_validation_codes(lib):
    f = lambda **a: attend(lib, **a)  # noqa: E731
    assert f(dtype=5) == A.ERR_UNSUPPORTED
    for bad in (dict(B=-1), dict(Q=-1), dict(heads=3), dict(heads=0), dict(table_width=0), dict(table_ld=3),
                dict(scale=float("nan")), dict(scale=3e38), dict(window=-1), dict(q_strides=None),
                dict(out_strides=None), dict(q_strides=(-1, 0, 0)), dict(out_strides=(0, 256, 64)),
                dict(out_strides=(512, 0, 64)), dict(out_strides=(512, 256, 0)), dict(q=0), dict(tables=0),
                dict(lens=0), dict(out=0), dict(out=FAKE)):
        assert f(**bad) == A.ERR_INVALID_ARG, bad
    for bad in (dict(q=FAKE + 1), dict(out=FAKE + 1), dict(tables=FAKE + 2), dict(lens=FAKE + 2), dict(lse=FAKE + 2),
                dict(err=FAKE + 1)):
        assert f(**bad) == A.ERR_MISALIGNED, bad
    assert f(B=S.CACHE_MAX_B + 1) == A.ERR_TOO_LARGE
    assert f(Q=1 << 19) == A.ERR_TOO_LARGE
    assert f(table_width=1 << 27, table_ld=1 << 27) == A.ERR_TOO_LARGE
    for bad in (dict(ws=0), dict(ws=FAKE + 128), dict(ws_bytes=1000)):
        assert f(**bad) == A.ERR_WORKSPACE, bad
    assert f(B=0, q=0, ws=0) == A.OK and f(Q=0, q=0, ws=0) == A.OK


def test_workspace_bytes(lib):
    f = S.cache4_attend_workspace_bytes
    assert f(0, 1, 8, 8, 64) == f(1, 1, 8, 3, 64) == f(1, 1, 8, 8, 80) == f(1, 1, 8, 8, 288) == 0
    assert f(S.CACHE_MAX_B + 1, 1, 8, 8, 64) == f(1, 1 << 18, 8, 8, 64) == 0
    sizes = [f(4, Q, 32, 8, 128) for Q in range(1, 40)]
    assert sizes == sorted(sizes) and sizes[0] > 0                       # one for more queries serves fewer


def test_workspaces_have_room_for_the_ctas_that_there_are(lib):
    """32 bytes a CTA, and for two parts of each a row's 2 numbers and its values: 456 CTAs for attention over the
    16-bit and 32-bit cache, whose callers may have laid out that; over the 4-bit one as many as its kernels have."""
    def nbytes(ctas, rows, D):
        whole = lambda n: -(-n // 256) * 256  # noqa: E731
        return whole(32 * ctas) + whole(2 * ctas * rows * 2 * 4) + 2 * ctas * rows * D * 4

    f, g = S.cache_attend_workspace_bytes, S.cache4_attend_workspace_bytes
    assert f(8, 8, 64, 8, 128) == nbytes(456, 64, 128) == 30365952
    assert f(64, 1, 32, 8, 128) == nbytes(456, 16, 128) and f(1, 4, 32, 8, 64) == nbytes(456, 16, 64)
    assert g(64, 1, 32, 8, 128) == nbytes(608, 8, 128)
    assert g(8, 8, 64, 8, 128) == nbytes(304, 64, 128)
    assert g(8, 8, 64, 8, 256) == max(nbytes(152, 64, 256), nbytes(304, 32, 256))  # (for up to 64 rows, or up to 32)
    for D in (32, 64, 96, 128, 160, 256):
        sizes = [g(4, Q, 8, 8, D) for Q in range(1, 200)]
        assert sizes == sorted(sizes)                                    # one for more queries serves fewer


# ---------------------------------------------------------------- the binding

torch = pytest.importorskip("torch")


class Placed(torch.Tensor):
    """A tensor that claims to be on cuda:`place`."""
    place = 0

    def get_device(self):
        return self.place


def placed(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Placed)


class Library:
    """Writes down each call's name and arguments, and launches nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return A.OK
        return call


@pytest.fixture
def library(lib, monkeypatch):
    S._begin()
    fake = Library()
    monkeypatch.setattr(S, "_lib", fake)
    monkeypatch.setattr(S.torch.cuda, "current_device", lambda: Placed.place)
    monkeypatch.setattr(S.torch._C, "_cuda_getCurrentRawStream", lambda dev: 0x5000 + dev, raising=False)
    return fake


def a_cache(**k):
    parts = (placed(3, 16, 2, n, dtype=torch.uint8) for n in (32, 4, 32, 4))
    return S.Cache4(*parts, **k)


def every_call(where):
    c, k, slots = a_cache(), placed(4, 2, 64), placed(4, dtype=torch.int64)
    over = S.Cache4Attend.__new__(S.Cache4Attend)
    over.B_max, over.Q_max, over.heads, over.kv_heads, over.head_dim = 2, 3, 4, 2, 64
    over.nbytes, over.workspace, over.device_index, over.scale = 256, placed(64), where, 1.0
    turn = S.Rotary.__new__(S.Rotary)
    turn.head_dim, turn.rotary_dim, turn.interleaved, turn.magnitude = 64, 32, False, 1.0
    turn.steps, turn.device_index = placed(16, dtype=torch.int64), where
    return {
        "asymspec_rotary": lambda: turn(k, placed(4, dtype=torch.int32), k, q_out=placed(4, 2, 64)),
        "asymspec_cache4_write": lambda: S.cache4_write(k, k, c, slots),
        "asymspec_cache4_read": lambda: S.cache4_read(c, slots),
        "asymspec_cache4_attend": lambda: over(placed(2, 3, 4, 64), c, placed(2, 3, dtype=torch.int32),
                                               placed(2, dtype=torch.int32)),
    }


@pytest.mark.parametrize("where", [0, 1])
@pytest.mark.parametrize("name", ["asymspec_rotary", "asymspec_cache4_write", "asymspec_cache4_read",
                                  "asymspec_cache4_attend"])
def test_tensors_on_another_device_than_the_current_one(library, monkeypatch, name, where):
    monkeypatch.setattr(Placed, "place", where)
    call = every_call(where)[name]
    monkeypatch.setattr(S.torch.cuda, "current_device", lambda: 1 - where)
    with pytest.raises(ValueError, match="cuda:%d" % where):
        call()
    assert not library.calls
    monkeypatch.setattr(S.torch.cuda, "current_device", lambda: where)
    call()
    (got, args), = library.calls
    assert got == name and args[-1] == 0x5000 + where


def test_the_view_of_a_cache(library):
    codes = placed(3, 2, 16, 32, dtype=torch.uint8).transpose(1, 2)
    scales = placed(3, 2, 16, 4, dtype=torch.uint8).transpose(1, 2)
    c = S.Cache4(codes, scales, codes, scales.view(torch.float8_e4m3fn), key_scale=0.5, value_scale=0.25)
    v = S.PackedCache.from_buffer_copy(c.view)
    assert (v.key_codes, v.value_scales) == (codes.data_ptr(), scales.data_ptr())
    assert tuple(v.key_code_strides) == (1024, 32, 512) and tuple(v.value_scale_strides) == (128, 4, 64)
    assert (v.num_blocks, v.block_size, v.kv_heads, v.head_dim) == (3, 16, 2, 64)
    assert (v.key_scale, v.value_scale) == (0.5, 0.25)
    # the stride of an axis of one entry is nobody's
    one = placed(3, 16, 1, 32, dtype=torch.uint8).as_strided((3, 16, 1, 32), (512, 32, 7, 1))
    few = placed(3, 16, 1, 4, dtype=torch.uint8).as_strided((3, 16, 1, 4), (64, 4, 3, 1))
    v = S.PackedCache.from_buffer_copy(S.Cache4(one, few, one, few).view)
    assert tuple(v.key_code_strides) == (512, 32, 0) and tuple(v.key_scale_strides) == (64, 4, 0)


def test_refusals_of_the_binding(library):
    codes, scales = placed(3, 16, 2, 32, dtype=torch.uint8), placed(3, 16, 2, 4, dtype=torch.uint8)
    for bad in ((codes.float(), scales, codes, scales), (codes, scales, codes[:2], scales),
                (codes, codes, codes, scales), (codes, scales, codes, scales.float()),
                (codes[0], scales, codes[0], scales), (torch.zeros(3, 16, 2, 32, dtype=torch.uint8), scales, codes, scales),
                (codes.transpose(2, 3), scales, codes.transpose(2, 3), scales)):
        with pytest.raises(ValueError):
            S.Cache4(*bad)
    c, k, slots = a_cache(), placed(4, 2, 64), placed(4, dtype=torch.int64)
    for bad in ((k, k[:3], slots), (k, k.float(), slots), (k, k, slots.int()), (k, k, slots[:3]), (k[0], k[0], slots),
                (k[..., :32], k[..., :32], slots), (k.transpose(0, 2), k.transpose(0, 2), slots)):
        with pytest.raises(ValueError):
            S.cache4_write(bad[0], bad[1], c, bad[2])
    with pytest.raises(TypeError):
        S.cache4_write(k.half(), k.half(), c, slots)
    with pytest.raises(ValueError):
        S.cache4_read(c, slots, out=(k, k[:3]))
    with pytest.raises(ValueError):
        S.cache4_read(c, slots, dtype=torch.float32, out=(k, k))
    with pytest.raises(TypeError):
        S.cache4_read(c, slots, dtype=torch.float16)
    turn = every_call(0)["asymspec_rotary"]
    turn()
    library.calls.clear()
    rotary_ = S.Rotary.__new__(S.Rotary)
    rotary_.head_dim, rotary_.rotary_dim, rotary_.interleaved, rotary_.magnitude = 64, 64, False, 1.0
    rotary_.steps, rotary_.device_index = placed(32, dtype=torch.int64), 0
    pos = placed(4, dtype=torch.int32)
    for bad in (dict(q=k, positions=pos.long()), dict(q=k, positions=pos[:3]), dict(q=k, positions=pos, k=k[:3]),
                dict(q=k, positions=pos, k=k.float()), dict(q=k[..., :32], positions=pos), dict(q=k[0], positions=pos),
                dict(q=k, positions=pos, k_out=k), dict(q=k, positions=pos, q_out=k[:3]),
                dict(q=k, positions=pos, q_out=k.float()), dict(q=k.transpose(0, 1)[:, :, :64], positions=pos)):
        with pytest.raises(ValueError):
            rotary_(**bad)
    assert not library.calls


def test_rotary_of_tensors_that_require_a_gradient(library):
    """Results that autograd knows, or a refusal; without gradients as ever."""
    turn = S.Rotary.__new__(S.Rotary)
    turn.head_dim, turn.rotary_dim, turn.interleaved, turn.magnitude = 64, 32, False, 1.0
    turn.steps, turn.device_index = placed(16, dtype=torch.int64), 0
    q, k, pos = placed(4, 2, 64), placed(4, 1, 64), placed(4, dtype=torch.int32)
    q.requires_grad_()
    for out in (turn(q, pos)[0], *turn(q, pos, k), *turn(k, pos, q)):
        assert out.requires_grad and out.grad_fn is not None
    for more in (dict(q_out=placed(4, 2, 64)), dict(k=k, k_out=placed(4, 1, 64)), dict(q_out=q)):
        n = len(library.calls)
        with pytest.raises(ValueError, match="without gradients"):
            turn(q, pos, **more)
        assert len(library.calls) == n
    with torch.no_grad():
        assert not turn(q, pos, q_out=placed(4, 2, 64))[0].requires_grad
    assert turn(k, pos)[0].grad_fn is None

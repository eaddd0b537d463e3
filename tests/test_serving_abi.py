"""The checks of arguments of the operators around the step, before any CUDA call."""
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


def constrain(lib, B=2, P=3, V=64, dtype=A.FP32, ld=64, out_ld=64, logits=FAKE, out=FAKE, null=False,
              **members):
    c = S.Constraints()
    c.mask_value = -S.FLT_MAX
    for name, v in members.items():
        setattr(c, name, v)
    return lib.asymspec_constrain_logits(None if null else ctypes.byref(c), logits, ld, out, out_ld, B,
                                         P, V, dtype, None, None)


def test_constrain_logits_validation_codes(lib):
    f = lambda **k: constrain(lib, **k)  # noqa: E731
    assert f(dtype=2) == A.ERR_UNSUPPORTED
    assert f(null=True) == A.ERR_INVALID_ARG
    assert f(B=-1) == A.ERR_INVALID_ARG
    assert f(P=-1) == A.ERR_INVALID_ARG
    assert f(V=1) == A.ERR_INVALID_ARG
    assert f(ld=63) == A.ERR_INVALID_ARG
    assert f(out_ld=63) == A.ERR_INVALID_ARG
    assert f(P=S.CONSTRAIN_MAX_P + 1) == A.ERR_TOO_LARGE
    assert f(B=65536) == A.ERR_TOO_LARGE
    assert f(V=(1 << 30) + 1, ld=1 << 31, out_ld=1 << 31) == A.ERR_TOO_LARGE
    assert f(logits=0) == A.ERR_INVALID_ARG
    assert f(out=0) == A.ERR_INVALID_ARG
    assert f(ld=80) == A.ERR_INVALID_ARG                                # in place, another stride
    assert f(out=FAKE + 2) == A.ERR_MISALIGNED
    assert f(logits=FAKE + 1, dtype=A.BF16) == A.ERR_MISALIGNED
    assert f(history=FAKE) == A.ERR_INVALID_ARG                         # without lengths
    assert f(history_len=FAKE) == A.ERR_INVALID_ARG                     # lengths of nothing
    assert f(history=FAKE, history_len=FAKE, history_width=-1) == A.ERR_INVALID_ARG
    assert f(history=FAKE + 2, history_len=FAKE) == A.ERR_MISALIGNED
    assert f(bias_offsets=FAKE, bias_count=2) == A.ERR_INVALID_ARG      # without entries
    assert f(bias_tokens=FAKE) == A.ERR_INVALID_ARG                     # entries of no request
    assert f(bias_offsets=FAKE, bias_tokens=FAKE, bias_values=FAKE, bias_count=-1) == A.ERR_INVALID_ARG
    assert f(mask=FAKE, mask_ld=1, mask_count=6) == A.ERR_INVALID_ARG   # 32 bits for 64 tokens
    assert f(mask=FAKE, mask_ld=2, mask_count=5) == A.ERR_INVALID_ARG   # 5 rows for 6 positions
    assert f(mask=FAKE, mask_ld=2, mask_count=6, mask_value=float("inf")) == A.ERR_INVALID_ARG
    assert f(mask_rows=FAKE) == A.ERR_INVALID_ARG
    assert f(repetition=FAKE + 1) == A.ERR_MISALIGNED
    assert f(B=0, logits=0, out=0) == A.OK
    assert f(P=0, logits=0, out=0) == A.OK


def plan(lib, B=2, block_size=16, num_blocks=8, table_ld=4, table_width=4, capacity=6, grow_all=3, **p):
    x = dict(lens=FAKE, accepted=0, grow=0, tables=FAKE, held=FAKE, free_list=FAKE, free_count=FAKE,
             start=FAKE, len=FAKE, out_held=FAKE, out_free=FAKE, offsets=FAKE, slots=FAKE, positions=0)
    x.update(p)
    return lib.asymspec_cache_plan(x["lens"], x["accepted"], x["grow"], grow_all, B, block_size,
                                   num_blocks, x["tables"], table_ld, table_width, x["held"],
                                   x["free_list"], x["free_count"], x["start"], x["len"], x["out_held"],
                                   x["out_free"], x["offsets"], x["slots"], x["positions"], capacity,
                                   None, None)


def test_cache_plan_validation_codes(lib):
    f = lambda **k: plan(lib, **k)  # noqa: E731
    for bad in (dict(B=-1), dict(block_size=0), dict(num_blocks=0), dict(table_width=0),
                dict(table_ld=3), dict(capacity=-1), dict(grow_all=-1), dict(lens=0), dict(tables=0),
                dict(held=0), dict(free_list=0), dict(free_count=0), dict(start=0), dict(len=0),
                dict(out_held=0), dict(out_free=0), dict(offsets=0), dict(slots=0)):
        assert f(**bad) == A.ERR_INVALID_ARG, bad
    for bad in (dict(B=S.CACHE_MAX_B + 1), dict(B=8192, table_width=1 << 19, table_ld=1 << 19),
                dict(block_size=1 << 30), dict(num_blocks=1 << 30), dict(capacity=1 << 31)):
        assert f(**bad) == A.ERR_TOO_LARGE, bad
    for bad in (dict(lens=FAKE + 2), dict(grow=FAKE + 1), dict(slots=FAKE + 4), dict(positions=FAKE + 2)):
        assert f(**bad) == A.ERR_MISALIGNED, bad


def cache(**k):
    x = dict(keys=FAKE, values=FAKE, key_strides=(1024, 64, 32), value_strides=(1024, 64, 32),
             num_blocks=8, block_size=16, kv_heads=2, head_dim=32, dtype=A.BF16)
    x.update(k)
    return S.Cache(x["keys"], x["values"], S._L3(*x["key_strides"]), S._L3(*x["value_strides"]),
                   x["num_blocks"], x["block_size"], x["kv_heads"], x["head_dim"], x["dtype"])


BAD_CACHES = ((dict(keys=0), A.ERR_INVALID_ARG), (dict(values=0), A.ERR_INVALID_ARG),
              (dict(num_blocks=0), A.ERR_INVALID_ARG), (dict(block_size=0), A.ERR_INVALID_ARG),
              (dict(kv_heads=0), A.ERR_INVALID_ARG), (dict(head_dim=0), A.ERR_INVALID_ARG),
              (dict(key_strides=(1024, -64, 32)), A.ERR_INVALID_ARG), (dict(dtype=5), A.ERR_UNSUPPORTED),
              (dict(num_blocks=1 << 30), A.ERR_TOO_LARGE), (dict(keys=FAKE + 1), A.ERR_MISALIGNED))


def write(lib, T=4, k=FAKE, v=FAKE, ks=(64, 32), slots=FAKE, null=False, **c):
    x = cache(**c)
    return lib.asymspec_cache_write(None if null else ctypes.byref(x), k, v, S._L2(*ks), S._L2(64, 32),
                                    slots, T, None, None)


def test_cache_write_validation_codes(lib):
    assert write(lib, null=True) == A.ERR_INVALID_ARG
    for bad, want in BAD_CACHES:
        assert write(lib, **bad) == want, bad
    for bad in (dict(T=-1), dict(k=0), dict(v=0), dict(slots=0), dict(ks=(-1, 32))):
        assert write(lib, **bad) == A.ERR_INVALID_ARG, bad
    assert write(lib, slots=FAKE + 4) == A.ERR_MISALIGNED
    assert write(lib, k=FAKE + 1) == A.ERR_MISALIGNED
    assert write(lib, T=0, k=0, v=0, slots=0) == A.OK


def attend(lib, B=2, Q=3, heads=4, qs=(384, 128, 32), scale=1.0, window=0, width=4, ld=4, ws=FAKE,
           nbytes=1 << 30, null=False, q=FAKE, out=FAKE, tables=FAKE, lens=FAKE, lse=0, **c):
    x = cache(**c)
    return lib.asymspec_cache_attend(None if null else ctypes.byref(x), q, S._L3(*qs), B, Q, heads,
                                     tables, ld, width, lens, scale, window, out, S._L3(384, 128, 32),
                                     lse, ws, nbytes, None, None)


def test_cache_attend_validation_codes(lib):
    assert attend(lib, null=True) == A.ERR_INVALID_ARG
    for bad, want in BAD_CACHES:
        assert attend(lib, **bad) == want, bad
    for bad in (dict(B=-1), dict(Q=-1), dict(heads=0), dict(heads=3), dict(width=0), dict(ld=3),
                dict(scale=float("nan")), dict(window=-1), dict(qs=(384, -128, 32)), dict(q=0),
                dict(out=0), dict(tables=0), dict(lens=0)):
        assert attend(lib, **bad) == A.ERR_INVALID_ARG, bad
    assert attend(lib, head_dim=264) == A.ERR_UNSUPPORTED
    for bad in (dict(B=S.CACHE_MAX_B + 1), dict(Q=1 << 19), dict(width=1 << 28, ld=1 << 28)):
        assert attend(lib, **bad) == A.ERR_TOO_LARGE, bad
    for bad in (dict(keys=FAKE + 2), dict(values=FAKE + 8), dict(head_dim=36),
                dict(key_strides=(1024, 64, 36)), dict(q=FAKE + 1), dict(lens=FAKE + 2), dict(lse=FAKE + 1)):
        assert attend(lib, **bad) == A.ERR_MISALIGNED, bad
    need = S.cache_attend_workspace_bytes(2, 3, 4, 2, 32)
    assert need > 0
    for bad in (dict(ws=0), dict(ws=FAKE + 16), dict(nbytes=need - 1)):
        assert attend(lib, **bad) == A.ERR_WORKSPACE, bad
    assert attend(lib, B=0, q=0) == A.OK
    assert attend(lib, Q=0, q=0) == A.OK


def test_cache_attend_refuses_its_queries_as_its_output(lib):
    """CTAs that share a request read its queries while others write: not in place."""
    assert attend(lib, q=FAKE, out=FAKE) == A.ERR_INVALID_ARG
    assert attend(lib, q=FAKE, out=FAKE, head_dim=36) == A.ERR_MISALIGNED    # (after all other checks)
    assert attend(lib, q=FAKE, out=FAKE, nbytes=0) == A.ERR_WORKSPACE


def test_cache_attend_workspace_of_no_shape(lib):
    n = S.cache_attend_workspace_bytes
    for shape in ((0, 1, 4, 2, 64), (1, 0, 4, 2, 64), (1, 1, 3, 2, 64), (1, 1, 4, 2, 257),
                  (S.CACHE_MAX_B + 1, 1, 4, 2, 64), (1, 1, 4, 0, 64), (1, 1 << 20, 4, 2, 64)):
        assert n(*shape) == 0, shape
    assert n(1, 1, 4, 2, 64) > 0


def test_structs_as_bytes_have_the_structures_layout():
    for packed, structure in ((S._CONSTRAINTS, S.Constraints), (S._CACHE, S.Cache)):
        assert packed.size == ctypes.sizeof(structure)
    n = [name for name, _ in S.Constraints._fields_]
    c = S.Constraints.from_buffer_copy(S._CONSTRAINTS.pack(*range(1, len(n)), 0.5))
    assert [getattr(c, name) for name in n] == list(range(1, len(n))) + [0.5]
    x = S.Cache.from_buffer_copy(S._CACHE.pack(*range(1, 14)))
    assert (x.keys, x.values, list(x.key_strides), list(x.value_strides)) == (1, 2, [3, 4, 5], [6, 7, 8])
    assert (x.num_blocks, x.block_size, x.kv_heads, x.head_dim, x.dtype) == (9, 10, 11, 12, 13)


def test_the_joining_kernel_waits_for_the_one_before():
    # attend_join is a programmatic dependent: resident while attend_split still runs
    import os
    import re
    with open(os.path.join(build.CSRC, "serving.cu")) as f:
        host = re.sub(r"//[^\n]*", "", f.read())
    assert host.count("programmaticStreamSerializationAllowed = 1") == 1
    with open(os.path.join(build.CSRC, "kernel_attend.cuh")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    body = text[text.index(" attend_join("):]
    first = re.search(r"griddepcontrol\.wait|\breturn;|p\.ws", body)
    assert first and first.group().startswith("griddep")


def test_arrays_that_vectors_read_lie_on_their_boundaries():
    import os
    import re
    for name in ("kernel_attend.cuh", "kernel_cache.cuh", "kernel_constrain.cuh"):
        with open(os.path.join(build.CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        arrays = set()
        for m in re.finditer(r"reinterpret_cast<(?:const )?(?:uint2|uint4|int4|float4|longlong2)\*>\((\w+)\b", text):
            # (the nearest declaration of that name before it, if that is an array)
            found = re.findall(r"[;{]([^;{}]*\b(?:T|float|int|unsigned)\b\*? [^;{}()]*\b%s\b[^;]*);" % m.group(1), text[:m.start()])
            if found and re.search(r"\b%s\[" % m.group(1), found[-1]):
                arrays.add(m.group(1))
                assert "__align__(16)" in found[-1], (name, found[-1].strip())
        assert arrays == {"kernel_attend.cuh": {"x", "y", "s_x"}, "kernel_cache.cuh": {"pos"},
                          "kernel_constrain.cuh": {"c_smem"}}[name]


def test_rows_that_share_memory():
    """Expanded views: rows that lie over one another are read where they are, never a row's
    width apart (which would be past the tensor's end); logits' rows must not be."""
    torch = pytest.importorskip("torch")
    one = torch.zeros(1, 9, dtype=torch.int32)
    assert S._rows("x", one.expand(5, 9), torch.int32, -1, 5)[1:] == (0, 9)
    assert S._rows("x", one, torch.int32, -1, 1)[1:] == (9, 9)
    assert S._rows("x", torch.zeros(3, 12, dtype=torch.int32)[:, :9], torch.int32, -1, 3)[1:] == (12, 9)
    z = torch.zeros(1, 1, 8)
    assert S._row_distance("z", z, 1, 1, 8) == 8
    assert S._row_distance("z", torch.zeros(2, 3, 10)[..., :8], 2, 3, 8) == 10
    for B, P in ((4, 1), (1, 4), (2, 3)):
        with pytest.raises(ValueError):
            S._row_distance("z", z.expand(B, P, 8), B, P, 8)
    with pytest.raises(ValueError):
        S._row_distance("z", torch.zeros(40).as_strided((2, 3, 8), (15, 5, 1)), 2, 3, 8)


def test_windows_of_any_size_stay_in_32_bits(tmp_path):
    """The host's bound of the window, compiled as it is, and the kernels' 32-bit sums with it: the
    first key, in request lengths from none to the table's; a window that spans the table is none."""
    import subprocess
    source = tmp_path / "window.cpp"
    source.write_text('''
        #include <cstdio>
        #include "k_attend.h"
        int main() {
          int window, width, block;
          while (std::scanf("%d %d %d", &window, &width, &block) == 3)
            std::printf("%d\\n", asymspec_impl::attend_window(window, width, block));
        }''')
    program = str(tmp_path / "window")
    subprocess.run(["g++", "-std=c++17", "-I", build.CSRC, str(source), "-o", program], check=True)
    top = 2 ** 31 - 1
    tables = [(1, 1), (4, 16), (64, 24), (1 << 26, 16), (1, 1 << 30)]
    asked = [(w, width, bs) for width, bs in tables
             for w in {0, 1, 16, width * bs - 1, width * bs, width * bs + 1, 1 << 30, top - 8, top} if w <= top]
    got = subprocess.run([program], input="\n".join("%d %d %d" % a for a in asked), capture_output=True,
                         text=True, check=True).stdout.split()
    assert len(got) == len(asked)
    for (w, width, bs), g in zip(asked, map(int, got)):
        assert g == (w if w < width * bs else 0), (w, width, bs)
        for n in (0, 1, width * bs):
            for Q in (1, 3, 1 << 20):
                first = max(0, n - Q - g + 1) if g else 0
                assert -2 ** 31 <= n - Q - g + 1 and 0 <= first <= n
                # of the key p that a query is at, with and without the bound: the same first key
                for p in (0, n - Q, n - 1):
                    if 0 <= p < width * bs:
                        assert (max(0, p - w + 1) if w else 0) == (max(0, p - g + 1) if g else 0)
    import os
    with open(os.path.join(build.CSRC, "serving.cu")) as f:
        assert f.read().count("p.window = attend_window(window, table_width, cache->block_size);") == 1


def test_cache_attend_refuses_outputs_that_lie_over_one_another(lib):
    def call(os, B=2, Q=3, heads=4):
        x = cache()
        return lib.asymspec_cache_attend(ctypes.byref(x), FAKE, S._L3(384, 128, 32), B, Q, heads, FAKE, 4, 4, FAKE,
                                         1.0, 0, FAKE, S._L3(*os), 0, 0, 0, None, None)
    for os in ((0, 128, 32), (384, 0, 32), (384, 128, 0)):
        assert call(os) == A.ERR_INVALID_ARG, os
    # an axis of one has any stride: what follows is the next check, of the workspace
    assert call((384, 128, 32)) == A.ERR_WORKSPACE
    assert call((0, 128, 32), B=1) == A.ERR_WORKSPACE
    assert call((384, 0, 32), Q=1) == A.ERR_WORKSPACE

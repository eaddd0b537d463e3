"""Attention over a cache in 4 bits against its definition in 64 bits."""
import math
import random

import pytest

from paper_2608_26004_gb300 import asymspec as A
from paper_2608_26004_gb300 import serving as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as _torch
    assert _torch.cuda.is_available(), "the gpu tests need a CUDA device"
    from paper_2608_26004_gb300 import build
    build.build_cuda()
    S.lib()
    return _torch


def inputs(torch, lens, Q, heads, kv, D, dtype, bs, seed, layout="hnd", spread=2.0, poison=True, slack=3, apart=0,
           key_scale=1.0, value_scale=1.0):
    """(q, cache, tables, lens): a pool in which every scale that no query may see is a NaN, and the codes are
    what the memory held; `apart`: bytes between the scales of a token's heads."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    B = len(lens)
    pages = [-(-max(n, 0) // bs) for n in lens]
    blocks = sum(pages) + slack
    width = max(pages + [1]) + 2
    ids = torch.randperm(blocks, generator=g, device="cuda").int()
    tables = torch.full((B, width + 3), -1, device="cuda", dtype=torch.int32)[:, :width]
    live = torch.zeros(blocks, bs, device="cuda", dtype=torch.bool)
    at = 0
    for b, n in enumerate(lens):
        mine = ids[at:at + pages[b]]
        at += pages[b]
        tables[b, :pages[b]] = mine
        j = torch.arange(max(n, 0), device="cuda")
        live[mine.long()[j // bs], j % bs] = True
    order = (blocks, kv, bs) if layout == "hnd" else (blocks, bs, kv)

    def part(width, room=0):
        x = torch.zeros(*order, width + room, dtype=torch.uint8, device="cuda")[..., :width]
        return x.transpose(1, 2) if layout == "hnd" else x

    cache = S.Cache4(part(D // 2), part(D // 16, apart), part(D // 2), part(D // 16, apart), key_scale=key_scale,
                     value_scale=value_scale)
    x = torch.randn(2, blocks * bs, kv, D, generator=g, device="cuda")
    S.cache4_write(x[0] * key_scale, x[1] * value_scale, cache, torch.arange(blocks * bs, device="cuda"))
    if poison:
        cache.key_scales[~live] = 0x7F
        cache.value_scales[~live] = 0xFF
        cache.key_codes[~live] = 0x77
    qkv = torch.randn(B, Q, (heads + 2) * D, generator=g, device="cuda").mul_(spread / key_scale).to(getattr(torch, dtype))
    q = qkv[..., :heads * D].unflatten(-1, (heads, D))
    return q, cache, tables, torch.tensor(lens, device="cuda", dtype=torch.int32)


def check(torch, x, out, lse, rows, scale=None, window=0):
    """Tolerances.  Keys and values enter as they are, queries to 2^-22, a score's factor and its distance from the
    reference are rounded three times: 2^-20 of the sum of magnitudes (`spread`), and its sum of D by D 2^-24 more:
    a score's error d.  Weights are then off by 2 d + 2^-20, as fp16 by 2^-11 more for bf16 (2^-22 for fp32, within
    that 2^-20) and, where they are small, by 2^-32 of the largest; sums of n of them by n 2^-24 where added one
    after another, products of the values 2^-22 more; the output is rounded once, so the bounds are rounded with
    it."""
    from tests._cache4 import values
    from tests._serving import attended
    q, cache, tables, lens = x
    D, bf16 = q.shape[3], q.dtype == torch.bfloat16
    keys, vals = (values(c, s, n) for c, s, n in ((cache.key_codes, cache.key_scales, cache.key_scale),
                                                  (cache.value_codes, cache.value_scales, cache.value_scale)))
    largest = float(vals.nan_to_num(0.0).abs().max())
    for b, i, h in rows:
        o, l, mag, spread, n = attended(q, keys, vals, tables, lens, b, i, h, scale=scale, window=window)
        got, gl = out[b, i, h].double().cpu(), float(lse[b, i, h])
        if n == 0:
            assert (got == 0).all() and gl == -math.inf, (b, i, h)
            continue
        d = spread * (2.0 ** -20 + D * 2.0 ** -24)
        tol = (2 * d + 2.0 ** -20 + 2.0 ** -22 + (2.0 ** -11 if bf16 else 0) + n * 2.0 ** -24) * mag \
            + n * 2.0 ** -32 * largest
        least, most = ((o + t).to(q.dtype).double() for t in (-tol, tol))
        bad = ~((least <= got) & (got <= most))
        assert not bad.any(), (b, i, h, n, got[bad][:5], o[bad][:5], tol[bad][:5])
        assert abs(gl - l) <= d + 2.0 ** -20 * (1 + abs(l)) + n * 2.0 ** -24, (b, i, h, gl, l)


def some_rows(B, Q, heads, seed, most=40):
    every = [(b, i, h) for b in range(B) for i in range(Q) for h in range(heads)]
    return every if len(every) <= most else random.Random(seed).sample(every, most)


CASES = [
    # lens, Q, heads, kv heads, D, dtype, block, layout, window
    ([1], 1, 1, 1, 64, "bfloat16", 16, "nhd", 0),
    ([1000], 1, 16, 8, 128, "bfloat16", 16, "hnd", 0),
    ([17, 0, 300, 64, 1, 2049], 1, 32, 8, 128, "bfloat16", 16, "nhd", 0),
    ([500, 3, 0, 8, 7, 4097], 8, 32, 8, 128, "bfloat16", 32, "hnd", 0),   # some shorter than Q
    ([129, 4000, 63], 8, 64, 8, 128, "bfloat16", 16, "nhd", 0),           # 64 rows a kv head
    ([777, 5], 9, 24, 3, 64, "bfloat16", 24, "nhd", 0),                   # blocks that no tile divides
    ([100, 333], 5, 8, 2, 96, "bfloat16", 7, "hnd", 0),
    ([211], 3, 6, 6, 32, "bfloat16", 1, "nhd", 0),
    ([1500, 40], 2, 4, 1, 256, "bfloat16", 16, "nhd", 0),
    ([1500, 40], 5, 8, 2, 256, "bfloat16", 16, "hnd", 0),                 # 20 rows of 256
    ([1500, 700], 10, 8, 2, 256, "bfloat16", 16, "hnd", 0),               # 40 rows of 256
    ([600], 4, 12, 4, 160, "bfloat16", 48, "nhd", 0),
    ([600, 77], 4, 12, 4, 128, "bfloat16", 8, "hnd", 0),                  # 12 rows
    ([90, 91], 2, 10, 2, 64, "bfloat16", 16, "hnd", 0),                   # 10 rows of 64
    ([90, 1291], 4, 20, 2, 64, "bfloat16", 16, "hnd", 0),                 # 40 rows of 64
    ([5000, 70], 5, 16, 8, 128, "bfloat16", 16, "nhd", 100),              # windows
    ([3000, 1], 1, 16, 2, 128, "bfloat16", 64, "hnd", 1),
    ([130, 2000], 8, 8, 8, 64, "bfloat16", 48, "nhd", 16),
    ([900, 300, 127], 9, 32, 4, 128, "bfloat16", 16, "hnd", 130),         # 72 rows, first keys inside a step
    ([2049, 128, 129, 255, 256, 257], 1, 8, 2, 128, "bfloat16", 16, "hnd", 0),
    ([1], 1, 2, 1, 64, "float32", 16, "nhd", 0),
    ([1000, 77], 1, 16, 8, 128, "float32", 16, "nhd", 0),
    ([300, 0, 2, 4100], 5, 8, 8, 64, "float32", 48, "hnd", 0),
    ([900, 30], 8, 32, 4, 128, "float32", 16, "nhd", 0),
    ([900, 30], 4, 16, 4, 128, "float32", 16, "hnd", 0),
    ([700, 30], 4, 32, 4, 128, "float32", 16, "hnd", 0),
    ([411], 2, 6, 2, 96, "float32", 5, "nhd", 33),
    ([260, 19], 3, 4, 2, 256, "float32", 16, "hnd", 0),
    ([260, 19], 5, 8, 2, 256, "float32", 16, "hnd", 0),
    ([50], 2, 3, 3, 32, "float32", 16, "nhd", 0),
    ([450, 60], 6, 12, 2, 64, "float32", 16, "nhd", 0),                   # 36 rows
    ([450, 60], 3, 12, 2, 64, "float32", 16, "nhd", 0),                   # 18 rows
    ([64] * 40 + [65] * 40, 1, 4, 2, 64, "bfloat16", 64, "nhd", 0),       # many short ones
    ([33000], 1, 2, 1, 128, "bfloat16", 16, "nhd", 0),                    # one long one
    ([20000, 9], 16, 32, 2, 64, "bfloat16", 16, "nhd", 0),                # 256 rows a kv head
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_rows_against_the_definition(torch, case):
    lens, Q, heads, kv, D, dtype, bs, layout, window = CASES[case]
    scales = ((1.0, 1.0), (0.25, 0.01), (3.0, 8.0))[case % 3]
    x = inputs(torch, lens, Q, heads, kv, D, dtype, bs, 200 + case, layout, apart=0 if case % 2 else 2,
               key_scale=scales[0], value_scale=scales[1])
    attend = S.Cache4Attend(len(lens), Q, heads, kv, D)
    attend.workspace.fill_(0xFF)                       # NaN wherever something is read unwritten
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    out, lse = attend(*x, window=window, error_word=err)
    check(torch, x, out, lse, some_rows(len(lens), Q, heads, case), window=window)
    assert int(err) == 0
    assert not out.isnan().any() and not lse.isnan().any()
    again, lse2 = attend(*x, window=window)
    assert torch.equal(out, again) and torch.equal(lse, lse2)   # the same bits each time


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_the_same_as_attention_over_what_is_read_back(torch, dtype):
    """cache_attend over the cache read back into one of `dtype`: each within its own tolerance of the definition."""
    lens, Q, H, kv, D, bs = [700, 33, 0, 4], 4, 8, 2, 128, 16
    q, cache, tables, n = x = inputs(torch, lens, Q, H, kv, D, dtype, bs, 77, poison=False)
    k, v = S.cache4_read(cache, torch.arange(cache.key_codes.shape[0] * bs, device="cuda"), dtype=q.dtype)
    k, v = (y.unflatten(0, (-1, bs)) for y in (k, v))
    out, lse = S.Cache4Attend(4, Q, H, kv, D)(*x)
    want, want_lse = S.CacheAttend(4, Q, H, kv, D)(q, k, v, tables, n)
    eps = torch.finfo(q.dtype).eps
    assert ((out - want).abs() <= (eps + 2.0 ** -10) * v.abs().max()).all()
    assert torch.equal(lse == -math.inf, want_lse == -math.inf)
    alive = lse != -math.inf
    assert ((lse - want_lse)[alive].abs() <= 2.0 ** -12).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lens,Q", [([0, 7, 1, 300], 8), ([0, 0], 3), ([3, 0, 2, 90, 1], 5), ([40], 1)])
def test_a_window_past_the_table_hides_nothing(torch, dtype, lens, Q):
    x = inputs(torch, lens, Q, 8, 4, 64, dtype, 16, 31)
    attend = S.Cache4Attend(len(lens), Q, 8, 4, 64)
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    want, want_lse = attend(*x)
    span = x[2].shape[1] * 16
    for window in (span, span + 1, 2 ** 30, 2 ** 31 - Q, 2 ** 31 - 1, 2 ** 40):
        out, lse = attend(*x, window=window, error_word=err)
        assert torch.equal(out, want) and torch.equal(lse, want_lse), window
    out, lse = attend(*x, window=span - 1, error_word=err)
    check(torch, x, out, lse, some_rows(len(lens), Q, 8, 3), window=span - 1)
    assert int(err) == 0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bs,n,Q,window", [(8, 155, 2, 50), (24, 400, 3, 55), (1, 60, 1, 7), (5, 90, 4, 30),
                                           (16, 200, 2, 41)])
def test_blocks_before_the_window_may_be_gone(torch, dtype, bs, n, Q, window):
    q, cache, tables, lens = x = inputs(torch, [n, 3], Q, 4, 2, 64, dtype, bs, 35)
    attend = S.Cache4Attend(2, Q, 4, 2, 64)
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    want, want_lse = attend(*x, window=window)
    first = n - Q - window + 1
    tables[0, :first // bs] = -1
    out, lse = attend(*x, window=window, error_word=err)
    assert int(err) == 0
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    check(torch, x, out, lse, some_rows(2, Q, 4, 5), window=window)
    tables[0, first // bs] = -1
    out, lse = attend(*x, window=window, error_word=err)
    assert int(err) == S.DATA_BAD_INDEX
    check(torch, x, out, lse, some_rows(2, Q, 4, 5), window=window)


def test_all_requests_empty(torch):
    x = inputs(torch, [0, 0, 0], 2, 8, 4, 64, "bfloat16", 16, 1)
    out, lse = S.Cache4Attend(3, 2, 8, 4, 64)(*x)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_scales_and_peaked_scores(torch, dtype):
    for scale, spread in ((0.0, 1.0), (1.0, 3.0), (-0.3, 1.0), (1e-3, 1.0), (2.0 ** -70, 2.0 ** 66)):
        x = inputs(torch, [700, 20], 3, 8, 4, 64, dtype, 16, 5, spread=spread)
        out, lse = S.Cache4Attend(2, 3, 8, 4, 64)(*x, scale=scale)
        check(torch, x, out, lse, some_rows(2, 3, 8, 1), scale=scale)


def test_rising_scores(torch):
    """A score that rises with every key, by less than raises the reference and by more."""
    for step in (0.05, 0.4, 3.0):
        q, cache, tables, lens = x = inputs(torch, [1500], 1, 4, 2, 64, "float32", 16, 6)
        slots = (tables[0, :94].long()[:, None] * 16 + torch.arange(16, device="cuda")).flatten()[:1500]
        k = torch.zeros(1500, 2, 64, device="cuda")
        k[..., 0] = torch.linspace(0, 1, 1500, device="cuda")[:, None] * 6
        q[..., 0] = step * 1500 / 6
        S.cache4_write(k, torch.randn(1500, 2, 64, device="cuda"), cache, slots)
        out, lse = S.Cache4Attend(1, 1, 4, 2, 64)(*x, scale=1.0)
        check(torch, x, out, lse, some_rows(1, 1, 4, 1), scale=1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_queries_of_every_size(torch, dtype):
    """Rows far apart in magnitude, elements far apart within a row, and rows of zeros."""
    q, cache, tables, lens = inputs(torch, [300, 40], 4, 8, 2, 64, dtype, 16, 15)
    q = q.clone()
    q[0, 0] *= 2.0 ** -90
    q[0, 1, :, 3] *= 2.0 ** 20
    q[0, 1] *= 2.0 ** -22
    q[0, 2] = 0
    q[1, 3] *= 2.0 ** -120
    x = (q, cache, tables, lens)
    out, lse = S.Cache4Attend(2, 4, 8, 2, 64)(*x)
    check(torch, x, out, lse, some_rows(2, 4, 8, 2, 64))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_a_later_tokens_keys_and_values_reach_no_earlier_query(torch, dtype):
    Q, n = 4, 150
    q, cache, tables, lens = x = inputs(torch, [n, 80], Q, 8, 2, 64, dtype, 16, 9)
    for back in (1, 2):                                # the last two of request 0's tokens
        at = n - back
        page = int(tables[0, at // 16])
        cache.key_scales[page, at % 16] = 0x7F
        cache.value_scales[page, at % 16] = 0xFF
    out, lse = S.Cache4Attend(2, Q, 8, 2, 64)(*x)
    rows = [(0, i, h) for i in (0, 1) for h in range(8)] + [(1, i, h) for i in range(Q) for h in range(8)]
    check(torch, x, out, lse, rows)
    assert out[0, 2:].isnan().all() and lse[0, 2:].isnan().all()
    # and with a window, values that fell out of it
    x = inputs(torch, [n, 80], Q, 8, 2, 64, dtype, 16, 10)
    for b, n_b in ((0, n), (1, 80)):
        at = n_b - Q - 20 + 1                           # the first key of query 0 alone
        x[1].value_scales[int(x[2][b, at // 16]), at % 16] = 0x7F
    out, lse = S.Cache4Attend(2, Q, 8, 2, 64)(*x, window=20)
    check(torch, x, out, lse, [(b, i, h) for b in (0, 1) for i in range(1, Q) for h in range(8)], window=20)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_nan_values_follow_the_formula(torch, dtype, D):
    """A value group that is a NaN makes those 16 elements of every query that sees it NaN, and no others."""
    Q, n = 3, 400
    x = inputs(torch, [n, 30], Q, 8, 4, D, dtype, 16, 19)
    want = torch.zeros(2, Q, 8, D, dtype=torch.bool, device="cuda")
    clean, lse = S.Cache4Attend(2, Q, 8, 4, D)(*x)
    for at, group in ((100, 1), (n - 2, D // 16 - 1)):   # seen by all queries; by the last two
        x[1].value_scales[int(x[2][0, at // 16]), at % 16, 1, group] = 0x7F
        want[0, 0 if at == 100 else 1:, 2:4, 16 * group:16 * group + 16] = True
    out, lse2 = S.Cache4Attend(2, Q, 8, 4, D)(*x)
    assert torch.equal(out.isnan(), want)
    assert torch.allclose(lse, lse2, rtol=0, atol=1e-5)
    # (rows without any are within the tolerance, the others' numbers close to what they were)
    check(torch, x, out, lse2, [(0, i, h) for i in range(Q) for h in (0, 1, 4, 7)] + [(1, 2, 3)])
    assert ((out - clean)[~want].abs() <= (torch.finfo(out.dtype).eps + 2.0 ** -10) * clean.abs().max()).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n", [90, 30000])              # one CTA's share, and joined ones
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_query_without_numbers_has_no_number(torch, dtype, n, bad):
    x = inputs(torch, [n, 0, 40], 3, 4, 2, 64, dtype, 16, 23)
    attend = S.Cache4Attend(3, 3, 4, 2, 64)
    q = x[0].clone()
    q[0, 1, 2, 5] = q[2, 0, 3, 63] = bad
    out, lse = attend(q, *x[1:])
    hit = torch.zeros(3, 3, 4, device="cuda", dtype=torch.bool)
    hit[0, 1, 2] = hit[2, 0, 3] = True
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    assert not out[~hit].isnan().any() and (lse[1] == -math.inf).all()
    check(torch, x, out, lse, [(b, i, h) for b in range(3) for i in range(3) for h in range(4) if not hit[b, i, h]])


def test_bad_data(torch):
    q, cache, tables, lens = inputs(torch, [100, 60, 40], 2, 4, 2, 64, "bfloat16", 16, 4)
    attend = S.Cache4Attend(3, 2, 4, 2, 64)
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    bad = lens.clone()
    bad[1] = -5
    out, lse = attend(q, cache, tables, bad, error_word=err)
    assert int(err) == S.DATA_BAD_LENGTH
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    check(torch, (q, cache, tables, bad), out, lse, [(0, 1, 3), (2, 0, 1)])
    err.zero_()
    t = tables.clone()
    t[0, 2], t[2, 0] = 10 ** 6, -3
    out, lse = attend(q, cache, t, lens, error_word=err)
    assert int(err) == S.DATA_BAD_INDEX
    check(torch, (q, cache, t, lens), out, lse, some_rows(3, 2, 4, 1))
    err.zero_()
    bad = lens.clone()
    bad[0] = 10 ** 9                                    # as much as its table: 9 blocks, 2 of them none
    out, lse = attend(q, cache, tables, bad, error_word=err)
    assert int(err) == S.DATA_BAD_LENGTH | S.DATA_BAD_INDEX
    check(torch, (q, cache, tables, lens), out, lse, [(1, 0, 0), (2, 1, 2)])


@pytest.mark.parametrize("layout", ["nhd", "hnd"])
def test_a_cache_past_32_bit_offsets(torch, layout):
    n, bs, H, D = 70000, 64, 8, 128
    cache = S.Cache4.zeros(n, bs, H, D)
    if layout == "nhd":
        parts = (torch.zeros(n, bs, H, w, dtype=torch.uint8, device="cuda") for w in (64, 8, 64, 8))
        cache = S.Cache4(*parts)
    assert cache.key_codes.numel() > 2 ** 31
    far = torch.tensor([[n - 1, n - 2, 1, n // 2 + 7]], device="cuda", dtype=torch.int32)
    slots = (far[0].long()[:, None] * bs + torch.arange(bs, device="cuda")).flatten()
    S.cache4_write(torch.randn(256, H, D, device="cuda"), torch.randn(256, H, D, device="cuda"), cache, slots)
    q = torch.randn(1, 2, 16, D, device="cuda").bfloat16()
    few = S.Cache4.zeros(4, bs, H, D)
    S.cache4_write(*S.cache4_read(cache, slots, dtype=torch.float32), few, torch.arange(256, device="cuda"))
    lens = torch.tensor([250], device="cuda", dtype=torch.int32)
    out, lse = S.Cache4Attend(1, 2, 16, H, D)(q, cache, far, lens)
    x = (q, few, torch.arange(4, device="cuda", dtype=torch.int32)[None], lens)
    check(torch, x, out, lse, some_rows(1, 2, 16, 3))


def test_other_streams_workspaces_and_a_graph(torch):
    """One workspace for calls of other sizes one after another, on a stream of its own, and
    replayed in a graph while the lengths change under it."""
    attend = S.Cache4Attend(8, 8, 16, 4, 128)
    big = inputs(torch, [3000, 50, 700, 1, 0, 9, 4000, 128], 8, 16, 4, 128, "bfloat16", 16, 7)
    small = inputs(torch, [90], 1, 16, 4, 128, "bfloat16", 16, 8)
    single = inputs(torch, [90, 300], 3, 16, 4, 128, "float32", 16, 8)
    want_big, want_small, want_single = attend(*big), attend(*small), attend(*single)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a, b, d, c = attend(*big), attend(*small), attend(*single), attend(*big)
    s.synchronize()
    assert torch.equal(a[0], want_big[0]) and torch.equal(b[0], want_small[0]) and torch.equal(d[0], want_single[0])
    assert torch.equal(c[0], want_big[0]) and torch.equal(c[1], want_big[1])
    out, lse = torch.empty_like(want_big[0]), torch.empty_like(want_big[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend(*big, out=out, lse=lse)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want_big[0])
    big[3].copy_(torch.tensor([10, 50, 699, 1, 0, 9, 3500, 100], device="cuda", dtype=torch.int32))
    g.replay()
    torch.cuda.synchronize()
    check(torch, big, out, lse, some_rows(8, 8, 16, 2))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("off", [1, 3])
def test_queries_and_outputs_off_the_16_byte_boundaries(torch, dtype, off):
    x = inputs(torch, [300, 20, 5000], 3, 8, 2, 64, dtype, 16, 13)
    attend = S.Cache4Attend(3, 3, 8, 2, 64)
    want, lse = attend(*x)
    room = torch.zeros(3 * 3 * (8 * 64 + 5) + off, device="cuda", dtype=x[0].dtype)
    q = room[off:].view(3, 3, 8 * 64 + 5)[..., :512].unflatten(-1, (8, 64))
    q.copy_(x[0])
    room = torch.zeros_like(room)
    out = room[off:].view(3, 3, 8 * 64 + 5)[..., :512].unflatten(-1, (8, 64))
    _, lse2 = attend(q, *x[1:], out=out)
    assert torch.equal(out, want) and torch.equal(lse, lse2)
    assert (room[:off] == 0).all() and (room[off:].view(3, 3, -1)[..., 512:] == 0).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("D", [64, 128])
def test_codes_and_scales_off_the_wide_boundaries(torch, dtype, D):
    """Codes on 16-byte boundaries but not on 32, scales on 2-byte ones: the same numbers."""
    q, cache, tables, lens = x = inputs(torch, [300, 20, 1000], 3, 8, 2, D, dtype, 16, 41)
    attend = S.Cache4Attend(3, 3, 8, 2, D)
    want, want_lse = attend(*x)

    def moved(t, room, off):
        y = torch.zeros(*t.shape[:3], t.shape[3] + room, dtype=torch.uint8, device="cuda")[..., off:off + t.shape[3]]
        y.copy_(t)
        return y

    for code_off, scale_off in ((16, 2), (0, 2), (16, 0)):
        other = S.Cache4(moved(cache.key_codes, 16, code_off), moved(cache.key_scales, 2, scale_off),
                         moved(cache.value_codes, 16, code_off), moved(cache.value_scales, 2, scale_off))
        out, lse = attend(q, other, tables, lens)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_a_step_whose_scores_are_far_from_the_first_reference(torch):
    """Rows whose scores are all far below or above what a first reference is good for, in the first steps or
    only later, for some rows of an item and not for others."""
    q, cache, tables, lens = inputs(torch, [900, 260], 4, 8, 2, 128, "bfloat16", 16, 43)
    k = torch.zeros(900, 2, 128, device="cuda")
    k[..., 0] = 6.0
    k[:, :, 1] = torch.where(torch.arange(900, device="cuda") < 640, 6.0, 0.5)[:, None]
    slots = (tables[0, :57].long()[:, None] * 16 + torch.arange(16, device="cuda")).flatten()[:900]
    S.cache4_write(k, torch.randn(900, 2, 128, device="cuda"), cache, slots)
    attend = S.Cache4Attend(2, 4, 8, 2, 128)
    for first, second in ((-20.0, 0.0), (20.0, 0.0), (0.0, -30.0), (0.0, 30.0), (-400.0, 1.0), (3.0, -4.0)):
        y = q.clone()
        y[0, 1:, :, 0], y[0, ::2, :4, 1] = first, second
        x = (y, cache, tables, lens)
        out, lse = attend(*x, scale=1.0)
        check(torch, x, out, lse, some_rows(2, 4, 8, 3, 64), scale=1.0)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_keys_far_below_a_few(torch, dtype):
    """Four keys of the first step, one of each warp's, and 32,764 whose weights are 2^-18.1 of theirs each: a
    30th of the result together, and of the only values that are not zero.  80 requests share the pages, so that a
    CTA takes most of an item's keys by itself."""
    n, B = 32768, 80
    q, cache, tables, _ = inputs(torch, [n], 1, 8, 8, 64, dtype, 16, 47)
    k, v = torch.zeros(2, n, 8, 64, device="cuda")
    few = torch.zeros(n, device="cuda", dtype=torch.bool)
    few[:128:32] = True
    k[..., 0] = 6.0
    k[~few, :, 1] = 6.0
    v[~few] = 6.0
    slots = (tables[0, :n // 16].long()[:, None] * 16 + torch.arange(16, device="cuda")).flatten()
    S.cache4_write(k, v, cache, slots)
    y = torch.zeros_like(q)
    y[..., 0], y[..., 1] = (-11.5 / 6 * math.log(2.0), -18.1 / 6 * math.log(2.0))
    x = (y.repeat(B, 1, 1, 1), cache, tables.repeat(B, 1), torch.full((B,), n, device="cuda", dtype=torch.int32))
    out, lse = S.Cache4Attend(B, 1, 8, 8, 64)(*x, scale=1.0)
    check(torch, x, out, lse, [(0, 0, 0), (41, 0, 3), (79, 0, 7)], scale=1.0)


def test_fp32_queries_with_elements_far_below_another(torch):
    """An element 2^26 times the others' size where the keys are zero: the score is the others' alone, and what is
    allowed of it (see check) goes by them.  Each request has one or two keys: lse is the score itself."""
    lens = [1, 2] * 24
    for D in (64, 128, 256):
        q, cache, tables, n = inputs(torch, lens, 2, 8, 2, D, "float32", 16, 51)
        k = torch.randn(cache.key_codes.shape[0] * 16, 2, D, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        k[..., 5] = 0.0
        S.cache4_write(k, torch.randn_like(k), cache, torch.arange(k.shape[0], device="cuda"))
        q = q.clone()
        q[..., 5] = 2.0 ** 26
        x = (q, cache, tables, n)
        out, lse = S.Cache4Attend(len(lens), 2, 8, 2, D)(*x)
        check(torch, x, out, lse, some_rows(len(lens), 2, 8, D, 80))


@pytest.mark.parametrize("heads,D", [(1, 64), (32, 128)])
def test_sums_over_a_million_keys(torch, heads, D):
    """Each request's 2^20 keys in one CTA's hands, with equal weights and positive values: what the tensor core cuts
    off its running sums all goes one way.  Tolerance: sums run over 8192 keys, 16 at a time, each cut by 2^-23 of the
    sum at most, 2^-14 in all; 128 such are added up with rounding, 2^-17; a key's weight is 2^7, exactly; two products
    at the end, 2^-22.  In all below 2^-13; the output is rounded once."""
    n, bs, B = 2 ** 20, 64, 608
    g = torch.Generator(device="cuda").manual_seed(17)
    cache = S.Cache4.zeros(n // bs, bs, 1, D)
    slots = torch.arange(n, device="cuda")
    for part in slots.split(2 ** 17):
        v = torch.rand(part.numel(), 1, D, generator=g, device="cuda") * torch.rand(part.numel(), 1, 1, generator=g, device="cuda").exp2()
        S.cache4_write(torch.zeros_like(v), v, cache, part)
    tables = torch.arange(n // bs, device="cuda", dtype=torch.int32).repeat(B, 1)
    q = torch.zeros(B, 1, heads, D, device="cuda", dtype=torch.bfloat16)
    attend = S.Cache4Attend(B, 1, heads, 1, D)
    out, lse = attend(q, cache, tables, torch.full((B,), n, device="cuda", dtype=torch.int32))
    total = torch.zeros(D, dtype=torch.float64, device="cuda")
    for part in slots.split(2 ** 17):
        total += S.cache4_read(cache, part, dtype=torch.float32)[1][:, 0].double().sum(0)
    mean = total / n
    least, most = ((mean * (1 + e)).bfloat16() for e in (-(2.0 ** -13), 2.0 ** -13))
    assert ((least <= out) & (out <= most)).all(), ((out.double() / mean - 1).mean(), (out.double() / mean - 1).abs().max())
    assert ((lse.double() - math.log(n)).abs() <= 2.0 ** -20 * 15).all()


@pytest.mark.parametrize("Q,heads,D", [(1, 8, 64), (8, 8, 128), (3, 4, 256)])
def test_references_that_rise_after_sums_were_put_by(torch, Q, heads, D):
    """Items of 157 steps in a CTA's hands whose scores rise all the way, slowly or by what raises a reference at most
    steps; and a NaN in a value that the last of them see, which makes those elements NaN and nothing else."""
    n, B = 20000, 400
    q, cache, tables, _ = inputs(torch, [n], Q, heads, 2, D, "bfloat16", 16, 53)
    slots = (tables[0, :n // 16].long()[:, None] * 16 + torch.arange(16, device="cuda")).flatten()
    k = torch.zeros(n, 2, D, device="cuda")
    k[..., 0] = torch.linspace(0, 6, n, device="cuda")[:, None]
    k[..., 1] = 6.0 * (torch.arange(n, device="cuda") % 3000 == 2999)[:, None]
    g = torch.Generator(device="cuda").manual_seed(54)
    S.cache4_write(k, torch.randn(n, 2, D, device="cuda", generator=g), cache, slots)
    attend = S.Cache4Attend(B, Q, heads, 2, D)
    tables, lens = tables.repeat(B, 1), torch.full((B,), n, device="cuda", dtype=torch.int32)
    for first, second in ((0.1, 0.0), (4.0, 0.0), (20.0, 2.0), (-3.0, 5.0)):
        y = torch.zeros_like(q)
        y[..., 0], y[..., 1] = first, second
        x = (y.repeat(B, 1, 1, 1), cache, tables, lens)
        out, lse = attend(*x, scale=1.0)
        check(torch, x, out, lse, [(0, 0, 0), (B // 2, Q - 1, heads - 1), (B - 1, Q // 2, 1)], scale=1.0)
    page = int(tables[0, (n - 1) // 16])
    cache.value_scales[page, (n - 1) % 16, 0, 1] = 0x7F
    bad, lse2 = attend(*x, scale=1.0)
    want = torch.zeros_like(bad, dtype=torch.bool)
    want[:, Q - 1, :heads // 2, 16:32] = True
    assert torch.equal(bad.isnan(), want) and torch.equal(lse, lse2)
    assert torch.equal(bad[~want], out[~want])


def test_calls_at_once_on_two_streams(torch):
    """Attention of other tiles at the same time, a workspace each: their CTAs meet on the SMs and share tensor
    memory."""
    calls = []
    for i, (lens, Q, heads, kv, D) in enumerate((([9000] * 12, 1, 32, 8, 128), ([7000, 30] * 8, 8, 32, 8, 128),
                                                 ([5000] * 20, 8, 8, 1, 256), ([3000] * 40, 4, 16, 4, 64))):
        x = inputs(torch, lens, Q, heads, kv, D, "bfloat16", 16, 60 + i)
        calls.append((S.Cache4Attend(len(lens), Q, heads, kv, D), x))
    want = [attend(*x) for attend, x in calls]
    torch.cuda.synchronize()
    streams, got, errs = [torch.cuda.Stream() for _ in calls], [[] for _ in calls], []
    for _ in range(6):
        for i, (s, (attend, x)) in enumerate(zip(streams, calls)):
            with torch.cuda.stream(s):
                errs.append(torch.zeros(1, device="cuda", dtype=torch.int32))
                got[i].append(attend(*x, error_word=errs[-1]))
    torch.cuda.synchronize()
    assert not any(int(e) for e in errs)
    for (out, lse), each in zip(want, got):
        assert all(torch.equal(a, out) and torch.equal(b, lse) for a, b in each)


def test_refusals_of_the_binding(torch):
    q, cache, tables, lens = inputs(torch, [100, 60], 2, 4, 2, 64, "bfloat16", 16, 4)
    attend = S.Cache4Attend(2, 2, 4, 2, 64)
    for bad in ((q, cache, tables.long(), lens), (q, cache, tables, lens.long()), (q, cache, tables[:1], lens),
                (q[:, :, :2], cache, tables, lens), (torch.cat([q, q]), cache, tables, lens),
                (q, S.Cache4.zeros(4, 16, 2, 128), tables, lens), (q.cpu(), cache, tables, lens)):
        with pytest.raises(ValueError):
            attend(*bad)
    with pytest.raises(TypeError):
        attend(q.half(), cache, tables, lens)
    with pytest.raises(ValueError):
        S.Cache4Attend(2, 2, 5, 2, 64)
    with pytest.raises(A.AsymSpecError):
        attend(q, cache, tables, lens, scale=math.nan)
    before = q.clone()
    with pytest.raises(A.AsymSpecError):
        attend(q, cache, tables, lens, out=q)
    assert torch.equal(q, before)
    with pytest.raises(A.AsymSpecError):
        attend(q, cache, tables, lens, out=torch.zeros(1, 2, 4, 64, device="cuda", dtype=torch.bfloat16).expand(2, 2, 4, 64))

"""cache_attend against its definition in 64 bits."""
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


def inputs(torch, lens, Q, heads, kv, D, dtype, bs, seed, layout="nhd", spread=2.0, poison=True, slack=3):
    """A pool in which every element that no query may see is NaN, tables with blocks in any
    order and indices of no block after them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = getattr(torch, dtype)
    B = len(lens)
    pages = [-(-max(n, 0) // bs) for n in lens]
    blocks = sum(pages) + slack
    width = max(pages + [1]) + 2
    ids = torch.randperm(blocks, generator=g, device="cuda").int()
    tables = torch.full((B, width + 3), -1, device="cuda", dtype=torch.int32)[:, :width]
    shape = {"nhd": (blocks, bs, kv, D), "hnd": (blocks, kv, bs, D)}[layout]
    keys = torch.randn(shape, generator=g, device="cuda").to(dt)
    values = torch.randn(shape, generator=g, device="cuda").to(dt)
    if layout == "hnd":
        keys, values = keys.transpose(1, 2), values.transpose(1, 2)
    live = torch.zeros(blocks, bs, device="cuda", dtype=torch.bool)
    at = 0
    for b, n in enumerate(lens):
        mine = ids[at:at + pages[b]]
        at += pages[b]
        tables[b, :pages[b]] = mine
        j = torch.arange(max(n, 0), device="cuda")
        live[mine.long()[j // bs], j % bs] = True
    if poison:
        keys[~live] = math.nan
        values[~live] = math.nan
    qkv = torch.randn(B, Q, (heads + 2) * D, generator=g, device="cuda").mul_(spread).to(dt)
    q = qkv[..., :heads * D].unflatten(-1, (heads, D))
    return q, keys, values, tables, torch.tensor(lens, device="cuda", dtype=torch.int32)


def check(torch, x, out, lse, rows, scale=None, window=0):
    """Tolerances.  Products of fp32 values are off by 2^-21 at most in whatever way they are
    formed, their sum of D by D 2^-24 more, of the sum of magnitudes (`spread`): a score's
    error d.  Weights are then off by 2 d + 2^-20, in two bf16 pieces by 2^-17 more, sums of
    n of them by n 2^-24 where added one after another; the output is rounded once, so the
    bounds are rounded with it."""
    from tests._serving import attended
    q, keys, values, tables, lens = x
    D, bf16 = q.shape[3], q.dtype == torch.bfloat16
    for b, i, h in rows:
        o, l, mag, spread, n = attended(q, keys, values, tables, lens, b, i, h, scale=scale, window=window)
        got, gl = out[b, i, h].double().cpu(), float(lse[b, i, h])
        if n == 0:
            assert (got == 0).all() and gl == -math.inf, (b, i, h)
            continue
        d = spread * (2.0 ** -21 + D * 2.0 ** -24)
        tol = (2 * d + 2.0 ** -20 + (2.0 ** -17 if bf16 else 0) + n * 2.0 ** -24) * mag
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
    ([1000], 1, 16, 8, 128, "bfloat16", 16, "nhd", 0),
    ([17, 0, 300, 64, 1, 2049], 1, 32, 8, 128, "bfloat16", 16, "nhd", 0),
    ([500, 3, 0, 8, 7, 4097], 8, 32, 8, 128, "bfloat16", 32, "hnd", 0),   # some shorter than Q
    ([129, 4000, 63], 8, 64, 8, 128, "bfloat16", 16, "nhd", 0),           # 64 rows a kv head
    ([777, 5], 9, 24, 3, 64, "bfloat16", 24, "nhd", 0),                   # blocks that no tile divides
    ([100, 333], 5, 8, 2, 96, "bfloat16", 7, "hnd", 0),
    ([211], 3, 6, 6, 80, "bfloat16", 1, "nhd", 0),
    ([1500, 40], 2, 4, 1, 256, "bfloat16", 16, "nhd", 0),
    ([600], 4, 12, 4, 136, "bfloat16", 48, "nhd", 0),
    ([90, 91], 2, 10, 2, 8, "bfloat16", 16, "nhd", 0),
    ([5000, 70], 5, 16, 8, 128, "bfloat16", 16, "nhd", 100),              # windows
    ([3000, 1], 1, 16, 2, 128, "bfloat16", 64, "hnd", 1),
    ([130, 2000], 8, 8, 8, 64, "bfloat16", 48, "nhd", 16),
    ([1], 1, 2, 1, 64, "float32", 16, "nhd", 0),
    ([1000, 77], 1, 16, 8, 128, "float32", 16, "nhd", 0),
    ([300, 0, 2, 4100], 5, 8, 8, 64, "float32", 48, "hnd", 0),
    ([900, 30], 8, 32, 4, 128, "float32", 16, "nhd", 0),
    ([411], 2, 6, 2, 100, "float32", 5, "nhd", 33),
    ([260, 19], 3, 4, 2, 256, "float32", 16, "hnd", 0),
    ([50], 2, 3, 3, 4, "float32", 16, "nhd", 0),
    ([64] * 40 + [65] * 40, 1, 4, 2, 64, "bfloat16", 64, "nhd", 0),       # many short ones
    ([33000], 1, 2, 1, 128, "bfloat16", 16, "nhd", 0),                    # one long one
    ([20000, 9], 16, 32, 2, 64, "bfloat16", 16, "nhd", 0),                # 256 rows a kv head
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_rows_against_the_definition(torch, case):
    lens, Q, heads, kv, D, dtype, bs, layout, window = CASES[case]
    x = inputs(torch, lens, Q, heads, kv, D, dtype, bs, 200 + case, layout)
    attend = S.CacheAttend(len(lens), Q, heads, kv, D)
    attend.workspace.fill_(0xFF)                       # NaN wherever something is read unwritten
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    out, lse = attend(*x, window=window, error_word=err)
    check(torch, x, out, lse, some_rows(len(lens), Q, heads, case), window=window)
    assert int(err) == 0
    assert not out.isnan().any() and not lse.isnan().any()
    again, lse2 = attend(*x, window=window)
    assert torch.equal(out, again) and torch.equal(lse, lse2)   # the same bits each time


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("lens,Q", [([0, 7, 1, 300], 8), ([0, 0], 3), ([3, 0, 2, 90, 1], 5), ([40], 1)])
def test_a_window_past_the_table_hides_nothing(torch, dtype, lens, Q):
    """Windows at and past what a table row holds, up to the largest number, with requests that
    have ended or are shorter than their queries: the bits of no window."""
    x = inputs(torch, lens, Q, 8, 4, 64, dtype, 16, 31)
    attend = S.CacheAttend(len(lens), Q, 8, 4, 64)
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    want, want_lse = attend(*x)
    span = x[3].shape[1] * 16
    for window in (span, span + 1, 2 ** 30, 2 ** 31 - Q, 2 ** 31 - 1):
        out, lse = attend(*x, window=window, error_word=err)
        assert torch.equal(out, want) and torch.equal(lse, want_lse), window
    check(torch, x, want, want_lse, some_rows(len(lens), Q, 8, 3))
    out, lse = attend(*x, window=span - 1, error_word=err)
    check(torch, x, out, lse, some_rows(len(lens), Q, 8, 3), window=span - 1)
    assert int(err) == 0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bs,n,Q,window", [(8, 155, 2, 50), (24, 400, 3, 55), (1, 60, 1, 7), (5, 90, 4, 30),
                                           (16, 200, 2, 41)])
def test_blocks_before_the_window_may_be_gone(torch, dtype, bs, n, Q, window):
    """What no query sees need not be in the table: no data error for it, but one for the first
    block that a query does see."""
    q, keys, values, tables, lens = x = inputs(torch, [n, 3], Q, 4, 2, 64, dtype, bs, 35)
    attend = S.CacheAttend(2, Q, 4, 2, 64)
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
    out, lse = S.CacheAttend(3, 2, 8, 4, 64)(*x)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_scales_and_peaked_scores(torch, dtype):
    for scale, spread in ((0.0, 1.0), (1.0, 3.0), (-0.3, 1.0)):
        x = inputs(torch, [700, 20], 3, 8, 4, 64, dtype, 16, 5, spread=spread)
        out, lse = S.CacheAttend(2, 3, 8, 4, 64)(*x, scale=scale)
        check(torch, x, out, lse, some_rows(2, 3, 8, 1), scale=scale)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_later_tokens_keys_and_values_reach_no_earlier_query(torch, dtype, bad):
    Q, n = 4, 150
    q, keys, values, tables, lens = inputs(torch, [n, 80], Q, 8, 2, 64, dtype, 16, 9)
    for back in (1, 2):                                # the last two of request 0's tokens
        at = n - back
        page = int(tables[0, at // 16])
        keys[page, at % 16] = bad
        values[page, at % 16] = bad
    x = (q, keys, values, tables, lens)
    out, lse = S.CacheAttend(2, Q, 8, 2, 64)(*x)
    rows = [(0, i, h) for i in (0, 1) for h in range(8)] + [(1, i, h) for i in range(Q) for h in range(8)]
    check(torch, x, out, lse, rows)
    # and with a window, keys that fell out of it
    x = inputs(torch, [n, 80], Q, 8, 2, 64, dtype, 16, 10)
    for b, n_b in ((0, n), (1, 80)):
        at = n_b - Q - 20 + 1                           # the first key of query 0 alone
        page = int(x[3][b, at // 16])
        x[2][page, at % 16] = bad
    out, lse = S.CacheAttend(2, Q, 8, 2, 64)(*x, window=20)
    check(torch, x, out, lse, [(b, i, h) for b in (0, 1) for i in range(1, Q) for h in range(8)], window=20)


def test_infinite_scores_follow_the_formula(torch):
    q, keys, values, tables, lens = x = inputs(torch, [100], 1, 2, 1, 64, "float32", 16, 3)
    page = int(tables[0, 1])
    keys[page, 3] = -math.inf * q[0, 0, 0].sign()       # head 0: a score of -infinity at key 19
    out, lse = S.CacheAttend(1, 1, 2, 1, 64)(*x)
    check(torch, x, out, lse, [(0, 0, 0)])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_infinite_values_follow_the_formula(torch, dtype):
    """A value of +infinity makes that element of every query that sees it +infinity, and no other."""
    Q, n = 3, 400
    x = inputs(torch, [n, 30], Q, 8, 4, 64, dtype, 16, 19)
    want, lse = S.CacheAttend(2, Q, 8, 4, 64)(*x)
    for at in (100, n - 2):                             # seen by all queries; by the last two
        x[2][int(x[3][0, at // 16]), at % 16, 1, 5] = math.inf
        want[0, 0 if at == 100 else 1:, 2:4, 5] = math.inf
    out, lse2 = S.CacheAttend(2, Q, 8, 4, 64)(*x)
    assert torch.equal(lse, lse2) or torch.allclose(lse, lse2, rtol=0, atol=1e-5)
    finite = want.isfinite()
    assert torch.equal(out.isfinite(), finite) and (out[~finite] == math.inf).all()
    check(torch, x, out, lse2, [(0, i, h) for i in range(Q) for h in (0, 1, 4, 7)] + [(1, 2, 3)])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n", [90, 30000])              # one CTA's share, and joined ones
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_query_without_numbers_has_no_number(torch, dtype, n, bad):
    """A NaN in a query makes its out and lse NaN, not -infinity, which says that it has no keys; so
    does an infinity, whose scores are infinities of both signs."""
    x = inputs(torch, [n, 0, 40], 3, 4, 2, 64, dtype, 16, 23)
    attend = S.CacheAttend(3, 3, 4, 2, 64)
    q = x[0].clone()
    q[0, 1, 2, 5] = q[2, 0, 3, 63] = bad
    out, lse = attend(q, *x[1:])
    hit = torch.zeros(3, 3, 4, device="cuda", dtype=torch.bool)
    hit[0, 1, 2] = hit[2, 0, 3] = True
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    assert not out[~hit].isnan().any() and (lse[1] == -math.inf).all()
    check(torch, x, out, lse, [(b, i, h) for b in range(3) for i in range(3) for h in range(4) if not hit[b, i, h]])


def test_bad_data(torch):
    q, keys, values, tables, lens = inputs(torch, [100, 60, 40], 2, 4, 2, 64, "bfloat16", 16, 4)
    attend = S.CacheAttend(3, 2, 4, 2, 64)
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    bad = lens.clone()
    bad[1] = -5
    out, lse = attend(q, keys, values, tables, bad, error_word=err)
    assert int(err) == S.DATA_BAD_LENGTH
    assert (out[1] == 0).all() and (lse[1] == -math.inf).all()
    check(torch, (q, keys, values, tables, bad), out, lse, [(0, 1, 3), (2, 0, 1)])
    err.zero_()
    t = tables.clone()
    t[0, 2], t[2, 0] = 10 ** 6, -3
    out, lse = attend(q, keys, values, t, lens, error_word=err)
    assert int(err) == S.DATA_BAD_INDEX
    check(torch, (q, keys, values, t, lens), out, lse, some_rows(3, 2, 4, 1))
    err.zero_()
    bad = lens.clone()
    bad[0] = 10 ** 9                                    # as much as its table: 9 blocks, 2 of them none
    out, lse = attend(q, keys, values, tables, bad, error_word=err)
    assert int(err) == S.DATA_BAD_LENGTH | S.DATA_BAD_INDEX
    check(torch, (q, keys, values, tables, lens), out, lse, [(1, 0, 0), (2, 1, 2)])


def test_a_cache_past_32_bit_offsets(torch):
    n, bs, H, D = 41000, 64, 8, 128
    keys = torch.zeros(n, bs, H, D, device="cuda", dtype=torch.bfloat16)
    assert keys.numel() * 2 > 2 ** 32
    far = torch.tensor([[n - 1, n - 2, 1, n // 2 + 7]], device="cuda", dtype=torch.int32)
    keys[far[0].long()] = torch.randn(4, bs, H, D, device="cuda").bfloat16()
    q = torch.randn(1, 2, 16, D, device="cuda").bfloat16()
    x = (q, keys, keys, far, torch.tensor([250], device="cuda", dtype=torch.int32))
    out, lse = S.CacheAttend(1, 2, 16, H, D)(*x)
    check(torch, x, out, lse, some_rows(1, 2, 16, 3))


def test_other_streams_workspaces_and_a_graph(torch):
    """One workspace for calls of other sizes one after another, on a stream of its own, and
    replayed in a graph while the lengths change under it."""
    attend = S.CacheAttend(8, 8, 16, 4, 128)
    big = inputs(torch, [3000, 50, 700, 1, 0, 9, 4000, 128], 8, 16, 4, 128, "bfloat16", 16, 7)
    small = inputs(torch, [90], 1, 16, 4, 128, "bfloat16", 16, 8)
    want_big, want_small = attend(*big), attend(*small)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a, b, c = attend(*big), attend(*small), attend(*big)
    s.synchronize()
    assert torch.equal(a[0], want_big[0]) and torch.equal(b[0], want_small[0])
    assert torch.equal(c[0], want_big[0]) and torch.equal(c[1], want_big[1])
    out, lse = torch.empty_like(want_big[0]), torch.empty_like(want_big[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend(*big, out=out, lse=lse)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want_big[0])
    big[4].copy_(torch.tensor([10, 50, 699, 1, 0, 9, 3500, 100], device="cuda", dtype=torch.int32))
    g.replay()
    torch.cuda.synchronize()
    check(torch, big, out, lse, some_rows(8, 8, 16, 2))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("off", [1, 3])
def test_queries_and_outputs_off_the_16_byte_boundaries(torch, dtype, off):
    x = inputs(torch, [300, 20, 5000], 3, 8, 2, 64, dtype, 16, 13)
    attend = S.CacheAttend(3, 3, 8, 2, 64)
    want, lse = attend(*x)
    room = torch.zeros(3 * 3 * (8 * 64 + 5) + off, device="cuda", dtype=x[0].dtype)
    q = room[off:].view(3, 3, 8 * 64 + 5)[..., :512].unflatten(-1, (8, 64))
    q.copy_(x[0])
    room = torch.zeros_like(room)
    out = room[off:].view(3, 3, 8 * 64 + 5)[..., :512].unflatten(-1, (8, 64))
    _, lse2 = attend(q, *x[1:], out=out)
    assert torch.equal(out, want) and torch.equal(lse, lse2)
    assert (room[:off] == 0).all() and (room[off:].view(3, 3, -1)[..., 512:] == 0).all()


def test_strided_outputs(torch):
    x = inputs(torch, [300, 20], 3, 8, 2, 64, "bfloat16", 16, 12)
    attend = S.CacheAttend(2, 3, 8, 2, 64)
    want, _ = attend(*x)
    room = torch.zeros(2, 8, 3, 65, device="cuda", dtype=torch.bfloat16)
    out = room[..., 1:].transpose(1, 2)
    attend(*x, out=out)
    assert torch.equal(out, want) and (room[..., 0] == 0).all()


def test_refusals_of_the_binding(torch):
    q, keys, values, tables, lens = inputs(torch, [100, 60], 2, 4, 2, 64, "bfloat16", 16, 4)
    attend = S.CacheAttend(2, 2, 4, 2, 64)
    for bad in ((q.float(), keys, values, tables, lens), (q, keys, values.float(), tables, lens),
                (q, keys, values[:, :8], tables, lens), (q, keys, values, tables.long(), lens),
                (q, keys, values, tables, lens.long()), (q, keys, values, tables[:1], lens),
                (q[:, :, :2], keys, values, tables, lens), (q, keys.cpu(), values.cpu(), tables, lens),
                (torch.cat([q, q]), keys, values, tables, lens)):
        with pytest.raises(ValueError):
            attend(*bad)
    with pytest.raises(ValueError):
        S.CacheAttend(2, 2, 5, 2, 64)
    with pytest.raises(A.AsymSpecError):
        attend(q, keys, values, tables, lens, scale=math.nan)
    with pytest.raises(A.AsymSpecError):               # rows off the 16-byte boundaries
        room = torch.zeros(keys.numel() + 1, device="cuda", dtype=torch.bfloat16)
        attend(q, room[1:].view(keys.shape), values, tables, lens)


def test_attention_in_place_is_refused(torch):
    q, keys, values, tables, lens = inputs(torch, [100, 60], 2, 4, 2, 64, "bfloat16", 16, 4)
    attend = S.CacheAttend(2, 2, 4, 2, 64)
    before = q.clone()
    with pytest.raises(A.AsymSpecError):
        attend(q, keys, values, tables, lens, out=q)
    assert torch.equal(q, before)


def test_an_expanded_output_is_refused(torch):
    x = inputs(torch, [100, 60], 2, 4, 2, 64, "bfloat16", 16, 4)
    attend = S.CacheAttend(2, 2, 4, 2, 64)
    for shape in ((1, 2, 4, 64), (2, 1, 4, 64), (2, 2, 1, 64)):
        with pytest.raises(A.AsymSpecError):
            attend(*x, out=torch.zeros(shape, device="cuda", dtype=torch.bfloat16).expand(2, 2, 4, 64))
    one = inputs(torch, [100], 1, 4, 2, 64, "bfloat16", 16, 5)
    out = torch.zeros(1, 4, 64, device="cuda", dtype=torch.bfloat16)[None].expand(1, 1, 4, 64)
    assert torch.equal(attend(*one, out=out)[0], attend(*one)[0])

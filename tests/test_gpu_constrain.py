"""constrain_logits against its definition in 64 bits."""
import math

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


def inputs(torch, B, P, V, dtype, N, seed, pad=0, masks=None, biased=7, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    base = torch.randn(B * P * (V + pad) + offset, generator=g, device="cuda").mul_(6).to(dtype)
    z = base[offset:].view(B, P, V + pad)[..., :V]
    i32 = dict(generator=g, device="cuda", dtype=torch.int32)
    x = dict(history=torch.randint(0, max(2, V // 7), (B, N), **i32) if N else None,
             drafts=torch.randint(0, max(2, V // 7), (B, P - 1), **i32) if P > 1 else None)
    if N:
        x["history_len"] = torch.randint(0, N + 1, (B,), **i32)
        x["prompt_len"] = (x["history_len"] * torch.rand(B, generator=g, device="cuda")).int()
    r = torch.rand(3, B, generator=g, device="cuda")
    x.update(repetition=0.7 + r[0], frequency=2 * r[1] - 0.5, presence=2 * r[2] - 0.5)
    if biased:
        x["bias"] = (torch.arange(0, B * biased + 1, biased, device="cuda", dtype=torch.int32),
                     torch.randint(0, V, (B * biased,), **i32),
                     8 * torch.randn(B * biased, generator=g, device="cuda"))
    if masks is not None:
        x["mask"] = torch.randint(-2 ** 31, 2 ** 31 - 1, (masks, (V + 31) // 32), **i32)
        x["mask_rows"] = torch.randint(-1, masks, (B, P), **i32)
    return z, x


def check(torch, z, x, y, rows=None):
    """Every entry within the roundings that its definition has in fp32 (four operations, each
    2^-24 of what enters it), those bounds rounded to the type as the result is."""
    B, P, V = z.shape
    from tests._serving import constrained
    for b in range(B):
        for k in range(P):
            if rows is not None and (b, k) not in rows:
                continue
            want, mag = constrained(z, b, k, **x)
            got = y[b, k].double().cpu()
            tol = 4 * 2.0 ** -24 * mag
            least, most = ((want + t).to(z.dtype).double() for t in (-tol, tol))
            bad = ~((got == want) | (got.isnan() & want.isnan()) | ((least <= got) & (got <= most)))
            assert not bad.any(), (b, k, bad.nonzero()[:5].tolist(), got[bad][:5], want[bad][:5])


CASES = [
    # B, P, V, dtype, history, pad, masks, biases, elements off the allocation's start
    (1, 5, 32000, "float32", 700, 0, None, 8, 0),
    (3, 8, 4096, "bfloat16", 900, 0, 9, 5, 0),
    (2, 9, 4099, "bfloat16", 300, 0, 5, 40, 0),      # rows at odd addresses
    (2, 2, 8193, "float32", 50, 3, 3, 0, 1),         # one entry in a last slice, rows apart, unaligned
    (5, 1, 1000, "bfloat16", 1, 24, 2, 1, 3),
    (1, 1, 2, "float32", 3, 0, 1, 1, 0),             # the smallest vocabulary
    (2, 3, 33, "bfloat16", 64, 31, 4, 2, 0),         # a mask that ends inside a word
    (3, 4, 12345, "float32", 0, 0, None, 0, 0),      # drafts alone
    (2, 256, 97, "bfloat16", 20, 0, 6, 3, 0),        # the most positions
    (2, 4, 40000, "bfloat16", 20000, 0, 2, 3, 0),    # a long history
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_rows_against_the_definition(torch, case):
    B, P, V, dtype, N, pad, masks, biased, offset = CASES[case]
    z, x = inputs(torch, B, P, V, getattr(torch, dtype), N, 100 + case, pad, masks, biased, offset)
    before = z.clone()
    y = S.constrain_logits(z, **x)
    assert torch.equal(z, before)
    rows = {(b, k) for b in (0, B - 1) for k in (0, 1, P // 2, P - 1)} if P > 20 else None
    check(torch, z, x, y, rows)


@pytest.mark.parametrize("name", ["repetition", "frequency", "presence", "bias", "mask", "drafts", "history"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_each_group_alone(torch, name, dtype):
    z, x = inputs(torch, 2, 4, 5001, getattr(torch, dtype), 400, 7, 0, 3, 6)
    groups = {"mask": ("mask", "mask_rows"), "bias": ("bias",), "drafts": ("drafts", "presence"),
              "history": ("history", "history_len", "prompt_len")}
    counted = ("repetition", "frequency", "presence")
    keep = groups.get(name, (name,) + groups["history"] if name in counted else (name,))
    x = {k: v for k, v in x.items() if k in keep}
    y = S.constrain_logits(z, **x)
    check(torch, z, x, y)
    if name == "history":  # nothing is penalised: the rows come back bit for bit
        assert torch.equal(y, z)


def test_nothing_at_all_copies_every_bit(torch):
    z = torch.randn(2, 3, 777, device="cuda", dtype=torch.bfloat16)
    z[0, 0, 5], z[1, 2, 0], z[0, 1, 7] = math.nan, math.inf, -0.0
    y = S.constrain_logits(z)
    assert torch.equal(y.view(torch.int16), z.view(torch.int16))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [4096, 4097])
def test_in_place(torch, dtype, V):
    z, x = inputs(torch, 3, 5, V, getattr(torch, dtype), 300, 8, 5, 4, 9)
    want = S.constrain_logits(z, **x)
    assert S.constrain_logits(z, out=z, **x) is z
    assert torch.equal(z, want)


def test_extremes_stay_finite_and_masks_replace_anything(torch):
    low = torch.finfo(torch.bfloat16).min
    V = 64
    z = torch.full((1, 2, V), 1.0, device="cuda", dtype=torch.bfloat16)
    z[..., 0], z[..., 1], z[..., 2], z[..., 3], z[..., 4] = low, -low, math.nan, math.inf, -math.inf
    z[..., 8:13] = z[..., :5]
    mask = torch.tensor([[-1 & ~0x1F00, -1]], device="cuda", dtype=torch.int32)  # 8..12 not allowed
    i32 = dict(device="cuda", dtype=torch.int32)
    x = dict(history=torch.arange(16, **i32)[None], history_len=torch.tensor([16], **i32),
             repetition=torch.tensor([1.5], device="cuda"), frequency=torch.tensor([3.0], device="cuda"),
             bias=(torch.tensor([0, 2], **i32), torch.tensor([0, 1], **i32),
                   torch.tensor([-3e38, 3e38], device="cuda")),
             mask=mask, mask_rows=torch.tensor([[0, -1]], **i32))
    y = S.constrain_logits(z, **x)
    check(torch, z, x, y)
    y = y.float().cpu()
    assert y[0, 0, 0] == low and y[0, 0, 1] == -low
    assert y[0, 0, 2].isnan() and y[0, 0, 3] == math.inf and y[0, 0, 4] == -math.inf
    assert (y[0, 0, 8:13] == low).all() and y[0, 1, 10].isnan()


@pytest.mark.parametrize("value,want", [(None, None), (-1e4, -9984.0), (0.0, 0.0), (-3.4e38, None)])
def test_mask_values_and_rows_that_allow_nothing(torch, value, want):
    z = torch.randn(2, 2, 100, device="cuda", dtype=torch.bfloat16)
    mask = torch.zeros(4, 4, device="cuda", dtype=torch.int32)
    mask[1:3] = -1
    y = S.constrain_logits(z, mask=mask, mask_value=value)
    want = torch.finfo(torch.bfloat16).min if want is None else want
    assert (y[0, 0] == want).all() and (y[1, 1] == want).all()
    assert torch.equal(y[0, 1], z[0, 1]) and torch.equal(y[1, 0], z[1, 0])


def test_the_last_bias_of_a_token_counts(torch):
    i32 = dict(device="cuda", dtype=torch.int32)
    z = torch.zeros(1, 1, 6000, device="cuda")
    tokens = torch.tensor([5, 5999, 5, 7, 5, 5999], **i32)
    values = torch.tensor([1.0, 2.0, 3.0, 4.0, 5.0, 6.0], device="cuda")
    y = S.constrain_logits(z, bias=(torch.tensor([0, 6], **i32), tokens, values)).cpu()
    assert y[0, 0, 5] == 5 and y[0, 0, 7] == 4 and y[0, 0, 5999] == 6 and y.sum() == 15


def test_more_biases_than_a_slice_holds(torch):
    i32 = dict(device="cuda", dtype=torch.int32)
    g = torch.Generator(device="cuda").manual_seed(77)
    z = torch.randn(2, 3, 1500, generator=g, device="cuda")
    tokens = torch.randint(0, 1500, (3000,), generator=g, **i32)
    x = dict(bias=(torch.tensor([0, 2900, 3000], **i32), tokens, torch.randn(3000, generator=g, device="cuda")))
    check(torch, z, x, S.constrain_logits(z, **x))


@pytest.mark.parametrize("B", [2, 33, 64, 65])
@pytest.mark.parametrize("in_place", [False, True])
def test_long_histories_of_many_lengths(torch, B, in_place):
    """Where histories may be long, some CTAs take the requests in the order of their lengths:
    none is left out or done twice, with equal lengths, empty ones and ones out of range."""
    V, P, N = 9001, 2, 16385
    z, x = inputs(torch, B, P, V, torch.float32, N, B, 0, None, 3)
    some = [0, N, 255, 256, 257, N, 4000, 0]
    x["history_len"][:min(B, 8)] = torch.tensor(some[:min(B, 8)], dtype=torch.int32)
    x["prompt_len"] = x["history_len"] // 3
    sound = x["history_len"].clone()
    x["history_len"][B - 1] = N + 5 if B % 2 else -3
    sound[B - 1] = N if B % 2 else 0
    x["prompt_len"][B - 1] = 0
    error = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = S.constrain_logits(z.clone(), **x, error_word=error) if not in_place else None
    if in_place:
        y = z.clone()
        S.constrain_logits(y, **x, out=y, error_word=error)
    assert int(error) == S.DATA_BAD_LENGTH
    check(torch, z, dict(x, history_len=sound), y, {(b, b % 2) for b in range(B)})


def test_bad_data_sets_bits_and_leaves_the_rest(torch):
    i32 = dict(device="cuda", dtype=torch.int32)
    z, x = inputs(torch, 2, 3, 500, torch.float32, 40, 21, 0, None, 0)

    def run(**change):
        err = torch.zeros(1, **i32)
        v = dict(x, **change)
        y = S.constrain_logits(z, error_word=err, **v)
        check(torch, z, v, y)
        return int(err)

    assert run() == 0
    h = x["history"].clone()
    h[0, 0], h[1, 1] = -1, 500
    full = torch.tensor([40, 40], **i32)
    assert run(history=h, history_len=full) == A.DATA_BAD_TOKEN
    d = x["drafts"].clone()
    d[1, 1] = 1 << 30
    assert run(drafts=d) == A.DATA_BAD_TOKEN
    assert run(history_len=torch.tensor([41, -3], **i32)) == S.DATA_BAD_LENGTH
    assert run(history_len=full, prompt_len=torch.tensor([-1, 41], **i32)) == S.DATA_BAD_LENGTH
    for rep in (0.0, -1.0, math.inf, math.nan):
        assert run(repetition=torch.tensor([1.2, rep], device="cuda")) == S.DATA_BAD_PENALTY
    assert run(presence=torch.tensor([math.nan, 1.0], device="cuda")) == S.DATA_BAD_PENALTY
    assert run(mask=torch.full((2, 16), -1, **i32),
               mask_rows=torch.tensor([[0, 1, -1], [2, -2, 0]], **i32)) == S.DATA_BAD_INDEX
    offsets, tokens = torch.tensor([-1, 1, 9], **i32), torch.tensor([3, 500], **i32)
    assert run(bias=(offsets, tokens, torch.ones(2, device="cuda"))) \
        == S.DATA_BAD_LENGTH | A.DATA_BAD_TOKEN


def test_another_stream_and_a_graph(torch):
    z, x = inputs(torch, 4, 8, 20000, torch.bfloat16, 2000, 31, 0, 6, 3)
    want = S.constrain_logits(z, **x)
    out = torch.empty_like(want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        S.constrain_logits(z, out=out, **x)
    s.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.constrain_logits(z, out=out, **x)
    for _ in range(3):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_refusals_of_the_binding(torch):
    z = torch.zeros(2, 3, 64, device="cuda")
    i32 = dict(device="cuda", dtype=torch.int32)
    for bad in (dict(history=torch.zeros(2, 4, **i32)), dict(history=torch.zeros(3, 4, **i32)),
                dict(drafts=torch.zeros(2, 1, **i32)), dict(drafts=torch.zeros(2, 2, device="cuda")),
                dict(presence=torch.zeros(3, device="cuda")), dict(mask=torch.zeros(6, 1, **i32)),
                dict(mask_rows=torch.zeros(2, 3, **i32)), dict(out=torch.zeros(2, 3, 65, device="cuda")),
                dict(repetition=torch.ones(2))):
        with pytest.raises(ValueError):
            S.constrain_logits(z, **bad)
    with pytest.raises(ValueError):
        S.constrain_logits(z.cpu())
    with pytest.raises(TypeError):
        S.constrain_logits(z.half())
    with pytest.raises(A.AsymSpecError):
        S.constrain_logits(z, mask=torch.zeros(5, 2, **i32))


def test_a_history_and_drafts_that_requests_share(torch):
    z, x = inputs(torch, 4, 3, 1500, torch.float32, 400, 41)
    x["history"], x["drafts"] = x["history"][:1].expand(4, 400), x["drafts"][1:2].expand(4, 2)
    error = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = S.constrain_logits(z, **x, error_word=error)
    assert int(error) == 0
    check(torch, z, x, y)
    with pytest.raises(ValueError):
        S.constrain_logits(z[:1, :1].expand(4, 3, 1500), **x)
    with pytest.raises(ValueError):
        S.constrain_logits(z, **x, out=z[:1].expand(4, 3, 1500))


def test_groups_that_are_empty_this_round(torch):
    """A history without room for a token and a mask tensor without a row are groups like others:
    nothing is said, no position has a grammar, and what goes past them is a data error."""
    i32 = dict(device="cuda", dtype=torch.int32)
    z, x = inputs(torch, 2, 3, 500, torch.float32, 40, 43, 0, None, 4)
    x.update(history=torch.zeros(2, 0, **i32), history_len=torch.zeros(2, **i32), prompt_len=torch.zeros(2, **i32),
             mask=torch.zeros(0, 16, **i32), mask_rows=torch.full((2, 3), -1, **i32))
    err = torch.zeros(1, **i32)
    y = S.constrain_logits(z, **x, error_word=err)
    assert int(err) == 0
    check(torch, z, x, y)
    x["history_len"][1], x["mask_rows"][0, 2] = 1, 0
    y = S.constrain_logits(z, **x, error_word=err)
    assert int(err) == S.DATA_BAD_LENGTH | S.DATA_BAD_INDEX
    check(torch, z, x, y)
    into = z.clone()
    S.constrain_logits(into, **x, out=into)
    assert torch.equal(into, y)
    with pytest.raises(ValueError):
        S.constrain_logits(z, mask=x["mask"])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("in_place", [False, True])
def test_biases_that_are_not_numbers(torch, dtype, in_place):
    """A NaN among the biases makes that entry NaN (it is neither kept nor taken for the lowest
    value); an infinite one stops at the type's range, also for a token that is penalised."""
    i32 = dict(device="cuda", dtype=torch.int32)
    z = torch.randn(1, 3, 3000, device="cuda").to(getattr(torch, dtype))
    x = dict(history=torch.tensor([[5, 2900, 7]], **i32), history_len=torch.tensor([3], **i32),
             repetition=torch.tensor([1.5], device="cuda"), presence=torch.tensor([0.5], device="cuda"),
             bias=(torch.tensor([0, 5], **i32), torch.tensor([5, 9, 7, 2999, 11], **i32),
                   torch.tensor([math.nan, math.nan, math.inf, -math.inf, 2.0], device="cuda")))
    z0 = z.clone()
    y = S.constrain_logits(z, out=z if in_place else None, **x)
    check(torch, z0, x, y)
    nan = y.isnan().nonzero()[:, 2].tolist()
    assert nan == [5, 9] * 3
    top = torch.finfo(z.dtype).max
    assert (y[..., 7] == top).all() and (y[..., 2999] == -top).all()


@pytest.mark.parametrize("B,P,V,dtype,pad", [(2, 2, 9001, "bfloat16", 0), (1, 13, 5000, "float32", 3),
                                             (2, 1, 20000, "float32", 0), (1, 40, 2560, "bfloat16", 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_biases_for_all_tokens(torch, B, P, V, dtype, pad, in_place):
    """Biases for every token, most of them several times, beside the other constraints: the last
    entry of each counts, in each batch of rows."""
    i32 = dict(device="cuda", dtype=torch.int32)
    z, x = inputs(torch, B, P, V, getattr(torch, dtype), 600, 51, pad, None if in_place else 3, 0)
    g = torch.Generator(device="cuda").manual_seed(52)
    tokens = torch.cat([torch.randint(-3, V + 3, (2 * V,), generator=g, **i32), torch.randperm(V, generator=g, **i32),
                        torch.randint(0, V, (V // 3,), generator=g, **i32)])
    m = tokens.numel()
    x["bias"] = (torch.tensor([0, m, m + 5][:B + 1], **i32), torch.cat([tokens, tokens[-5:]]),
                 torch.randn(m + 5, generator=g, device="cuda"))
    z0, err = z.clone(), torch.zeros(1, **i32)
    y = S.constrain_logits(z, out=z if in_place else None, error_word=err, **x)
    assert int(err) == A.DATA_BAD_TOKEN
    check(torch, z0, x, y, {(b, k) for b in range(B) for k in (0, P // 2, P - 1)})


def test_many_biases_take_no_square_of_their_number(torch):
    """Sixteen times the biases take at most 64 times as long (a search of the list for each token
    takes 256 times as long)."""
    B, V = 64, 128256
    z = torch.randn(B, 1, V, device="cuda").bfloat16()
    out = torch.empty_like(z)

    def us(m):
        off = torch.arange(0, B * m + 1, m, device="cuda", dtype=torch.int32)
        tok = (torch.arange(m, device="cuda", dtype=torch.int32) * (V // m)).repeat(B)
        val = torch.randn(B * m, device="cuda")
        best = math.inf
        for _ in range(3):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            S.constrain_logits(z, bias=(off, tok, val), out=out)
            end.record()
            end.synchronize()
            best = min(best, begin.elapsed_time(end) * 1e3)
        return best

    few, all_ = us(V // 16), us(V)
    assert all_ < 64 * few, (few, all_)

"""Writing and reading a cache in 4 bits against its definition."""
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


def pool(torch, blocks, bs, kv, D, layout="hnd", fill=0xA5, **k):
    """A cache whose every byte is `fill`, scales apart by more than they are long."""
    shape = (blocks, kv, bs) if layout == "hnd" else (blocks, bs, kv)
    parts = [torch.full((*shape, w), fill, dtype=torch.uint8, device="cuda") for w in (D // 2, D // 16 + 2) * 2]
    parts = [x[..., :w] for x, w in zip(parts, (D // 2, D // 16) * 2)]
    if layout == "hnd":
        parts = [x.transpose(1, 2) for x in parts]
    return S.Cache4(*parts, **k)


def at(cache, slots):
    bs = cache.key_codes.shape[1]
    page, i = slots // bs, slots % bs
    return [x[page, i] for x in (cache.key_codes, cache.key_scales, cache.value_codes, cache.value_scales)]


CASES = [
    # T, kv heads, D, block, layout, dtype, key_scale, value_scale
    (1, 1, 32, 1, "hnd", "bfloat16", 1.0, 1.0),
    (3, 2, 64, 16, "hnd", "bfloat16", 1.0, 0.25),
    (130, 8, 128, 16, "nhd", "bfloat16", 0.03, 5.0),
    (57, 3, 96, 7, "nhd", "float32", 1.0, 2.0 ** -20),
    (40, 1, 160, 24, "hnd", "float32", 0.7, 1.0),
    (9, 5, 256, 64, "nhd", "bfloat16", 2.0 ** -60, 2.0 ** 60),
    (2000, 4, 128, 32, "hnd", "float32", 1.0, 1.0),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_written_and_read(torch, case):
    """Codes and scales bit for bit; what is read back is what they stand for, rounded once, or twice to
    bf16; everything else is left alone."""
    from tests._cache4 import values, written
    T, kv, D, bs, layout, dtype, ks, vs = CASES[case]
    g = torch.Generator(device="cuda").manual_seed(60 + case)
    blocks = -(-T // bs) + 3
    cache = pool(torch, blocks, bs, kv, D, layout, key_scale=ks, value_scale=vs)
    kv_in = torch.randn(T, 2, kv, D, generator=g, device="cuda") * torch.randn(T, 2, kv, D, generator=g, device="cuda").mul(2).exp()
    kv_in[:, 0] *= ks
    kv_in[:, 1] *= vs
    kv_in = kv_in.to(getattr(torch, dtype))
    k, v = kv_in[:, 0], kv_in[:, 1]
    slots = torch.randperm(blocks * bs, generator=g, device="cuda")[:T]
    if T > 2:
        slots[1] = -1
    live = slots >= 0
    before = [x.clone() for x in (cache.key_codes, cache.key_scales, cache.value_codes, cache.value_scales)]
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    S.cache4_write(k, v, cache, slots, error_word=err)
    assert int(err) == 0
    got = at(cache, slots[live])
    for x, scale, codes, scales in ((k, ks, got[0], got[1]), (v, vs, got[2], got[3])):
        want_codes, want_scales = written(x[live], scale)
        assert torch.equal(scales.cpu(), want_scales)
        assert torch.equal(codes.cpu(), want_codes)
    page, i = slots[live] // bs, slots[live] % bs
    for x, old in zip((cache.key_codes, cache.key_scales, cache.value_codes, cache.value_scales), before):
        old[page, i] = x[page, i]
        assert torch.equal(x, old)
    for out_type in (torch.float32, torch.bfloat16):
        a, b = S.cache4_read(cache, slots, dtype=out_type)
        for y, scale, codes, scales in ((a, ks, got[0], got[1]), (b, vs, got[2], got[3])):
            assert torch.equal(y[live], values(codes, scales, scale).float().to(out_type))
            assert (y[~live] == 0).all()


def test_every_code_and_scale(torch):
    """All 256 bytes of codes under all 256 scales."""
    from tests._cache4 import values
    c = torch.arange(256, device="cuda", dtype=torch.uint8)
    codes = c.view(8, 1, 1, 32).expand(8, 256, 1, 32).contiguous()       # a block per eighth, a token per scale
    scales = c.view(1, 256, 1, 1).expand(8, 256, 1, 4).contiguous()
    cache = S.Cache4(codes, scales, codes, scales, key_scale=1.0, value_scale=0.3)
    k, v = S.cache4_read(cache, torch.arange(8 * 256, device="cuda"), dtype=torch.float32)
    for x, scale in ((k, 1.0), (v, 0.3)):
        want = values(codes, scales, scale).float().view(2048, 1, 64)
        assert torch.equal(x.isnan(), want.isnan()) and torch.equal(x.nan_to_num(0.0), want.nan_to_num(0.0))


def test_edges_of_the_types(torch):
    """Halfway values, zeros of both signs, values too small and too large, infinities and NaN."""
    from tests._cache4 import values, written
    rows = []
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    rows.append(ties + [-x for x in ties] + [6.0, -0.0])                 # under a scale of 1
    rows.append([0.0, -0.0] * 8)
    rows.append([6.0 * 2.0 ** -10 * f for f in (1.0, 1.0001, 0.9999, -0.5)] + [0.0] * 12)   # the smallest scale's half
    rows.append([6.0 * 2.0 ** -9 * f for f in (1.5, 1.0, -0.3, 0.05)] + [0.0] * 12)         # between two of the smallest
    rows.append([2688.0, -2688.0, 1.0, 400.0] + [0.0] * 12)
    rows.append([1e30, -1e30, 3000.0, 2.0] + [0.0] * 12)                 # past the largest
    rows.append([math.inf, -math.inf, 5.0, 1e38] + [1.0] * 12)
    rows.append([math.nan] + [1.0] * 15)
    rows.append([1e-40, 2e-39] + [0.0] * 14)
    rows.append([6.0 * (1 + 1 / 16), 1.0] + [0.1] * 14)                  # a scale halfway between two
    rows.append([6.0 * (1 + 3 / 16), 1.0] + [0.1] * 14)
    rows += [[1.0] * 16] * (-len(rows) % 2)
    x = torch.tensor(rows, device="cuda").view(1, len(rows) // 2, 32)
    kv = x.shape[1]
    cache = pool(torch, 1, 1, kv, 32)
    S.cache4_write(x, -x, cache, torch.zeros(1, device="cuda", dtype=torch.int64))
    got = at(cache, torch.zeros(1, device="cuda", dtype=torch.int64))
    a, b = S.cache4_read(cache, torch.zeros(1, device="cuda", dtype=torch.int64), dtype=torch.float32)
    for y, codes, scales, back in ((x, got[0], got[1], a), (-x, got[2], got[3], b)):
        want_codes, want_scales = written(y, 1.0)
        assert torch.equal(scales.cpu(), want_scales)
        fine = ~y.unflatten(-1, (-1, 16)).isnan().any(-1)
        assert torch.equal(codes.cpu().unflatten(-1, (-1, 8))[fine.cpu()], want_codes.unflatten(-1, (-1, 8))[fine.cpu()])
        groups = back.unflatten(-1, (-1, 16))
        assert groups[~fine].isnan().all() and int((~fine).sum()) == 1 and groups[fine].isfinite().all()
        assert groups[fine].abs().max() == 2688.0
        assert torch.equal(back.nan_to_num(9.0), values(codes, scales, 1.0).float().nan_to_num(9.0))


def test_error_of_a_group_is_half_a_step(torch):
    """An element is off by half of its step at most (the largest one's is 2 scales, so 1 / 6 of the largest), and
    a rounded scale by 2^-4 of the largest more."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(500, 2, 128, generator=g, device="cuda")
    cache = S.Cache4.zeros(32, 16, 2, 128)
    slots = torch.arange(500, device="cuda")
    S.cache4_write(x, x, cache, slots)
    k, v = S.cache4_read(cache, slots, dtype=torch.float32)
    assert torch.equal(k, v)
    most = x.unflatten(-1, (-1, 16)).abs().amax(-1, keepdim=True)
    assert ((k - x).unflatten(-1, (-1, 16)).abs() <= most * (1 / 6 + 2.0 ** -4)).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_strides_and_alignments(torch, dtype):
    """Tokens off the 16-byte boundaries, apart and heads first: the same bits, and nothing beside."""
    T, kv, D = 33, 3, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(T, kv, D, generator=g, device="cuda").to(getattr(torch, dtype))
    slots = torch.randperm(48, generator=g, device="cuda")[:T]
    a, b = (S.Cache4.zeros(3, 16, kv, D) for _ in range(2))
    S.cache4_write(x, x, a, slots)
    room = torch.zeros(kv * T * (D + 1) + 1, device="cuda", dtype=x.dtype)
    y = room[1:].view(kv, T, D + 1)[..., :D].transpose(0, 1)
    y.copy_(x)
    S.cache4_write(y, y, b, slots)
    for n in ("key_codes", "key_scales", "value_codes", "value_scales"):
        assert torch.equal(getattr(a, n), getattr(b, n))
    want, _ = S.cache4_read(a, slots, dtype=x.dtype)
    room.zero_()
    v = torch.zeros_like(want)
    k2, v2 = S.cache4_read(a, slots, out=(y, v))
    assert k2 is y and v2 is v and torch.equal(y, want) and torch.equal(v, want)
    assert room[0] == 0 and (room[1:].view(kv, T, D + 1)[..., D:] == 0).all()
    one = x[:1, :1].expand(T, kv, D)                    # one head for all
    S.cache4_write(one, one, b, slots)
    k, _ = S.cache4_read(b, slots, dtype=x.dtype)
    assert torch.equal(k, k[:1, :1].expand(T, kv, D))


def test_slots_past_the_pool(torch):
    x = torch.ones(5, 2, 64, device="cuda")
    cache = S.Cache4.zeros(2, 16, 2, 64)
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    S.cache4_write(x, x, cache, torch.tensor([3, 32, -5, 10 ** 12, 31], device="cuda"), error_word=err)
    assert int(err) == S.DATA_BAD_INDEX
    hit = cache.key_scales.flatten(0, 1).any(-1).any(-1)
    assert hit.nonzero().flatten().tolist() == [3, 31]
    err.zero_()
    k, v = S.cache4_read(cache, torch.tensor([31, 32, -1, 2 ** 40, 3], device="cuda"), error_word=err)
    assert int(err) == S.DATA_BAD_INDEX
    # 1 / 6 lies between the scales 10 / 64 and 11 / 64, nearer the second; its code of 6 stands for 66 / 64
    assert (k[[0, 4]] == 66 / 64).all() and (k[1:4] == 0).all() and (v[1:4] == 0).all()
    err.zero_()
    S.cache4_read(cache, torch.tensor([-1, 5], device="cuda"), error_word=err)
    assert int(err) == 0


def test_a_pool_past_32_bit_offsets(torch):
    n, bs, H, D = 35000, 64, 8, 256
    cache = S.Cache4.zeros(n, bs, H, D)
    assert cache.key_codes.numel() > 2 ** 31
    slots = torch.tensor([n * bs - 1, 5, (n - 3) * bs + 17, n // 2 * bs + 1], device="cuda")
    x = torch.randn(4, H, D, device="cuda")
    S.cache4_write(x, -x, cache, slots)
    k, v = S.cache4_read(cache, slots, dtype=torch.float32)
    few = S.Cache4.zeros(1, 4, H, D)
    S.cache4_write(x, -x, few, torch.arange(4, device="cuda"))
    k2, v2 = S.cache4_read(few, torch.arange(4, device="cuda"), dtype=torch.float32)
    assert torch.equal(k, k2) and torch.equal(v, v2) and torch.equal(v, -k)


def test_no_tokens_streams_and_a_graph(torch):
    x = torch.randn(20, 2, 64, device="cuda").bfloat16()
    slots = torch.arange(20, device="cuda")
    cache = S.Cache4.zeros(2, 16, 2, 64)
    S.cache4_write(x[:0], x[:0], cache, slots[:0])
    assert S.cache4_read(cache, slots[:0])[0].shape == (0, 2, 64)
    assert not cache.key_scales.any()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        S.cache4_write(x, x, cache, slots)
        want, _ = S.cache4_read(cache, slots)
    s.synchronize()
    out = torch.zeros_like(want), torch.zeros_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.cache4_write(x, x, cache, slots)
        S.cache4_read(cache, slots, out=out)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], want)
    x.mul_(2)                                           # twice the values: twice the scales
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], want * 2) and torch.equal(out[1], want * 2)


def test_refusals(torch):
    x = torch.ones(5, 2, 64, device="cuda")
    slots = torch.arange(5, device="cuda")
    with pytest.raises(A.AsymSpecError):                # codes off the 16-byte boundaries
        room = torch.zeros(16 * 2 * 32 + 8, dtype=torch.uint8, device="cuda")[8:].view(1, 16, 2, 32)
        scales = torch.zeros(1, 16, 2, 4, dtype=torch.uint8, device="cuda")
        S.cache4_write(x, x, S.Cache4(room, scales, room, scales), slots)
    with pytest.raises(A.AsymSpecError):                # heads that no 32 divides
        S.cache4_write(x[..., :48], x[..., :48], S.Cache4.zeros(1, 16, 2, 48), slots)
    cache = S.Cache4.zeros(1, 16, 2, 64)
    with pytest.raises(A.AsymSpecError):
        S.cache4_read(cache, slots, out=(x, x))
    with pytest.raises(A.AsymSpecError):
        S.cache4_read(cache, slots, out=(x, torch.ones(5, 1, 64, device="cuda").expand(5, 2, 64)))
    with pytest.raises(A.AsymSpecError):
        S.cache4_write(x, x, S.Cache4.zeros(1, 16, 2, 64, key_scale=0.0), slots)

"""cache_plan and cache_write against their definitions; whole numbers and copies: equal."""
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


def state(seed, B, bs, longest, spare, width=None, hold=None):
    """Requests of any length up to `longest`, some of them empty, holding what they need (or a
    number of blocks more), and a pool with `spare` free blocks in any order."""
    r = random.Random(seed)
    lens = [0 if r.random() < 0.2 else r.randint(0, longest) for _ in range(B)]
    held = [-(-t // bs) + (r.randint(0, hold) if hold else 0) for t in lens]
    width = width or max(held + [1]) + 24
    ids = list(range(sum(held) + spare))
    r.shuffle(ids)
    tables, at = [], 0
    for h in held:
        tables.append(ids[at:at + h] + [-7] * (width - h))
        at += h
    return lens, held, tables, ids[at:], len(ids)


def run(torch, lens, held, tables, free, blocks, *, block_size, accepted=None, grow=0, capacity=None,
        pad=0, in_place=False):
    i32 = dict(device="cuda", dtype=torch.int32)
    B, width = len(lens), len(tables[0])
    t = torch.full((B, width + pad), -9, **i32)
    t[:, :width] = torch.tensor(tables, **i32)
    t = t[:, :width]
    fl = torch.full((blocks,), -5, **i32)
    fl[:len(free)] = torch.tensor(free, **i32)
    x = dict(lens=torch.tensor(lens, **i32), held=torch.tensor(held, **i32),
             free_count=torch.tensor([len(free)], **i32))
    g = torch.tensor(grow, **i32) if isinstance(grow, list) else grow
    if capacity is None:
        capacity = sum(grow) if isinstance(grow, list) else B * grow
    err = torch.zeros(1, **i32)
    out = None
    if in_place:
        out = dict(start=x["lens"], len=torch.empty(B, **i32), held=x["held"], free_count=x["free_count"],
                   offsets=torch.empty(B + 1, **i32), positions=torch.empty(capacity, **i32),
                   slots=torch.empty(capacity, device="cuda", dtype=torch.int64))
    r = S.cache_plan(x["lens"], t, x["held"], fl, x["free_count"], block_size=block_size,
                     accepted=None if accepted is None else torch.tensor(accepted, **i32), grow=g,
                     capacity=capacity, out=out, error_word=err)
    got = {k: v.tolist() for k, v in r.items()}
    got.update(tables=t.tolist(), free=fl.tolist()[:got["free_count"][0]], err=int(err))
    return got


def compare(got, want, capacity=None):
    start, ends, kept, free, offsets, slots, positions, tables = want
    n = len(slots) if capacity is None else capacity
    fill = [-1] * max(0, n - len(slots))
    assert got["start"] == start and got["len"] == ends and got["held"] == kept
    assert got["offsets"] == offsets
    assert got["slots"] == (slots + fill)[:n] and got["positions"] == (positions + fill)[:n]
    assert got["tables"] == tables and got["free"] == free


@pytest.mark.parametrize("seed,B,bs,longest,K", [
    (1, 1, 16, 100, 4), (2, 64, 16, 3000, 7), (3, 37, 1, 60, 8), (4, 200, 24, 5000, 1),
    (5, 1024, 64, 700, 4), (6, 1025, 8, 90, 3), (7, 5, 4096, 9000, 7), (8, 8192, 32, 40, 2)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rounds(torch, seed, B, bs, longest, K, in_place):
    from tests._serving import planned
    r = random.Random(seed)
    lens, held, tables, free, blocks = state(seed, B, bs, longest, B * (2 * K // bs + 3), hold=2)
    accepted = [r.randint(-1, K) for _ in range(B)]
    want = planned(lens, tables, held, free, block_size=bs, accepted=accepted, grow=K + 1)
    got = run(torch, lens, held, tables, free, blocks, block_size=bs, accepted=accepted, grow=K + 1,
              pad=seed % 3, in_place=in_place)
    compare(got, want)
    assert got["err"] == 0
    live = [s for s in got["slots"] if s >= 0]
    assert len(set(live)) == len(live) == B * (K + 1)      # no slot twice


@pytest.mark.parametrize("seed,B,bs,longest,spare,extra", [
    (11, 1, 16, 50, 400, 0), (12, 30, 16, 3000, 6000, 100), (13, 300, 24, 500, 3000, 0),
    (19, 100, 16, 900, 30, 5),       # a pool that runs out
    (15, 50, 1, 40, 0, 3),            # none at all, but for what is given back
    (16, 3, 16, 60000, 12000, 0), (17, 2000, 8, 30, 2000, 1)])
def test_requests_begin_end_and_go_on(torch, seed, B, bs, longest, spare, extra):
    from tests._serving import planned
    r = random.Random(seed)
    lens, held, tables, free, blocks = state(seed, B, bs, longest, spare, width=2 * (longest // bs + 2))
    grow = []
    for b in range(B):
        what = r.random()
        if what < 0.3:
            lens[b] = 0
        grow.append(0 if what < 0.4 else r.randint(0, longest) if what < 0.6 else r.randint(0, 9))
    want = planned(lens, tables, held, free, block_size=bs, grow=grow)
    got = run(torch, lens, held, tables, free, blocks, block_size=bs, grow=grow,
              capacity=sum(grow) + extra, pad=5)
    compare(got, want, sum(grow) + extra)
    unserved = any(e != s + g for s, e, g in zip(want[0], want[1], grow))
    assert got["err"] == (S.DATA_NO_BLOCKS if unserved else 0)
    assert unserved == (seed in (15, 19))


def test_no_blocks_no_requests_no_tokens(torch):
    from tests._serving import planned
    i32 = dict(device="cuda", dtype=torch.int32)
    r = S.cache_plan(torch.empty(0, **i32), torch.empty(0, 4, **i32), torch.empty(0, **i32),
                     torch.tensor([2, 1, 0], **i32), torch.tensor([3], **i32), block_size=16, grow=3,
                     capacity=2)
    assert r["offsets"].tolist() == [0] and r["free_count"].tolist() == [3]
    assert r["slots"].tolist() == [-1, -1]
    lens, held, tables, free, blocks = state(9, 6, 16, 100, 4)
    want = planned(lens, tables, held, free, block_size=16, grow=0)
    compare(run(torch, lens, held, tables, free, blocks, block_size=16, grow=0), want)


def test_a_request_keeps_its_place_over_many_rounds(torch):
    """The state of one call into the next, requests ending and beginning: no block is lost or
    held twice, and what stays cached keeps its slot."""
    i32 = dict(device="cuda", dtype=torch.int32)
    r = random.Random(5)
    B, bs, blocks, width, K = 24, 16, 400, 40, 4
    tables = torch.full((B, width), -1, **i32)
    free = torch.randperm(blocks, device="cuda").int()
    s = dict(start=torch.zeros(B, **i32), held=torch.zeros(B, **i32),
             free_count=torch.tensor([blocks], **i32))
    place = [dict() for _ in range(B)]
    for step in range(40):
        acc = [r.randint(-1, K) for _ in range(B)]
        lens = s["start"].tolist()
        for b in range(B):
            if lens[b] > width * bs - 40 or r.random() < 0.05:
                lens[b], acc[b], place[b] = 0, -1, {}
        s = S.cache_plan(torch.tensor(lens, **i32), tables, s["held"], free, s["free_count"],
                         block_size=bs, accepted=torch.tensor(acc, **i32), grow=K + 1)
        start, slots, pos = s["start"].tolist(), s["slots"].tolist(), s["positions"].tolist()
        table = tables.tolist()
        held = s["held"].tolist()
        inside = [x for b in range(B) for x in table[b][:held[b]]]
        outside = free.tolist()[:int(s["free_count"])]
        assert sorted(inside + outside) == list(range(blocks)), step
        for b in range(B):
            place[b] = {p: x for p, x in place[b].items() if p < start[b]}
            for i in range(K + 1):
                assert pos[b * (K + 1) + i] == start[b] + i
                place[b][start[b] + i] = slots[b * (K + 1) + i]
            for p, x in place[b].items():
                assert table[b][p // bs] * bs + p % bs == x, (step, b, p)


def test_bad_data(torch):
    i32 = dict(device="cuda", dtype=torch.int32)

    def plan(lens=(5, 20), held=(1, 2), free=(9, 8, 7), accepted=None, grow=4, tables=None, capacity=8,
             count=None):
        err = torch.zeros(1, **i32)
        t = torch.tensor(tables or [[0, 1, 2], [3, 4, 5]], **i32)
        fl = torch.tensor(list(free) + [-1] * (10 - len(free)), **i32)
        r = S.cache_plan(torch.tensor(lens, **i32), t, torch.tensor(held, **i32), fl,
                         torch.tensor([len(free) if count is None else count], **i32), block_size=16,
                         accepted=None if accepted is None else torch.tensor(accepted, **i32),
                         grow=grow if isinstance(grow, int) else torch.tensor(grow, **i32),
                         capacity=capacity, error_word=err)
        return {k: v.tolist() for k, v in r.items()}, int(err)

    r, e = plan()
    assert e == 0 and r["start"] == [5, 20] and r["len"] == [9, 24] and r["held"] == [1, 2]
    r, e = plan(lens=(-3, 20))
    assert e == S.DATA_BAD_LENGTH and r["start"] == [0, 20] and r["len"] == [4, 24]
    r, e = plan(accepted=(-2, 0))
    assert e == S.DATA_BAD_LENGTH and r["start"] == [5, 21]
    r, e = plan(grow=[-1, 4])
    assert e == S.DATA_BAD_LENGTH and r["offsets"] == [0, 0, 4]
    r, e = plan(lens=(5, 46))                       # 46 + 4 tokens do not fit three blocks of 16
    assert e == S.DATA_BAD_LENGTH and r["len"] == [9, 46] and r["held"] == [1, 2]
    assert r["slots"][4:] == [-1] * 4 and r["slots"][:4] == [5, 6, 7, 8]
    r, e = plan(lens=(5, 1 << 30), grow=[4, 2 ** 31 - 1])
    assert e == S.DATA_BAD_LENGTH and r["start"] == [5, 48] and r["held"] == [1, 2]
    r, e = plan(held=(1, 7))
    assert e == S.DATA_BAD_LENGTH and r["held"] == [1, 2]
    r, e = plan(capacity=6)
    assert e == S.DATA_BAD_LENGTH and len(r["slots"]) == 6 and r["offsets"] == [0, 4, 8]
    r, e = plan(count=-4, grow=30)
    assert e == S.DATA_BAD_LENGTH | S.DATA_NO_BLOCKS and r["free_count"] == [0]
    r, e = plan(tables=[[10, 1, 2], [3, -1, 5]])    # a block that does not exist
    assert e == S.DATA_BAD_INDEX and r["slots"] == [-1] * 8
    r, e = plan(free=(9, 8, 77), grow=12, capacity=24)           # nor in the list
    assert e == S.DATA_BAD_INDEX


def test_more_blocks_than_there_are(torch):
    """Blocks given back to a list that is full already (bad data) go nowhere, in a pool of so many
    that the place after the list's end does not fit 32 bits either."""
    i32 = dict(device="cuda", dtype=torch.int32)
    for blocks in (40, 2 ** 31 - 1):
        room = torch.empty(blocks + 64, **i32)
        room[:32] = -77
        room[32 + blocks:] = -77
        free = room[32:32 + blocks]
        free[-40:] = torch.arange(40, **i32)
        tables = torch.arange(40, **i32).view(2, 20)
        err = torch.zeros(1, **i32)
        r = S.cache_plan(torch.tensor([0, 3], **i32), tables, torch.tensor([20, 15], **i32), free,
                         torch.tensor([blocks], **i32), block_size=1, grow=2, error_word=err)
        assert int(err) == S.DATA_BAD_LENGTH
        assert r["held"].tolist() == [2, 5] and r["free_count"].tolist() == [blocks]
        assert r["slots"].tolist() == [0, 1, 23, 24]
        assert (room[:32] == -77).all() and (room[32 + blocks:] == -77).all()
        assert torch.equal(free[-40:], torch.arange(40, **i32))
        # and requests that need some take none of what was not put there
        err.zero_()
        r = S.cache_plan(torch.tensor([0, 3], **i32), tables, torch.tensor([20, 3], **i32), free,
                         torch.tensor([blocks], **i32), block_size=1, grow=torch.tensor([0, 4], **i32),
                         capacity=4, error_word=err)
        assert int(err) == S.DATA_BAD_LENGTH | S.DATA_BAD_INDEX
        assert r["held"].tolist() == [0, 7] and r["slots"].tolist() == [-1] * 4
        assert tables[1, 3:7].tolist() == [-1] * 4
        assert (room[:32] == -77).all() and (room[32 + blocks:] == -77).all()
        del room, free


WRITES = [
    # T, heads, D, block, dtype, layout, offset of k in its allocation
    (1, 1, 64, 16, "bfloat16", "nhd", 0), (513, 8, 128, 16, "bfloat16", "nhd", 0),
    (100, 3, 80, 24, "float32", "hnd", 0), (77, 2, 5, 7, "bfloat16", "nhd", 0),
    (300, 4, 64, 16, "bfloat16", "hnd", 1), (65, 1, 1, 1, "float32", "nhd", 0),
    (50, 5, 36, 3, "float32", "hnd", 2), (5000, 2, 96, 32, "bfloat16", "dnh", 0)]


@pytest.mark.parametrize("case", range(len(WRITES)))
def test_writes(torch, case):
    T, H, D, bs, dtype, layout, off = WRITES[case]
    dt = getattr(torch, dtype)
    g = torch.Generator(device="cuda").manual_seed(case)
    blocks = T // bs + 5

    def pool():
        shape = {"nhd": (blocks, bs, H, D), "hnd": (blocks, H, bs, D), "dnh": (H, blocks, bs, D)}[layout]
        x = torch.randn(shape, generator=g, device="cuda").to(dt)
        return {"nhd": x, "hnd": x.transpose(1, 2), "dnh": x.permute(1, 2, 0, 3)}[layout]

    keys, values = pool(), pool()
    qkv = torch.randn(T * 3 * H * D + off, generator=g, device="cuda").to(dt)[off:].view(T, 3, H, D)
    slots = torch.randperm(blocks * bs, generator=g, device="cuda")[:T]
    slots[::7] = -1
    want_k, want_v = keys.clone(), values.clone()
    for t, s in enumerate(slots.tolist()):
        if s >= 0:
            want_k[s // bs, s % bs] = qkv[t, 1]
            want_v[s // bs, s % bs] = qkv[t, 2]
    S.cache_write(qkv[:, 1], qkv[:, 2], keys, values, slots)
    assert torch.equal(keys, want_k) and torch.equal(values, want_v)


def test_a_slot_past_the_pool_is_skipped(torch):
    keys, values = torch.zeros(4, 16, 2, 64, device="cuda"), torch.zeros(4, 16, 2, 64, device="cuda")
    k = torch.ones(4, 2, 64, device="cuda")
    err = torch.zeros(1, device="cuda", dtype=torch.int32)
    S.cache_write(k, k, keys, values, torch.tensor([63, 64, 2 ** 40, -2 ** 40], device="cuda"), error_word=err)
    assert int(err) == S.DATA_BAD_INDEX
    assert keys.sum() == 128 and keys[3, 15].sum() == 128 and values.sum() == 128


def test_a_cache_past_32_bit_offsets(torch):
    """Element offsets beyond 2^32: 5 GiB of bf16 keys that are also the values."""
    n, bs, H, D = 41000, 64, 8, 128
    keys = torch.zeros(n, bs, H, D, device="cuda", dtype=torch.bfloat16)
    assert keys.numel() > 2 ** 31 and keys.numel() * 2 > 2 ** 32
    k = torch.randn(3, H, D, device="cuda").bfloat16()
    slots = torch.tensor([n * bs - 1, 0, n * bs // 2 + 5], device="cuda")
    S.cache_write(k, k, keys, keys, slots)
    flat = keys.view(-1, H, D)
    assert torch.equal(flat[slots], k)
    assert int((flat.view(-1, 1024)[::4096] != 0).any(-1).sum()) <= 3


def test_refusals_of_the_binding(torch):
    i32 = dict(device="cuda", dtype=torch.int32)
    one, t = torch.zeros(2, **i32), torch.zeros(2, 3, **i32)
    c = torch.zeros(1, **i32)
    for bad in (dict(accepted=torch.zeros(3, **i32)), dict(accepted=torch.zeros(2, device="cuda")),
                dict(grow=torch.zeros(2, **i32)), dict(grow=torch.zeros(1, **i32), capacity=3)):
        with pytest.raises(ValueError):
            S.cache_plan(one, t, one, t[0], c, block_size=16, **bad)
    with pytest.raises(A.AsymSpecError):
        S.cache_plan(one, t, one, t[0], c, block_size=0)
    with pytest.raises(ValueError):
        S.cache_plan(one, t[:1], one, t[0], c, block_size=16)
    k = torch.zeros(4, 2, 64, device="cuda")
    cache = torch.zeros(3, 16, 2, 64, device="cuda")
    slots = torch.zeros(4, device="cuda", dtype=torch.int64)
    for bad in ((k.bfloat16(), k, cache, cache, slots), (k, k, cache, cache.bfloat16(), slots),
                (k, k, cache, cache, slots.int()), (k, k, cache, cache, slots[:3]),
                (k[:, :1], k[:, :1], cache, cache, slots), (k, k, cache.cpu(), cache.cpu(), slots),
                (k, k, cache.transpose(2, 3), cache.transpose(2, 3), slots)):
        with pytest.raises((ValueError, TypeError)):
            S.cache_write(*bad)
    with pytest.raises(TypeError):
        S.cache_write(k.half(), k.half(), cache.half(), cache.half(), slots)

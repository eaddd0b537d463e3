"""Rotary positions and the cache in 4 bits as a serving loop uses them: by themselves over a plan's rounds,
and in examples/serving_round.py."""
import importlib.util
import os

import pytest

from paper_2608_26004_gb300 import serving as S

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def torch():
    import torch as _torch
    assert _torch.cuda.is_available(), "the gpu tests need a CUDA device"
    from paper_2608_26004_gb300 import build
    build.build_cuda()
    S.lib()
    return _torch


@pytest.fixture(scope="module")
def example(torch):
    spec = importlib.util.spec_from_file_location("serving_round", os.path.join(ROOT, "examples", "serving_round.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rounds_of_plan_rotary_write_and_attention(torch, dtype):
    """A prompt and three rounds with rejected drafts: each round's queries over what the cache holds of the
    committed tokens' turned keys, both from their definitions."""
    from tests._cache4 import values, written
    from tests.test_gpu_attend4 import check, some_rows
    from tests.test_gpu_rotary import check as check_turned
    B, Q, H, kv, D, bs = 4, 3, 8, 2, 64, 16
    dt, i32 = getattr(torch, dtype), dict(dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(31)
    tables = torch.full((B, 12), -1, **i32)
    free = torch.randperm(B * 12, generator=gen, device="cuda").int()
    state = dict(start=torch.zeros(B, **i32), held=torch.zeros(B, **i32), free_count=torch.tensor([B * 12], **i32))
    rotary = S.Rotary(D, rotary_dim=48, scaling=dict(kind="wavelength", factor=4.0, original_length=256, fast=4.0, slow=1.0))
    cache = S.Cache4.zeros(B * 12, bs, kv, D)
    attend = S.Cache4Attend(B, Q, H, kv, D)
    err = torch.zeros(1, **i32)
    prompt = torch.tensor([70, 5, 33, 16], **i32)
    accepted = None
    kept = [[] for _ in range(B)]                       # each request's turned keys and values, one a token
    for r in range(4):
        grow = prompt if r == 0 else Q
        T = int(prompt.sum()) if r == 0 else B * Q
        state = S.cache_plan(state["start"], tables, state["held"], free, state["free_count"], block_size=bs,
                             accepted=accepted, grow=grow, capacity=T + 2, error_word=err)
        qkv = torch.randn(T + 2, (H + 2 * kv) * D, generator=gen, device="cuda").to(dt)
        q, k, v = (x.unflatten(-1, (-1, D)) for x in qkv.split([H * D, kv * D, kv * D], -1))
        q2, k2 = rotary(q, state["positions"], k)
        check_turned(torch, k2, k, state["positions"], rotary)
        S.cache4_write(k2, v, cache, state["slots"], error_word=err)
        offsets = state["offsets"].tolist()
        for b in range(B):
            kept[b] += [(k2[i], v[i]) for i in range(offsets[b], offsets[b + 1])]
            assert len(kept[b]) == int(state["len"][b])
            page = tables[b].long()[torch.arange(len(kept[b]), device="cuda") // bs]
            at = torch.arange(len(kept[b]), device="cuda") % bs
            for x, codes, scales in ((0, cache.key_codes, cache.key_scales), (1, cache.value_codes, cache.value_scales)):
                want = written(torch.stack([t[x] for t in kept[b]]), 1.0)
                assert torch.equal(codes[page, at].cpu(), want[0]) and torch.equal(scales[page, at].cpu(), want[1])
        if r > 0:
            x = (q2[:T].view(B, Q, H, D), cache, tables, state["len"])
            out, lse = attend(*x, error_word=err)
            check(torch, x, out, lse, some_rows(B, Q, H, r))
            # of the round's tokens the first and 0 to Q - 1 more stay
            accepted = torch.randint(0, Q, (B,), generator=gen, **i32)
            for b in range(B):
                kept[b] = kept[b][:int(state["start"][b]) + int(accepted[b]) + 1]
        else:
            state = dict(state, start=state["len"])
            accepted = None
    assert int(err) == 0
    assert values(cache.key_codes, cache.key_scales, 1.0).isfinite().all()


@pytest.mark.parametrize("rotary,four_bits", [(True, False), (False, True), (True, True)])
def test_the_loop_commits_what_the_rules_allow(torch, example, rotary, four_bits):
    B, K, rounds = 5, 3, 6
    loop = example.Loop(B=B, K=K, V=1024, prompt=(30, 70), rounds=rounds, seed=B, rotary=rotary, four_bits=four_bits)
    for _ in range(rounds):
        assert int(loop.round()) == 0
        assert (loop.accepted >= 0).all()
    loop.raise_errors(torch.zeros(1, dtype=torch.int32))
    said = (loop.history_len - loop.prompt_len).tolist()
    assert all(rounds <= n <= rounds * (K + 1) for n in said)
    # what is cached of each request: its tokens' keys at their positions, as the cache holds them.  (Another
    # shape of matrix product may round a projection otherwise: 2 %; a value in 4 bits is off by a sixth of its
    # group's largest at most, and by what its scale is rounded, 2^-4 of it.)
    for c in loop.contexts:
        for b in range(B):
            n = int(c.state["start"][b] + loop.accepted[b] + 1)
            tokens = loop.history[b, int(loop.history_len[b]) - 1 - n:int(loop.history_len[b]) - 1]
            at = torch.arange(n, device="cuda")
            _, _, k, v = c.project(tokens)
            _, k = c.placed(None, k[None], at.int())
            k = k[0]
            slots = c.tables[b].long()[at // c.block_size] * c.block_size + at % c.block_size
            if four_bits:
                got = S.cache4_read(c.cache, slots)
            else:
                got = tuple(x.flatten(0, 1)[slots] for x in (c.keys, c.values))
            for x, y in zip(got, (k, v)):
                y = y.float()
                most = y.unflatten(-1, (-1, 16)).abs().amax(-1, keepdim=True).expand(*y.shape[:-1], -1, 16).flatten(-2)
                room = 0.02 + 0.02 * y.abs() + (most * (1 / 6 + 2.0 ** -4) if four_bits else 0)
                assert ((x.float() - y).abs() <= room).all()


def test_rotary_attention_of_the_loop_equals_attention_without_a_cache(torch, example):
    """The verifier's logits of a round against dense attention over the cache's turned keys (see the same test
    without positions for the 5 %)."""
    for four_bits in (False, True):
        loop = example.Loop(B=4, K=3, V=512, prompt=(25, 50), rounds=4, seed=9, rotary=True, four_bits=four_bits)
        for _ in range(3):
            loop.round()
        c, m = loop.verifier, loop.verifier.model
        c.plan(loop.K + 1, loop.accepted)
        tokens = torch.randint(0, 512, (4, loop.K + 1), device="cuda")
        got = c.logits(tokens).float()
        start = c.state["start"].tolist()
        for b in range(4):
            n = start[b]
            at = torch.arange(n + loop.K + 1, device="cuda")
            slots = c.tables[b].long()[at // 16] * 16 + at % 16
            k, v = S.cache4_read(c.cache, slots) if four_bits else (x.flatten(0, 1)[slots] for x in (c.keys, c.values))
            x, q, k0, _ = c.project(tokens[b])
            q, _ = c.placed(q[None], k0[None], at[n:].int())
            for i in range(loop.K + 1):
                kk, vv = (t[:n + i + 1].double().repeat_interleave(m.heads // m.kv_heads, 1) for t in (k, v))
                s = torch.einsum("hd,nhd->hn", q[0, i].double(), kk) / m.dim ** 0.5
                o = torch.einsum("hn,nhd->hd", s.softmax(-1), vv).reshape(-1).bfloat16()
                want = m.logits(x[i], o).float()
                assert (got[b, i] - want).abs().max() <= 0.05 * want.abs().max()


def test_the_program_takes_both(example, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["serving_round.py", "--requests", "2", "--rounds", "3", "--rotary", "--four-bits"])
    example.main()
    assert "tokens committed per request" in capsys.readouterr().out

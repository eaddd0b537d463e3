"""The serving loop of examples/serving_round.py: what is committed keeps the rules, and every
cache holds exactly the committed tokens' keys and values."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import torch
    assert torch.cuda.is_available(), "the gpu tests need a CUDA device"
    from paper_2608_26004_gb300 import build
    build.build_cuda()
    spec = importlib.util.spec_from_file_location("serving_round", os.path.join(ROOT, "examples", "serving_round.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("B,K,rounds", [(6, 4, 10), (1, 1, 6), (17, 7, 5)])
def test_rounds_commit_what_the_rules_allow(example, B, K, rounds):
    import torch
    loop = example.Loop(B=B, K=K, V=1024, prompt=(30, 70), rounds=rounds, seed=B)
    accepted = 0
    for _ in range(rounds):
        error = loop.round()
        assert int(error) == 0
        assert (loop.accepted >= 0).all()
        accepted += int(loop.accepted.sum())
    assert [int(c.error) for c in loop.contexts] == [0, 0, 0]
    for b in range(B):
        said = loop.history[b, int(loop.prompt_len[b]):int(loop.history_len[b])]
        assert rounds <= said.numel() <= rounds * (K + 1)
        assert (said != 0).all()
        if b % 2 == 0:
            assert (said < 512).all()
    # cached: the prompt, then the round's first token (the prompt's last, again) and what was
    # accepted; the last next token is not cached yet
    for c in loop.contexts:
        length = c.state["start"] + loop.accepted + 1
        for b in range(B):
            n = int(length[b])
            committed = loop.history[b, int(loop.prompt_len[b]) - 1:int(loop.history_len[b]) - 1]
            at = torch.arange(n - committed.numel(), n, device="cuda")
            page = c.tables[b].long()[at // c.block_size]
            _, _, k, v = c.project(committed)
            close = dict(rtol=0.02, atol=0.02)  # (another shape of matrix product may round otherwise)
            assert torch.allclose(c.keys[page, at % c.block_size].float(), k.float(), **close)
            assert torch.allclose(c.values[page, at % c.block_size].float(), v.float(), **close)


def test_attention_of_the_loop_equals_attention_without_a_cache(example):
    """The verifier's logits of a round against dense attention over the committed tokens.  The
    attention's output is rounded to bf16 (2^-8) before two bf16 products; a logit sums 128
    terms of either sign, so 5 % of the largest logit is ample for it and far below what a
    wrong key or position does."""
    import torch
    loop = example.Loop(B=4, K=3, V=512, prompt=(25, 50), rounds=4, seed=9)
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
        page = c.tables[b].long()[at // 16]
        k, v = c.keys[page, at % 16].double(), c.values[page, at % 16].double()
        x, q, _, _ = c.project(tokens[b])
        for i in range(loop.K + 1):
            kk, vv = (t[:n + i + 1].repeat_interleave(m.heads // m.kv_heads, 1) for t in (k, v))
            s = torch.einsum("hd,nhd->hn", q[i].double(), kk) / m.dim ** 0.5
            o = torch.einsum("hn,nhd->hd", s.softmax(-1), vv).reshape(-1).bfloat16()
            want = m.logits(x[i], o).float()
            assert (got[b, i] - want).abs().max() <= 0.05 * want.abs().max()


@pytest.mark.parametrize("B,K,rounds", [(5, 3, 6), (1, 2, 3)])
def test_every_token_is_cached_once_at_its_place(example, B, K, rounds):
    """The prompt's last token is the first round's first: it has one place, like all others."""
    import torch
    loop = example.Loop(B=B, K=K, V=1024, prompt=(30, 70), rounds=rounds, seed=B)
    prompt = [c.state["len"].tolist() for c in loop.contexts]
    for _ in range(rounds):
        loop.round()
    for c, lengths in zip(loop.contexts, prompt):
        cached = (c.state["start"] + loop.accepted + 1).tolist()
        for b in range(B):
            begin, end = int(loop.prompt_len[b]), int(loop.history_len[b])
            tokens = loop.history[b, begin - lengths[b]:end - 1]  # (the last one waits for the next round)
            assert cached[b] == tokens.numel() == lengths[b] + (end - begin) - 1
            at = torch.arange(cached[b], device="cuda")
            page = c.tables[b].long()[at // c.block_size]
            _, _, k, v = c.project(tokens)
            close = dict(rtol=0.02, atol=0.02)
            assert torch.allclose(c.keys[page, at % c.block_size].float(), k.float(), **close)
            assert torch.allclose(c.values[page, at % c.block_size].float(), v.float(), **close)


def test_requests_that_the_pool_has_no_blocks_for_sit_out(example):
    """The verifier's pool runs out: what it cannot serve attends over none but its own tokens,
    commits nothing and stays as it is; the others go on."""
    import torch
    from paper_2608_26004_gb300 import serving as S
    B, K, rounds = 6, 4, 8
    loop = example.Loop(B=B, K=K, V=1024, prompt=(30, 70), rounds=rounds, seed=2)
    prompt = [c.state["len"].tolist() for c in loop.contexts]
    loop.verifier.state["free_count"].fill_(4)
    calls = []
    for c in loop.contexts:
        def recorded(q, keys, values, tables, lens, c=c, call=c.attend, **more):
            calls.append((lens.clone(), c.state["len"]))
            return call(q, keys, values, tables, lens, **more)
        c.attend = recorded
    sat_out = 0
    for _ in range(rounds):
        before = loop.history_len.clone()
        assert int(loop.round()) == 0
        v = loop.verifier.state
        unserved = v["len"] == v["start"]
        sat_out += int(unserved.sum())
        assert torch.equal(loop.history_len == before, unserved)
    assert 0 < sat_out < B * rounds and int(unserved.sum()) < B
    assert int(loop.verifier.error) == S.DATA_NO_BLOCKS
    assert [int(c.error) for c in loop.contexts[:2]] == [0, 0]
    for lens, room in calls:
        assert (lens <= room).all()
    for c, lengths in zip(loop.contexts, prompt):
        cached = (c.state["start"] + loop.accepted + 1).tolist()
        for b in range(B):
            begin, end = int(loop.prompt_len[b]), int(loop.history_len[b])
            tokens = loop.history[b, begin - lengths[b]:end - 1]
            assert cached[b] == tokens.numel()
            at = torch.arange(cached[b], device="cuda")
            page = c.tables[b].long()[at // c.block_size]
            _, _, k, _ = c.project(tokens)
            assert torch.allclose(c.keys[page, at % c.block_size].float(), k.float(), rtol=0.02, atol=0.02)


@pytest.mark.parametrize("K,rounds", [(4, 16), (7, 200)])
def test_tables_hold_all_rounds(example, K, rounds):
    loop = example.Loop(B=2, K=K, V=1024, rounds=rounds)
    most = loop.history.shape[1] + K + 1  # everything that may be said, and the last round's drafts
    for c in loop.contexts:
        assert c.tables.shape[1] * c.block_size >= most
        assert c.keys.shape[0] >= 2 * -(-most // c.block_size)


def test_the_program_says_when_its_data_was_bad(example, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["serving_round.py", "--requests", "2", "--rounds", "3"])
    example.main()
    assert "tokens committed per request" in capsys.readouterr().out

    class Starved(example.Loop):
        def __init__(self, **kw):
            super().__init__(**kw)
            self.verifier.state["free_count"].zero_()

    monkeypatch.setattr(example, "Loop", Starved)
    monkeypatch.setattr("sys.argv", ["serving_round.py", "--requests", "2", "--rounds", "12"])
    with pytest.raises(RuntimeError, match="verifier.*0x200"):
        example.main()

    class Unseen(example.Loop):
        def __init__(self, **kw):
            super().__init__(**kw)
            self.history[0, 0] = -1  # (no token: what the constraints read)

    monkeypatch.setattr(example, "Loop", Unseen)
    with pytest.raises(RuntimeError, match="constraints.*0x"):
        example.main()

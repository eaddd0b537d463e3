"""A serving loop around the verification step, on the GPU from end to end.

Three contexts per request, as the method has them: the drafter on the full context, the
drafter and the verifier on the compressed one, each a small one-layer model with random
weights over a paged key-value cache of its own.  A round of every request:

  cache_plan         blocks and slots for the K + 1 tokens of the round, the tokens that the
                     round before rejected given up (its accept_len never leaves the GPU)
  cache_write,       keys and values of the new tokens, attention over the cached ones: one
  CacheAttend        token at a time while drafting, K + 1 at once while verifying
  constrain_logits   penalties for what the request has said, its biases and its grammar
  draft_tokens       the drafter's draw
  FuseVerify         the accepted drafts and the next token

    python examples/serving_round.py [--requests 8] [--drafts 4] [--rounds 16]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_26004_gb300 import asymspec as A  # noqa: E402
from paper_2608_26004_gb300 import serving as S  # noqa: E402


class Model:
    """One attention layer between random embeddings and an output layer; `near`: another model
    whose weights these are a noisy copy of, as a drafter's answers are of its verifier's."""

    def __init__(self, V, gen, width=128, heads=8, kv_heads=2, dim=64, near=None):
        def weights(name, *shape, scale):
            w = torch.randn(shape, generator=gen, device="cuda") * scale
            return (w if near is None else getattr(near, name).float() + 0.3 * w).bfloat16()

        self.heads, self.kv_heads, self.dim, self.width = heads, kv_heads, dim, width
        self.embed = weights("embed", V, width, scale=1.0)
        self.qkv = weights("qkv", width, (heads + 2 * kv_heads) * dim, scale=width ** -0.5)
        self.out = weights("out", heads * dim, width, scale=(heads * dim) ** -0.5)
        self.head = weights("head", width, V, scale=4.0 * width ** -0.5)

    def logits(self, x, o):
        h = x.float() + (o @ self.out).float()
        return (h * h.square().mean(-1, keepdim=True).rsqrt()).bfloat16() @ self.head


class Context:
    """A model on one context of every request, of `tokens` tokens at most: its paged cache and the state
    of its plan."""

    def __init__(self, model, B, most_new, tokens, block_size=16):
        i32 = dict(dtype=torch.int32, device="cuda")
        width = -(-tokens // block_size)
        blocks = B * width
        shape = (blocks, block_size, model.kv_heads, model.dim)
        self.model, self.B, self.block_size = model, B, block_size
        self.keys = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        self.values = torch.empty_like(self.keys)
        self.tables = torch.full((B, width), -1, **i32)
        self.free = torch.randperm(blocks, device="cuda").to(torch.int32)
        self.state = dict(start=torch.zeros(B, **i32), held=torch.zeros(B, **i32),
                          free_count=torch.tensor([blocks], **i32))
        self.attend = S.CacheAttend(B, most_new, model.heads, model.kv_heads, model.dim)
        self.error = torch.zeros(1, **i32)

    def plan(self, grow, accepted=None, capacity=None):
        s = self.state
        self.state = S.cache_plan(s["start"], self.tables, s["held"], self.free, s["free_count"],
                                  block_size=self.block_size, accepted=accepted, grow=grow,
                                  capacity=capacity, error_word=self.error)

    def project(self, tokens):
        m = self.model
        x = m.embed[tokens.long()]
        q, k, v = (x @ m.qkv).split([m.heads * m.dim, m.kv_heads * m.dim, m.kv_heads * m.dim], -1)
        return x, q.unflatten(-1, (m.heads, m.dim)), k.unflatten(-1, (m.kv_heads, m.dim)), \
            v.unflatten(-1, (m.kv_heads, m.dim))

    def prefill(self, prompts, lengths):
        """prompts: [tokens of all requests, one after another].  (One layer: its keys and values
        are all that later tokens need of a prompt.)"""
        self.plan(lengths, capacity=prompts.numel())
        _, _, k, v = self.project(prompts)
        S.cache_write(k, v, self.keys, self.values, self.state["slots"], error_word=self.error)
        # the next plan keeps what was just written, but for the last token: that is the first
        # round's first, which writes it again, at its place
        self.state = dict(self.state, start=(self.state["len"] - 1).clamp(min=0))

    def logits(self, tokens, first=0):
        """[B, n, V] after each of the round's tokens first .. first + n - 1."""
        B, n = tokens.shape
        x, q, k, v = self.project(tokens)
        slots = self.state["slots"].view(B, -1)[:, first:first + n].contiguous().view(-1)
        S.cache_write(k.flatten(0, 1), v.flatten(0, 1), self.keys, self.values, slots, error_word=self.error)
        # (no more than its blocks hold: where the pool had none for a request, the table's entries
        # from there on are another's)
        seen = torch.minimum(self.state["start"] + (first + n), self.state["len"])
        o, _ = self.attend(q, self.keys, self.values, self.tables, seen, error_word=self.error)
        return self.model.logits(x, o.flatten(2))


class Loop:
    def __init__(self, B=8, K=4, V=4096, prompt=(40, 200), rounds=16, seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.B, self.K, self.V = B, K, V
        drafter = Model(V, gen)
        verifier = Model(V, gen, near=drafter)
        full, short = prompt[1], prompt[0]  # tokens of a full context, and of a compressed one
        tokens = full + (K + 1) * (rounds + 1)
        self.drafter_full = Context(drafter, B, 1, tokens)
        self.drafter_comp = Context(drafter, B, K + 1, tokens)
        self.verifier = Context(verifier, B, K + 1, tokens)
        self.contexts = (self.drafter_full, self.drafter_comp, self.verifier)
        lengths = torch.randint(short // 2, short + 1, (B,), generator=gen, **i32)
        prompts = torch.randint(0, V, (B, full), generator=gen, **i32)
        everything = torch.full((B,), full, **i32)
        self.drafter_full.prefill(prompts.reshape(-1), everything)
        tail = torch.arange(full, device="cuda") >= (full - lengths)[:, None]
        compressed = prompts[tail]  # (of the ends of the full contexts)
        for c in (self.drafter_comp, self.verifier):
            c.prefill(compressed, lengths)
        # what the constraints go by: the full context is the prompt, then what is committed
        self.history = torch.zeros(B, full + (K + 1) * rounds, **i32)
        self.history[:, :full] = prompts
        self.history_len, self.prompt_len = everything.clone(), everything
        self.last = prompts[:, -1].contiguous()  # the round's first token
        self.penalties = dict(repetition=torch.full((B,), 1.2, device="cuda"),
                              frequency=torch.full((B,), 0.3, device="cuda"),
                              presence=torch.full((B,), 0.2, device="cuda"))
        # every other request answers in the first half of the vocabulary
        words = torch.zeros(1, V // 32, **i32)
        words[0, :V // 64] = -1
        self.mask = words
        self.mask_rows = torch.where(torch.arange(B, device="cuda") % 2 == 0, 0, -1).to(torch.int32)
        self.mask_rows = self.mask_rows[:, None].expand(B, K + 1).contiguous()
        # nobody says token 0
        self.bias = (torch.arange(B + 1, **i32), torch.zeros(B, **i32), torch.full((B,), -1e4, device="cuda"))
        self.step = A.FuseVerify(B, K)
        self.error = torch.zeros(1, **i32)  # of the constraints
        self.accepted = None

    def raise_errors(self, step):
        """Raises what the error words of the loop (and `step`, of its steps) hold, if anything."""
        words = dict(step=step, constraints=self.error, drafter_full=self.drafter_full.error,
                     drafter_comp=self.drafter_comp.error, verifier=self.verifier.error)
        bad = {name: hex(int(w)) for name, w in words.items() if int(w)}
        if bad:
            raise RuntimeError(f"bad data: {bad}")

    def constrained(self, logits, drafts=None, first=0):
        n = logits.shape[1]
        return S.constrain_logits(
            logits, history=self.history, history_len=self.history_len, prompt_len=self.prompt_len,
            drafts=drafts, bias=self.bias, mask=self.mask,
            mask_rows=self.mask_rows[:, first:first + n].contiguous(), mask_value=-1e4,
            error_word=self.error, **self.penalties)

    def round(self):
        B, K = self.B, self.K
        for c in self.contexts:
            c.plan(K + 1, self.accepted)
        served = torch.stack([c.state["len"] > c.state["start"] for c in self.contexts]).all(0)
        # drafting: each token's constraints count the drafts before it as said
        said = self.history.clone()
        rows, drafts, token = [], [], self.last
        for i in range(K + 1):
            raw = self.drafter_full.logits(token[:, None], first=i)
            at = torch.arange(said.shape[1], device="cuda") == (self.history_len + (i - 1))[:, None]
            if i > 0:
                said = torch.where(at, token[:, None], said)
            row = S.constrain_logits(raw, history=said, history_len=self.history_len + i,
                                     prompt_len=self.prompt_len, bias=self.bias, mask=self.mask,
                                     mask_rows=self.mask_rows[:, i:i + 1].contiguous(), mask_value=-1e4,
                                     error_word=self.error, **self.penalties)
            rows.append(row)
            if i < K:
                token, _ = A.draft_tokens(row[:, 0].contiguous())
                drafts.append(token)
        drafts = torch.stack(drafts, 1)
        inputs = torch.cat([self.last[:, None], drafts], 1)
        full = torch.cat(rows, 1)
        comp = self.constrained(self.drafter_comp.logits(inputs), drafts)
        ver = self.constrained(self.verifier.logits(inputs), drafts)
        r = self.step(full, comp, ver, drafts)
        # a request that a context had no blocks for sits the round out: nothing of it is kept
        self.accepted = torch.where(served, r["accept_len"], -1)
        next_token = torch.where(served, r["next_token"], self.last)
        # the accepted drafts and the next token join the history
        j = torch.arange(K + 1, device="cuda")
        new = torch.where(j < self.accepted[:, None], torch.cat([drafts, drafts[:, :1]], 1), next_token[:, None])
        at = (self.history_len[:, None] + j).clamp(max=self.history.shape[1] - 1).long()
        kept = self.history.gather(1, at)
        self.history.scatter_(1, at, torch.where(j <= self.accepted[:, None], new, kept))
        self.history_len = self.history_len + self.accepted + 1
        self.last = next_token
        return r["error_word"]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--rounds", type=int, default=16)
    a = ap.parse_args()
    loop = Loop(B=a.requests, K=a.drafts, rounds=a.rounds)
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    for _ in range(a.rounds):
        step |= loop.round()
    loop.raise_errors(step)
    said = loop.history_len - loop.prompt_len
    print("tokens committed per request:", said.tolist(), "in", a.rounds, "rounds")
    print("request 0:", loop.history[0, int(loop.prompt_len[0]):int(loop.history_len[0])].tolist())


if __name__ == "__main__":
    main()

"""The operators around the verification step, as cases that can be timed and compared.

Between two calls of the step a serving loop does four things on the GPU, none of which
needs the host to read anything back:

  constrain  penalties for repeated tokens, biases and grammar masks on the logits of every
             position of a round (position k has the history and the drafts before k);
  plan       block tables and slot maps of a paged key-value cache from the requests' lengths
             and the accepted lengths of the round before: blocks taken from and given back
             to the pool;
  write      keys and values of the new tokens into the cache at their slots;
  attend     attention of one or a few new tokens of each request over its cached tokens.

``run`` computes a case by elementary torch operations in 32 bits, or, where ``own`` is set,
by the package's kernels.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
ELT = {"fp32": 4, "bf16": 2}


# ---------------------------------------------------------------- cases

def _constrain(name, B, P, V, dtype, hist, masked, biased, pad=0, low=0.0):
    """hist: the longest history (they are spread from 1 to it); masked: the share of rows
    under a grammar mask; biased: bias entries of each request; pad: extra entries per row;
    low: what a masked logit becomes (0: the type's lowest value)."""
    return dict(name=name, kind="constrain", B=B, P=P, V=V, dtype=dtype, hist=hist, masked=masked,
                biased=biased, pad=pad, low=low)


def _plan(name, B, P, block, longest, mode, scarce=False):
    """mode "round": P tokens more for every request after a verified round; "admit": a third
    of the requests start with a prompt of up to `longest` tokens, a third end, a third go on."""
    return dict(name=name, kind="plan", B=B, P=P, block=block, longest=longest, mode=mode,
                scarce=scarce)


def _write(name, T, kv_heads, D, dtype, block, layout):
    return dict(name=name, kind="write", T=T, kv_heads=kv_heads, D=D, dtype=dtype, block=block,
                layout=layout)


def _attend(name, B, Q, heads, kv_heads, D, dtype, block, shortest, longest, layout="nhd",
            window=0, ended=0):
    return dict(name=name, kind="attend", B=B, Q=Q, heads=heads, kv_heads=kv_heads, D=D,
                dtype=dtype, block=block, shortest=shortest, longest=longest, layout=layout,
                window=window, ended=ended)


def listed():
    return [
        # one request, fp32: a round of four drafts and the bonus position, a short chat
        _constrain("constrain-1x5-fp32", 1, 5, 32000, "fp32", 700, 0.0, 8),
        # a full batch: histories up to a few thousand tokens, half of the rows under a grammar
        _constrain("constrain-64x8-bf16", 64, 8, 128256, "bf16", 8192, 0.5, 16),
        # agents with long transcripts, every answer structured
        _constrain("constrain-32x9-long-bf16", 32, 9, 151936, "bf16", 65536, 1.0, 0),
        # a vocabulary that no vector divides (added tokens), one drafted position at a time
        _constrain("constrain-64x1-odd-bf16", 64, 1, 100003, "bf16", 4096, 0.25, 300, low=-10000.0),
        # between two rounds of a full batch: the rejected tail is given up, K + 1 slots more
        _plan("plan-64x8-round", 64, 8, 16, 32768, "round"),
        # continuous batching: prompts admitted, finished requests give their blocks back
        _plan("plan-256-admit", 256, 8, 16, 8192, "admit"),
        # the new tokens of a round
        _write("write-512-bf16", 512, 8, 128, "bf16", 16, "nhd"),
        # a prompt's chunk, heads outside the tokens of a block
        _write("write-16384-bf16", 16384, 8, 128, "bf16", 32, "hnd"),
        # one request drafting: one token, a short context (latency)
        _attend("attend-1x1-bf16", 1, 1, 16, 8, 128, "bf16", 16, 1000, 1000),
        # a drafted position of a full batch, ragged contexts, two requests just ended
        _attend("attend-64x1-bf16", 64, 1, 32, 8, 128, "bf16", 16, 64, 8192, ended=2),
        # verification of K = 7 drafts over agents' long contexts
        _attend("attend-16x8-long-bf16", 16, 8, 32, 8, 128, "bf16", 32, 4096, 131072),
        # fp32, no shared heads, a sliding window, heads outside the tokens of a block
        _attend("attend-32x5-window-fp32", 32, 5, 8, 8, 64, "fp32", 48, 100, 16384, "hnd",
                window=2000),
    ]


LARGEST_BYTES = 2.0e9  # cached bytes that a drawn attention reads at most
LARGEST_FLOPS = 6.0e10


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("constrain", "plan", "write", "attend"), (3, 2, 1, 4))[0]
    dtype = rng.choices(("bf16", "fp32"), (2, 1))[0]
    if kind == "constrain":
        V, P = _log_uniform(rng, 32000, 151936), rng.randint(1, 9)
        V = V // 64 * 64 if rng.random() < 2 / 3 else V
        most = min(64, int(64 * 8 * 128256 * 2 / (P * V * ELT[dtype])))
        c = _constrain("", _log_uniform(rng, 1, most), P, V, dtype, _log_uniform(rng, 1, 65536),
                       rng.choice((0.0, 0.25, 0.5, 1.0)), rng.choice((0, 1, 16, 300)),
                       rng.choice((0, 0, 64, 5)), rng.choice((0.0, -10000.0, -100.0)))
    elif kind == "plan":
        mode = rng.choice(("round", "admit"))
        c = _plan("", _log_uniform(rng, 1, 1024), rng.randint(1, 9), rng.choice((8, 16, 24, 64)),
                  _log_uniform(rng, 64, 32768 if mode == "round" else 8192), mode,
                  rng.random() < 0.25)
    elif kind == "write":
        c = _write("", _log_uniform(rng, 1, 16384), rng.choice((1, 2, 4, 8)), rng.choice((64, 96, 128)),
                   dtype, rng.choice((8, 16, 24, 64)), rng.choice(("nhd", "hnd")))
    else:
        kv, G = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 8))
        Q = 1 if rng.random() < 0.5 else rng.randint(2, 9)
        D = rng.choice((64, 96, 128))
        longest = _log_uniform(rng, 16, 131072)
        key_bytes, key_flops = 2 * kv * D * ELT[dtype], 4 * Q * kv * G * D
        tokens = min(LARGEST_BYTES / key_bytes, LARGEST_FLOPS / key_flops)
        B = _log_uniform(rng, 1, max(1, min(64, int(tokens / longest))))
        c = _attend("", B, Q, kv * G, kv, D, dtype, rng.choice((8, 16, 24, 64)),
                    min(longest, _log_uniform(rng, Q, max(Q, longest))), longest,
                    rng.choice(("nhd", "hnd")), rng.choice((0, 0, 0, _log_uniform(rng, 16, 4096))),
                    1 if B > 8 and rng.random() < 0.5 else 0)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def _spread(n, lo, hi):
    """n whole numbers from lo to hi, even over their logarithm, the last of them hi."""
    lo = max(1, min(lo, hi))
    return [round(lo * (hi / lo) ** (i / (n - 1))) if n > 1 else hi for i in range(n)]


def _permuted(values, gen, dtype=torch.int32):
    order = torch.randperm(len(values), generator=gen, device="cuda")
    return torch.tensor(values, dtype=dtype, device="cuda")[order]


def _ints(lo, hi, shape, gen):
    """Whole numbers in [lo, hi]."""
    return torch.randint(lo, hi + 1, shape, generator=gen, device="cuda", dtype=torch.int32)


def _normal(shape, gen, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _cache(case, blocks, gen):
    """A pool of `blocks` blocks, seen as [blocks, block, kv_heads, D] whatever its layout."""
    n, h, d, dt = case["block"], case["kv_heads"], case["D"], DTYPE[case["dtype"]]
    if case["layout"] == "hnd":
        return torch.randn(blocks, h, n, d, generator=gen, device="cuda", dtype=dt).transpose(1, 2)
    return torch.randn(blocks, n, h, d, generator=gen, device="cuda", dtype=dt)


def _constrain_inputs(case, gen):
    B, P, V, n = case["B"], case["P"], case["V"], case["hist"]
    x = {}
    # a language model's next-token logits: a few tokens hold most of the mass
    u = torch.rand(B, P, V + case["pad"], generator=gen, device="cuda")
    x["logits"] = u.mul_(V).add_(1.0).log_().mul_(-2.5).add_(12.0).to(DTYPE[case["dtype"]])[..., :V]
    # text repeats itself: token ids of a history are heavy-tailed
    x["history"] = (V * torch.rand(B, n, generator=gen, device="cuda") ** 3).int().clamp_(max=V - 1)
    x["history_len"] = _permuted(_spread(B, 1, n), gen)
    x["prompt_len"] = (x["history_len"] * torch.rand(B, generator=gen, device="cuda")).int()
    x["drafts"] = _ints(0, V - 1, (B, P - 1), gen) if P > 1 else None
    r = torch.rand(3, B, generator=gen, device="cuda")
    x["repetition"], x["frequency"], x["presence"] = 1.0 + 0.5 * r[0], 1.5 * r[1], 1.5 * r[2]
    if case["biased"]:
        m = case["biased"]
        x["bias_offsets"] = torch.arange(0, B * m + 1, m, device="cuda", dtype=torch.int32)
        # one entry in each m-th of the vocabulary: no token twice
        step = V // m
        tok = torch.arange(m, device="cuda", dtype=torch.int32) * step + _ints(0, step - 1, (B, m), gen)
        x["bias_tokens"] = tok.reshape(-1)
        x["bias_values"] = 10.0 * torch.randn(B * m, generator=gen, device="cuda")
    rows = B * P
    masks = round(case["masked"] * rows)
    if masks:
        # every other grammar allows few tokens, the others most
        w = _ints(-2 ** 31, 2 ** 31 - 2, (2, masks, (V + 31) // 32), gen)
        few = torch.arange(masks, device="cuda")[:, None] % 2 == 0
        few_words = w[0] & w[1] & w[0].roll(1, 1) & w[1].roll(3, 1) & w[0].roll(5, 1)
        x["mask"] = torch.where(few, few_words, w[0] | w[1] | w[0].roll(1, 1))
        at = _permuted(list(range(masks)) + [-1] * (rows - masks), gen)
        x["mask_rows"] = at.view(B, P)
    return x


def _plan_lengths(case):
    """Of each request: tokens cached, drafts accepted (-1: its data was bad), tokens more, blocks held."""
    B, P, bs, n = case["B"], case["P"], case["block"], case["longest"]
    up = lambda t: -(-t // bs)  # noqa: E731
    lens = _spread(B, 16, n)
    if case["mode"] == "round":
        return [(t, 7 * i % (P + 1) - 1, P, up(t + P)) for i, t in enumerate(lens)]
    return [(0, -1, t, 0) if i % 3 == 0 else (0, -1, 0, up(t)) if i % 3 == 1 else (t, -1, 1, up(t))
            for i, t in enumerate(lens)]


def _plan_moved(case):
    """Blocks that each request takes (or, negative, gives back)."""
    return [-(-(t + a + 1 + g) // case["block"]) - h for t, a, g, h in _plan_lengths(case)]


def _plan_inputs(case, gen):
    B, P, bs = case["B"], case["P"], case["block"]
    order = torch.randperm(B, generator=gen, device="cuda")
    lens, accepted, grow, held = torch.tensor(_plan_lengths(case), dtype=torch.int32,
                                              device="cuda")[order].T.contiguous()
    x = dict(lens=lens, held=held, accepted=None, grow=None)
    if case["mode"] == "round":
        x["accepted"] = accepted
    else:
        x["grow"] = grow
    width = -(-(case["longest"] + 2 * P + 1) // bs)
    taken = sum(h for *_, h in _plan_lengths(case))
    wanted = sum(max(0, m) for m in _plan_moved(case))
    spare = wanted // 2 if case["scarce"] else wanted + 64
    ids = torch.randperm(taken + spare, generator=gen, device="cuda", dtype=torch.int32)
    x["tables"] = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    filled = torch.arange(width, device="cuda") < held[:, None]
    x["tables"][filled] = ids[:taken]
    x["free_list"] = torch.full((taken + spare,), -1, dtype=torch.int32, device="cuda")
    x["free_list"][:spare] = ids[taken:]
    x["free_count"] = torch.tensor([spare], dtype=torch.int32, device="cuda")
    x["capacity"] = B * P if case["mode"] == "round" else sum(g for _, _, g, _ in _plan_lengths(case)) + 100
    return x


def _write_inputs(case, gen):
    T, h, d, bs = case["T"], case["kv_heads"], case["D"], case["block"]
    blocks = -(-T // bs) + 32
    # keys and values as a projection leaves them, side by side
    kv = _normal((T, 2, h, d), gen, DTYPE[case["dtype"]])
    slots = torch.randperm(blocks * bs, generator=gen, device="cuda")[:T]
    slots[torch.rand(T, generator=gen, device="cuda") < 0.05] = -1  # padding of a captured batch
    return dict(k=kv[:, 0], v=kv[:, 1], slots=slots, key_cache=_cache(case, blocks, gen),
                value_cache=_cache(case, blocks, gen))


def _attend_lengths(case):
    n = case["B"] - case["ended"]
    return _spread(n, max(case["shortest"], case["Q"]), case["longest"]) + [0] * case["ended"]


def _attend_inputs(case, gen):
    B, Q, bs, d = case["B"], case["Q"], case["block"], case["D"]
    lens = _permuted(_attend_lengths(case), gen)
    width = -(-max(case["longest"], Q) // bs)
    pages = (lens + bs - 1) // bs
    total = sum(-(-t // bs) for t in _attend_lengths(case))
    blocks = total + 16
    tables = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    ids = torch.randperm(blocks, generator=gen, device="cuda", dtype=torch.int32)
    tables[torch.arange(width, device="cuda") < pages[:, None]] = ids[:total]
    # queries as a projection leaves them, with the new keys and values beside them;
    # scores a few nats apart, as trained heads have them
    qkv = _normal((B, Q, (case["heads"] + 2 * case["kv_heads"]) * d), gen, DTYPE[case["dtype"]], 2.0)
    q = qkv[..., :case["heads"] * d].unflatten(-1, (case["heads"], d))
    return dict(q=q, key_cache=_cache(case, blocks, gen), value_cache=_cache(case, blocks, gen),
                tables=tables, lens=lens)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"constrain": _constrain_inputs, "plan": _plan_inputs, "write": _write_inputs,
            "attend": _attend_inputs}[case["kind"]](case, gen)


def prepare(case, seed):
    return dict(case=case, x=_inputs(case, seed))


# ---------------------------------------------------------------- one pass, plain

def _constrain_plain(case, x):
    B, P, V, dev = case["B"], case["P"], case["V"], x["logits"].device
    n = x["history"].shape[1]
    at = torch.arange(n, device=dev)
    live, out = at < x["history_len"][:, None], at >= x["prompt_len"][:, None]
    tok = x["history"].long()
    prompt = torch.zeros(B, V, device=dev).scatter_add_(1, tok, (live & ~out).float()) > 0
    count = torch.zeros(B, V, device=dev).scatter_add_(1, tok, (live & out).float())
    count = count[:, None].expand(B, P, V).contiguous()
    if P > 1:  # position k has the drafts before it
        before = torch.ones(P, P - 1, device=dev).tril_(-1).expand(B, P, P - 1)
        count.scatter_add_(2, x["drafts"].long()[:, None].expand(B, P, P - 1).contiguous(), before)
    z = x["logits"].float()
    f = lambda v: v[:, None, None]  # noqa: E731
    rep = f(x["repetition"])
    y = torch.where(prompt[:, None] | (count > 0), torch.where(z > 0, z / rep, z * rep), z)
    y = y - f(x["frequency"]) * count - f(x["presence"]) * (count > 0)
    if case["biased"]:
        b = torch.zeros(B, V, device=dev)
        row = torch.arange(B, device=dev).repeat_interleave(case["biased"])
        b[row, x["bias_tokens"].long()] = x["bias_values"]
        y = y + b[:, None]
    low = torch.finfo(x["logits"].dtype).min
    y = torch.where(z.isfinite(), y.clamp(low, -low), y)  # a finite logit stays finite
    if "mask" in x:
        v = torch.arange(V, device=dev)
        allowed = (x["mask"][:, v // 32] >> (v % 32)) & 1 != 0
        allowed = allowed[x["mask_rows"].long().clamp(min=0)] | (x["mask_rows"] < 0)[..., None]
        y = torch.where(allowed, y, case["low"] or low)
    return y.to(x["logits"].dtype)


def _plan_plain(case, x):
    bs, dev, tables = case["block"], x["lens"].device, x["tables"]
    B, width = tables.shape
    keep = x["lens"] if x["accepted"] is None else x["lens"] + x["accepted"] + 1
    grow = x["grow"] if x["grow"] is not None else torch.full_like(keep, case["P"])
    blocks = (keep + grow + bs - 1) // bs
    more = (blocks - x["held"]).clamp(min=0)
    less = (x["held"] - blocks).clamp(min=0)
    top = x["free_count"] + less.sum()
    upto = more.cumsum(0)
    served = (more == 0) | (upto <= top)
    more = torch.where(served, more, 0)
    # blocks given back go on the stack in the order of the requests, then blocks are taken off it
    j = torch.arange(width, device=dev)
    back = (j >= blocks[:, None]) & (j < x["held"][:, None])
    at = x["free_count"] + (less.cumsum(0) - less)[:, None] + j - blocks[:, None]
    x["free_list"][at[back].long()] = tables[back]
    new = (j >= x["held"][:, None]) & (j < blocks[:, None]) & served[:, None]
    at = top - 1 - (more.cumsum(0) - more)[:, None] - (j - x["held"][:, None])
    tables[new] = x["free_list"][at[new].long()]
    offsets = torch.zeros(B + 1, dtype=torch.int32, device=dev)
    offsets[1:] = grow.cumsum(0)
    t = torch.arange(x["capacity"], device=dev, dtype=torch.int32)
    b = torch.searchsorted(offsets[1:], t, right=True).clamp(max=B - 1)
    position = keep[b] + t - offsets[b]
    live = (t < offsets[-1]) & served[b]
    page = tables[b, (position // bs).clamp(max=width - 1).long()].long()
    slots = torch.where(live, page * bs + position % bs, -1)
    return dict(start=keep, len=torch.where(served, keep + grow, keep),
                held=torch.where(served, blocks, x["held"]),
                free_count=(top - more.sum()).int(), offsets=offsets, slots=slots,
                positions=torch.where(live, position, -1), tables=tables, free_list=x["free_list"])


def _write_plain(case, x):
    t = (x["slots"] >= 0).nonzero()[:, 0]
    page, at = x["slots"][t] // case["block"], x["slots"][t] % case["block"]
    x["key_cache"][page, at] = x["k"][t]
    x["value_cache"][page, at] = x["v"][t]
    return x["key_cache"], x["value_cache"]


def _attend_plain(case, x):
    B, Q, h, d, bs = case["B"], case["Q"], case["kv_heads"], case["D"], case["block"]
    dev = x["q"].device
    n = case["longest"]
    j = torch.arange(n, device=dev)
    page, at = x["tables"][:, j // bs].clamp(min=0).long(), j % bs
    live = (j < x["lens"][:, None])[..., None, None]
    k = x["key_cache"][page, at].float().masked_fill_(~live, 0.0)
    v = x["value_cache"][page, at].float().masked_fill_(~live, 0.0)
    q = x["q"].float().view(B, Q, h, -1, d) / math.sqrt(d)
    s = torch.einsum("bqhgd,bnhd->bhgqn", q, k)
    own_at = (x["lens"][:, None] - Q + torch.arange(Q, device=dev))[..., None]
    seen = (j <= own_at) & (j > own_at - (case["window"] or 2 ** 30))
    s.masked_fill_(~seen[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True).clamp_(min=torch.finfo(torch.float32).min)
    p = (s - m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.einsum("bhgqn,bnhd->bqhgd", p, v)
    o = o / total.permute(0, 3, 1, 2, 4).clamp(min=torch.finfo(torch.float32).tiny)
    lse = (total.log() + m).squeeze(-1).permute(0, 3, 1, 2)
    return o.reshape(B, Q, -1, d).to(x["q"].dtype), lse.reshape(B, Q, -1)


# ---------------------------------------------------------------- one pass

def run(state):
    case, x, kind = state["case"], state["x"], state["case"]["kind"]
    if not own:
        return {"constrain": _constrain_plain, "plan": _plan_plain, "write": _write_plain,
                "attend": _attend_plain}[kind](case, x)
    from paper_2608_26004_gb300 import serving as S
    if kind == "constrain":
        bias = (x["bias_offsets"], x["bias_tokens"], x["bias_values"]) if case["biased"] else None
        return S.constrain_logits(
            x["logits"], history=x["history"], history_len=x["history_len"],
            prompt_len=x["prompt_len"], drafts=x["drafts"], repetition=x["repetition"],
            frequency=x["frequency"], presence=x["presence"], bias=bias, mask=x.get("mask"),
            mask_rows=x.get("mask_rows"), mask_value=case["low"] or None)
    if kind == "plan":
        r = S.cache_plan(x["lens"], x["tables"], x["held"], x["free_list"], x["free_count"],
                         block_size=case["block"], accepted=x["accepted"],
                         grow=case["P"] if x["grow"] is None else x["grow"],
                         capacity=x["capacity"])
        return dict(r, tables=x["tables"], free_list=x["free_list"])
    if kind == "write":
        S.cache_write(x["k"], x["v"], x["key_cache"], x["value_cache"], x["slots"])
        return x["key_cache"], x["value_cache"]
    if "attend" not in state:  # the workspace that a serving loop keeps
        state["attend"] = S.CacheAttend(case["B"], case["Q"], case["heads"], case["kv_heads"], case["D"])
    return state["attend"](x["q"], x["key_cache"], x["value_cache"], x["tables"], x["lens"],
                           window=case["window"])


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "constrain":
        rows = case["B"] * case["P"]
        masks, hist = round(case["masked"] * rows), sum(_spread(case["B"], 1, case["hist"]))
        small = case["B"] * (20 + 8 * case["biased"] + 4 * case["P"])
        return {"bytes": 2 * rows * case["V"] * ELT[case["dtype"]] + masks * ((case["V"] + 31) // 32) * 4
                + 4 * hist + small, "flops": 4 * rows * case["V"]}
    if case["kind"] == "plan":
        moved = sum(abs(m) for m in _plan_moved(case))
        tokens = sum(g for _, _, g, _ in _plan_lengths(case))
        return {"bytes": case["B"] * 28 + 8 * moved + 16 * tokens, "flops": 8 * tokens + 8 * case["B"]}
    if case["kind"] == "write":
        n = case["T"] * case["kv_heads"] * case["D"]
        return {"bytes": 4 * n * ELT[case["dtype"]] + 8 * case["T"], "flops": 0}
    Q, d, elt = case["Q"], case["D"], ELT[case["dtype"]]
    keys = [min(t, case["window"] + Q - 1) if case["window"] else t for t in _attend_lengths(case)]
    rows = case["B"] * Q * case["heads"]
    return {"bytes": 2 * sum(keys) * case["kv_heads"] * d * elt + rows * (2 * d * elt + 4)
            + 4 * sum(-(-t // case["block"]) for t in keys) + 4 * case["B"],
            "flops": 4 * sum(keys) * Q * case["heads"] * d}


# ---------------------------------------------------------------- the same in 64 bits

def _constrain_exact(case, x):
    B, P, V = case["B"], case["P"], case["V"]
    low = torch.finfo(x["logits"].dtype).min
    rows = []
    for b in range(B):
        n, m = int(x["history_len"][b]), int(x["prompt_len"][b])
        past = x["history"][b, :n].long()
        base = torch.bincount(past[m:], minlength=V)
        in_prompt = torch.bincount(past[:m], minlength=V) > 0
        rep, freq, pres = (float(x[k][b]) for k in ("repetition", "frequency", "presence"))
        for k in range(P):
            y = x["logits"][b, k].double()
            c = base + torch.bincount(x["drafts"][b, :k].long(), minlength=V) if k else base
            seen = (c > 0) | in_prompt
            y[seen & (y > 0)] /= rep
            y[seen & (x["logits"][b, k] <= 0)] *= rep
            y -= freq * c + pres * (c > 0)
            if case["biased"]:
                i, e = (int(v) for v in x["bias_offsets"][b:b + 2])
                y[x["bias_tokens"][i:e].long()] += x["bias_values"][i:e].double()
            y.clamp_(low, -low)
            at = int(x["mask_rows"][b, k]) if "mask" in x else -1
            if at >= 0:
                bits = (x["mask"][at][:, None] >> torch.arange(32, device=y.device)) & 1
                y[bits.reshape(-1)[:V] == 0] = case["low"] or low
            rows.append(y)
    return torch.stack(rows).view(B, P, V)


def _attend_exact(case, x):
    Q, bs, d, g = case["Q"], case["block"], case["D"], case["heads"] // case["kv_heads"]
    out, lse = [], []
    for b in range(case["B"]):
        n = int(x["lens"][b])
        o = torch.zeros(Q, case["heads"], d, dtype=torch.float64, device="cuda")
        l = torch.full((Q, case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
        if n:
            t = x["tables"][b, :-(-n // bs)].long()
            for h in range(case["kv_heads"]):
                k = x["key_cache"][t, :, h].reshape(-1, d)[:n].double()
                v = x["value_cache"][t, :, h].reshape(-1, d)[:n].double()
                for i in range(Q):
                    last = n - Q + i
                    first = max(0, last - case["window"] + 1) if case["window"] else 0
                    s = x["q"][b, i, h * g:(h + 1) * g].double() @ k[first:last + 1].T / math.sqrt(d)
                    l[i, h * g:(h + 1) * g] = s.logsumexp(-1)
                    o[i, h * g:(h + 1) * g] = s.softmax(-1) @ v[first:last + 1]
        out.append(o)
        lse.append(l)
    return torch.stack(out), torch.stack(lse)


def exact(case, seed):
    if case["kind"] not in ("constrain", "attend"):
        return None  # whole numbers and copies
    x = _inputs(case, seed)
    return (_constrain_exact if case["kind"] == "constrain" else _attend_exact)(case, x)

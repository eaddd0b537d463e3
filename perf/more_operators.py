"""Rotary positions and a key-value cache held in 4 bits, as cases that can be timed and compared.

What a serving loop does with a token's queries, keys and values before and in its attention:

  rotary  queries and keys turned by their positions: the halves of a head or neighbouring
          elements as pairs, the whole head or its first part, frequencies stretched for long
          contexts; and the transpose, which is the gradient;
  store   new keys and values written into a paged cache of 4 bits (16 elements of a head share a
          scale of 8 bits), and read back as the attention will see them;
  read    cached tokens read back at their slots (a context that is moved or compressed);
  attend  attention of one or a few new tokens of each request over its cached ones.

``run`` computes a case by elementary torch operations in 32 bits (angles in 64), or, where
``own`` is set, by the package's kernels.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
ELT = {"fp32": 4, "bf16": 2}
GROUP = 16  # elements of a head that share a scale


# ---------------------------------------------------------------- cases

def _rotary(name, T, heads, kv_heads, D, dtype, longest, rot=0, interleaved=False, scaling="none",
            factor=1.0, inverse=False, padding=0.0):
    """rot: elements of a head that are turned (0: all); scaling: how the frequencies are
    stretched by `factor`; padding: the share of tokens without a position (-1)."""
    return dict(name=name, kind="rotary", T=T, heads=heads, kv_heads=kv_heads, D=D, dtype=dtype,
                longest=longest, rot=rot or D, interleaved=interleaved, scaling=scaling,
                factor=factor, inverse=inverse, padding=padding)


def _store(name, T, kv_heads, D, dtype, block, layout, key_scale=1.0, value_scale=1.0):
    return dict(name=name, kind="store", T=T, kv_heads=kv_heads, D=D, dtype=dtype, block=block,
                layout=layout, key_scale=key_scale, value_scale=value_scale)


def _read(name, T, kv_heads, D, dtype, block, layout, key_scale=1.0, value_scale=1.0):
    return dict(_store(name, T, kv_heads, D, dtype, block, layout, key_scale, value_scale), kind="read")


def _attend(name, B, Q, heads, kv_heads, D, dtype, block, shortest, longest, layout="hnd", window=0,
            ended=0, key_scale=1.0, value_scale=1.0):
    return dict(name=name, kind="attend", B=B, Q=Q, heads=heads, kv_heads=kv_heads, D=D, dtype=dtype,
                block=block, shortest=shortest, longest=longest, layout=layout, window=window,
                ended=ended, key_scale=key_scale, value_scale=value_scale)


def listed():
    return [
        # one request's round of four drafts and the bonus position, a short chat (latency)
        _rotary("rotary-5-bf16", 5, 16, 8, 128, "bf16", 1000),
        # a full batch's round, part of each head turned, neighbouring elements, a captured
        # batch's padding
        _rotary("rotary-512-part-fp32", 512, 16, 4, 96, "fp32", 32768, rot=64, interleaved=True,
                padding=0.1),
        # a chunk of prompts behind long contexts, frequencies stretched past the trained length
        _rotary("rotary-16384-long-bf16", 16384, 32, 8, 128, "bf16", 500000, scaling="ramp", factor=8.0),
        # the gradient of a drafter's training batch
        _rotary("rotary-4099-gradient-bf16", 4099, 32, 8, 64, "bf16", 8192, scaling="wavelength",
                factor=4.0, inverse=True),
        # the new tokens of one round of a full batch
        _store("store-512-bf16", 512, 8, 128, "bf16", 16, "hnd"),
        # a prompt's chunk, heads inside the tokens of a block, scales set for small values
        _store("store-16384-bf16", 16384, 8, 128, "bf16", 32, "nhd", 0.25, 0.0625),
        # a short context's tokens, fp32 out, a head size and block size of their own
        _read("read-1500-fp32", 1500, 2, 96, "fp32", 24, "nhd", 0.5, 0.5),
        # long contexts moved: what a compressed context keeps of a full one
        _read("read-100003-bf16", 100003, 8, 128, "bf16", 16, "hnd"),
        # one request drafting: one token, a short context (latency)
        _attend("attend4-1x1-bf16", 1, 1, 16, 8, 128, "bf16", 16, 1000, 1000),
        # a drafted position of a full batch, ragged contexts, two requests just ended
        _attend("attend4-64x1-bf16", 64, 1, 32, 8, 128, "bf16", 16, 64, 8192, ended=2),
        # verification of K = 7 drafts over agents' long contexts
        _attend("attend4-16x8-long-bf16", 16, 8, 32, 8, 128, "bf16", 32, 4096, 131072),
        # fp32, no shared heads, a sliding window, heads inside the tokens of a block
        _attend("attend4-32x5-window-fp32", 32, 5, 8, 8, 64, "fp32", 48, 100, 16384, "nhd", window=2000,
                value_scale=0.25),
    ]


LARGEST_BYTES = 7.0e8  # cached bytes that a drawn attention reads at most
LARGEST_FLOPS = 6.0e10
LARGEST_ELEMENTS = 8.0e7  # of a drawn rotary's queries and keys
LARGEST_TOKENS = 1.0e8    # elements of keys that a drawn store or read moves


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("rotary", "store", "read", "attend"), (3, 2, 1, 4))[0]
    dtype = rng.choices(("bf16", "fp32"), (2, 1))[0]
    scales = rng.choice((1.0, 0.5, 0.0625)), rng.choice((1.0, 0.25, 0.046875))
    block, layout = rng.choice((8, 16, 24, 32, 64)), rng.choice(("nhd", "hnd"))
    if kind == "rotary":
        kv, G, D = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 8)), rng.choice((64, 80, 96, 128, 256))
        most = min(16384, int(LARGEST_ELEMENTS / ((kv * G + kv) * D * ELT[dtype] / 2)))
        rot = D if rng.random() < 0.5 else rng.choice((D // 4, D // 2, D * 3 // 4)) // 2 * 2
        c = _rotary("", _log_uniform(rng, 1, most), kv * G, kv, D, dtype, _log_uniform(rng, 64, 1000000),
                    rot, rng.random() < 0.4, rng.choice(("none", "linear", "base", "ramp", "wavelength")),
                    rng.choice((2.0, 4.0, 8.0, 32.0)), rng.random() < 0.3, rng.choice((0.0, 0.0, 0.1, 0.5)))
    elif kind in ("store", "read"):
        kv, D = rng.choice((1, 2, 4, 8)), rng.choice((64, 96, 128, 256))
        most = min(16384 if kind == "store" else 131072, int(LARGEST_TOKENS / (kv * D)))
        c = (_store if kind == "store" else _read)("", _log_uniform(rng, 1, most), kv, D, dtype, block, layout,
                                                   *scales)
    else:
        kv, G = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 8))
        Q = 1 if rng.random() < 0.5 else rng.randint(2, 9)
        D = rng.choice((64, 96, 128, 128, 256))
        longest = _log_uniform(rng, 16, 131072)
        key_bytes, key_flops = 2 * kv * D * 0.5625, 4 * Q * kv * G * D
        tokens = min(LARGEST_BYTES / key_bytes, LARGEST_FLOPS / key_flops)
        B = _log_uniform(rng, 1, max(1, min(64, int(tokens / longest))))
        c = _attend("", B, Q, kv * G, kv, D, dtype, block, min(longest, _log_uniform(rng, Q, max(Q, longest))),
                    longest, layout, rng.choice((0, 0, 0, _log_uniform(rng, 16, 4096))),
                    1 if B > 8 and rng.random() < 0.5 else 0, *scales)
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


def _normal(shape, gen, dtype, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def _channels(n, gen):
    """What a projection's channels come out as: most alike, some several times as large."""
    return torch.randn(n, generator=gen, device="cuda").mul_(0.5).exp_()


def _quantised(x, scale):
    """Codes [.., D / 2] and scales [.., D / 16] (bytes) of x [.., D]: of each 16 elements, s = e4m3
    of the largest magnitude over 6 scale, and e2m1 of x / (s scale), two in a byte, the first in its
    low bits.  Every operation is rounded to fp32 as it is written here."""
    y = x.float().unflatten(-1, (-1, GROUP))
    s = (y.abs().amax(-1) * (1.0 / (6.0 * scale))).clamp_(max=448.0).to(torch.float8_e4m3fn)
    step = s.float() * scale
    z = y * torch.where(step > 0, 1.0 / step, 0.0)[..., None]
    m = z.abs()
    # magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6; halfway to the even code
    c = (m > 0.25).to(torch.uint8)
    for more in (m >= 0.75, m > 1.25, m >= 1.75, m > 2.5, m >= 3.5, m > 5.0):
        c += more
    c = (c + 8 * torch.signbit(z)).to(torch.uint8).flatten(-2)
    return c[..., ::2] | (c[..., 1::2] << 4), s.view(torch.uint8)


def _values(codes, scales, scale):
    """What codes [.., D / 2] and scales [.., D / 16] stand for, in fp32."""
    level = torch.tensor((0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0), device=codes.device)
    level = torch.cat((level, -level))
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    s = scales.view(torch.float8_e4m3fn).float()
    return (level[c.int()].unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2) * scale


def _cache(case, blocks, gen):
    """A pool of `blocks` blocks of keys and values, each as codes and scales, seen as [blocks,
    block, kv_heads, ..] whatever its layout."""
    n, h, d = case["block"], case["kv_heads"], case["D"]
    out = {}
    for name, scale in (("key", case["key_scale"]), ("value", case["value_scale"])):
        width = {"codes": d // 2, "scales": d // GROUP}
        parts = {part: torch.empty((blocks, h, n, w) if case["layout"] == "hnd" else (blocks, n, h, w),
                                   dtype=torch.uint8, device="cuda") for part, w in width.items()}
        if case["layout"] == "hnd":
            parts = {part: x.transpose(1, 2) for part, x in parts.items()}
        channel = _channels((h, d), gen) * scale
        step = max(1, 2 ** 26 // (n * h * d))
        for i in range(0, blocks, step):
            m = min(step, blocks - i)
            x = torch.randn(m, n, h, d, generator=gen, device="cuda") * channel
            parts["codes"][i:i + m], parts["scales"][i:i + m] = _quantised(x, scale)
        out |= {f"{name}_{part}": x for part, x in parts.items()}
    return out


def _rotary_inputs(case, gen):
    T, h, hk, d = case["T"], case["heads"], case["kv_heads"], case["D"]
    # queries and keys as a projection leaves them, with the values behind them
    qkv = _normal((T, (h + 2 * hk) * d), gen, DTYPE[case["dtype"]])
    q = qkv[:, :h * d].unflatten(-1, (h, d))
    k = qkv[:, h * d:(h + hk) * d].unflatten(-1, (hk, d))
    # tokens of a few requests one after another, each from a position of its own on
    at = torch.arange(T, device="cuda")
    start = torch.randint(0, max(1, case["longest"] - T), (T // 64 + 1,), generator=gen, device="cuda")
    positions = (start[at // 64] + at % 64).int()
    positions[torch.rand(T, generator=gen, device="cuda") < case["padding"]] = -1
    return dict(q=q, k=k, positions=positions, q_out=torch.empty_like(q, memory_format=torch.contiguous_format),
                k_out=torch.empty_like(k, memory_format=torch.contiguous_format))


def _slots(T, total, gen):
    slots = torch.randperm(total, generator=gen, device="cuda")[:T]
    slots[torch.rand(T, generator=gen, device="cuda") < 0.05] = -1  # padding of a captured batch
    return slots


def _store_inputs(case, gen):
    T, h, d = case["T"], case["kv_heads"], case["D"]
    blocks = -(-T // case["block"]) + 32
    x = _cache(case, blocks, gen)
    # keys and values as a projection leaves them, side by side
    kv = torch.randn(T, 2, h, d, generator=gen, device="cuda") * _channels((2, h, d), gen)
    kv[:, 0] *= case["key_scale"]
    kv[:, 1] *= case["value_scale"]
    kv = kv.to(DTYPE[case["dtype"]])
    return dict(x, k=kv[:, 0], v=kv[:, 1], slots=_slots(T, blocks * case["block"], gen))


def _read_inputs(case, gen):
    blocks = -(-case["T"] // case["block"]) + 32
    return dict(_cache(case, blocks, gen), slots=_slots(case["T"], blocks * case["block"], gen))


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
    qkv = _normal((B, Q, (case["heads"] + 2 * case["kv_heads"]) * d), gen, DTYPE[case["dtype"]],
                  1.5 / case["key_scale"])
    q = qkv[..., :case["heads"] * d].unflatten(-1, (case["heads"], d))
    return dict(_cache(case, blocks, gen), q=q, tables=tables, lens=lens)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"rotary": _rotary_inputs, "store": _store_inputs, "read": _read_inputs,
            "attend": _attend_inputs}[case["kind"]](case, gen)


# what the scalings take beside their factor
RAMP = dict(original_length=4096, fast=32.0, slow=1.0)
WAVELENGTH = dict(original_length=8192, fast=4.0, slow=1.0)
BASE = 10000.0


def prepare(case, seed):
    return dict(case=case, x=_inputs(case, seed))


# ---------------------------------------------------------------- one pass, plain

def _frequencies(case):
    """Radians a position, fp64, of each pair; and what turned elements are multiplied by."""
    rot, kind, f = case["rot"], case["scaling"], case["factor"]
    base = BASE * f ** (rot / (rot - 2)) if kind == "base" and rot > 2 else BASE
    i = torch.arange(0, rot, 2, dtype=torch.float64, device="cuda")
    w = base ** (-i / rot)
    if kind == "linear":
        return w / f, 1.0
    if kind == "ramp":
        # pairs that turn more than `fast` times within the original length stay, those that turn
        # less than `slow` times are stretched, between them by the pair's index
        pair = lambda turns: rot * math.log(RAMP["original_length"] / (turns * 2 * math.pi)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(math.floor(pair(RAMP["fast"])), 0), min(math.ceil(pair(RAMP["slow"])), rot - 1)
        kept = 1.0 - ((i / 2 - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return w / f * (1.0 - kept) + w * kept, 0.1 * math.log(f) + 1.0
    if kind == "wavelength":
        # the same by the number of turns
        turns = WAVELENGTH["original_length"] * w / (2 * math.pi)
        kept = ((turns - WAVELENGTH["slow"]) / (WAVELENGTH["fast"] - WAVELENGTH["slow"])).clamp(0.0, 1.0)
        return w / f * (1.0 - kept) + w * kept, 1.0
    return w, 1.0


def _rotary_plain(case, x):
    w, magnitude = _frequencies(case)
    angle = x["positions"].double()[:, None] * w * (-1.0 if case["inverse"] else 1.0)
    c, s = (magnitude * angle.cos()).float()[:, None], (magnitude * angle.sin()).float()[:, None]
    rot, live = case["rot"], (x["positions"] >= 0)[:, None, None]
    for name in ("q", "k"):
        z, out = x[name], x[name + "_out"]
        y = z.float()
        if case["interleaved"]:
            a, b = y[..., :rot:2], y[..., 1:rot:2]
            turned = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
        else:
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            turned = torch.cat((a * c - b * s, a * s + b * c), -1)
        out[..., rot:] = z[..., rot:]
        out[..., :rot] = torch.where(live, turned.to(z.dtype), z[..., :rot])
    return x["q_out"], x["k_out"]


def _at(case, x, slots):
    return slots // case["block"], slots % case["block"]


def _read_plain(case, x):
    live = (x["slots"] >= 0)[:, None, None]
    page, at = _at(case, x, x["slots"].clamp(min=0))
    return tuple(torch.where(live, _values(x[n + "_codes"][page, at], x[n + "_scales"][page, at], case[n + "_scale"]),
                             0.0).to(DTYPE[case["dtype"]]) for n in ("key", "value"))


def _store_plain(case, x):
    t = (x["slots"] >= 0).nonzero()[:, 0]
    page, at = _at(case, x, x["slots"][t])
    for n in ("key", "value"):
        x[n + "_codes"][page, at], x[n + "_scales"][page, at] = _quantised(x[n[0]][t], case[n + "_scale"])
    return _read_plain(case, x)


def _attend_plain(case, x):
    B, Q, h, d = case["B"], case["Q"], case["kv_heads"], case["D"]
    dev = x["q"].device
    n = case["longest"]
    j = torch.arange(n, device=dev)
    page, at = x["tables"][:, j // case["block"]].clamp(min=0).long(), j % case["block"]
    live = (j < x["lens"][:, None])[..., None, None]
    k, v = (torch.empty(B, n, h, d, device=dev) for _ in range(2))
    for name, to in (("key", k), ("value", v)):
        for b in range(B):
            to[b] = _values(x[name + "_codes"][page[b], at], x[name + "_scales"][page[b], at], case[name + "_scale"])
        to.masked_fill_(~live, 0.0)
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

def _scaling(case):
    kind, f = case["scaling"], case["factor"]
    if kind == "none":
        return None
    return dict(kind=kind, factor=f, **(RAMP if kind == "ramp" else WAVELENGTH if kind == "wavelength" else {}))


def run(state):
    case, x, kind = state["case"], state["x"], state["case"]["kind"]
    if not own:
        return {"rotary": _rotary_plain, "store": _store_plain, "read": _read_plain,
                "attend": _attend_plain}[kind](case, x)
    from paper_2608_26004_gb300 import serving as S
    if kind == "rotary":
        if "rotary" not in state:  # the frequencies that a model keeps
            state["rotary"] = S.Rotary(case["D"], rotary_dim=case["rot"], base=BASE,
                                       interleaved=case["interleaved"], scaling=_scaling(case))
        return state["rotary"](x["q"], x["positions"], x["k"], transpose=case["inverse"], q_out=x["q_out"],
                               k_out=x["k_out"])
    if "cache" not in state:  # the view of the pool that a serving loop keeps
        state["cache"] = S.Cache4(x["key_codes"], x["key_scales"], x["value_codes"], x["value_scales"],
                                  key_scale=case["key_scale"], value_scale=case["value_scale"])
    if kind in ("store", "read"):
        if kind == "store":
            S.cache4_write(x["k"], x["v"], state["cache"], x["slots"])
        return S.cache4_read(state["cache"], x["slots"], dtype=DTYPE[case["dtype"]])
    if "attend" not in state:  # the workspace that a serving loop keeps
        state["attend"] = S.Cache4Attend(case["B"], case["Q"], case["heads"], case["kv_heads"], case["D"])
    return state["attend"](x["q"], state["cache"], x["tables"], x["lens"], window=case["window"])


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    d, elt = case["D"], ELT[case["dtype"]]
    if case["kind"] == "rotary":
        n = case["T"] * (case["heads"] + case["kv_heads"])
        return {"bytes": 2 * n * d * elt + 4 * case["T"], "flops": 3 * n * case["rot"]}
    packed = d // 2 + d // GROUP  # bytes of a head's keys, or values
    if case["kind"] in ("store", "read"):
        n = case["T"] * case["kv_heads"] * 2
        moved = n * (d * elt + packed) + 8 * case["T"]
        return {"bytes": 2 * moved if case["kind"] == "store" else moved,
                "flops": (5 if case["kind"] == "store" else 2) * n * d}
    Q = case["Q"]
    keys = [min(t, case["window"] + Q - 1) if case["window"] else t for t in _attend_lengths(case)]
    rows = case["B"] * Q * case["heads"]
    return {"bytes": 2 * sum(keys) * case["kv_heads"] * packed + rows * (2 * d * elt + 4)
            + 4 * sum(-(-t // case["block"]) for t in keys) + 4 * case["B"],
            "flops": 4 * sum(keys) * Q * case["heads"] * d}


# ---------------------------------------------------------------- the same in 64 bits

def _rotary_exact(case, x):
    w, magnitude = _frequencies(case)
    rot, out = case["rot"], []
    turn = torch.polar(torch.full_like(w, magnitude), w * 0.0)
    angle = torch.outer(x["positions"].double(), w)
    z = torch.polar(torch.ones_like(angle), -angle if case["inverse"] else angle) * turn
    z[x["positions"] < 0] = 1.0
    for name in ("q", "k"):
        y = x[name].double().clone()
        # pairs as complex numbers
        pairs = y[..., :rot].unflatten(-1, (-1, 2)) if case["interleaved"] \
            else y[..., :rot].unflatten(-1, (2, -1)).transpose(-1, -2)
        r = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z[:, None])
        y[..., :rot] = (r if case["interleaved"] else r.transpose(-1, -2)).flatten(-2)
        out.append(y)
    return tuple(out)


# values of codes and scales in 64 bits, from their bits: sign, exponent, fraction
_E2M1 = [(-1.0 if c & 8 else 1.0) * ((c & 1) * 0.5 if c & 6 == 0 else math.ldexp(2 + (c & 1), (c >> 1 & 3) - 2))
         for c in range(16)]
_E4M3 = [math.nan if c & 127 == 127 else (-1.0 if c & 128 else 1.0)
         * math.ldexp(c & 7 if c & 120 == 0 else 8 + (c & 7), max(c >> 3 & 15, 1) - 10) for c in range(256)]


def _power_of_two(x):
    """The largest power of two that is no larger than x (fp64, positive and normal)."""
    return (x.view(torch.int64) & (0x7FF << 52)).view(torch.float64)


def _stored_exact(x, scale):
    """What is read back of x [.., D]: the definition's four roundings to fp32 (of the largest magnitude
    over 6 scale, of the step, its reciprocal and the quotient), every product before one in 64 bits."""
    r32 = lambda t: t.float().double()  # noqa: E731
    y = x.double().unflatten(-1, (-1, GROUP))
    most = r32(y.abs().amax(-1) * float(torch.tensor(1.0 / (6.0 * scale), dtype=torch.float32)))
    # the nearest e4m3 value, halfway to the even one: multiples of 2^-9 up to 2^-6, then of an
    # eighth of the value's power of two
    unit = _power_of_two(most.clamp(min=2.0 ** -6)) / 8.0
    s = ((most / unit).round() * unit).clamp(max=448.0)
    step = r32(s * scale)
    z = r32(y * torch.where(step > 0, r32(1.0 / step), 0.0)[..., None]).clamp(-6.0, 6.0)
    # the nearest e2m1 value likewise
    unit = torch.where(z.abs() < 2.0, 0.5, torch.where(z.abs() < 4.0, 1.0, 2.0))
    return ((z / unit).round() * unit * s[..., None]).flatten(-2) * scale


def _read_exact(case, x):
    if case["kind"] == "store":
        k, v = (_stored_exact(x[n[0]], case[n + "_scale"]) for n in ("key", "value"))
    else:
        page, at = _at(case, x, x["slots"].clamp(min=0))
        k, v = (_cached_exact(x, n, case[n + "_scale"], page, at) for n in ("key", "value"))
    gone = x["slots"] < 0
    for t in (k, v):
        t[gone] = 0.0
    return k, v


def _cached_exact(x, name, scale, page, at, head=slice(None)):
    codes, scales = x[name + "_codes"][page, at, head], x[name + "_scales"][page, at, head]
    e2m1, e4m3 = (torch.tensor(t, dtype=torch.float64, device=codes.device) for t in (_E2M1, _E4M3))
    e = e2m1[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return e * e4m3[scales.int()].repeat_interleave(GROUP, -1) * scale


def _attend_exact(case, x):
    Q, bs, d, g = case["Q"], case["block"], case["D"], case["heads"] // case["kv_heads"]
    out, lse = [], []
    for b in range(case["B"]):
        n = int(x["lens"][b])
        o = torch.zeros(Q, case["heads"], d, dtype=torch.float64, device="cuda")
        l = torch.full((Q, case["heads"]), -math.inf, dtype=torch.float64, device="cuda")
        if n:
            j = torch.arange(n, device="cuda")
            page, at = x["tables"][b].long()[j // bs], j % bs
            for h in range(case["kv_heads"]):
                k, v = (_cached_exact(x, name, case[name + "_scale"], page, at, h) for name in ("key", "value"))
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
    x = _inputs(case, seed)
    return {"rotary": _rotary_exact, "store": _read_exact, "read": _read_exact,
            "attend": _attend_exact}[case["kind"]](case, x)

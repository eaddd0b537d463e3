"""The operators around the verification step from their definitions, in 64 bits (or, for
whole numbers, in Python), one request and one position at a time."""
import math

import torch

LOWEST = {torch.float32: torch.finfo(torch.float32).min, torch.bfloat16: torch.finfo(torch.bfloat16).min}


def constrained(logits, b, k, *, history=None, history_len=None, prompt_len=None, drafts=None,
                repetition=None, frequency=None, presence=None, bias=None, mask=None, mask_rows=None,
                mask_value=None):
    """(values, sum of the magnitudes that enter each) of row (b, k), fp64 on the CPU."""
    x = logits[b, k].double().cpu()
    V, low = x.numel(), LOWEST[logits.dtype]
    n, seen = torch.zeros(V, dtype=torch.float64), torch.zeros(V, dtype=torch.bool)
    if history is not None:
        length = min(max(int(history_len[b]), 0), history.shape[1])
        m = min(max(int(prompt_len[b]), 0), length) if prompt_len is not None else 0
        for i, v in enumerate(history[b, :length].tolist()):
            if 0 <= v < V:
                seen[v] = True
                n[v] += i >= m
    if drafts is not None:
        for v in drafts[b, :k].tolist():
            if 0 <= v < V:
                seen[v] = True
                n[v] += 1
    rep, freq, pres = (d if p is None else float(p[b])
                       for p, d in ((repetition, 1.0), (frequency, 0.0), (presence, 0.0)))
    if not (0 < rep < math.inf and abs(freq) < math.inf and abs(pres) < math.inf):
        rep, freq, pres = 1.0, 0.0, 0.0
    y = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    mag = y.abs()
    y = y - freq * n - pres * (n > 0)
    mag = mag + abs(freq) * n + abs(pres) * (n > 0)
    if bias is not None:
        offsets, tokens, values = (t.cpu() for t in bias)
        add = {}
        for i in range(max(int(offsets[b]), 0), min(int(offsets[b + 1]), tokens.numel())):
            if 0 <= int(tokens[i]) < V:
                add[int(tokens[i])] = float(values[i])
        for v, a in add.items():
            y[v] += a
            mag[v] += abs(a)
    y = torch.where(x.isfinite(), y.clamp(low, -low), y)
    if mask is not None:
        at = int(mask_rows[b, k]) if mask_rows is not None else b * logits.shape[1] + k
        value = min(max(low if mask_value is None else mask_value, low), -low)
        if at < -1 or at >= mask.shape[0]:
            y[:] = value
        elif at >= 0:
            words = mask[at].cpu().tolist()
            bits = torch.tensor([(words[v // 32] >> (v % 32)) & 1 for v in range(V)])
            y[bits == 0] = value
    return y, mag


def planned(lens, tables, held, free, *, block_size, accepted=None, grow=0):
    """The plan of B requests: lists in, and (start, len, held, free, offsets, slots, positions,
    tables) out; `free` is the stack."""
    B, width = len(lens), len(tables[0]) if lens else 0
    tables, free = [list(t) for t in tables], list(free)
    start, more = [], []
    for b in range(B):
        start.append(lens[b] + (accepted[b] + 1 if accepted else 0))
        g = grow[b] if isinstance(grow, list) else grow
        more.append(g)
    want = [-(-(start[b] + more[b]) // block_size) for b in range(B)]
    kept, fits = list(held), [start[b] + more[b] <= width * block_size for b in range(B)]
    for b in range(B):
        if fits[b] and want[b] < held[b]:
            free += tables[b][want[b]:held[b]]
            kept[b] = want[b]
    upto, left, ok = 0, len(free), []
    for b in range(B):
        need = max(want[b] - held[b], 0) if fits[b] else 0
        upto += need
        ok.append(fits[b] and (need == 0 or upto <= left))
        if ok[-1] and need:
            for j in range(held[b], want[b]):
                tables[b][j] = free.pop()
            kept[b] = want[b]
    offsets, slots, positions = [0], [], []
    for b in range(B):
        for i in range(more[b]):
            p = start[b] + i
            positions.append(p if ok[b] else -1)
            slots.append(tables[b][p // block_size] * block_size + p % block_size if ok[b] else -1)
        offsets.append(offsets[-1] + more[b])
    ends = [start[b] + (more[b] if ok[b] else 0) for b in range(B)]
    return start, ends, kept, free, offsets, slots, positions, tables


def attended(q, keys, values, tables, lens, b, i, h, *, scale=None, window=0):
    """Of query i of request b, head h, in 64 bits: (out, lse, sum of |weight * value|, largest
    score error per unit of relative error in its products, keys seen)."""
    Q, heads, D = q.shape[1:]
    bs, kh = keys.shape[1], h // (heads // keys.shape[2])
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    last = int(lens[b]) - Q + i
    first = max(0, last - window + 1) if window else 0
    j = torch.arange(first, max(first, last + 1), device=q.device)
    page = tables[b].long()[j // bs] if j.numel() else j
    live = (page >= 0) & (page < keys.shape[0])
    j, page = j[live], page[live]
    if not j.numel():
        return torch.zeros(D, dtype=torch.float64), -math.inf, torch.zeros(D, dtype=torch.float64), 0.0, 0
    k, v = keys[page, j % bs, kh].double(), values[page, j % bs, kh].double()
    x = q[b, i, h].double()
    s = k @ x * scale
    spread = float(((k.abs() @ x.abs()) * abs(scale)).max())
    w = s.softmax(-1)
    return (w @ v).cpu(), float(s.logsumexp(-1)), (w @ v.abs()).cpu(), spread, j.numel()

"""Plain references of the calls before the attention (hisparse_plan_tokens, hisparse_rotate_tokens,
hisparse_summarize_records, hisparse_select_records): loops over whole numbers and 64-bit arithmetic, on
CPU tensors."""
from __future__ import annotations

import math

import torch

from paper_2608_07009_amd import hisparse as hs

KEYS, BOUNDS, MEANS = hs.HISPARSE_INDEX_KEYS, hs.HISPARSE_INDEX_BOUNDS, hs.HISPARSE_INDEX_MEANS
INDEX_ROWS = {KEYS: 1, BOUNDS: 2, MEANS: 1}  # of 128, per token (KEYS) or record


def clamp(x, lo, hi):
    return min(max(x, lo), hi)


def plan(new, kv, t, max_chunk, max_records, total, free, used, table):
    """start, kv_len, used, positions, slots; writes into table [requests][>= max_records] (lists)."""
    cap = max_records * t
    used0 = used = clamp(used, 0, len(free or []))
    start, out, pos, slots = [0], [], [], []
    for r, n in enumerate(new):
        old = clamp(kv[r] if kv else 0, 0, cap)
        n = min(clamp(n, 0, max_chunk), cap - old, total - start[-1])
        for p in range(old, old + n):
            if p % t == 0:
                if free:
                    table[r][p // t] = free[used] if used < len(free) else -1
                used += 1
            rec = table[r][p // t]
            pos.append(p)
            slots.append(rec * t + p % t if rec >= 0 else -1)
        start.append(start[-1] + n)
        out.append(old + n)
    assert used - used0 <= total
    tail = total - start[-1]
    return start, out, used, pos + [0] * tail, slots + [-1] * tail


def frequencies(d: hs.RotaryDesc):
    out = []
    for i in range(d.dims // 2):
        f = d.theta ** (-2.0 * i / d.dims)
        if d.scaling == hs.HISPARSE_ROTARY_LINEAR:
            f /= d.factor
        elif d.scaling == hs.HISPARSE_ROTARY_BY_PARTS:
            turns = d.original_tokens * f / (2 * math.pi)
            s = clamp((turns - d.low_turns) / (d.high_turns - d.low_turns), 0.0, 1.0)
            f = s * f + (1 - s) * f / d.factor
        out.append(f)
    return out


def rotate(d: hs.RotaryDesc, positions, x, first):
    """float64 [tokens][heads][dims] of rows x, and what the result is made of: |a| + |b| of each
    rotated element's pair (0 for the others), the scale of its fp32 roundings."""
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    back = -1.0 if d.flags & hs.HISPARSE_ROTARY_BACK else 1.0
    half = d.dims // 2
    for i, f in enumerate(frequencies(d)):
        a, b = (i, i + half) if d.layout == hs.HISPARSE_ROTARY_HALF else (2 * i, 2 * i + 1)
        a, b = a + first, b + first
        angle = positions.double()[:, None] * f
        c, s = torch.cos(angle) * d.magnitude, back * torch.sin(angle) * d.magnitude
        xa, xb = x[..., a].double(), x[..., b].double()
        y[..., a], y[..., b] = xa * c - xb * s, xb * c + xa * s
        size[..., a] = size[..., b] = (xa.abs() + xb.abs()) * abs(d.magnitude)
    return y, size


def request_rows(start, kv_len, r, max_chunk, max_len, total):
    """First row, new tokens and cached tokens of request r, as the calls hold them."""
    if start is None:
        begin, n = r * max_chunk, max_chunk
    else:
        begin = clamp(start[r], 0, total)
        n = min(clamp(start[r + 1], begin, total) - begin, max_chunk)
    return begin, n, max_len if kv_len is None else clamp(kv_len[r], 0, max_len)


def scores(kind, q, w, rows):
    """float64 [candidates] of queries q [q_heads][128], weights w or None, rows [cand][1 or 2][128]."""
    q, rows = q.double(), rows.double()
    if kind == KEYS:
        dot = rows[:, 0] @ q.t().contiguous()
        dot = torch.where(dot > 0, dot, torch.where(dot == dot, torch.zeros_like(dot), dot))
        return (dot * (1.0 if w is None else w.double())).sum(1)
    if kind == MEANS:
        return rows[:, 0] @ q.sum(0)
    neg, pos = torch.where(q < 0, q, 0.0).sum(0), torch.where(q < 0, 0.0, q).sum(0)
    return rows[:, 0] @ neg + rows[:, 1] @ pos


def select_row(kind, q, w, rows, valid, k, first, last):
    """The list of one new token and kv head: rows of the candidates it sees, valid [cand]."""
    seen = valid.numel()
    K = min(k, seen)
    own = seen - 1 if last else None
    forced = {j for j in range(seen) if j < first or j >= seen - last}
    if seen <= k:
        chosen = [j for j in range(seen) if valid[j]]
    else:
        chosen = [j for j in forced if valid[j] or j == own]
        m = k - len(chosen)
        chosen = [j for j in chosen if valid[j]]
        x = scores(kind, q, w, rows)
        free = [j for j in range(seen) if valid[j] and j not in forced]
        if free and m > 0:
            y = x[free]
            y = torch.where(y != y, math.inf, y)  # NaN above +inf: by a second key
            nan = (x[free] != x[free])
            order = sorted(range(len(free)),
                           key=lambda i: (not nan[i], -y[i].item() if not nan[i] else 0.0, free[i])) \
                if bool(nan.any()) else torch.sort(y, descending=True, stable=True)[1].tolist()
            chosen += [free[i] for i in order[:m]]
    others = sorted(j for j in chosen if j != own)
    out = others + [-1] * (k - len(others))
    if own is not None and K > 0:
        assert len(others) < K
        out[K - 1] = own if valid[own] else -1
    return out

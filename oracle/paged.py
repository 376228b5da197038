"""CPU ORACLE of the paged key/value cache -- TEST INFRASTRUCTURE, NOT PRODUCT CODE.

Plain restatements, row by row and in float64, of the rules in ``include/ds.h``: the page bookkeeping of one step,
the per-head norm with rotary position and the cache write, and attention over pages.  Nothing here imports the
CUDA package.
"""
from __future__ import annotations

import math

import numpy as np


def page_update(kv_len, n_new, done, table, free_list, free_cnt, page_size, max_rows):
    """One step's bookkeeping on copies of table and free_list.  Returns a dict with the results and ``refused``."""
    B = len(kv_len)
    table, free = np.array(table, dtype=np.int64), list(free_list[:free_cnt])
    tail = list(free_list[free_cnt:])
    pages = lambda n: -(-n // page_size)  # noqa: E731
    old = []
    for b in range(B):
        if done is not None and done[b]:
            back = table[b, :pages(kv_len[b])].tolist()
            free += back
            tail = tail[len(back):]
            old.append(0)
        else:
            old.append(int(kv_len[b]))
    stack = free + tail          # the array as it stands: handing pages out does not erase them
    top = len(free)
    length, row_start, positions, slots, refused = [], [0], [], [], []
    asked_pages = asked_rows = taken = 0
    for b in range(B):
        need, n = pages(old[b] + int(n_new[b])) - pages(old[b]), int(n_new[b])
        asked_pages += need
        asked_rows += n
        if (need and asked_pages > top) or (n and asked_rows > max_rows):
            refused.append(b)
            need = n = 0
        for j in range(need):
            table[b, pages(old[b]) + j] = stack[top - 1 - taken]
            taken += 1
        for i in range(n):
            pos = old[b] + i
            positions.append(pos)
            slots.append(int(table[b, pos // page_size]) * page_size + pos % page_size)
        length.append(old[b] + n)
        row_start.append(row_start[-1] + n)
    pad = max_rows - len(slots)
    return dict(kv_len=np.array(length), free_cnt=top - taken, row_start=np.array(row_start),
                positions=np.array(positions + [0] * pad), slot_map=np.array(slots + [-1] * pad),
                block_table=table, free_list=np.array(stack), refused=refused)


def rope_frequencies(rotary_dim, theta, scaling=None, factor=1.0, orig_len=0, beta_fast=32.0, beta_slow=1.0):
    """(radians per position of each pair, factor on the rotated values)."""
    R = rotary_dim
    d = np.arange(R // 2, dtype=np.float64)
    if scaling == "ntk":
        theta = theta * factor ** (R / (R - 2))
    f = theta ** (-2.0 * d / R)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling != "yarn":
        return f, 1.0
    c = lambda turns: R * math.log(orig_len / (2 * math.pi * turns)) / (2 * math.log(theta))  # noqa: E731
    lo, hi = max(math.floor(c(beta_fast)), 0), min(math.ceil(c(beta_slow)), R - 1)
    r = np.clip((d - lo) / max(hi - lo, 1e-3), 0, 1)
    return f * (1 - r) + f / factor * r, (0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0)


def norm_rope(x, weight, eps, positions, freq, mscale, interleaved):
    """x [N, H, D] float64 -> normed (weight given) and rotated.  Also returns the length of each element's pair
    (the element itself outside the rotated part), the scale of the rounding errors."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64)
    out, size = x.copy(), np.abs(x)
    half = len(freq)
    for n, pos in enumerate(positions):
        a = float(pos) * freq
        first = np.arange(half) * 2 if interleaved else np.arange(half)
        second = first + 1 if interleaved else first + half
        lo, hi = x[n][:, first], x[n][:, second]
        out[n][:, first] = mscale * (lo * np.cos(a) - hi * np.sin(a))
        out[n][:, second] = mscale * (hi * np.cos(a) + lo * np.sin(a))
        size[n][:, first] = size[n][:, second] = mscale * np.hypot(lo, hi)
    return out, size


def visible(length, count, i, causal, window, sinks):
    """The cache rows that query i of count sees, as a list."""
    end = length - count + 1 + i if causal else length
    return [t for t in range(max(0, end)) if window == 0 or t < sinks or t >= end - window]


def attn_paged(q, k_cache, v_cache, table, kv_len, row_start, scale, causal, window=0, sinks=0, rows=None):
    """q [N, Hq, D], caches [pages, Hkv, ps, D], all float64.  Returns out, lse, spread (sum_t p_t |v_t|) and reach
    (scale * max_t sum_d |q_d k_td|), the last two the scales of the rounding errors.  Rows of no sequence: NaN."""
    N, Hq, D = q.shape
    Hkv, ps = k_cache.shape[1], k_cache.shape[2]
    out, spread = np.full((N, Hq, D), np.nan), np.full((N, Hq, D), np.nan)
    lse, reach = np.full((N, Hq), np.nan), np.zeros((N, Hq))
    for b, length in enumerate(kv_len):
        count = row_start[b + 1] - row_start[b]
        for i in range(count):
            r = row_start[b] + i
            see = np.array(visible(int(length), int(count), i, causal, window, sinks), dtype=np.int64)
            if len(see) == 0:
                out[r], spread[r], lse[r] = 0.0, 0.0, -np.inf
                continue
            page, off = table[b, see // ps], see % ps
            for g in range(Hkv):
                heads = slice(g * (Hq // Hkv), (g + 1) * (Hq // Hkv))
                k, v = k_cache[page, g, off], v_cache[page, g, off]
                z = scale * (q[r, heads] @ k.T)
                top = z.max(-1, keepdims=True)
                p = np.exp(z - top)
                lse[r, heads] = (top + np.log(p.sum(-1, keepdims=True)))[:, 0]
                p /= p.sum(-1, keepdims=True)
                out[r, heads], spread[r, heads] = p @ v, p @ np.abs(v)
                reach[r, heads] = abs(scale) * (np.abs(q[r, heads]) @ np.abs(k).T).max(-1)
    return out, lse, spread, reach

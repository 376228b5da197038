"""CPU ORACLE of the 8-bit paged cache -- TEST INFRASTRUCTURE, NOT PRODUCT CODE.

Plain restatements, block by block and in float64, of the rules in ``include/ds.h``: quantising rows into their pages, reading
them back, and the values that attention sees.  Nothing here imports the CUDA package.
"""
from __future__ import annotations

import math

import numpy as np
import torch


def _value(byte):
    sign, exponent, fraction = -1.0 if byte & 0x80 else 1.0, (byte >> 3) & 15, byte & 7
    if byte & 0x7f == 0x7f:
        return math.nan
    return sign * (fraction * 2.0 ** -9 if exponent == 0 else (8 + fraction) * 2.0 ** (exponent - 10))


E4M3 = np.array([_value(b) for b in range(256)])
_UP = E4M3[:0x7f]                                          # 0 .. 448, ascending


def encode(x):
    """Nearest e4m3 byte, ties to the even one; beyond 448 the largest, NaN and infinities NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.where(np.isfinite(x), np.abs(x), 0.0), 448.0)
    lo = np.clip(np.searchsorted(_UP, a, side="right") - 1, 0, 0x7d)
    below, above = a - _UP[lo], _UP[lo + 1] - a
    byte = np.where((above < below) | ((above == below) & (lo % 2 == 1)), lo + 1, lo)
    byte = np.where(np.signbit(x) & np.isfinite(x), byte | 0x80, byte)
    return np.where(np.isfinite(x), byte, 0x7f).astype(np.uint8)


MOST = 1.875 * 2.0 ** 127


def exponent(a):
    """The smallest e >= -126 with a <= 448 * 2^e."""
    e = -126
    while a > 448.0 * 2.0 ** e:
        e += 1
    return e


def exponents(a):
    """``exponent`` of an array."""
    m, e = np.frexp(np.asarray(a, dtype=np.float64))               # a = m 2^e, 448 = 0.875 * 2^9
    return np.where(np.asarray(a) == 0, -126, np.maximum(e - 9 + (m > 0.875), -126))


def write(x, codes, scales, T, table, kv_len, row_start, page_size):
    """Rows x [N, Hkv, D] (float64) into copies of codes (bytes) [pages, Hkv, ps, D] and scales [pages, Hkv, ps / T].  Sequences with
    impossible lengths or pages are the tests' business.  Returns codes, scales."""
    codes, scales = codes.copy(), scales.copy()
    for b, length in enumerate(kv_len):
        n = int(row_start[b + 1] - row_start[b])
        old = int(length) - n
        for block in range(old // T, -(-int(length) // T) if n else 0):
            first = block * T
            held, new = np.arange(first, max(first, old)), np.arange(max(first, old), min(first + T, int(length)))
            page, s_at = int(table[b, first // page_size]), (first % page_size) // T
            y = x[int(row_start[b]) + new - old]                    # [rows, Hkv, D]
            fin = np.where(np.isfinite(y), np.minimum(np.abs(y), MOST), 0.0)
            e = exponents(fin.max((0, 2)))                          # [Hkv]
            s = scales[page, :, s_at].astype(np.float64)
            if len(held):
                counts = np.isfinite(s) & (np.abs(s) <= 2.0 ** 127) & (s != 0)
                m, up = np.frexp(np.where(counts, np.abs(s), 1.0))
                e = np.where(counts, np.maximum(e, up - (m == 0.5)), e)
                with np.errstate(invalid="ignore", over="ignore"):
                    v = E4M3[codes[page][:, held % page_size]] * (s / 2.0 ** e)[:, None, None]
                changed = s != 2.0 ** e
                again = codes[page][:, held % page_size]
                again[changed] = encode(v)[changed]
                codes[page, :, held % page_size] = again.transpose(1, 0, 2)
            v = np.where(np.isfinite(y), np.clip(y, -MOST, MOST), y)
            codes[page, :, new % page_size] = encode(v / (2.0 ** e)[:, None])
            scales[page, :, s_at] = 2.0 ** e
    return codes, scales


def values(codes, scales):
    """What the cache stands for: float64 [pages, Hkv, ps, D]."""
    T = codes.shape[2] // scales.shape[2]
    with np.errstate(invalid="ignore"):
        return E4M3[codes] * np.repeat(scales.astype(np.float64), T, axis=2)[..., None]


def attn_paged(q, k_cache, v_cache, table, kv_len, row_start, scale, causal, window=0, sinks=0):
    """``paged.attn_paged`` with all queries of a sequence and KV head at once, on float64 tensors wherever they live (the caches may hold
    anything where no query looks)."""
    N, Hq, D = q.shape
    Hkv, ps = k_cache.shape[1], k_cache.shape[2]
    G, dev = Hq // Hkv, q.device
    out, spread = q.new_full((N, Hq, D), math.nan), q.new_full((N, Hq, D), math.nan)
    lse, reach = q.new_full((N, Hq), math.nan), q.new_zeros((N, Hq))
    table = torch.as_tensor(table, device=dev).long()
    for b, length in enumerate(kv_len):
        lo, hi = int(row_start[b]), int(row_start[b + 1])
        count, length = hi - lo, int(length)
        if count == 0:
            continue
        t, i = torch.arange(length, device=dev), torch.arange(count, device=dev)[:, None]
        end = length - count + 1 + i if causal else torch.full((count, 1), length, device=dev)
        see = t < end
        if window:
            see &= (t < sinks) | (t >= end - window)
        used = see.any(0)
        t, see = t[used], see[:, used]
        if len(t) == 0:
            out[lo:hi], spread[lo:hi], lse[lo:hi] = 0.0, 0.0, -math.inf
            continue
        k, v = (c[table[b, t // ps], :, t % ps].transpose(0, 1) for c in (k_cache, v_cache))             # [Hkv, keys, D]
        qq = q[lo:hi].view(count, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, count * G, D)
        shape = (Hkv, count, G, len(t))
        z = (scale * (qq @ k.transpose(1, 2))).view(shape).masked_fill(~see[:, None], -math.inf)
        far = (abs(scale) * (qq.abs() @ k.abs().transpose(1, 2))).view(shape).masked_fill(~see[:, None], 0.0).amax(-1)
        top = z.amax(-1, keepdim=True)
        top = torch.where(torch.isneginf(top), 0.0, top)
        p = torch.exp(z - top)
        total = p.sum(-1, keepdim=True)
        p = (p / torch.where(total == 0, 1.0, total)).view(Hkv, count * G, -1)
        back = lambda x: x.view(Hkv, count, G, -1).permute(1, 0, 2, 3).reshape(count, Hq, -1)  # noqa: E731
        out[lo:hi], spread[lo:hi] = back(p @ v), back(p @ v.abs())
        lse[lo:hi], reach[lo:hi] = back(top + total.log())[..., 0], back(far)[..., 0]
    return tuple(x.cpu().numpy() for x in (out, lse, spread, reach))

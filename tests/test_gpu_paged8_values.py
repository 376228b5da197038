"""The 8-bit paged cache where values lie far apart or next to a border of the type.

Scales of V: a weight enters its product as a 16-bit float, relative to the largest weight times scale that the query itself sees, which
stands at 2^3 .. 2^15 (fp32 outputs 2^9 .. 2^15, two parts, the second times 2^11).  So a term is off by half a step, 2^-11 (2^-22) of
itself, or by 2^-25 of those units (2^-36), 2^-28 (2^-45) of the largest, where it is too small for that."""
import copy
import math

import numpy as np
import pytest
import torch

from oracle import paged8 as oracle8
from test_gpu_paged import BF, DEV, F32, U, f64
from test_gpu_paged8 import PATHS, Case8, Pool, every_path, read_back

pytestmark = pytest.mark.gpu


def tokens(path, seed, at_least=4, **kw):
    """A case with a scale for every token; its first sequence has at_least new rows."""
    dtype, D, Hq, Hkv, lens, counts, room = PATHS[path]
    return Case8(lens, [max(at_least, counts[0]), *counts[1:]], Hq, Hkv, D, 16, 1, dtype, seed=seed, room=room, **kw)


def with_scale(c, t, by):
    d = copy.copy(c)
    d.scales = [x.clone() for x in c.scales]
    page, off = d.place(0, t)
    d.scales[1][page, :, off] *= by
    return d


@every_path
@pytest.mark.parametrize("by", [2.0 ** 40, -2.0 ** 12, 2.0 ** 110])
def test_large_values_of_a_hidden_row_leave_the_other_queries_as_they_are(path, by):
    """The last new row, and rows at and outside a window's edge, with a scale of V far above the others."""
    c = tokens(path, 3)
    n, count = c.lens[0], c.counts[0]
    clean, clean_lse, scale = c.run()
    d = with_scale(c, n - 1, by)
    out, lse, _ = d.run()
    assert torch.equal(out[:count - 1], clean[:count - 1]) and torch.equal(out[count:], clean[count:]) and torch.equal(lse, clean_lse)
    keep = np.zeros(c.N, dtype=bool)
    keep[count - 1] = True
    d.compare(out, lse, d.reference(scale), scale, keep)
    edge = n - count + 1 - 5                     # window 5: of all queries the first alone sees this row
    clean, clean_lse, _ = c.run(window=5)
    out, lse, _ = with_scale(c, edge, by).run(window=5)
    assert torch.equal(out[1:], clean[1:]) and torch.equal(lse, clean_lse)
    out, lse, _ = with_scale(c, edge - 1, by).run(window=5)
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


def weight_error(dtype, E, n):
    bf = dtype == BF
    return 2 * (2 * E + 2.0 ** -21 + (2.0 ** -11 if bf else 2.0 ** -22)) + 4 * (16 + math.sqrt(n)) * U


@every_path
def test_a_large_value_of_small_weight_does_not_take_the_others_bits(path):
    """A row with 2^30 times the scale of V and weights near 2^-45: the largest terms are the others'."""
    c = tokens(path, 5, 1)
    D, rows = c.D, c.counts[0]
    c.q = (c.q.float().abs() + 0.1).to(c.dtype)
    page, off = c.place(0, 7)
    c.codes[0][page, :, off] = 0xfe                                        # -448 each
    c.scales[0][page, :, off] = 45 * math.log(2) * math.sqrt(D) / (0.9 * D * 448)
    c.scales[1][page, :, off] = 0.01 * 2.0 ** 30
    out, lse, scale = c.run(causal=False)
    want, want_lse, spread, reach = (x[:rows] for x in c.reference(scale, causal=False))
    k, v = c.values()
    by_scale = [v, c.scales[1].abs().double().to(DEV)[..., None].expand(*c.codes[1].shape)]
    most = oracle8.attn_paged(c.q[:c.N].double().to(DEV), k, by_scale[1], c.table, c.lens, c.starts, scale, False)[0][:rows]
    q = f64(c.q)[:rows]
    most_k = float(torch.where(torch.isfinite(k), k.abs(), 0.0).sum(-1).max())
    bf, n = c.dtype == BF, max(c.lens)
    E = (D + 4) * U * reach + (2.0 ** -21 if bf else 2.0 ** -39) * scale * np.abs(q).max(-1) * most_k + (0.0 if bf else 2.0 ** -22 * reach)
    tol = (2.0 ** -8 if bf else U) * np.abs(want) + weight_error(c.dtype, E, n)[..., None] * spread + n * 448 * (2.0 ** -28 if bf else 2.0 ** -45) * most
    err = np.abs(f64(out)[:rows] - want)
    assert (err <= tol).all(), (err - tol).max()


@pytest.mark.parametrize("path,below", [(p, b) for p in PATHS for b in ((16, 24) if PATHS[p][0] == BF else (16, 24, 38))])
def test_scales_far_below_the_largest(path, below):
    """In the upper half of the dimensions one row alone has values, under a scale of V 2^-below times the others'; weights near 1 / n."""
    bf = PATHS[path][0] == BF
    c = tokens(path, 6, 1, sharp=0.02)
    D, rows, n = c.D, c.counts[0], c.lens[0]
    t = torch.arange(n)
    page, off = c.place(0, t)
    c.codes[1][page, :, off, D // 2:] = 0
    c.scales[1][page, :, off] = 0.01
    page, off = c.place(0, n // 2)
    c.codes[1][page, :, off, D // 2:] = 0x7e                               # 448
    c.scales[1][page, :, off] = 0.01 * 2.0 ** -below
    out, lse, scale = c.run(causal=False)
    want, _, spread, reach = (x[:rows] for x in c.reference(scale, causal=False))
    assert (reach < 0.3).all()                                             # so that a weight is at most e^0.6 < 2 times another
    q = f64(c.q)[:rows]
    k = c.values()[0]
    most_k = float(torch.where(torch.isfinite(k), k.abs(), 0.0).sum(-1).max())
    E = (D + 4) * U * reach + (2.0 ** -21 if bf else 2.0 ** -39) * scale * np.abs(q).max(-1) * most_k + (0.0 if bf else 2.0 ** -22 * reach)
    rel = (2.0 ** -8 if bf else U) + weight_error(c.dtype, E, n) + 2 * 2.0 ** (below - (28 if bf else 45))
    err = np.abs(f64(out)[:rows] - want)[..., D // 2:]
    assert (err <= rel[..., None] * np.abs(want[..., D // 2:])).all(), (err / np.abs(want[..., D // 2:])).max()


# ------------------------------------------------------------------------------------------------ one rounding
def near_ties(n, ties, low, high, seed):
    """n pairs of an e4m3 byte and an fp32 scale in (low, high] whose product lies within 2^-24 of a tie, or on it."""
    rng = np.random.default_rng(seed)
    codes, scales = [], []
    while len(codes) < n:
        c, tie = int(rng.integers(1, 0x7f)), float(rng.choice(ties))
        s = np.float32(tie / oracle8.E4M3[c])
        if low < s <= high:
            codes.append(c | (0x80 if rng.random() < 0.5 else 0))
            scales.append(s)
    return np.array(codes, np.uint8), np.array(scales, np.float32)


def test_rows_held_under_foreign_scales_are_rounded_once():
    """Scales in (1/2, 1] become 1: products next to the border between two e4m3 values."""
    B = 400
    p = Pool([7] * B, [1] * B, 1, 32, 8, 8, seed=2)
    mid = (oracle8.E4M3[1:0x7f] + oracle8.E4M3[:0x7e]) / 2
    for i in range(2):
        codes, scales = near_ties(B, mid, 0.5, 1.0, seed=i)
        codes[0], scales[0] = 0x09, 0.6111111
        assert oracle8.E4M3[codes[0]] == 0.017578125
        pages = p.table[:, 0].long()
        p.codes[i][pages, 0, :, ::2] = torch.from_numpy(codes)[:, None, None].expand(B, 8, 16)
        p.scales[i][pages, 0, 0] = torch.from_numpy(scales)
    for dtype in (BF, F32):
        p.check(torch.zeros(p.N + 3, 2, 32, dtype=dtype))


@pytest.mark.parametrize("s", [1.5 * 2.0 ** 127, -1.0000001 * 2.0 ** 127, 2.0 ** 127, 2.0 ** -149, -1.7 * 2.0 ** -130])
@pytest.mark.parametrize("new", [0.0, 1.0, 2.0 ** 100, 2.0 ** 127])
def test_rows_held_under_the_largest_and_smallest_scales(s, new):
    """Every byte, rescaled from s to what the new row needs: beyond 448 the largest, far below nothing."""
    p = Pool([8], [1], 1, 256, 16, 16)
    page = p.table[0, 0].long()
    for i in range(2):
        p.codes[i][page] = torch.arange(256, dtype=torch.int32).to(torch.uint8)
        p.scales[i][page] = s
    p.check(torch.full((4, 2, 256), new, dtype=F32))
    long = Pool([8], [40], 1, 256, 64, 64)                                 # the kernel for long runs
    page = long.table[0, 0].long()
    for i in range(2):
        long.codes[i][page] = torch.arange(256, dtype=torch.int32).to(torch.uint8)
        long.scales[i][page] = s
    long.check(torch.full((43, 2, 256), new, dtype=F32))


def nearest_bf16(x):
    """float64 -> the nearest bf16 value, ties to even; beyond the largest infinite."""
    unit = np.exp2(np.maximum(np.frexp(x)[1], -125) - 8.0)
    y = np.rint(x / unit) * unit
    return np.where(np.abs(y) >= 2.0 ** 128, np.sign(y) * np.inf, y)


@pytest.mark.parametrize("shift", [0, 60, 115, -100, -118, -125, -130])
def test_rows_read_back_in_bf16_are_rounded_once(shift):
    """Products next to the border between two bf16 values, ordinary ones and some that are next to the type's ends."""
    n = 600
    rng = np.random.default_rng(7)
    ties = (256 + rng.integers(0, 256, 4000) + 0.5) * 2.0 ** (shift - 8)   # halfway between neighbours of 8 bits
    if shift < -110:
        ties = (rng.integers(1, 256, 4000) + 0.5) * 2.0 ** -133            # of the smallest
        if shift < -118:
            ties = ties + rng.choice([-1, 1], 4000) * 2.0 ** (-149 if shift == -125 else -153)
    p = Pool([n], [0], 1, 16, 8, 1)
    t = np.arange(n)
    page, off = p.table[0].long()[torch.from_numpy(t // 8)], torch.from_numpy(t % 8)
    want = []
    for i in range(2):
        codes, scales = near_ties(n, ties, 2.0 ** -149, 3e38, seed=i)
        if shift == 0:
            codes[0], scales[0] = 0x09, 58.444443
        p.codes[i][page, 0, off] = torch.from_numpy(codes)[:, None].expand(n, 16)
        p.scales[i][page, 0, off] = torch.from_numpy(scales)
        want.append(nearest_bf16(oracle8.E4M3[codes] * scales.astype(np.float64)))
    out, _ = read_back(p, [c.to(DEV) for c in p.codes], [s.to(DEV) for s in p.scales], BF)
    for i in range(2):
        got = f64(out[i])[:, 0]
        assert np.array_equal(got, np.repeat(want[i][:, None], 16, 1)), np.argwhere(got[:, 0] != want[i])[:4]


# ------------------------------------------------------------------------------------------------ NaN in partly visible tiles
@pytest.mark.parametrize("D,Hq,count", [(128, 2, 20), (64, 4, 20), (128, 4, 60), (64, 8, 30)])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False, window=900), dict(window=300, sinks=4)])
@pytest.mark.parametrize("workspace", [True, False])
def test_nan_in_one_sequence_costs_the_others_nothing(D, Hq, count, kw, workspace):
    """NaN in V at the edge of what the first sequence's queries see, long sequences behind it in the same CTAs: status 0, their outputs
    as they were, and in the first sequence NaN where the formula has it."""
    n, lens = 330, [330, 40000, 333, 20000, 7, 331]
    counts = [count, count, count, count, 3, count]
    c = Case8(lens, counts, Hq, 1, D, 64, 1, BF, seed=count)
    ws = None if workspace else torch.empty(0, dtype=torch.uint8, device=DEV)
    clean, clean_lse, _ = c.run(workspace=ws, **kw)
    d = copy.copy(c)
    d.codes = [x.clone() for x in c.codes]
    marks = {t: slice(j, None, 7 + j) for j, t in enumerate((n - 1, n - 2, n - 9, n - count, 3, 40))}
    for b in (0, 2):
        for t, dims in marks.items():
            page, off = d.place(b, t)
            d.codes[1][page, :, off, dims] = 0x7f
    out, lse, _ = d.run(workspace=ws, **kw)
    want, want_lse = clean.clone(), clean_lse
    for b in (0, 2):
        for i in range(count):
            end = lens[b] - count + 1 + i if kw.get("causal", True) else lens[b]
            for t, dims in marks.items():
                if t < end and ("window" not in kw or t < kw.get("sinks", 0) or t >= end - kw["window"]):
                    want[int(c.starts[b]) + i, :, dims] = math.nan
    assert torch.isnan(want).any() and torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(out.nan_to_num(9.0), want.nan_to_num(9.0)) and torch.equal(lse, want_lse)


def test_a_whole_prompt_of_nan_ends():
    """Every byte of V NaN, hundreds of rows: each row that sees a key is NaN, within the kernel's limits of waiting."""
    c = Case8([1500, 9], [1500, 9], 4, 1, 128, 16, 16, BF, seed=2)
    c.codes[1].fill_(0xff)
    out, lse, _ = c.run(window=700)
    assert torch.isnan(out).all() and torch.isfinite(lse).all()


# ------------------------------------------------------------------------------------------------ items of many and of few rows in turn
@pytest.mark.parametrize("D,Hq,most", [(128, 2, 128), (64, 4, 64), (128, 8, 25), (64, 2, 30)])
@pytest.mark.parametrize("workspace", [True, False])
def test_items_of_many_rows_and_of_few_behind_each_other(D, Hq, most, workspace):
    """256, 100 or 60 rows, then 1 to 4, over 1 to 3 tiles, several items to a CTA: the streams of a CTA end and begin at different times."""
    B = 330
    counts = [most if b % 2 == 0 else 1 for b in range(B)]
    lens = [(150, 40, 260, 390, 120)[b % 5] + b % 7 for b in range(B)]
    c = Case8(lens, counts, Hq, 1, D, 16, 16, BF, seed=most)
    ws = None if workspace else torch.empty(0, dtype=torch.uint8, device=DEV)
    out, lse = c.check(workspace=ws)
    for _ in range(5):
        again, lse2, _ = c.run(workspace=ws)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


# ------------------------------------------------------------------------------------------------ long prompts
@pytest.mark.parametrize("dtype,D,Hq,Hkv", [(BF, 128, 2, 2), (BF, 64, 4, 1), (F32, 64, 2, 1)])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False), dict(window=150, sinks=5)])
def test_prompts_of_hundreds_of_rows(dtype, D, Hq, Hkv, kw):
    Case8([700, 513, 1000], [700, 513, 300], Hq, Hkv, D, 16, 16, dtype, seed=D).check(**kw)

"""GPU parity of the 8-bit paged cache (``ds_kv8_write``, ``ds_kv8_read``, ``ds_attn_paged8``) against the float64 oracle.

Writing and reading have one rounding of an exact quotient or product each (scales are powers of two, or the product of 4 and 24
bits is rounded to 24 and then to the type), so bytes, scales and bf16 rows are equal, fp32 rows within u = 2^-24.

Attention: tolerances as in ``test_gpu_paged.py`` (an output is rounded once; scores, weights and sums count against
spread = sum_t p_t |v_t|), with what is different here:
* queries are scaled by a power of two per row.  bf16: exact in fp16, or as e4m3 plus e5m2 (rows scaled to 2^7) but for elements below
  2^-6, whose e4m3 part is a multiple of 2^-9 and whose rest, at most 2^-10, is rounded to 3 bits, half a step 2^-14: 2^-21 max|q| sum|k|.
  fp32: two fp16 parts, the second rounded at 2^-11 of at most 2^-11 of the value: 2^-22 reach; what fp16 drops below 2^-25 of a
  row scaled to 2^14: 2^-39 max|q| sum|k|;
* weights are fp16, half a step 2^-11, for fp32 outputs two parts, 2^-22; what is dropped below 2^-25 of weights scaled by 2^6 (fp32: 2^10),
  of values up to 448 times the largest scale's next power of two, at most 4 max|v|: n 2^-29 (2^-33) max|v| (the sum of weights is at
  least 1).
"""
import copy
import math

import numpy as np
import pytest
import torch

import paper_2601_17917_b200 as ds
from oracle import paged8 as oracle8
from test_gpu_paged import BF, DEV, F32, U, f64, status_word

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def strided(shape, order, fill, dtype):
    """[pages, Hkv, n, ..] with the memory order page, head, row ("head"), or page, row, head ("row")."""
    if order == "head":
        return torch.full(shape, fill, dtype=dtype)
    return torch.full((shape[0], shape[2], shape[1], *shape[3:]), fill, dtype=dtype).transpose(1, 2)


# ------------------------------------------------------------------------------------------------ writing and reading
class Pool:
    """An 8-bit cache whose sequences hold `old` rows each, everything else in it garbage."""

    def __init__(self, old, new, Hkv, D, ps, T, seed=0, order="head", spare=2, power=True):
        g = torch.Generator().manual_seed(seed)
        B, self.T, self.ps, self.D, self.Hkv = len(old), T, ps, D, Hkv
        self.old, self.new = old, new
        width = max(1, max(-(-(o + n) // ps) for o, n in zip(old, new)))
        n_pages = B * width + spare
        self.table = torch.randperm(n_pages, generator=g)[:B * width].view(B, width).to(torch.int32)
        self.codes = [strided((n_pages, Hkv, ps, D), order, 0, torch.uint8) for _ in range(2)]
        self.scales = [strided((n_pages, Hkv, ps // T), order, 0.0, torch.float32) for _ in range(2)]
        for c, s in zip(self.codes, self.scales):
            c.copy_(torch.randint(0, 256, c.shape, generator=g, dtype=torch.uint8))
            e = torch.randint(-9, 4, s.shape, generator=g).float()
            s.copy_(torch.exp2(e) if power else torch.exp(torch.randn(s.shape, generator=g)) * (1 - 2 * (torch.rand(s.shape, generator=g) < 0.1).float()))
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.N = int(self.starts[-1])
        self.lens = [o + n for o, n in zip(old, new)]
        self.g = g

    def rows(self, dtype, spread=1.5):
        x = torch.randn(self.N + 3, 2 * self.Hkv, self.D, generator=self.g) * torch.exp(spread * torch.randn(self.N + 3, 2 * self.Hkv, 1, generator=self.g))
        return x.to(dtype)

    def write(self, kv, codes=None, scales=None, table=None, lens=None, starts=None, uniform=False, status=0, stream=None, **kw):
        """Runs the entry point on copies of codes and scales (their strides kept).  kv [N.., 2 Hkv, D] as K beside V."""
        codes = [(c if codes is None else x).to(DEV) for c, x in zip(self.codes, codes or self.codes)]
        scales = [(s if scales is None else x).to(DEV) for s, x in zip(self.scales, scales or self.scales)]
        kv, st = kv.to(DEV), status_word()
        ds.ds_kv8_write(kv[:, :self.Hkv], kv[:, self.Hkv:], *codes, *scales, (self.table if table is None else table).to(DEV),
                        i32(self.lens if lens is None else lens), None if uniform else i32(self.starts if starts is None else starts),
                        **dict(dict(max_q=max(1, max(self.new))), **kw), status=st, stream=stream)
        assert ds.ds_read_status(st) == status
        return codes, scales

    def want(self, kv, skip=()):
        kv = f64(kv)
        keep = [b for b in range(len(self.old)) if b not in skip]
        out = []
        for i in range(2):
            c, s = self.codes[i].numpy(), self.scales[i].numpy()
            for b in keep:
                lo, hi = int(self.starts[b]), int(self.starts[b + 1])
                c, s = oracle8.write(kv[lo:hi, i * self.Hkv:(i + 1) * self.Hkv], c, s, self.T, self.table.numpy()[b:b + 1], [self.lens[b]],
                                     [0, hi - lo], self.ps)
            out.append((c, s))
        return [x[0] for x in out], [x[1] for x in out]

    def check(self, kv, skip=(), **kw):
        codes, scales = self.write(kv, **kw)
        want_c, want_s = self.want(kv, skip)
        for i in range(2):
            assert np.array_equal(scales[i].cpu().numpy(), want_s[i], equal_nan=True)
            got = codes[i].cpu().numpy()
            nan = np.isnan(oracle8.E4M3[want_c[i]])
            assert np.array_equal(np.isnan(oracle8.E4M3[got]), nan) and np.array_equal(got[~nan], want_c[i][~nan])
        return codes, scales


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ps,T", [(1, 1), (16, 16), (16, 1), (24, 12), (64, 64), (8, 2), (500, 100)])
@pytest.mark.parametrize("Hkv,D", [(2, 64), (1, 128), (5, 96), (3, 16), (2, 256)])
def test_written_bytes_and_scales(dtype, ps, T, Hkv, D):
    """Rows behind nothing, behind part of a block, whole blocks, single rows and none."""
    p = Pool([0, 5, 33, 16, 0, 130, 7], [40, 1, 3, 0, 1, 70, 17], Hkv, D, ps, T, seed=ps + D)
    p.check(p.rows(dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("old,new", [([100] * 70, [1] * 70), ([3 * b for b in range(300)], [b % 3 for b in range(300)]), ([0, 0], [2000, 1500]),
                                     ([5], [1]), ([0] * 1100, [1] * 1100)])
def test_written_rows_of_many_sequences_and_long_ones(dtype, old, new):
    p = Pool(old, new, 2, 64, 16, 8, seed=len(old))
    p.check(p.rows(dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_writing_with_foreign_scales_layouts_and_uniform_rows(dtype):
    """Blocks begun under scales that are no powers of two, some negative; pages row by row; K and V as slices of a wider
    projection; row_start left out."""
    p = Pool([5, 20, 0, 47], [3, 3, 3, 3], 3, 64, 16, 8, seed=1, order="row", power=False)
    kv = p.rows(dtype)
    wide = torch.full((p.N + 3, 2 * p.Hkv + 5, p.D), float("nan"), dtype=dtype)
    wide[:, 2:2 + 2 * p.Hkv] = kv
    want = p.check(wide[:, 2:2 + 2 * p.Hkv])
    got = p.write(kv, uniform=True)
    for a, b in zip(want[0] + want[1], got[0] + got[1]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_at_the_borders(dtype):
    """Blocks of nothing but zeros, of the smallest and largest values, with infinities and NaN; rows held under scales that are
    zero, infinite or NaN; the exponent's border at 448 times a power of two; every tie of the type."""
    p = Pool([3, 3, 3, 3, 0, 0, 0, 0, 0, 0, 0], [2, 2, 2, 2, 4, 4, 4, 4, 4, 4, 4], 1, 64, 8, 8, seed=3)
    kv = p.rows(dtype)
    for b, s in enumerate((0.0, math.inf, math.nan, 2.0 ** 100)):
        for t in p.scales:
            t[p.table[b, 0].long()] = s
    at = lambda b: kv[int(p.starts[b]):int(p.starts[b + 1])]  # noqa: E731
    fi = torch.finfo(dtype)
    at(4).zero_()
    at(5).copy_(torch.full((64,), fi.smallest_normal) * torch.randn(4, 2, 64).sign())
    at(5)[0, 0, 0] = fi.smallest_normal * fi.eps                       # the smallest of all
    at(6)[0, :, :] = fi.max
    at(6)[1, :, :] = fi.min
    at(6)[2, :, 3] = 1.875 * 2.0 ** 127
    at(7)[1, 0, 5], at(7)[1, 1, 6], at(7)[2, :, 7] = math.inf, -math.inf, math.nan
    at(8).fill_(math.nan)
    at(9)[:] = torch.linspace(-1, 1, 64)
    at(9)[0, :, 0], at(9)[0, :, 1] = 448.0, -448.0
    mid = torch.tensor(oracle8.E4M3[:0x7f])
    ties = ((mid[1:] + mid[:-1]) / 2)
    at(10)[:] = 0
    at(10)[0, :, 0] = 448.0
    at(10)[1:3] = torch.cat([ties, ties.new_zeros(2)])[:128].view(2, 1, 64).expand(2, 2, 64).to(dtype)
    p.check(kv)


def test_a_block_that_grows_keeps_its_rows():
    """Rows appended one at a time, each larger than the last: what was held stays within half a step of the final scale, twice."""
    Hkv, D, ps, T = 1, 64, 16, 16
    p = Pool([0], [1], Hkv, D, ps, T)
    codes, scales = [c.to(DEV) for c in p.codes], [s.to(DEV) for s in p.scales]
    g = torch.Generator().manual_seed(0)
    rows = torch.randn(T, 2 * Hkv, D, generator=g) * torch.exp2(torch.arange(T).float()).view(-1, 1, 1)
    table = p.table.to(DEV)
    for t in range(T):
        x = rows[t:t + 1].to(DEV)
        ds.ds_kv8_write(x[:, :Hkv], x[:, Hkv:], *codes, *scales, table, i32([t + 1]))
    page = int(p.table[0, 0])
    for i in range(2):
        s = float(scales[i][page, 0, 0])
        peak = float(rows[:, i].abs().max())
        assert s == 2.0 ** oracle8.exponent(peak)
        got = oracle8.E4M3[codes[i][page, 0].cpu().numpy()] * s
        x = f64(rows[:, i])
        assert (np.abs(got - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -9 * s).all()      # a second rounding only below 2^-6 s


def test_writes_with_bad_lengths_rows_and_pages_are_flagged_and_left_out():
    p = Pool([20, 5, 9, 0], [4, 3, 2, 6], 2, 64, 8, 4, seed=5)
    kv = p.rows(BF)
    flag = ds.DS_DEV_INDEX
    for n in (-1, 2, p.table.shape[1] * p.ps + 1, 2 ** 31 - 1, -2 ** 31):      # 2: fewer than its new rows
        lens = list(p.lens)
        lens[1] = n
        p.check(kv, skip=[1], lens=lens, status=flag)
    p.check(kv, skip=[0], max_len=23, status=flag)
    for entry in (-1, p.codes[0].shape[0], 2 ** 31 - 1, -2 ** 31):
        t = p.table.clone()
        t[2, 1] = entry                                                        # rows 9 and 10 of sequence 2
        p.check(kv, skip=[2], table=t, status=flag)
    got = p.write(kv, max_q=3, status=flag)                                    # sequences 0 and 3 have more
    want_c, want_s = p.want(kv, skip=[0, 3])
    for i in range(2):
        assert np.array_equal(got[0][i].cpu().numpy(), want_c[i]) and np.array_equal(got[1][i].cpu().numpy(), want_s[i])
    starts = p.starts.copy()
    for last in (2 ** 31 - 1, -5, kv.shape[0] + 1):
        starts[-1] = last
        p.check(kv, skip=[3], starts=starts, status=flag)
    starts = p.starts.copy()
    starts[0] = -2
    p.check(kv, skip=[0], starts=starts, status=flag)


def read_back(p, codes, scales, dtype, first=None, dense=None, extra=0, status=0, lens=None, out_start=None, table=None):
    B, D, Hkv = len(p.old), p.D, p.Hkv
    lens = p.lens if lens is None else lens
    st = status_word()
    if dense is not None:
        out = [torch.full((B, dense, Hkv, D), 7.0, dtype=dtype, device=DEV) for _ in range(2)]
        start = None
    else:
        take = [max(0, n - (first[b] if first is not None else 0)) for b, n in enumerate(p.lens)]
        start = np.concatenate([[0], np.cumsum(take)]) if out_start is None else out_start
        out = [torch.full((sum(take) + extra, Hkv, D), 7.0, dtype=dtype, device=DEV) for _ in range(2)]
    ds.ds_kv8_read(*codes, *scales, (p.table if table is None else table).to(DEV), i32(lens), *out, out_start=None if start is None else i32(start),
                   first=None if first is None else i32(first), status=st)
    assert ds.ds_read_status(st) == status
    return out, start


def same_rows(got, want, dtype):
    """bf16: the product (exact, or rounded to 24 bits first) rounded to 8; fp32: half a step."""
    got = f64(got)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    err = np.abs(got - want)[~nan]
    assert (err <= (2.0 ** -8 if dtype == BF else U) * np.abs(want[~nan]) + 2.0 ** -134).all(), err.max()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ps,T", [(1, 1), (16, 16), (24, 3), (64, 64)])
@pytest.mark.parametrize("Hkv,D,order", [(2, 64, "head"), (1, 128, "row"), (5, 96, "head"), (3, 16, "row"), (2, 256, "head"), (32, 128, "head")])
def test_rows_read_back(dtype, ps, T, Hkv, D, order):
    p = Pool([0, 5, 33, 0, 130, 7], [40, 1, 3, 0, 70, 17], Hkv, D, ps, T, seed=ps + D, order=order, power=D != 96)
    codes, scales = [c.to(DEV) for c in p.codes], [s.to(DEV) for s in p.scales]
    val = [oracle8.values(c.numpy(), s.numpy()) for c, s in zip(p.codes, p.scales)]

    def rows(i, b, lo, hi):
        t = np.arange(lo, hi)
        return val[i][p.table.numpy()[b, t // ps], :, t % ps]
    for first in (None, [0, 3, 30, 0, 199, 0]):
        (ko, vo), start = read_back(p, codes, scales, dtype, first, extra=2)
        for i, o in enumerate((ko, vo)):
            assert (o[start[-1]:] == 7.0).all()
            for b, n in enumerate(p.lens):
                same_rows(o[start[b]:start[b + 1]], rows(i, b, first[b] if first else 0, n), dtype)
        for width in (50, 300):
            out, _ = read_back(p, codes, scales, dtype, first, dense=width)
            for i, o in enumerate(out):
                for b, n in enumerate(p.lens):
                    lo = first[b] if first else 0
                    there = min(width, n - lo)
                    same_rows(o[b, :there], rows(i, b, lo, lo + there), dtype)
                    assert (o[b, there:] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_every_byte_under_extreme_scales(dtype):
    """Products of 2^-135 and of 2^128: the smallest values round to the type's, the largest become infinite."""
    p = Pool([0], [8], 1, 256, 8, 1)
    for i in range(2):
        p.codes[i][:] = torch.arange(256, dtype=torch.int32).to(torch.uint8)
        p.scales[i][:] = torch.tensor([2.0 ** -126, 2.0 ** -120, 1.0, 3.0, -0.7, 2.0 ** 119, 0.0, 2.0 ** 120])
    (k, v), _ = read_back(p, [c.to(DEV) for c in p.codes], [s.to(DEV) for s in p.scales], dtype)
    s = p.scales[0][int(p.table[0, 0]), 0].numpy().astype(np.float64)
    want = oracle8.E4M3[None, :] * s[:, None]
    with np.errstate(over="ignore", invalid="ignore"):
        want = np.where(np.abs(want) >= 2.0 ** 128, np.sign(want) * np.inf, want)
    got = f64(k)[:, 0]
    inf = np.isinf(want)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(np.sign(got[inf]), np.sign(want[inf]))
    same_rows(torch.from_numpy(np.where(inf, 0, got)), np.where(inf, 0, want), dtype)
    assert torch.equal(k.view(torch.int32 if dtype == F32 else torch.int16), v.view(torch.int32 if dtype == F32 else torch.int16))


def test_reads_into_the_dense_prefix_cache():
    """[B, Hkv, P, D], as the attention over a dense prefix cache takes it, and a slice of a larger one."""
    p = Pool([30, 12], [0, 0], 2, 64, 16, 16, seed=2)
    args = [c.to(DEV) for c in p.codes] + [s.to(DEV) for s in p.scales]
    want, _ = read_back(p, args[:2], args[2:], BF, dense=32)
    big = [torch.full((2, 2, 40, 64), 7.0, dtype=BF, device=DEV) for _ in range(2)]
    view = [x[:, :, 4:36].transpose(1, 2) for x in big]
    got = ds.ds_kv8_read(*args, p.table.to(DEV), i32(p.lens), *view)
    for i in range(2):
        assert torch.equal(got[i].nan_to_num(9.0), want[i].nan_to_num(9.0)) and (big[i][:, :, :4] == 7.0).all() and (big[i][:, :, 36:] == 7.0).all()


def test_reads_with_bad_lengths_rows_and_pages_are_flagged_and_left_out():
    p = Pool([20, 5, 9], [0, 0, 0], 2, 64, 8, 4, seed=5)
    args = [c.to(DEV) for c in p.codes], [s.to(DEV) for s in p.scales]
    flag = ds.DS_DEV_INDEX
    want, start = read_back(p, *args, BF)
    for n in (-1, 25, 2 ** 31 - 1):
        got, _ = read_back(p, *args, BF, lens=[20, n, 9], status=flag)
        for w, g in zip(want, got):
            assert (g[20:25] == 7.0).all() and torch.equal(g[:20].nan_to_num(9.0), w[:20].nan_to_num(9.0)) and torch.equal(g[25:].nan_to_num(9.0), w[25:].nan_to_num(9.0))
    got, _ = read_back(p, *args, BF, lens=[20, 3, 9], status=flag)             # two rows beyond the length
    assert (got[0][23:25] == 7.0).all() and torch.equal(got[0][:23].nan_to_num(9.0), want[0][:23].nan_to_num(9.0))
    t = p.table.clone()
    t[0, 1] = -3
    got, _ = read_back(p, *args, BF, table=t, status=flag)
    assert (got[1][8:16] == 7.0).all() and torch.equal(got[1][16:].nan_to_num(9.0), want[1][16:].nan_to_num(9.0))
    out = [torch.full((34, 2, 64), 7.0, dtype=BF, device=DEV) for _ in range(2)]
    for s, f in (([0, 20, 25, 999], [0, 0, 0]), ([0, 20, 19, 34], [0, 0, 0]), ([-4, 20, 25, 34], [0, 0, 0]), ([0, 20, 25, 34], [0, -1, 0])):
        st = status_word()
        ds.ds_kv8_read(*args[0], *args[1], p.table.to(DEV), i32(p.lens), *out, out_start=i32(s), first=i32(f), status=st)
        assert ds.ds_read_status(st) == flag, s


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_beyond_32_bit_offsets(dtype):
    small = Pool([20, 5], [4, 30], 4, 128, 64, 16, seed=5)
    n_pages = (1 << 31) // (64 * 128 * 4) + 40
    kv = small.rows(dtype)
    want = small.check(kv)
    far = small.table + (n_pages - small.codes[0].shape[0])
    codes = [torch.zeros(n_pages, 4, 64, 128, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.zeros(n_pages, 4, 4, device=DEV) for _ in range(2)]
    lo = n_pages - small.codes[0].shape[0]
    for big, x in zip(codes + scales, small.codes + small.scales):
        big[lo:] = x.to(DEV)
    got = small.write(kv, codes=codes, scales=scales, table=far)
    for a, b in zip(got[0] + got[1], want[0] + want[1]):
        assert torch.equal(a[lo:].nan_to_num(9.0) if a.is_floating_point() else a[lo:], b.nan_to_num(9.0) if b.is_floating_point() else b)
        assert not (a[:lo] != 0).any()
    out, _ = read_back(small, *got, dtype, table=far)
    ref, _ = read_back(small, *want, dtype)
    assert all(torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0)) for a, b in zip(out, ref))


# ------------------------------------------------------------------------------------------------ attention
class Case8:
    """A pool of 8-bit pages with shuffled tables; unused rows, blocks, pages and table entries hold what must not be used."""

    def __init__(self, lens, counts, Hq, Hkv, D, ps, T, dtype, seed=0, sharp=1.0, order="head", spare=2, room=0):
        g = torch.Generator().manual_seed(seed)
        B = len(lens)
        width = max(1, max(-(-n // ps) for n in lens))
        n_pages = B * width + spare
        self.table = torch.randperm(n_pages, generator=g)[:B * width].view(B, width).to(torch.int32)
        if room:      # columns of the table beyond every length: a call that may turn out long is divided otherwise
            self.table = torch.cat([self.table, torch.full((B, room), -7, dtype=torch.int32)], 1)
        self.lens, self.counts, self.ps, self.T, self.dtype, self.D = lens, counts, ps, T, dtype, D
        self.starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.N = int(self.starts[-1])
        self.q = (torch.randn(self.N + 3, Hq, D, generator=g) * sharp).to(dtype)      # three rows of nobody at the end
        used = torch.zeros(n_pages, ps, dtype=torch.bool)
        for b, n in enumerate(lens):
            t = torch.arange(n)
            used[self.table[b].long()[t // ps], t % ps] = True
        block = used.view(n_pages, ps // T, T).any(-1)
        self.codes, self.scales = [], []
        for junk in (math.nan, math.inf):
            scale = strided((n_pages, Hkv, ps // T), order, 0.0, torch.float32)
            scale.copy_(0.01 * torch.exp(0.7 * torch.randn(scale.shape, generator=g)))
            x = torch.randn(n_pages, Hkv, ps, D, generator=g) / scale.repeat_interleave(T, 2)[..., None]
            code = strided((n_pages, Hkv, ps, D), order, 0, torch.uint8)
            code.copy_(x.clamp(-448, 448).to(F8).view(torch.uint8))
            code.masked_fill_(~used[:, None, :, None], 0x7f)
            scale.masked_fill_(~block[:, None, :], junk)
            self.codes.append(code)
            self.scales.append(scale)

    def values(self):
        """What the cache stands for, float64, on the GPU (the bytes' values are checked against the table in test_oracle_paged8.py)."""
        return [c.to(DEV).view(F8).double() * s.to(DEV).double().repeat_interleave(self.T, 2)[..., None] for c, s in zip(self.codes, self.scales)]

    def place(self, b, t):
        return self.table[b, t // self.ps].long(), t % self.ps

    def run(self, scale=None, causal=True, window=0, sinks=0, max_len=0, workspace=None, stream=None, uniform=False, lens=None, starts=None,
            table=None, status=0):
        d = lambda t: t.to(DEV)  # noqa: E731  (keeps strides)
        out = torch.full((self.N + 3, self.q.shape[1], self.D), 7.0, dtype=self.dtype, device=DEV)
        lse = torch.full((self.N + 3, self.q.shape[1]), 7.0, dtype=F32, device=DEV)
        st = status_word()
        scale = 1 / math.sqrt(self.D) if scale is None else scale
        ds.ds_attn_paged8(d(self.q), *map(d, self.codes), *map(d, self.scales), d(self.table if table is None else table),
                          i32(self.lens if lens is None else lens), scale, None if uniform else i32(self.starts if starts is None else starts),
                          max_q=max(1, max(self.counts)), max_len=max_len, causal=causal, window=window, sinks=sinks, out=out, lse=lse, status=st,
                          workspace=workspace, stream=stream)
        torch.cuda.synchronize()
        assert ds.ds_read_status(st) == status
        assert (out[self.N:] == 7.0).all() and (lse[self.N:] == 7.0).all()       # rows of no sequence
        return out[:self.N], lse[:self.N], scale

    def reference(self, scale, causal=True, window=0, sinks=0, lens=None):
        k, v = self.values()
        return oracle8.attn_paged(self.q[:self.N].double().to(DEV), k, v, self.table, self.lens if lens is None else lens, self.starts, scale, causal,
                                  window, sinks)

    def check(self, **kw):
        out, lse, scale = self.run(**kw)
        ref = self.reference(scale, **{n: kw[n] for n in ("causal", "window", "sinks") if n in kw})
        self.compare(out, lse, ref, scale)
        return out, lse

    def extremes(self):
        """max|v| and sum|k| of a row at most, of what is used."""
        k, v = (torch.where(torch.isfinite(x), x.abs(), 0.0) for x in self.values())
        return float(v.max()), float(k.sum(-1).max())

    def compare(self, out, lse, ref, scale, keep=None):
        compare8(out, lse, ref, self.dtype, self.D, max(self.lens + [1]), f64(self.q)[:self.N], scale, *self.extremes(), keep)


def compare8(out, lse, ref, dtype, D, n, q, scale, most_v, most_k, keep=None):
    want, want_lse, spread, reach = ref
    got, got_lse, most_q = f64(out), f64(lse), np.abs(q).max(-1)
    if keep is not None:
        want, want_lse, spread, reach, got, got_lse, most_q = (x[keep] for x in (want, want_lse, spread, reach, got, got_lse, most_q))
    bf = dtype == BF
    E = (D + 4) * U * reach + (2.0 ** -21 if bf else 2.0 ** -39) * abs(scale) * most_q * most_k + (0.0 if bf else 2.0 ** -22 * reach)
    weights = 2 * (2 * E + 2.0 ** -21 + (2.0 ** -11 if bf else 2.0 ** -22)) + 4 * (16 + math.sqrt(n)) * U
    tol = (2.0 ** -8 if bf else U) * np.abs(want) + weights[..., None] * spread + n * (2.0 ** -29 if bf else 2.0 ** -33) * most_v
    assert np.isfinite(want).all()
    err = np.abs(got - want)
    assert (err <= tol).all(), (np.nanmax(err - tol), np.isnan(got).sum(), np.argwhere(~(err <= tol))[:4])
    empty = np.isneginf(want_lse)
    assert (np.isneginf(got_lse) == empty).all()
    fin = ~empty
    err = np.abs(got_lse[fin] - want_lse[fin])
    assert (err <= (E + 2.0 ** -21 + 4 * (16 + math.sqrt(n)) * U)[fin] + 4 * U * np.abs(want_lse[fin])).all(), err.max()


TYPES = [(BF, 128), (BF, 64), (F32, 64), (F32, 128)]


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (7, 1), (16, 2)])
def test_one_new_token_over_uneven_lengths(dtype, D, Hq, Hkv):
    Case8([1, 15, 16, 17, 63, 64, 65, 200, 0], [1] * 9, Hq, Hkv, D, 16, 16, dtype, seed=Hq + D).check()


@pytest.mark.parametrize("ps,T", [(1, 1), (3, 3), (8, 2), (24, 12), (64, 64), (128, 1), (500, 100)])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
def test_page_and_block_sizes(ps, T, dtype, D):
    Case8([1, 130, 77, 0, 257], [1, 2, 1, 1, 3], 6, 2, D, ps, T, dtype, seed=ps).check()


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("counts", [[4, 0, 1, 9, 2], [33, 40, 1, 16, 17]])
@pytest.mark.parametrize("room", [0, 500])
def test_several_new_rows(dtype, D, causal, counts, room):
    """Uneven numbers of new rows, none at all, and more rows than the cache holds (the first ones see nothing)."""
    lens = [70, 5, 129, 200, 1] if counts[0] == 4 else [33, 300, 65, 10, 131]
    Case8(lens, counts, 8, 4, D, 16, 8, dtype, seed=sum(counts), room=room).check(causal=causal)


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("Hq,Hkv,counts", [(8, 1, [3, 16, 0, 17]), (28, 4, [32, 1, 33, 5]), (2, 2, [64, 65, 128, 129]), (16, 1, [8, 9, 1, 24])])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False), dict(window=100, sinks=9), dict(window=300, sinks=130, causal=False)])
@pytest.mark.parametrize("room", [0, 500])
def test_many_rows_per_head(dtype, D, Hq, Hkv, counts, kw, room):
    """From a fraction of a 128-row tile to several of them, peaked and flat scores, ends inside tiles."""
    Case8([129, 600, 1000, 257], counts, Hq, Hkv, D, 16, 16, dtype, seed=Hq, sharp=2.0, room=room).check(**kw)
    Case8([3000, 64, 0, 1], counts, Hq, Hkv, D, 24, 12, dtype, seed=Hq + 1, sharp=4.0, room=room).check(**kw)


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (50, 4), (64, 64), (100, 17), (1000, 3), (7, 1000), (2 ** 31 - 1, 0)])
def test_window_and_first_tokens(dtype, D, causal, window, sinks):
    Case8([400, 3, 64, 129, 0, 250], [3, 1, 5, 2, 1, 20], 4, 2, D, 16, 4, dtype, seed=window % 1001).check(causal=causal, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,D,Hq,Hkv,lens,counts", [
    (BF, 128, 28, 4, [3000, 17, 900], [1, 1, 1]), (BF, 64, 2, 1, [20000], [2]), (BF, 128, 8, 8, [5000, 4999, 1], [5, 1, 1]),
    (F32, 128, 4, 2, [2500, 6000], [1, 3]), (BF, 128, 4, 1, [9000], [9]), (F32, 64, 8, 1, [7001], [1]), (BF, 128, 8, 2, [4000, 3100], [40, 64])])
@pytest.mark.parametrize("kw", [dict(), dict(window=2100, sinks=5)])
def test_long_lengths_are_split_and_joined(dtype, D, Hq, Hkv, lens, counts, kw):
    c = Case8(lens, counts, Hq, Hkv, D, 64, 64, dtype, seed=len(lens))
    out, lse = c.check(**kw)
    # the same bits again, and without a workspace (unsplit) the same within the tolerance
    again, lse2, _ = c.run(**kw)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    c.check(workspace=torch.empty(0, dtype=torch.uint8, device=DEV), **kw)


# dtype, D, Hq, Hkv, lengths, new rows, spare columns of the table (what a call may turn out to need decides its division)
PATHS = {
    "clusters": (BF, 128, 2, 2, [300, 70], [1, 1], 0),
    "clusters, 16 rows": (BF, 64, 8, 1, [300, 70], [2, 1], 0),
    "clusters, 32 rows": (BF, 128, 8, 1, [300, 70], [4, 3], 0),
    "an item per CTA": (BF, 64, 32, 32, [300, 70] * 8, [1] * 16, 0),
    "an item per CTA by the lengths": (BF, 128, 32, 32, [2900, 2800] * 4, [1] * 8, 0),
    "ranges": (BF, 128, 4, 2, [3000, 70], [1, 1], 1000),
    "ranges, 32 rows": (BF, 64, 16, 2, [3000, 70], [4, 1], 1000),
    "ranges, many sequences": (BF, 64, 8, 8, [1500] * 36, [1] * 36, 1000),
    "40 rows, clusters": (BF, 128, 2, 2, [300, 70], [40, 1], 0),
    "40 rows": (BF, 128, 8, 2, [3000, 70], [10, 1], 1000),
    "64 rows": (BF, 64, 4, 2, [300, 70], [32, 1], 1000),
    "100 rows": (BF, 128, 8, 2, [3000, 70], [25, 1], 1000),
    "200 rows": (BF, 64, 8, 2, [500, 70], [50, 1], 1000),
    "many rows of many sequences": (BF, 128, 8, 4, [600] * 36, [20] * 36, 1000),
    "40 rows, items that are not split": (BF, 128, 8, 4, [200, 70] * 12, [10, 20] * 12, 0),
    "100 rows, items that are not split": (BF, 64, 8, 2, [200, 100] * 10, [25, 1] * 10, 0),
    "200 rows, items that are not split": (BF, 128, 8, 2, [250, 1] * 10, [50, 50] * 10, 0),
    "fp32 clusters": (F32, 128, 2, 2, [300, 70], [1, 1], 0),
    "fp32 clusters, 16 rows": (F32, 64, 8, 2, [300, 70], [4, 1], 0),
    "fp32 ranges, 40 rows": (F32, 64, 8, 2, [3000, 70], [10, 1], 1000),
    "fp32 ranges": (F32, 128, 2, 2, [3000, 70], [1, 1], 1000),
}
every_path = pytest.mark.parametrize("path", list(PATHS))


def path_case(path, seed=0, T=8, **kw):
    dtype, D, Hq, Hkv, lens, counts, room = PATHS[path]
    return Case8(lens, counts, Hq, Hkv, D, 16, T, dtype, seed=seed, room=room, **kw)


@every_path
@pytest.mark.parametrize("scale", [None, 0.0, -0.2, 3.0, 1e-30])
def test_any_scale_on_every_path(path, scale):
    c = path_case(path, seed=5)
    out, lse = c.check(scale=scale)
    again, lse2, _ = c.run(scale=scale)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@every_path
def test_scales_of_blocks_that_differ_by_powers_of_ten(path):
    """V's scales over 2^-20 .. 1, K's over 2^-6 .. 1 with values to match; some negative, some zero."""
    c = path_case(path, seed=7, T=4)
    g = torch.Generator().manual_seed(1)
    for i, low in ((0, 6), (1, 20)):
        s = c.scales[i]
        fin = torch.isfinite(s)
        f = torch.exp2(-low * torch.rand(s.shape, generator=g)) * (1 - 2 * (torch.rand(s.shape, generator=g) < 0.2).float())
        f[torch.rand(s.shape, generator=g) < 0.05] = 0.0
        s.copy_(torch.where(fin, s * f, s))
    c.check(causal=False)


@every_path
@pytest.mark.parametrize("where", [2.0 ** 90, 2.0 ** -90, 2.0 ** 118])
def test_very_large_and_very_small_scales_of_values(path, where):
    c = path_case(path, seed=8)
    fin = torch.isfinite(c.scales[1])
    c.scales[1].copy_(torch.where(fin, (c.scales[1] / 0.1 * where).clamp(max=2.0 ** 119), c.scales[1]))
    c.check()


@every_path
def test_rising_scores_and_large_queries(path):
    """Scores that rise along the keys, so fast that no reference holds for long; queries of 2^60 against scales of 2^-60."""
    c = path_case(path, seed=9)
    c.q = (c.q.abs().float() * 2.0 ** 60).to(c.dtype)
    for b, n in enumerate(c.lens):
        t = torch.arange(n)
        page, off = c.table[b].long()[t // c.ps], t % c.ps
        c.codes[0][page, :, off] = torch.from_numpy(oracle8.encode((0.02 * t.numpy()).clip(max=60.0)))[:, None, None].expand(n, c.codes[0].shape[1], c.D)
    fin = torch.isfinite(c.scales[0])
    c.scales[0].copy_(torch.where(fin, torch.tensor(2.0 ** -60), c.scales[0]))
    c.check()


@every_path
def test_equal_keys_give_the_plain_average_at_any_size(path):
    """Every key the same, so large that scores are 1e36 and the like: weights alike, the plain average.  Tolerance: the weights'
    parts and the sums (2^-11 or 2^-22, 4 (16 + sqrt(n)) u) against the mean of |v|."""
    c = path_case(path, seed=2)
    b, n, rows = 0, c.lens[0], c.counts[0]
    c.q = (c.q.abs().float() + 0.1).to(c.dtype)
    t = torch.arange(n)
    c.codes[0][c.table[b].long()[t // c.ps], :, t % c.ps] = 0xfe
    fin = torch.isfinite(c.scales[0])
    c.scales[0].copy_(torch.where(fin, torch.tensor(2.0 ** 108), c.scales[0]))
    out, lse, scale = c.run(causal=False)
    v = c.values()[1][c.table[b].long()[t // c.ps].to(DEV), :, (t % c.ps).to(DEV)].cpu().numpy()      # [n, Hkv, D]
    G = c.q.shape[1] // c.codes[0].shape[1]
    want, spread = (x.mean(0).repeat(G, 0) for x in (v, np.abs(v)))
    w = 2.0 ** -11 if c.dtype == BF else 2.0 ** -22
    tol = (2.0 ** -8 if c.dtype == BF else U) * np.abs(want) + (2 * w + 4 * (16 + math.sqrt(n)) * U) * spread + n * (2.0 ** -29 if c.dtype == BF else 2.0 ** -33) * c.extremes()[0]
    assert (np.abs(f64(out[:rows]) - want) <= tol).all()
    assert torch.isfinite(lse[:rows]).all() and (lse[:rows] < -1e30).all()


@every_path
def test_what_a_query_does_not_see_cannot_reach_it(path):
    """NaN in K, V and the scales of the later new rows, and at a window's edge: the queries before them, and other sequences, must
    not notice; those that see them get NaN."""
    dtype, D, Hq, Hkv, lens, counts, room = PATHS[path]
    n, count = lens[0], max(4, counts[0])
    last, edge, everything = n - 1, n - count + 1 - 5, slice(None)

    c = Case8(lens, [count, *counts[1:]], Hq, Hkv, D, 16, 1, dtype, seed=3, room=room)
    for t in (last, edge - 1, edge):      # not the largest of V's scales, to which weights are relative: the others' bits stay
        page, off = c.place(0, t)
        c.scales[1][page, :, off] *= 1e-3
    clean, clean_lse, _ = c.run()

    def dirty(t, codes=(), scales=(), junk=math.nan):
        d = copy.copy(c)
        d.codes, d.scales = [x.clone() for x in c.codes], [x.clone() for x in c.scales]
        page, off = d.place(0, t)
        for i, dims in codes:
            d.codes[i][page, :, off, dims] = 0xff
        for i in scales:
            d.scales[i][page, :, off] = junk
        return d
    for d in (dirty(last, [(0, everything)]), dirty(last, [(1, everything)]), dirty(last, scales=[0]), dirty(last, scales=[1]),
              dirty(last, scales=[1], junk=math.inf), dirty(last, [(0, slice(3, 4))])):
        out, lse, _ = d.run()
        assert torch.equal(out[:count - 1], clean[:count - 1]) and torch.equal(lse[:count - 1], clean_lse[:count - 1])
        assert torch.equal(out[count:], clean[count:]) and torch.equal(lse[count:], clean_lse[count:])
        assert (~torch.isfinite(out[count - 1])).any()
    out, lse, _ = dirty(last, [(1, slice(1, None, 3))]).run()                     # V alone, some dimensions: only there
    assert torch.isnan(out[count - 1, :, 1::3]).all() and torch.equal(out[count - 1, :, 0::3], clean[count - 1, :, 0::3])
    assert torch.equal(out[:count - 1], clean[:count - 1]) and torch.equal(lse, clean_lse)
    # window 5: query 0 alone sees row end_0 - 5
    clean, clean_lse, _ = c.run(window=5)
    for d in (dirty(edge, [(1, everything)]), dirty(edge, scales=[1]), dirty(edge, [(0, everything)])):
        out, lse, _ = d.run(window=5)
        assert torch.isnan(out[0]).all() and torch.equal(out[1:], clean[1:]) and torch.equal(lse[1:], clean_lse[1:])
    out, lse, _ = dirty(edge - 1, [(0, everything), (1, everything)], [0, 1]).run(window=5)      # a row that nobody sees
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


@every_path
def test_nan_that_every_query_sees_is_in_every_output(path):
    c = path_case(path, seed=4)
    page, off = c.place(0, 5)
    c.codes[1][page, :, off, ::7] = 0x7f
    out, lse, scale = c.run(causal=False)
    rows = c.counts[0]
    assert torch.isnan(out[:rows, :, ::7]).all()
    keep = torch.ones(c.D, dtype=torch.bool)
    keep[::7] = False
    assert torch.isfinite(out[:rows][:, :, keep]).all() and torch.isfinite(out[rows:]).all() and torch.isfinite(lse).all()


@every_path
def test_bad_pages_lengths_and_rows_are_flagged_and_reach_no_other_sequence(path):
    c = path_case(path, seed=3)
    want, want_lse, scale = c.run()
    flag = ds.DS_DEV_INDEX
    mine = slice(int(c.starts[1]), int(c.starts[2]))
    for entry in (-5, 10 ** 6, c.codes[0].shape[0], -2 ** 31, 2 ** 31 - 1):
        t = c.table.clone()
        t[1, min(2, (c.lens[1] - 1) // c.ps)] = entry
        out, lse, _ = c.run(table=t, status=flag)
        out[mine], lse[mine] = want[mine], want_lse[mine]      # whatever page is read in its place, the others are as they were
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    keep = np.ones(c.N, dtype=bool)
    keep[mine] = False
    for n in (-1, -2 ** 31, c.table.shape[1] * c.ps + 1, 2 ** 31 - 1):
        out, lse, _ = c.run(lens=[n if b == 1 else x for b, x in enumerate(c.lens)], status=flag)
        c.compare(out, lse, c.reference(scale, lens=[0 if b == 1 else x for b, x in enumerate(c.lens)]), scale, keep)
    for at, value in ((-1, -2 ** 31), (0, -3)):                 # the last sequence's rows run backwards, the first one's begin before the array
        starts = c.starts.copy()
        starts[at] = value
        c.run(starts=starts, status=flag)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
def test_layouts_bytes_and_uniform_rows(dtype, D):
    """Row-major pages, slices of larger buffers (strides), float8 and byte tensors, row_start left out, the output in the queries' place."""
    c = Case8([100, 30, 7], [3, 3, 3], 6, 2, D, 16, 8, dtype, seed=8, order="row")
    want, _ = c.check()
    c.check(uniform=True, causal=False)
    both = torch.full((*c.codes[0].shape[:3], 2 * D), 0x7f, dtype=torch.uint8)
    both[..., :D], both[..., D:] = c.codes[0], c.codes[1]
    both = both.to(DEV).view(F8)
    scales = torch.stack(c.scales, -1).to(DEV)
    wide = torch.full((c.q.shape[0], 10, D), float("nan"), dtype=dtype)
    wide[:, 2:8] = c.q
    wide = wide.to(DEV)
    out = ds.ds_attn_paged8(wide[:, 2:8], both[..., :D], both[..., D:], scales[..., 0], scales[..., 1], c.table.to(DEV), i32(c.lens), 1 / math.sqrt(D),
                            i32(c.starts), max_q=3, out=wide[:, 2:8])
    assert torch.equal(out[:c.N], want) and torch.isnan(wide[:, :2]).all() and torch.isnan(wide[:, 8:]).all()


@every_path
def test_far_pages(path):
    """Pages of codes beyond 2^31 bytes."""
    c = path_case(path, seed=4)
    want, want_lse, _ = c.run()
    n_small, Hkv, ps, D = c.codes[0].shape
    n_pages = (1 << 31) // (Hkv * ps * D) + n_small + 5
    codes = [torch.zeros(n_pages, Hkv, ps, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.zeros(n_pages, Hkv, c.scales[0].shape[2], device=DEV) for _ in range(2)]
    for big, x in zip(codes + scales, c.codes + c.scales):
        big[n_pages - n_small:] = x.to(DEV)
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    ds.ds_attn_paged8(c.q[:c.N].to(DEV), *codes, *scales, (c.table + (n_pages - n_small)).to(DEV), i32(c.lens), 1 / math.sqrt(D), i32(c.starts),
                      max_q=max(c.counts), out=out, lse=lse)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_refusals_of_the_binding():
    c = Case8([40, 40], [1, 1], 4, 2, 64, 16, 8, BF)
    q, k, v, ks, vs, t = (x.to(DEV) for x in (c.q, *c.codes, *c.scales, c.table))
    n = i32(c.lens)
    call = lambda q=q, k=k, v=v, ks=ks, vs=vs, t=t, n=n, **kw: ds.ds_attn_paged8(q, k, v, ks, vs, t, n, 0.1, **kw)  # noqa: E731
    call()
    for bad in (dict(k=k.float()), dict(v=v[:, :, :8]), dict(v=v.transpose(0, 1).contiguous().transpose(0, 1)), dict(n=n.long()), dict(t=t.long()),
                dict(t=t[:1]), dict(out=q.float()), dict(lse=torch.zeros(2, device=DEV)), dict(row_start=n[:1]), dict(q=q.transpose(1, 2)),
                dict(q=q.half()), dict(ks=ks.double()), dict(ks=ks[:, :, :1]), dict(ks=ks[..., None]), dict(ks=ks[:1]), dict(vs=vs.cpu()),
                dict(ks=torch.cat([ks, ks, ks], 2)[:, :, :3], vs=torch.cat([vs, vs, vs], 2)[:, :, :3]), dict(status=torch.zeros(1, device=DEV))):
        with pytest.raises((ValueError, TypeError)):
            call(**bad)
    for bad in (dict(max_q=30), dict(window=-1), dict(max_q=0)):
        with pytest.raises(ds.DsError):
            call(**bad)
    x = torch.zeros(2, 2, 64, dtype=BF, device=DEV)
    write = lambda k=x, v=x, kc=k, ks=ks, n=n, **kw: ds.ds_kv8_write(k, v, kc, kc, ks, ks, t, n, **kw)  # noqa: E731
    for bad in (dict(k=x.half()), dict(k=x[0]), dict(v=x[:, :1]), dict(kc=k.float()), dict(ks=ks.int()), dict(n=n[:1]), dict(row_start=n),
                dict(k=x.transpose(0, 1).contiguous().transpose(0, 1))):
        with pytest.raises((ValueError, TypeError)):
            write(**bad)
    for bad in (dict(max_q=2), dict(max_q=0), dict(max_len=-1)):
        with pytest.raises(ds.DsError):
            write(**bad)
    read = lambda ko=x, vo=x, **kw: ds.ds_kv8_read(k, v, ks, vs, t, n, ko, vo, **kw)  # noqa: E731
    for bad in (dict(), dict(ko=x[None], vo=x[None]), dict(out_start=n), dict(out_start=i32([0, 1, 2]), first=n[:1]), dict(ko=x.half(), vo=x.half(), out_start=i32([0, 1, 2])),
                dict(vo=x.float(), out_start=i32([0, 1, 2]))):
        with pytest.raises((ValueError, TypeError)):
            read(**bad)


@every_path
@pytest.mark.parametrize("junk", [math.nan, math.inf, -math.inf])
def test_a_query_that_is_not_finite_is_its_own_output_only(path, junk):
    c = path_case(path, seed=12)
    clean, clean_lse, _ = c.run(causal=False)
    row, head = int(c.starts[1]) - 1, c.q.shape[1] - 1
    c.q[row, head, 5] = junk
    out, lse, _ = c.run(causal=False)
    assert torch.isnan(out[row, head]).all() and torch.isnan(lse[row, head])
    out[row, head], lse[row, head] = clean[row, head], clean_lse[row, head]
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


@every_path
def test_outputs_in_the_place_of_the_queries(path):
    c = path_case(path, seed=13)
    want, _, scale = c.run()
    q = c.q.to(DEV)
    ds.ds_attn_paged8(q, *(x.to(DEV) for x in (*c.codes, *c.scales, c.table)), i32(c.lens), scale, i32(c.starts), max_q=max(c.counts), out=q)
    assert torch.equal(q[:c.N], want) and torch.equal(q[c.N:].cpu(), c.q[c.N:])


# ------------------------------------------------------------------------------------------------ graphs, streams, a serving loop
@pytest.mark.parametrize("dtype,D,G,n,lens", [(BF, 128, 4, 1, [2000, 300, 77]), (BF, 128, 1, 1, [3000] * 30), (BF, 128, 4, 16, [2000, 300, 77]),
                                              (BF, 64, 4, 16, [9000, 300, 77]),
                                              (BF, 128, 4, 16, [200, 30] * 12), (F32, 64, 2, 2, [900, 5000, 1])])
def test_a_captured_call_reads_lengths_rows_and_tables_at_replay(dtype, D, G, n, lens):
    """Captured once with the longest lengths, replayed with others, which put the work on the CTAs differently."""
    B = len(lens)
    c = Case8(lens, [n] * B, 4 * G, 4, D, 16, 16, dtype, seed=3)
    args = [x.to(DEV) for x in (c.q, *c.codes, *c.scales, c.table)]
    length, rows = i32(lens), torch.tensor(c.starts, device=DEV)
    plan = ds.PagedAttn8Plan(*args, length, 0.1, row_start=rows, max_q=n, max_len=max(lens))
    plan.launch()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.launch()
        plan.launch()
    for step in range(3):
        new = [0 if step == 2 else max(0, x // (1 + (b + step) % 5) - step) for b, x in enumerate(lens)]
        starts = [0]
        for b in range(B):
            starts.append(starts[-1] + (n if (b + step) % 3 else n - 1))
        length.copy_(torch.tensor(new, dtype=torch.int32))
        rows.copy_(torch.tensor(starts, dtype=torch.int32))
        plan.out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = plan.out.clone()
        eager, lse = torch.full_like(got, 7.0), torch.zeros(got.shape[:2], device=DEV)
        ds.ds_attn_paged8(*args, length, 0.1, rows, max_q=n, max_len=max(lens), out=eager, lse=lse)
        assert torch.equal(got, eager) and (got[starts[-1]:] == 7.0).all()
        k, v = c.values()
        ref = oracle8.attn_paged(c.q[:starts[-1]].double().to(DEV), k, v, c.table, new, starts, 0.1, True)
        compare8(got[:starts[-1]], lse[:starts[-1]], ref, dtype, D, max(lens), f64(c.q)[:starts[-1]], 0.1, *c.extremes())


def test_two_captured_calls_side_by_side_and_another_stream():
    c = Case8([3000, 17], [1, 1], 4, 1, 64, 16, 16, BF, seed=9)
    want, _, _ = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _, _ = c.run(stream=side)
    assert torch.equal(got, want)
    args = [x.to(DEV) for x in (c.q, *c.codes, *c.scales, c.table)]
    plans = [ds.PagedAttn8Plan(*args, i32(c.lens), 0.125, row_start=i32(c.starts), out=torch.zeros_like(args[0])) for _ in range(2)]
    graphs = []
    for p in plans:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            p.launch()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, gr in zip(streams, graphs):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    for p in plans:
        assert torch.equal(p.out[:c.N], want[:c.N])
    if torch.cuda.device_count() > 1:
        with torch.cuda.device(1):
            assert torch.equal(plans[0].launch()[:c.N], want[:c.N])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,causal,block", [(8, True, 1), (1, True, 3), (8, False, 20)])
def test_serving_steps_end_to_end(dtype, T, causal, block):
    """Prompts, then steps of one row, of a few, or of a block that is denoised (rewritten) twice before the next; a finished request whose
    pages another takes.  Every step runs page bookkeeping, norm + rotary, the 8-bit write and attention on device state alone, from the third on
    as a captured graph; the cache equals the oracle's writes byte for byte, attention float64 attention over it, and reading back gives its rows."""
    B, Hq, Hkv, D, ps, max_rows, width = 4, 4, 2, 64, 8, 96, 16
    n_pages = B * width
    g = torch.Generator().manual_seed(T)
    rope = ds.RopeTable(D, 1e4)
    table = torch.zeros(B, width, dtype=torch.int32, device=DEV)
    free, cnt = torch.randperm(n_pages, generator=g).to(torch.int32).to(DEV), i32([n_pages])
    kv_len, n_new, done = i32([0] * B), i32([0] * B), torch.zeros(B, dtype=torch.uint8, device=DEV)
    codes = [torch.full((n_pages, Hkv, ps, D), 0x7f, dtype=torch.uint8, device=DEV).view(F8) for _ in range(2)]
    scales = [torch.full((n_pages, Hkv, ps // T), 2.0 ** 60, device=DEV) for _ in range(2)]      # of former owners
    st, w = status_word(), torch.ones(D, dtype=dtype, device=DEV)
    qkv = torch.zeros(max_rows, Hq + 2 * Hkv, D, dtype=dtype, device=DEV)
    ko, vo = (torch.zeros(max_rows, Hkv, D, dtype=dtype, device=DEV) for _ in range(2))
    pages = ds.PageUpdatePlan(kv_len, n_new, table, free, cnt, ps, max_rows, done, kv_len_out=kv_len, free_cnt_out=cnt, status=st)
    rotate = ds.QkNormRopePlan(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], pages.positions, rope, w, w, k_out=ko, v_out=vo,
                               n_rows=pages.row_start[B:], status=st)
    write = ds.Kv8WritePlan(ko, vo, *codes, *scales, table, kv_len, row_start=pages.row_start, max_q=40, status=st)
    attend = ds.PagedAttn8Plan(rotate.q_out, *codes, *scales, table, kv_len, 0.125, row_start=pages.row_start, max_q=40, causal=causal, status=st,
                               lse=torch.zeros(max_rows, Hq, dtype=F32, device=DEV))
    back = torch.zeros(2, B, width * ps, Hkv, D, dtype=dtype, device=DEV)
    read = ds.Kv8ReadPlan(*codes, *scales, table, kv_len, back[0], back[1], status=st)

    def append():
        pages.launch()
        denoise()

    def denoise():
        rotate.launch()
        write.launch()
        attend.launch()
        read.launch()
    graphs = {}
    held_c, held_s = [c.view(torch.uint8).cpu().numpy() for c in codes], [s.cpu().numpy() for s in scales]
    steps = [([5, 17, 0, 40], [], append)] + [([block] * B, [], append), ([block] * B, [], denoise)] * 2 + [([block, 0, block, 30], [3], append)]
    for t, (new, over, step) in enumerate(steps + [([block] * B, [], append)]):
        n_new.copy_(torch.tensor(new))
        done.zero_()
        done[over] = 1
        qkv.copy_(torch.randn(qkv.shape, generator=g) * torch.exp(torch.randn(max_rows, 1, 1, generator=g)))
        if t >= 3 and step not in graphs:
            graphs[step] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graphs[step]):
                step()
        if t >= 3:
            graphs[step].replay()
        else:
            step()
        assert ds.ds_read_status(st) == 0
        starts, lens, tab = pages.row_start.cpu().numpy(), kv_len.tolist(), table.cpu().numpy()
        assert starts.tolist() == [0, *np.cumsum(new)]
        for i, x in enumerate((ko, vo)):
            held_c[i], held_s[i] = oracle8.write(f64(x), held_c[i], held_s[i], T, tab, lens, starts, ps)
            assert np.array_equal(codes[i].view(torch.uint8).cpu().numpy(), held_c[i]) and np.array_equal(scales[i].cpu().numpy(), held_s[i])
        k, v = (oracle8.values(c, s) for c, s in zip(held_c, held_s))
        n = int(starts[-1])
        for i, x in enumerate((k, v)):
            for b, length in enumerate(lens):
                at = np.arange(length)
                same_rows(back[i, b, :length], x[tab[b, at // ps], :, at % ps], dtype)
        ref = oracle8.attn_paged(rotate.q_out[:n].double(), torch.from_numpy(k).to(DEV), torch.from_numpy(v).to(DEV), tab, lens, starts, 0.125, causal)
        most = [np.abs(np.concatenate([x[tab[b, np.arange(length) // ps], :, np.arange(length) % ps] for b, length in enumerate(lens)])) for x in (k, v)]
        compare8(attend.out[:n], attend.lse[:n], ref, dtype, D, max(lens), f64(rotate.q_out)[:n], 0.125, most[1].max(), most[0].sum(-1).max())

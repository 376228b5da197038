"""GPU parity of the paged-cache entry points against the float64 oracle, through the C ABI.

Tolerances, from arithmetic (u = 2^-24, half a unit of fp32):
* attention: an output is rounded once to its type (2^-8 |ref| in bf16, u |ref| in fp32).  Before that, a weight's
  relative error is twice the score's error E (a dot product of D terms, scaled: (D + 4) u reach, reach =
  scale max_t sum_d |q_d k_td|) plus the exponential's own 2^-21, and 2^-16 where the weights are split into two bf16
  halves for the tensor cores (bf16 only); the sums over n keys add 4 (16 + sqrt(n)) u.  Each counts against
  spread = sum_t p_t |v_t|, not against |ref|, which cancels.  The sum of weights doubles them.
* lse: E + 2^-21 + 4 (16 + sqrt(n)) u + 4 u |lse|.
* norm + rotary: 2^-8 |ref| or u |ref|, plus 64 u times the length of the rotated pair (sum of squares, root, division
  and weight 20 u; the angle's 2^-26 turns are 2 pi 2^-26 = 1.6 u; sine and cosine 2 units, two products, one sum,
  mscale).
Whole numbers are equal.
"""
import math

import numpy as np
import pytest
import torch

import paper_2601_17917_b200 as ds
from oracle import paged as oracle

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24


def f64(t):
    return t.detach().double().cpu().numpy()


def status_word():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------------------ attention
class Case:
    """A pool of pages with shuffled tables; unused rows, pages and table entries hold what must not be used."""

    def __init__(self, lens, counts, Hq, Hkv, D, ps, dtype, seed=0, sharp=1.0, order="head", spare=2, cap=None, room=0):
        g = torch.Generator().manual_seed(seed)
        B = len(lens)
        width = max(1, max(-(-n // ps) for n in lens)) if cap is None else cap
        n_pages = B * width + spare
        shape = (n_pages, Hkv, ps, D) if order == "head" else (n_pages, ps, Hkv, D)
        kc = torch.randn(shape, generator=g)
        vc = torch.randn(shape, generator=g)
        if order == "row":
            kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
        self.table = torch.randperm(n_pages, generator=g)[:B * width].view(B, width).to(torch.int32)
        if room:      # columns of the table beyond every length: a call that may turn out long is divided otherwise
            self.table = torch.cat([self.table, torch.full((B, room), -7, dtype=torch.int32)], 1)
        self.lens, self.counts, self.ps, self.dtype, self.D = lens, counts, ps, dtype, D
        starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.starts, self.N = starts, int(starts[-1])
        self.q = (torch.randn(self.N + 3, Hq, D, generator=g) * sharp).to(dtype)      # three rows of nobody at the end
        self.k, self.v = kc.to(dtype), vc.to(dtype)
        used = torch.zeros(n_pages, ps, dtype=torch.bool)
        for b, n in enumerate(lens):
            t = torch.arange(n)
            used[self.table[b].long()[t // ps], t % ps] = True
        hidden = ~used[:, None, :, None].expand(n_pages, Hkv, ps, D)
        self.k[hidden] = float("nan")
        self.v[hidden] = float("inf")

    def run(self, scale=None, causal=True, window=0, sinks=0, max_len=0, workspace=None, stream=None, uniform=False):
        d = lambda t: t.to(DEV)  # noqa: E731  (keeps strides)
        out = torch.full((self.N + 3, self.q.shape[1], self.D), 7.0, dtype=self.dtype, device=DEV)
        lse = torch.full((self.N + 3, self.q.shape[1]), 7.0, dtype=F32, device=DEV)
        st = status_word()
        scale = 1 / math.sqrt(self.D) if scale is None else scale
        ds.ds_attn_paged(d(self.q), d(self.k), d(self.v), d(self.table), torch.tensor(self.lens, dtype=torch.int32, device=DEV),
                         scale, None if uniform else torch.tensor(self.starts, device=DEV), max_q=max(1, max(self.counts)),
                         max_len=max_len, causal=causal, window=window, sinks=sinks, out=out, lse=lse, status=st,
                         workspace=workspace, stream=stream)
        torch.cuda.synchronize()
        assert ds.ds_read_status(st) == 0
        assert (out[self.N:] == 7.0).all() and (lse[self.N:] == 7.0).all()       # rows of no sequence
        return out[:self.N], lse[:self.N], scale

    def check(self, **kw):
        out, lse, scale = self.run(**kw)
        ref = oracle.attn_paged(f64(self.q)[:self.N], f64(self.k), f64(self.v), self.table.numpy(), self.lens, self.starts,
                                scale, kw.get("causal", True), kw.get("window", 0), kw.get("sinks", 0))
        compare(out, lse, ref, self.dtype, self.D, max(self.lens + [1]))
        return out, lse


def compare(out, lse, ref, dtype, D, n):
    want, want_lse, spread, reach = ref
    bf = dtype == BF
    E = (D + 4) * U * reach
    weights = 2 * (2 * E + 2.0 ** -21 + (2.0 ** -16 if bf else 0.0)) + 4 * (16 + math.sqrt(n)) * U
    tol = (2.0 ** -8 if bf else U) * np.abs(want) + weights[..., None] * spread
    got = f64(out)
    assert np.isfinite(want).all()
    err = np.abs(got - want)
    assert (err <= tol).all(), (np.nanmax(err - tol), np.isnan(got).sum(), np.argwhere(~(err <= tol))[:4])
    got, empty = f64(lse), np.isneginf(want_lse)
    assert (np.isneginf(got) == empty).all()
    fin = ~empty
    err = np.abs(got[fin] - want_lse[fin])
    assert (err <= (E + 2.0 ** -21 + 4 * (16 + math.sqrt(n)) * U)[fin] + 4 * U * np.abs(want_lse[fin])).all(), err.max()


TYPES = [(BF, 128), (BF, 64), (F32, 32), (F32, 64), (F32, 128), (F32, 256)]


@pytest.mark.parametrize("dtype,D", TYPES)
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 4), (7, 1), (16, 2)])
def test_one_new_token_over_uneven_lengths(dtype, D, Hq, Hkv):
    Case([1, 15, 16, 17, 63, 64, 65, 200, 0], [1] * 9, Hq, Hkv, D, 16, dtype, seed=Hq + D).check()


@pytest.mark.parametrize("ps", [1, 3, 8, 24, 64, 128, 500])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
def test_page_sizes(ps, dtype, D):
    Case([1, 130, 77, 0, 257], [1, 2, 1, 1, 3], 6, 2, D, ps, dtype, seed=ps).check()


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 64)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("counts", [[4, 0, 1, 9, 2], [33, 40, 1, 16, 17]])
@pytest.mark.parametrize("room", [0, 500])
def test_several_new_rows(dtype, D, causal, counts, room):
    """Uneven numbers of new rows, none at all, and more rows than the cache holds (the first ones see nothing)."""
    lens = [70, 5, 129, 200, 1] if counts[0] == 4 else [33, 300, 65, 10, 131]
    Case(lens, counts, 8, 4, D, 16, dtype, seed=sum(counts), room=room).check(causal=causal)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,counts", [(8, 1, [3, 16, 0, 17]), (28, 4, [32, 1, 33, 5]), (2, 2, [64, 65, 128, 129]),
                                           (16, 1, [8, 9, 1, 24])])
@pytest.mark.parametrize("kw", [dict(), dict(causal=False), dict(window=100, sinks=9), dict(window=300, sinks=130, causal=False)])
@pytest.mark.parametrize("room", [0, 500])
def test_many_rows_per_head(D, Hq, Hkv, counts, kw, room):
    """From a fraction of a 128-row tile to several of them, peaked and flat scores, ends inside tiles."""
    Case([129, 600, 1000, 257], counts, Hq, Hkv, D, 16, BF, seed=Hq, sharp=2.0, room=room).check(**kw)
    Case([5000, 64, 0, 1], counts, Hq, Hkv, D, 24, BF, seed=Hq + 1, sharp=4.0, room=room).check(**kw)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kw", [dict(), dict(window=100, sinks=9), dict(window=1), dict(window=300, sinks=130, causal=False)])
def test_many_rows_of_many_sequences(D, kw):
    lens = [(37 * b) % 450 for b in range(80)]
    Case(lens, [20 - b % 9 if b % 13 else 0 for b in range(80)], 8, 4, D, 16, BF, seed=D).check(**kw)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (50, 4), (64, 64), (100, 17), (1000, 3), (7, 1000)])
def test_window_and_first_tokens(dtype, D, causal, window, sinks):
    Case([400, 3, 64, 129, 0, 250], [3, 1, 5, 2, 1, 20], 4, 2, D, 16, dtype, seed=window).check(causal=causal, window=window,
                                                                                              sinks=sinks)


@pytest.mark.parametrize("dtype,D,Hq,Hkv,lens,counts", [
    (BF, 128, 28, 4, [3000, 17, 900], [1, 1, 1]), (BF, 64, 2, 1, [20000], [2]), (BF, 128, 8, 8, [5000, 4999, 1], [5, 1, 1]),
    (F32, 128, 4, 2, [2500, 6000], [1, 3]), (BF, 128, 4, 1, [9000], [9]), (F32, 64, 8, 1, [7001], [1])])
@pytest.mark.parametrize("kw", [dict(), dict(window=2100, sinks=5)])
def test_long_lengths_are_split_and_joined(dtype, D, Hq, Hkv, lens, counts, kw):
    c = Case(lens, counts, Hq, Hkv, D, 64, dtype, seed=len(lens))
    out, lse = c.check(**kw)
    # the same bits again, and without a workspace (unsplit) the same within the tolerance
    again, lse2, _ = c.run(**kw)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    c.check(workspace=torch.empty(0, dtype=torch.uint8, device=DEV), **kw)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,Hkv,n", [
    ([900, 1280, 30, 0, 1100, 700, 64, 65, 1000], 32, 1),       # short enough for a CTA each, whatever their lengths
    ([1400, 1500, 1450, 1321, 1490, 1500, 1333, 1404], 32, 1),   # longer, even: a CTA each, by the lengths on the device
    ([3000, 50, 1, 0, 300, 20, 64, 90], 32, 2),                  # longer, uneven: equal ranges
    ([2500] + [40] * 39, 4, 1), ([1500] * 36, 8, 2),             # more than 32 sequences: the search goes through shared memory
    ([700, 100, 2000], 2, 5), ([64] * 3, 1, 1)])                 # clusters of eight, of two
def test_how_the_work_is_divided(dtype, lens, Hkv, n):
    c = Case(lens, [min(n, 1 + b % 3) if n < 5 else n for b in range(len(lens))], 2 * Hkv, Hkv, 64, 16, dtype, seed=len(lens))
    out, lse = c.check()
    again, lse2, _ = c.run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,Hkv,n", [([1400] * 100, 4, 1), ([1400 - 7 * b for b in range(100)], 4, 2), ([0] * 20 + [3000] + [90] * 60, 5, 1),
                                        ([2000] * 33, 8, 3), ([1500, 0] * 50 + [1600], 4, 1)])
def test_how_the_work_of_many_sequences_is_divided(dtype, lens, Hkv, n):
    """An item per CTA where the lengths are even enough, equal ranges else: with empty sequences, and sequences
    without rows, among them."""
    c = Case(lens, [0 if b % 11 == 5 else n for b in range(len(lens))], 2 * Hkv, Hkv, 64, 16, dtype, seed=len(lens))
    out, lse = c.check()
    again, lse2, _ = c.run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype,D,G,n", [(BF, 128, 1, 1), (BF, 128, 4, 8), (BF, 128, 4, 9), (BF, 64, 2, 40), (F32, 64, 2, 3), (F32, 256, 1, 1)])
@pytest.mark.parametrize("length", [40, 5000])
def test_the_output_may_be_the_queries(dtype, D, G, n, length):
    c = Case([length, 0, length // 3, n], [n, n, n - 1, n], 2 * G, 2, D, 16, dtype, seed=n, room=500 if length > 40 else 0)
    want, _, scale = c.run()
    q = c.q.to(DEV)
    k, v, t = (x.to(DEV) for x in (c.k, c.v, c.table))
    got = ds.ds_attn_paged(q, k, v, t, torch.tensor(c.lens, dtype=torch.int32, device=DEV), scale, torch.tensor(c.starts, device=DEV),
                           max_q=n, out=q)
    assert got is q and torch.equal(q[:c.N], want) and torch.equal(q[c.N:].cpu(), c.q[c.N:])


@pytest.mark.parametrize("dtype,D,G", [(BF, 128, 1), (BF, 128, 8), (F32, 64, 2)])
@pytest.mark.parametrize("causal", [True, False])
def test_windows_and_first_tokens_of_any_size(dtype, D, G, causal):
    """2^31 - 1 as window or number of first tokens hides nothing, also from queries of sequences shorter than their
    rows (whose first rows see nothing)."""
    c = Case([700, 3, 0, 64], [5, 5, 5, 5], 2 * G, 2, D, 16, dtype, seed=G)
    want, want_lse = c.check(causal=causal)
    top = (1 << 31) - 1
    c.check(causal=causal, window=1, sinks=top)
    for kw in (dict(window=top), dict(window=top, sinks=top), dict(window=704), dict(window=top - 5)):
        got, lse, _ = c.run(causal=causal, **kw)
        assert torch.equal(got, want) and torch.equal(lse, want_lse), kw


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_sequences_and_peaked_scores(dtype):
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 300, 150)]
    Case(lens, [1] * 150, 4, 2, 64, 16, dtype, seed=5, sharp=6.0).check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_negative_and_zero_scale(dtype):
    c = Case([100, 3], [2, 1], 2, 1, 64, 16, dtype, seed=2)
    c.check(scale=-0.2)
    c.check(scale=0.0)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
def test_layouts_and_uniform_rows(dtype, D):
    """Row-major pages, slices of larger buffers (strides), and row_start left out."""
    c = Case([100, 30, 7], [3, 3, 3], 6, 2, D, 16, dtype, seed=8, order="row")
    c.check()
    c.check(uniform=True, causal=False)
    # both caches as slices of one buffer, queries as a slice of a fused projection
    both = torch.full((*c.k.shape[:3], 2 * D), float("nan"), dtype=dtype)
    both[..., :D], both[..., D:] = c.k, c.v
    wide = torch.full((c.q.shape[0], 10, D), float("nan"), dtype=dtype)
    wide[:, 2:8] = c.q
    both, wide = both.to(DEV), wide.to(DEV)
    c2 = Case([100, 30, 7], [3, 3, 3], 6, 2, D, 16, dtype, seed=8, order="row")
    big = torch.zeros(c2.N + 3, 9, 2 * D, dtype=dtype, device=DEV)
    out = big[:, 1:7, D:]
    ds.ds_attn_paged(wide[:, 2:8], both[..., :D], both[..., D:], c2.table.to(DEV), torch.tensor(c2.lens, dtype=torch.int32, device=DEV),
                     1 / math.sqrt(D), torch.tensor(c2.starts, device=DEV), max_q=3, out=out)
    want, _, _ = c2.run()
    assert torch.equal(out[:c2.N], want)
    assert (big[:, 0] == 0).all() and (big[:, 7:] == 0).all() and (big[:, :, :D] == 0).all()


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 64)])
@pytest.mark.parametrize("Hq", [2, 4, 12, 40])
@pytest.mark.parametrize("room", [0, 500])
def test_what_a_query_does_not_see_cannot_reach_it(dtype, D, Hq, room):
    """NaN and infinities in K and V of the later new rows: a causal query before them must not notice; those that see
    them get NaN.  The same at the window's edge."""
    c = Case([70, 40], [6, 1], Hq, 2, D, 16, dtype, seed=3, room=room)
    clean, _, _ = c.run()
    dirty = Case([70, 40], [6, 1], Hq, 2, D, 16, dtype, seed=3, room=room)
    page, off = dirty.table[0, 67 // 16].long(), 67 % 16
    dirty.v[page, :, off] = float("nan")
    dirty.k[page, :, off] = float("inf")
    page, off = dirty.table[0, 69 // 16].long(), 69 % 16
    dirty.v[page, :, off, ::3] = float("inf")
    out, lse, _ = dirty.run()
    assert torch.equal(out[:3], clean[:3]) and torch.equal(out[6:], clean[6:])     # rows 64, 65, 66 and the other sequence
    assert torch.isnan(out[3:6]).all()
    # V alone infinite, at the last row: only the last query, only there
    dirty = Case([70, 40], [6, 1], Hq, 2, D, 16, dtype, seed=3, room=room)
    dirty.v[page, :, off, 1::3] = float("inf")
    out, lse, _ = dirty.run()
    assert torch.equal(out[:5], clean[:5]) and torch.isinf(out[5, :, 1::3]).all()
    assert torch.equal(out[5, :, 0::3], clean[5, :, 0::3]) and torch.equal(out[5, :, 2::3], clean[5, :, 2::3])
    # window 5: query 0 (row 64) sees rows 60 .. 64, query 1 rows 61 .. 65: row 60 belongs to query 0 alone
    clean, _, _ = c.run(window=5)
    dirty = Case([70, 40], [6, 1], Hq, 2, D, 16, dtype, seed=3, room=room)
    page, off = dirty.table[0, 60 // 16].long(), 60 % 16
    dirty.v[page, :, off] = float("nan")
    out, _, _ = dirty.run(window=5)
    assert torch.isnan(out[0]).all() and torch.equal(out[1:], clean[1:])
    # a row that no query of a window sees
    dirty = Case([70, 40], [6, 1], Hq, 2, D, 16, dtype, seed=3, room=room)
    for r in (0, 33, 58, 59):
        dirty.v[dirty.table[0, r // 16].long(), :, r % 16] = float("nan")
        dirty.k[dirty.table[0, r // 16].long(), :, r % 16] = float("nan")
    out, _, _ = dirty.run(window=5)
    assert torch.equal(out, clean)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scores_of_minus_infinity_have_no_weight(dtype):
    """K rows of the type's lowest value against positive queries: -inf or hugely negative scores."""
    c = Case([50, 20], [1, 1], 2, 1, 64, 16, dtype, seed=4)
    c.q.abs_()
    low = torch.finfo(dtype).min
    for b, rows in ((0, range(0, 50, 3)), (1, range(20))):
        for r in rows:
            c.k[c.table[b, r // 16].long(), :, r % 16] = low
    out, lse, scale = c.run()
    keep = [r for r in range(50) if r % 3]
    kk = torch.stack([c.k[c.table[0, r // 16].long(), 0, r % 16] for r in keep]).double()
    vv = torch.stack([c.v[c.table[0, r // 16].long(), 0, r % 16] for r in keep]).double()
    p = torch.softmax(scale * c.q[0].double() @ kk.T, -1)
    assert (out[0].double().cpu() - p @ vv).abs().max() <= 2.0 ** -7
    assert (out[1] == 0).all() and torch.isneginf(lse[1]).all()       # every score -inf: as if nothing were seen


def test_large_offsets_in_the_cache():
    """Pages whose offset passes 2^31 elements (a pool of 5 GB)."""
    ps, D, Hkv = 64, 128, 4
    n_pages = (1 << 31) // (ps * D * Hkv) + 40
    k = torch.zeros(n_pages, Hkv, ps, D, dtype=BF, device=DEV)
    small = Case([150, 64], [1, 2], 8, Hkv, D, ps, BF, seed=6)
    far = small.table + (n_pages - 10)
    assert int(far.max()) < n_pages
    k[far.view(-1).long()] = small.k[small.table.view(-1).long()].to(DEV)
    v = k.clone()
    v[far.view(-1).long()] = small.v[small.table.view(-1).long()].to(DEV)
    st = status_word()
    got = ds.ds_attn_paged(small.q.to(DEV), k, v, far.to(DEV), torch.tensor(small.lens, dtype=torch.int32, device=DEV),
                           1 / math.sqrt(D), torch.tensor(small.starts, device=DEV), max_q=2, status=st)
    assert ds.ds_read_status(st) == 0
    assert torch.equal(got[:small.N], small.run()[0])


def test_bad_lengths_pages_and_rows_are_flagged_and_clamped():
    c = Case([40, 40, 40], [1, 1, 1], 2, 1, 64, 16, BF, seed=1)
    base = dict(q=c.q.to(DEV), k=c.k.to(DEV), v=c.v.to(DEV), table=c.table.to(DEV),
                lens=torch.tensor(c.lens, dtype=torch.int32, device=DEV), starts=torch.tensor(c.starts, device=DEV))

    def flagged(max_len=0, **kw):
        a, st = {**base, **kw}, status_word()
        out = ds.ds_attn_paged(a["q"], a["k"], a["v"], a["table"], a["lens"], 0.1, a["starts"], max_len=max_len, status=st)
        return ds.ds_read_status(st), out
    ok, want = flagged()
    assert ok == 0
    for entry in (-5, 10 ** 6, 9 + 2):
        t = base["table"].clone()
        t[1, 1] = entry
        s, out = flagged(table=t)
        assert s == ds.DS_DEV_INDEX and torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])
    for n in (-1, 49, 2 ** 31 - 1):
        l = base["lens"].clone()
        l[1] = n
        s, out = flagged(lens=l)
        assert s == ds.DS_DEV_INDEX and torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])
    assert flagged(max_len=39)[0] == ds.DS_DEV_INDEX
    for rows in ([0, 2, 3, 4], [0, 1, 2, 99], [-1, 1, 2, 3], [0, 1, 0, 1]):      # two rows with max_q = 1, past N, negative
        assert flagged(starts=torch.tensor(rows, dtype=torch.int32, device=DEV))[0] == ds.DS_DEV_INDEX, rows


def test_refusals_of_the_binding():
    c = Case([40, 40], [1, 1], 4, 2, 64, 16, BF)
    q, k, v, t = (x.to(DEV) for x in (c.q, c.k, c.v, c.table))
    n = torch.tensor(c.lens, dtype=torch.int32, device=DEV)
    call = lambda q=q, k=k, v=v, t=t, n=n, **kw: ds.ds_attn_paged(q, k, v, t, n, 0.1, **kw)  # noqa: E731
    call()
    for bad in (dict(k=k.float()), dict(v=v[:, :, :8]), dict(v=v.transpose(0, 1).contiguous().transpose(0, 1)), dict(n=n.long()),
                dict(t=t.long()), dict(t=t[:1]), dict(out=q.float()), dict(lse=torch.zeros(2, device=DEV)),
                dict(row_start=n[:1]), dict(q=q.transpose(1, 2)), dict(k=k[0], v=v[0]), dict(status=torch.zeros(1, device=DEV))):
        with pytest.raises((ValueError, TypeError)):
            call(**bad)
    for bad in (dict(max_q=3), dict(window=-1), dict(max_q=0)):
        with pytest.raises(ds.DsError):
            call(**bad)
    with pytest.raises(ds.DsError):
        call(q=q[..., :40], k=k[..., :40], v=v[..., :40])


# ------------------------------------------------------------------------------------------------ norm + rotary + write
def rope_case(N, Hq, Hkv, D, dtype, seed, ps=16, spare=3):
    g = torch.Generator().manual_seed(seed)
    qkv = (2 * torch.randn(N, Hq + 2 * Hkv, D, generator=g)).to(dtype).to(DEV)
    w = [(1 + 0.2 * torch.randn(D, generator=g)).to(dtype).to(DEV) for _ in range(2)]
    pos = torch.randint(0, 200000, (N,), generator=g, dtype=torch.int32)
    n_pages = -(-N // ps) + spare
    slots = torch.randperm(n_pages * ps, generator=g)[:N]
    return qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], w, pos, slots, n_pages


def rope_close(got, x, w, eps, pos, table, dtype):
    f, m, inter = table
    want, size = oracle.norm_rope(f64(x), None if w is None else f64(w), eps, pos.tolist(), f, m, inter)
    err = np.abs(f64(got) - want)
    tol = (2.0 ** -8 if dtype == BF else U) * np.abs(want) + 64 * U * size
    assert (err <= tol).all(), (err - tol).max()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,Hq,Hkv,D,R", [(1, 1, 1, 128, 128), (5, 4, 2, 64, 64), (33, 7, 1, 128, 64), (130, 3, 3, 256, 256),
                                          (17, 4, 4, 96, 32), (9, 2, 1, 48, 16), (20, 28, 4, 128, 128), (3, 2, 2, 32, 16),
                                          (6, 2, 2, 80, 80), (2, 1, 1, 16, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rotation_and_cache_write(dtype, N, Hq, Hkv, D, R, interleaved):
    q, k, v, w, pos, slots, n_pages = rope_case(N, Hq, Hkv, D, dtype, seed=N + D)
    kw = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=2.0),
          dict(scaling="yarn", factor=8.0, orig_len=4096)][(N + D) % 4]
    rope = ds.RopeTable(R, 1e5, interleaved=interleaved, **kw)
    table = (*oracle.rope_frequencies(R, 1e5, **kw), interleaved)
    for weights in ((None, None), tuple(w), (w[0], None)):
        kc = torch.full((n_pages, Hkv, 16, D), 5.0, dtype=dtype, device=DEV)
        vc = torch.full_like(kc, 6.0)
        ko, vo = (torch.empty(N, Hkv, D, dtype=dtype, device=DEV) for _ in range(2))
        st = status_word()
        out = ds.ds_qk_norm_rope(q, k, v, pos.to(DEV), rope, *weights, eps=1e-5, k_out=ko, v_out=vo, k_cache=kc,
                                 v_cache=vc, slot_map=slots.to(DEV), status=st)
        assert ds.ds_read_status(st) == 0
        rope_close(out, q, weights[0], 1e-5, pos, table, dtype)
        rope_close(ko, k, weights[1], 1e-5, pos, table, dtype)
        assert torch.equal(vo, v)
        for cache, rows, fill in ((kc, ko, 5.0), (vc, v, 6.0)):
            flat = cache.transpose(1, 2).reshape(-1, Hkv, D)
            assert torch.equal(flat[slots], rows)
            rest = torch.ones(n_pages * 16, dtype=torch.bool)
            rest[slots] = False
            assert (flat[rest] == fill).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rope_in_place_rows_in_use_unset_slots_and_layouts(dtype):
    N, Hq, Hkv, D = 21, 4, 2, 64
    q, k, v, w, pos, slots, n_pages = rope_case(N, Hq, Hkv, D, dtype, seed=1)
    rope = ds.RopeTable(64)
    want = ds.ds_qk_norm_rope(q, k, v, pos.to(DEV), rope, *w)
    ko, vo = torch.empty(N, Hkv, D, dtype=dtype, device=DEV), torch.empty(N, Hkv, D, dtype=dtype, device=DEV)
    ds.ds_qk_norm_rope(q, k, v, pos.to(DEV), rope, *w, k_out=ko, v_out=vo)
    # in place on the fused buffer, 13 of 21 rows in use, two rows without a slot, row-major pages in one buffer
    fused = torch.cat([q, k, v], 1)
    q2, k2, v2 = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    slots = slots.clone()
    slots[3] = slots[12] = -1
    both = torch.full((n_pages, 16, Hkv, 2 * D), 9.0, dtype=dtype, device=DEV).transpose(1, 2)
    st = status_word()
    ds.ds_qk_norm_rope(q2, k2, v2, pos.to(DEV), rope, *w, q_out=q2, k_out=k2, v_out=v2, k_cache=both[..., :D],
                       v_cache=both[..., D:], slot_map=slots.to(DEV), n_rows=torch.tensor([13], dtype=torch.int32, device=DEV),
                       status=st)
    assert ds.ds_read_status(st) == 0
    assert torch.equal(q2[:13], want[:13]) and torch.equal(q2[13:], q[13:])
    assert torch.equal(k2[:13], ko[:13]) and torch.equal(k2[13:], k[13:]) and torch.equal(v2, v)
    flat = both.transpose(1, 2).reshape(-1, Hkv, 2 * D)
    keep = [n for n in range(13) if n not in (3, 12)]
    assert torch.equal(flat[slots[keep]], torch.cat([ko, v], -1)[keep])
    rest = torch.ones(n_pages * 16, dtype=torch.bool)
    rest[slots[keep]] = False
    assert (flat[rest] == 9.0).all()
    for count in (0, -4, 99):      # nothing; nothing; all
        fresh = torch.full_like(want, 3.0)
        ds.ds_qk_norm_rope(q, k, v, pos.to(DEV), rope, *w, q_out=fresh, n_rows=torch.tensor([count], dtype=torch.int32, device=DEV))
        assert torch.equal(fresh, want) if count == 99 else (fresh == 3.0).all()


def test_rope_far_and_negative_positions_and_extreme_values():
    D = 64
    q = torch.randn(6, 2, D, generator=torch.Generator().manual_seed(0)).to(DEV)
    q[4] = 0.0
    q[5] *= 1e18
    pos = torch.tensor([2 ** 31 - 1, -(2 ** 31), -7, 16777217, 5, 9], dtype=torch.int32)
    w = torch.ones(D, device=DEV)
    rope = ds.RopeTable(D, 10000.0)
    f, m = oracle.rope_frequencies(D, 10000.0)
    # the reference's angle in 64 bits is itself off by pos 2^-53 radians and more: exact phases instead
    turn = np.array([x for x in rope.struct.turn[:D // 2]], dtype=object)
    want = np.empty((6, 2, D))
    x = f64(q)
    y = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + 1e-6)
    for n in range(6):
        a = np.array([((int(pos[n]) * int(t)) % 2 ** 64) / 2.0 ** 64 * 2 * math.pi for t in turn])
        want[n, :, :32] = y[n, :, :32] * np.cos(a) - y[n, :, 32:] * np.sin(a)
        want[n, :, 32:] = y[n, :, 32:] * np.cos(a) + y[n, :, :32] * np.sin(a)
    got = f64(ds.ds_qk_norm_rope(q, q, q, pos.to(DEV), rope, w, w))
    size = np.tile(np.hypot(y[..., :32], y[..., 32:]), 2)
    assert (np.abs(got - want) <= 65 * U * size + 1e-30).all()
    assert (got[4] == 0).all()


def test_rope_bad_slots_are_flagged_and_not_written():
    N, D = 4, 64
    q, k, v, w, pos, slots, n_pages = rope_case(N, 2, 1, D, BF, seed=2)
    kc, vc = torch.zeros(n_pages, 1, 16, D, dtype=BF, device=DEV), torch.zeros(n_pages, 1, 16, D, dtype=BF, device=DEV)
    for bad in (-2, n_pages * 16, 2 ** 40):
        s, st = slots.clone(), status_word()
        s[2] = bad
        kc.zero_()
        ds.ds_qk_norm_rope(q, k, v, pos.to(DEV), ds.RopeTable(64), k_cache=kc, v_cache=vc, slot_map=s.to(DEV), status=st)
        assert ds.ds_read_status(st) == ds.DS_DEV_INDEX
        assert int((kc != 0).any(-1).sum()) == 3


# ------------------------------------------------------------------------------------------------ page bookkeeping
def page_case(B, ps, old_hi, new_hi, seed, done_share=0.3, tight=False):
    rng = np.random.default_rng(seed)
    old, new = rng.integers(0, old_hi + 1, B), rng.integers(0, new_hi + 1, B)
    done = (rng.random(B) < done_share).astype(np.uint8)
    width = max(1, -(-(old_hi + new_hi) // ps))
    held = -(-old // ps)
    n_pages = int(held.sum()) + (int(rng.integers(0, 4)) if tight else B * width + 1)
    n_pages = max(n_pages, 1)
    perm = rng.permutation(n_pages)
    table = np.full((B, width), -1)
    at = 0
    for b in range(B):
        table[b, :held[b]] = perm[at:at + held[b]]
        at += held[b]
    free = np.full(n_pages, -1)
    free[:n_pages - at] = perm[at:]
    return old, new, done, table, free, n_pages - at


def page_run(old, new, done, table, free, cnt, ps, max_rows, in_place=False, **kw):
    i = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)  # noqa: E731
    st, t, fl, n, c = status_word(), i(table), i(free), i(old), i([cnt])
    wide = torch.full((t.shape[0], t.shape[1] + 3), 77, dtype=torch.int32, device=DEV)
    wide[:, :t.shape[1]] = t
    t = wide[:, :t.shape[1]]
    pos = torch.full((max_rows + 5,), 77, dtype=torch.int32, device=DEV)
    slot = torch.full((max_rows + 5,), 77, dtype=torch.int64, device=DEV)
    r = ds.ds_page_update(n, i(new), t, fl, c, ps, max_rows=max_rows, done=None if done is None else torch.tensor(done, device=DEV),
                          kv_len_out=n if in_place else None, free_cnt_out=c if in_place else None,
                          positions=pos, slot_map=slot, status=st, **kw)
    s = ds.ds_read_status(st)
    assert (pos[max_rows:] == 77).all() and (slot[max_rows:] == 77).all() and (wide[:, -3:] == 77).all()
    h = lambda x: x.cpu().numpy().astype(np.int64)  # noqa: E731
    return dict(kv_len=h(r["kv_len_out"]), free_cnt=int(r["free_cnt_out"]), row_start=h(r["row_start"]),
                positions=h(pos[:max_rows]), slot_map=h(slot[:max_rows]), block_table=h(t), free_list=h(fl)), s


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,ps,old_hi,new_hi", [(1, 16, 0, 1), (1, 1, 5, 3000), (3, 4, 20, 9), (64, 16, 300, 40),
                                                (257, 24, 100, 33), (1500, 16, 90, 3), (1025, 1, 3, 2), (8192, 32, 40, 2),
                                                (5, 128, 70000, 20000)])
def test_page_update_matches_oracle(B, ps, old_hi, new_hi, in_place):
    for seed, tight in ((0, False), (1, True), (2, True)):
        old, new, done, table, free, cnt = page_case(B, ps, old_hi, new_hi, seed, tight=tight)
        if seed == 2:
            done = None
        max_rows = max(0, int(new.sum()) + (7 if not tight else -5))
        want = oracle.page_update(old, new, done, table, free, cnt, ps, max_rows)
        got, s = page_run(old, new, done, table, free, cnt, ps, max_rows, in_place)
        refused = want.pop("refused")
        assert s == (ds.DS_DEV_PAGES if refused else 0)
        for name, value in want.items():
            assert np.array_equal(got[name], value), (name, seed)


def test_page_update_without_sequences_rows_or_row_arrays():
    got, s = page_run(np.zeros(0, int), np.zeros(0, int), None, np.zeros((0, 4), int), [3, 1], 2, 16, 6)
    assert s == 0 and got["free_cnt"] == 2 and got["row_start"].tolist() == [0] and (got["slot_map"] == -1).all()
    i = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    table = torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    r = ds.ds_page_update(i([5, 0]), i([1, 2]), table, i([4, 6, 9, 0, 0, 0, 0, 0, 0, 0]), i([3]), 4, max_rows=8)
    assert r["kv_len_out"].tolist() == [6, 2] and table[1, 0] == 9 and r["slot_map"].tolist() == [1, 36, 37] + [-1] * 5


def test_page_update_flags_bad_input():
    old, new, done, table, free, cnt = page_case(6, 4, 20, 9, 3)
    ok, s = page_run(old, new, None, table, free, cnt, 4, 60)
    assert s == 0
    bad = old.copy()
    bad[2] = -3                                   # as if it held nothing
    got, s = page_run(bad, new, None, table, free, cnt, 4, 60)
    assert s == ds.DS_DEV_INDEX and got["kv_len"][2] == new[2]
    bad = new.copy()
    bad[1] = -1
    got, s = page_run(old, bad, None, table, free, cnt, 4, 60)
    assert s == ds.DS_DEV_INDEX and got["kv_len"][1] == old[1]
    bad[1] = 2 ** 31 - 1                          # beyond the table
    got, s = page_run(old, bad, None, table, free, cnt, 4, 60)
    assert s == ds.DS_DEV_INDEX and got["kv_len"][1] == old[1]
    for c in (-1, len(free) + 1):
        assert page_run(old, 0 * new, None, table, free, c, 4, 60)[1] & ds.DS_DEV_INDEX
    f = np.array(free)
    f[cnt - 1] = 10 ** 6                          # the first page handed out does not exist
    got, s = page_run([0], [3], None, np.zeros((1, 4), int), f, cnt, 4, 5)
    assert s == ds.DS_DEV_INDEX and got["slot_map"].tolist() == [-1] * 5 and got["positions"].tolist() == [0, 1, 2, 0, 0]
    # more pages come back than the list has room for
    got, s = page_run([16, 16], [0, 0], np.ones(2, np.uint8), np.arange(8).reshape(2, 4), [0, 1, 2], 2, 4, 5)
    assert s & ds.DS_DEV_INDEX and got["free_cnt"] == 3


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", [BF, F32])
def test_serving_steps_end_to_end(dtype):
    """Prompts, decode steps, a finished request whose slot and pages a new one takes: every step runs the three entry
    points on device state alone, and each step's attention equals float64 attention over the rows that were appended."""
    B, Hq, Hkv, D, ps, max_rows = 4, 4, 2, 64, 8, 64
    n_pages, width = 24, 8
    g = torch.Generator().manual_seed(0)
    rope = ds.RopeTable(D, 1e4)
    table = torch.zeros(B, width, dtype=torch.int32, device=DEV)
    free = torch.randperm(n_pages, generator=g).to(torch.int32).to(DEV)
    cnt = torch.tensor([n_pages], dtype=torch.int32, device=DEV)
    kv_len = torch.zeros(B, dtype=torch.int32, device=DEV)
    n_new, done = torch.zeros_like(kv_len), torch.zeros(B, dtype=torch.uint8, device=DEV)
    kc, vc = (torch.full((n_pages, Hkv, ps, D), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    st, w = status_word(), torch.ones(D, dtype=dtype, device=DEV)
    qkv = torch.zeros(max_rows, Hq + 2 * Hkv, D, dtype=dtype, device=DEV)
    pages = ds.PageUpdatePlan(kv_len, n_new, table, free, cnt, ps, max_rows, done, kv_len_out=kv_len, free_cnt_out=cnt, status=st)
    write = ds.QkNormRopePlan(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], pages.positions, rope, w, w,
                              k_cache=kc, v_cache=vc, slot_map=pages.slot_map, n_rows=pages.row_start[B:], status=st)
    attend = ds.PagedAttnPlan(write.q_out, kc, vc, table, kv_len, 0.125, row_start=pages.row_start, max_q=40, status=st,
                              lse=torch.zeros(max_rows, Hq, dtype=F32, device=DEV))

    def step():
        pages.launch()
        write.launch()
        attend.launch()
    held = [[] for _ in range(B)]           # (k, v) rows of every sequence, as the device rounded them
    graph = None
    for t, (new, over) in enumerate([([5, 17, 0, 40], []), ([1, 1, 0, 1], []), ([1, 1, 3, 1], []), ([1, 0, 1, 30], [3]),
                                     ([2, 1, 1, 1], []), ([1, 0, 1, 1], [1])]):
        n_new.copy_(torch.tensor(new))
        done.zero_()
        done[over] = 1
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        if t == 3:                           # from here on the step is one captured graph
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is not None:
            graph.replay()
        else:
            step()
        assert ds.ds_read_status(st) == 0
        starts = [0] + np.cumsum(new).tolist()
        assert pages.row_start.tolist() == starts
        f, m = oracle.rope_frequencies(D, 1e4)
        for b in range(B):
            if b in over:
                held[b] = []
            pos = range(len(held[b]), len(held[b]) + new[b])
            x = f64(qkv)[starts[b]:starts[b + 1]]
            kk, size = oracle.norm_rope(x[:, Hq:Hq + Hkv], np.ones(D), 1e-6, pos, f, m, False)
            slots = pages.slot_map[starts[b]:starts[b + 1]].cpu()
            got = kc.transpose(1, 2).reshape(-1, Hkv, D)[slots]
            assert (np.abs(f64(got) - kk) <= (2.0 ** -8 if dtype == BF else U) * np.abs(kk) + 64 * U * size).all()
            held[b] += [(f64(got[i]), x[i, Hq + Hkv:]) for i in range(new[b])]
            assert int(kv_len[b]) == len(held[b])
        # a dense cache of what was appended, one page per sequence, as the oracle's input
        top = max(len(h) for h in held)
        dk, dv = np.zeros((2, B, Hkv, top, D))
        for b in range(B):
            for i, (kk, vv) in enumerate(held[b]):
                dk[b, :, i], dv[b, :, i] = kk, vv
        n = starts[-1]
        ref = oracle.attn_paged(f64(write.q_out)[:n], dk, dv, np.arange(B)[:, None], [len(h) for h in held], starts, 0.125, True)
        compare(attend.out[:n], attend.lse[:n], ref, dtype, D, top)


@pytest.mark.parametrize("dtype,D,G,n,lens", [(BF, 128, 4, 1, [2000, 300, 77]), (BF, 128, 1, 1, [3000] * 30), (BF, 128, 4, 16, [2000, 300, 77]),
                                              (BF, 64, 4, 16, [9000, 300, 77]), (F32, 64, 2, 2, [900, 5000, 1])])
def test_a_captured_call_reads_lengths_rows_and_tables_at_replay(dtype, D, G, n, lens):
    """Captured once with the longest lengths, replayed with others, which put the work on the CTAs differently."""
    B = len(lens)
    c = Case(lens, [n] * B, 8 * G, 8, D, 16, dtype, seed=3)
    q, k, v, t = (x.to(DEV) for x in (c.q, c.k, c.v, c.table))
    length, rows = torch.tensor(lens, dtype=torch.int32, device=DEV), torch.tensor(c.starts, device=DEV)
    plan = ds.PagedAttnPlan(q, k, v, t, length, 0.1, row_start=rows, max_q=n, max_len=max(lens))
    plan.launch()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.launch()
        plan.launch()
    for step in range(4):
        new = [0 if step == 3 else max(0, x // (1 + (b + step) % 5) - step) for b, x in enumerate(lens)]
        starts = [0]
        for b in range(B):
            starts.append(starts[-1] + (n if (b + step) % 3 else n - 1))
        length.copy_(torch.tensor(new, dtype=torch.int32))
        rows.copy_(torch.tensor(starts, dtype=torch.int32))
        plan.out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = plan.out.clone()
        ref = oracle.attn_paged(f64(c.q)[:starts[-1]], f64(c.k), f64(c.v), c.table.numpy(), new, np.array(starts, np.int32), 0.1, True)
        eager, lse = torch.full_like(got, 7.0), torch.zeros(got.shape[:2], device=DEV)
        ds.ds_attn_paged(q, k, v, t, length, 0.1, rows, max_q=n, max_len=max(lens), out=eager, lse=lse)
        compare(got[:starts[-1]], lse[:starts[-1]], ref, dtype, D, max(lens))
        assert torch.equal(got, eager) and (got[starts[-1]:] == 7.0).all()


def test_streams_devices_and_plans_that_share_nothing():
    c = Case([3000, 17], [1, 1], 4, 1, 64, 16, BF, seed=9)
    want, _, _ = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _, _ = c.run(stream=side)
    assert torch.equal(got, want)
    q, k, v, t = (x.to(DEV) for x in (c.q, c.k, c.v, c.table))
    n, r = torch.tensor(c.lens, dtype=torch.int32, device=DEV), torch.tensor(c.starts, device=DEV)
    # two captured graphs of the same call, each with its own workspace, replayed side by side on two streams
    plans = [ds.PagedAttnPlan(q, k, v, t, n, 0.125, row_start=r, out=torch.zeros_like(q)) for _ in range(2)]
    want = plans[0].launch().clone()
    graphs = []
    for p in plans:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            p.launch()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for p in plans:
        p.out.zero_()
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

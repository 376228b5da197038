"""``ds_attn_paged`` on infinite and very large values and scores, on every way that a call may be divided and for every
kernel.  Tolerances: those of ``test_gpu_paged.py`` where nothing else is said."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as oracle
from test_gpu_paged import BF, F32, U, Case, compare, f64

pytestmark = pytest.mark.gpu

# dtype, D, Hq, Hkv, lengths, new rows, spare columns of the table (what a call may turn out to need decides its division)
PATHS = {
    "bf16 clusters": (BF, 128, 2, 2, [300, 70], [1, 1], 0),
    "bf16 clusters, 16 rows": (BF, 64, 8, 1, [300, 70], [2, 1], 0),
    "bf16 clusters, 32 rows": (BF, 128, 8, 1, [300, 70], [4, 3], 0),
    "bf16 an item per CTA": (BF, 64, 32, 32, [300, 70] * 8, [1] * 16, 0),
    "bf16 an item per CTA by the lengths": (BF, 128, 32, 32, [1450, 1400] * 4, [1] * 8, 0),
    "bf16 ranges": (BF, 128, 4, 2, [3000, 70], [1, 1], 1000),
    "bf16 ranges, 32 rows": (BF, 64, 16, 2, [3000, 70], [4, 1], 1000),
    "bf16 ranges, many sequences": (BF, 64, 8, 8, [1500] * 36, [1] * 36, 0),
    "bf16 33 rows, clusters": (BF, 128, 2, 2, [300, 70], [33, 1], 0),
    "bf16 tcgen05, 40 rows": (BF, 128, 8, 2, [3000, 70], [10, 1], 1000),
    "bf16 tcgen05, 64 rows": (BF, 64, 4, 2, [300, 70], [32, 1], 1000),
    "bf16 tcgen05, 100 rows": (BF, 128, 8, 2, [3000, 70], [25, 1], 1000),
    "bf16 tcgen05, 200 rows": (BF, 64, 8, 2, [500, 70], [50, 1], 1000),
    "bf16 tcgen05, many sequences": (BF, 128, 8, 4, [600] * 36, [20] * 36, 1000),
    "fp32 clusters": (F32, 128, 2, 2, [300, 70], [1, 1], 0),
    "fp32 clusters, 8 rows": (F32, 64, 8, 2, [300, 70], [2, 1], 0),
    "fp32 ranges, 20 rows": (F32, 32, 8, 2, [3000, 70], [5, 1], 1000),
    "fp32 ranges": (F32, 256, 2, 2, [3000, 70], [1, 1], 1000),
}
every_path = pytest.mark.parametrize("path", list(PATHS))


def case(path, seed=0, **kw):
    dtype, D, Hq, Hkv, lens, counts, room = PATHS[path]
    return Case(lens, counts, Hq, Hkv, D, 16, dtype, seed=seed, room=room, **kw)


def reference(c, scale, causal):
    with np.errstate(invalid="ignore"):
        return oracle.attn_paged(f64(c.q)[:c.N], f64(c.k), f64(c.v), c.table.numpy(), c.lens, c.starts, scale, causal)


@every_path
@pytest.mark.parametrize("causal", [True, False])
def test_an_infinite_value_that_every_query_sees_is_in_every_output(path, causal):
    """Rows in tiles without any hidden key: the average is infinite where V is, NaN where infinities of both signs meet,
    and what it was everywhere else."""
    c = case(path)
    clean, clean_lse, scale = c.run(causal=causal)
    for row, dims, value in ((5, slice(0, None, 7), math.inf), (100, slice(1, None, 7), -math.inf), (101, slice(2, None, 7), math.inf),
                             (130, slice(2, None, 7), math.inf), (199, slice(3, None, 7), math.inf), (200, slice(3, None, 7), -math.inf)):
        c.v[c.table[0, row // 16].long(), :, row % 16, dims] = value
    out, lse, _ = c.run(causal=causal)
    want = reference(c, scale, causal)[0]
    assert np.isposinf(want[:c.counts[0]]).any() and np.isneginf(want[:c.counts[0]]).any() and np.isnan(want[:c.counts[0]]).any()
    got = f64(out)
    for kind in (np.isposinf, np.isneginf, np.isnan):
        assert np.array_equal(kind(got), kind(want)), kind
    finite = torch.from_numpy(np.isfinite(want))
    assert torch.equal(out.cpu()[finite], clean.cpu()[finite]) and torch.equal(lse, clean_lse)


@every_path
def test_averages_of_very_large_values_are_finite(path):
    """|V| up to 0.95 2^127, of either sign and of one: no sum may pass the average it leads to.  Scores that rise along the
    keys, and so fast that no maximum holds for long, are what a lagging reference is worst for."""
    for rising in (False, True):
        c = case(path, seed=1)
        page, off = c.table.long(), c.ps
        finite = torch.isfinite(c.v)
        big = (c.v.float().clamp(-1.9, 1.9) * 2.0 ** 126).to(c.dtype)
        c.v = torch.where(finite, big.abs() if rising else big, c.v)
        if rising:
            c.q = c.q.abs()
            for b, n in enumerate(c.lens):
                t = torch.arange(n)
                c.k[page[b, t // off], :, t % off] = (0.02 * t)[:, None, None].expand(n, c.k.shape[1], c.D).to(c.dtype)
        c.check()


@every_path
def test_rows_whose_keys_are_all_of_the_lowest_values(path):
    """Scores of -1e36 and the like (queries of sums 1/200), all the same (K is the type's lowest value everywhere): the plain average.  And with one
    key at half of that: its value.  Equal keys have equal scores whatever their rounding, so the weights are 2^-20 or so
    all alike, kept to 2^-22 in two bf16 halves; the sums add 4 (16 + sqrt(n)) u."""
    c = case(path, seed=2)
    c.q = (c.q.abs().float() / c.q.abs().float().sum(-1, keepdim=True) / 200).to(c.dtype)
    low, b = torch.finfo(c.dtype).min, 0
    t = torch.arange(c.lens[b])
    place = (c.table[b].long()[t // c.ps], slice(None), t % c.ps)
    c.k[place] = low
    n, rows = c.lens[b], c.counts[b]
    out, lse, scale = c.run(causal=False)
    v = f64(c.v[place])                                                   # [n, Hkv, D]
    G = c.q.shape[1] // c.k.shape[1]
    want, spread = (x.mean(0).repeat(G, 0) for x in (v, np.abs(v)))
    tol = (2.0 ** -8 if c.dtype == BF else U) * np.abs(want) + (2.0 ** -22 + 4 * (16 + math.sqrt(n)) * U) * spread
    assert (np.abs(f64(out[:rows]) - want) <= tol).all()
    assert torch.isfinite(lse[:rows]).all() and (lse[:rows] < -1e34).all()
    one = n // 3
    c.k[c.table[b, one // c.ps].long(), :, one % c.ps] = low / 2
    out, _, _ = c.run(causal=False)
    assert torch.equal(out[:rows].cpu(), c.v[c.table[b, one // c.ps].long(), :, one % c.ps].repeat_interleave(G, 0)[None].expand(rows, -1, -1))


@every_path
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-30])
def test_any_scale(path, scale):
    case(path, seed=5).check(scale=scale)


@every_path
def test_an_infinite_value_of_small_weight(path):
    """A key some 10 to 40 nats below the others (2^-60 at the least): its infinity is in the output all the same."""
    c = case(path, seed=6)
    c.q = c.q.abs()
    page, off = c.table[0, 6].long(), 5
    c.k[page, :, off] = -3.0
    c.v[page, :, off, 1::5] = -math.inf
    out, lse, scale = c.run(causal=False)
    want, want_lse = reference(c, scale, False)[:2]
    got = f64(out)
    assert np.isneginf(want[:c.counts[0], :, 1::5]).all()
    assert np.array_equal(np.isneginf(got), np.isneginf(want)) and not np.isnan(got).any()

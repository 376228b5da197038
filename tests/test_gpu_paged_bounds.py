"""``ds_attn_paged`` with lengths, row ranges and page numbers that are out of bounds, and with pages far into a large pool, on
every way that a call may be divided and for every kernel: each has its own loads, scans and flags."""
import math

import numpy as np
import pytest
import torch

import paper_2601_17917_b200 as ds
from oracle import paged as oracle
from test_gpu_paged import DEV, F32, compare, f64, status_word
from test_gpu_paged_values import case, every_path

pytestmark = pytest.mark.gpu


def run(c, lens=None, starts=None, table=None, max_len=0, k=None, v=None):
    st = status_word()
    i32 = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32), device=DEV)  # noqa: E731
    out = torch.full(c.q.shape, 7.0, dtype=c.dtype, device=DEV)
    lse = torch.full(c.q.shape[:2], 7.0, dtype=F32, device=DEV)
    ds.ds_attn_paged(c.q.to(DEV), c.k.to(DEV) if k is None else k, c.v.to(DEV) if v is None else v, (c.table if table is None else table).to(DEV),
                     i32(c.lens if lens is None else lens), 1 / math.sqrt(c.D), i32(c.starts if starts is None else starts),
                     max_q=max(c.counts), max_len=max_len, out=out, lse=lse, status=st)
    return out, lse, ds.ds_read_status(st)


def others(c, out, lse, lens):
    """Every sequence but the second one, whose lengths are these, against the oracle."""
    lens = [0 if b == 1 else n for b, n in enumerate(lens)]
    ref = oracle.attn_paged(f64(c.q)[:c.N], f64(c.k), f64(c.v), c.table.numpy(), lens, c.starts, 1 / math.sqrt(c.D), True)
    keep = np.ones(c.N, dtype=bool)
    keep[c.starts[1]:c.starts[2]] = False
    compare(out[:c.N][torch.from_numpy(keep)], lse[:c.N][torch.from_numpy(keep)], [x[keep] for x in ref], c.dtype, c.D, max(lens))
    assert (out[c.N:] == 7.0).all() and (lse[c.N:] == 7.0).all()


@every_path
def test_bad_pages_lengths_and_rows_are_flagged_and_reach_no_other_sequence(path):
    c = case(path, seed=3)
    want, want_lse, s = run(c)
    assert s == 0
    mine = slice(int(c.starts[1]), int(c.starts[2]))
    for entry in (-5, 10 ** 6, c.k.shape[0], -2 ** 31, 2 ** 31 - 1):
        t = c.table.clone()
        t[1, 2] = entry
        out, lse, s = run(c, table=t)
        assert s == ds.DS_DEV_INDEX
        out[mine], lse[mine] = want[mine], want_lse[mine]      # whatever page is read in its place, the others are as they were
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    for n in (-1, -2 ** 31, c.table.shape[1] * c.ps + 1, 2 ** 31 - 1):
        lens = list(c.lens)
        lens[1] = n
        out, lse, s = run(c, lens=lens)
        assert s == ds.DS_DEV_INDEX
        others(c, out, lse, c.lens)
    top = max(c.lens) - 1
    out, lse, s = run(c, max_len=top)
    assert s == ds.DS_DEV_INDEX
    others(c, out, lse, [min(n, top) for n in c.lens])
    # the last sequence's rows run backwards (none are left), or past the end of the arrays; the first one's begin before it
    starts = c.starts.copy()
    starts[-1] = -2 ** 31
    out, lse, s = run(c, starts=starts)
    last = int(c.starts[-2])
    assert s == ds.DS_DEV_INDEX and (out[last:] == 7.0).all() and (lse[last:] == 7.0).all()
    starts[-1] = 2 ** 31 - 1
    assert run(c, starts=starts)[2] == ds.DS_DEV_INDEX
    starts = c.starts.copy()
    starts[0] = -3
    assert run(c, starts=starts)[2] == ds.DS_DEV_INDEX


@every_path
def test_pages_beyond_32_bit_offsets(path):
    c = case(path, seed=4)
    n_small, Hkv, ps, D = c.k.shape
    n_pages = (1 << 31) // (Hkv * ps * D) + n_small + 5
    k, v = (torch.full((n_pages, Hkv, ps, D), 3.0, dtype=c.dtype, device=DEV) for _ in range(2))
    k[n_pages - n_small:], v[n_pages - n_small:] = c.k.to(DEV), c.v.to(DEV)
    want, want_lse, s = run(c)
    out, lse, far = run(c, table=c.table + (n_pages - n_small), k=k, v=v)
    assert s == far == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)
    del k, v

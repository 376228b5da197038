"""Pins of the 8-bit cache's oracle (no GPU): every byte against the library's type, hand-worked values, invariants; and the
argument checks of the entry points and the layout of their structs, which need no GPU either."""
import ctypes
import math
import subprocess
from pathlib import Path

import numpy as np
import pytest
import torch

import paper_2601_17917_b200 as ds
from oracle import paged as rows
from oracle import paged8 as oracle
from paper_2601_17917_b200 import build as ds_build
from paper_2601_17917_b200 import paged, paged8

ROOT = Path(__file__).resolve().parents[1]
FAKE = 0x7f0000000000      # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    ds_build.build()
    return ds.lib()


# ------------------------------------------------------------------------------------------------ oracle
def test_every_byte_and_rounding_against_the_library_type():
    byte = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = byte.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.E4M3, want, equal_nan=True)
    x = torch.cat([torch.linspace(-460, 460, 4001), torch.logspace(-12, 3, 2000, base=2.0), -torch.logspace(-12, 3, 2000, base=2.0)]).float()
    between = torch.tensor(sorted(oracle.E4M3[:0x7f]))
    x = torch.cat([x, ((between[1:] + between[:-1]) / 2).float(), between.float()])      # ties
    x = x[x.abs() <= 448]
    got = oracle.encode(x.double().numpy())
    assert np.array_equal(got, x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert oracle.encode([math.nan, math.inf, -math.inf, 1000.0, -1000.0, -0.0]).tolist() == [0x7f, 0x7f, 0x7f, 0x7e, 0xfe, 0x80]


def test_exponents_by_hand():
    several = np.concatenate([np.exp2(np.arange(-148, 128, 0.37)), 448.0 * np.exp2(np.arange(-130.0, 119))])
    assert oracle.exponents(several).tolist() == [oracle.exponent(a) for a in several] and oracle.exponents(0.0) == -126
    assert [oracle.exponent(a) for a in (448.0, 448.1, 224.0, 224.1, 1.75, 1.76, 0.0, 2.0 ** -140, oracle.MOST)] == [0, 1, -1, 0, -8, -7, -126, -126, 120]


def test_write_by_hand():
    """Two rows at the end of a block of four that holds two: the second is larger, the block is rescaled."""
    codes, scales = np.zeros((2, 1, 4, 16), np.uint8), np.ones((2, 1, 1), np.float32)
    codes[1, 0, 0, :2], codes[1, 0, 1, 0] = oracle.encode([448.0, 3.0]), oracle.encode(0.0078125)
    x = np.zeros((2, 1, 16))
    x[0, 0, 0], x[1, 0, 0], x[1, 0, 1] = 1.0, -900.0, math.nan
    c, s = oracle.write(x, codes, scales, 4, np.array([[1]]), [4], [0, 2], 4)
    assert s[1, 0, 0] == 4.0 and s[0, 0, 0] == 1.0 and (c[0] == 0).all()           # 448 * 2 = 896 < 900
    v = oracle.values(c, s)[1, 0]
    assert v[0, 0] == 448.0 and v[0, 1] == 3.0 and v[1, 0] == 0.0078125 and v[2, 0] == 1.0 and v[3, 0] == -896.0 and math.isnan(v[3, 1])
    # all four rows anew: the scale follows them down
    c, s = oracle.write(np.full((4, 1, 16), 0.5), c, s, 4, np.array([[1]]), [4], [0, 4], 4)
    assert s[1, 0, 0] == 2.0 ** -9 and (oracle.values(c, s)[1] == 0.5).all()


@pytest.mark.parametrize("T", [1, 2, 8])
def test_written_rows_are_within_half_a_step(T):
    """Half a step: 2^-4 of the value, or 2^-10 of the scale where that is more."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((11, 2, 16)) * np.exp(2 * rng.standard_normal((11, 2, 1)))
    c, s = oracle.write(x, np.zeros((3, 2, 8, 16), np.uint8), np.ones((3, 2, 8 // T), np.float32), T, np.array([[2, 0]]), [11], [0, 11], 8)
    v = oracle.values(c, s)
    got = np.concatenate([v[2], v[0]], 1).transpose(1, 0, 2)[:11]
    step = np.concatenate([s[2], s[0]], 1).repeat(T, 1).T[:11][..., None]
    assert (np.abs(got - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * step)).all()


@pytest.mark.parametrize("kw", [dict(causal=True), dict(causal=False), dict(causal=True, window=7, sinks=3), dict(causal=False, window=2, sinks=0)])
def test_attention_of_all_queries_at_once_is_that_of_one_after_the_other(kw):
    rng = np.random.default_rng(1)
    lens, starts, table = [23, 2, 0, 9], [0, 5, 9, 10, 10], rng.permutation(16).reshape(4, 4)
    k, v, q = rng.standard_normal((16, 2, 6, 8)), rng.standard_normal((16, 2, 6, 8)), rng.standard_normal((11, 6, 8))
    a = rows.attn_paged(q, k, v, table, lens, starts, 0.4, kw["causal"], kw.get("window", 0), kw.get("sinks", 0))
    b = oracle.attn_paged(torch.from_numpy(q), torch.from_numpy(k), torch.from_numpy(v), table, lens, starts, 0.4, **kw)
    for x, y in zip(a, b):
        assert np.allclose(x, y, rtol=1e-13, atol=1e-14, equal_nan=True)


# ------------------------------------------------------------------------------------------------ entry points
def test_structs_match_the_header(tmp_path):
    names = {"ds_kv8_write_params": paged8.Kv8WriteParams, "ds_kv8_read_params": paged8.Kv8ReadParams, "ds_paged8_params": paged8.Paged8Params,
             "ds_paged_params": paged.PagedParams}
    lines = [f'printf("{n} %zu", sizeof({n}));' + "".join(f'printf(" %zu", offsetof({n}, {f[0]}));' for f in s._fields_) + 'printf("\\n");'
             for n, s in names.items()]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ds.h"\nint main(void) {' + "\n".join(lines) + "return 0; }")
    subprocess.run(["gcc", "-I", str(ROOT / "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.strip().splitlines():
        name, *numbers = line.split()
        s = names[name]
        assert [int(x) for x in numbers] == [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_], name


def fill(p, **kw):
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    return p


def write_params(**kw):
    p = fill(paged8.Kv8WriteParams(), B=2, Hkv=2, D=64, dtype=1, N=4, max_q=2, page_size=16, max_pages=3, n_pages=8, scale_block=4, kv_len=FAKE,
             block_table=FAKE, table_stride=3, k=FAKE, v=FAKE, kv_stride=(128, 64), k_cache=FAKE, v_cache=FAKE, cache_stride=(2048, 1024, 64),
             k_scale=FAKE, v_scale=FAKE, scale_stride=(8, 4, 1))
    return fill(p, **kw)


def read_params(**kw):
    p = fill(paged8.Kv8ReadParams(), B=2, Hkv=2, D=64, dtype=1, N=4, page_size=16, max_pages=3, n_pages=8, scale_block=4, kv_len=FAKE,
             block_table=FAKE, table_stride=3, k_cache=FAKE, v_cache=FAKE, cache_stride=(2048, 1024, 64), k_scale=FAKE, v_scale=FAKE,
             scale_stride=(8, 4, 1), k_out=FAKE, v_out=FAKE, out_stride=(512, 128, 64))
    return fill(p, **kw)


def attn_params(a=None, **kw):
    p = paged8.Paged8Params()
    fill(p.a, B=2, Hq=4, Hkv=2, D=64, dtype=1, N=4, max_q=2, page_size=16, max_pages=3, n_pages=8, causal=1, scale=0.1, kv_len=FAKE,
         block_table=FAKE, table_stride=3, q=FAKE, q_stride=(256, 64), k_cache=FAKE, v_cache=FAKE, cache_stride=(2048, 1024, 64), out=FAKE,
         out_stride=(256, 64))
    fill(p, scale_block=4, k_scale=FAKE, v_scale=FAKE, scale_stride=(8, 4, 1))
    fill(p.a, **(a or {}))
    return fill(p, **kw)


BAD_POOL = [dict(page_size=0), dict(max_pages=0), dict(n_pages=0), dict(scale_block=0), dict(scale_block=5), dict(scale_block=32), dict(table_stride=2),
            dict(dtype=2), dict(N=-1), dict(B=-1), dict(Hkv=0), dict(D=0), dict(kv_len=None), dict(block_table=None), dict(k_cache=None), dict(v_scale=None),
            dict(k_cache=FAKE + 8), dict(k_scale=FAKE + 2), dict(kv_len=FAKE + 2), dict(status=FAKE + 1), dict(cache_stride=(2048, 1024, 72)),
            dict(cache_stride=(2048, -1024, 64)), dict(scale_stride=(8, 4, -1))]
BIG = [dict(D=72), dict(D=272), dict(B=8193), dict(Hkv=32768), dict(page_size=1 << 20, scale_block=1 << 17), dict(max_pages=1 << 28, table_stride=1 << 28),
       dict(n_pages=1 << 28)]


def test_refusals_of_writing_and_reading(L):
    call = lambda name, p: getattr(L, name)(ctypes.byref(p), None)  # noqa: E731
    for kw in BAD_POOL + [dict(k=None), dict(v=FAKE + 2), dict(kv_stride=(128, 60)), dict(max_q=0), dict(max_q=3), dict(max_len=-1), dict(row_start=FAKE + 2)]:
        assert call("ds_kv8_write", write_params(**kw)) == ds.DS_ERR_INVALID_ARG, kw
    for kw in BAD_POOL + [dict(k_out=None), dict(v_out=FAKE + 2), dict(out_stride=(512, 128, 60)), dict(out_stride=(510, 128, 64)), dict(out_start=FAKE + 2),
                          dict(first=FAKE + 2)]:
        assert call("ds_kv8_read", read_params(**kw)) == ds.DS_ERR_INVALID_ARG, kw
    for kw in BIG:
        kw = dict(dict(row_start=FAKE), **kw)
        assert call("ds_kv8_write", write_params(**kw)) == ds.DS_ERR_UNSUPPORTED, kw
        kw["out_start"] = kw.pop("row_start")
        assert call("ds_kv8_read", read_params(**kw)) == ds.DS_ERR_UNSUPPORTED, kw
    assert call("ds_kv8_read", read_params(B=8192, N=1 << 19)) == ds.DS_ERR_UNSUPPORTED
    assert L.ds_kv8_write(None, None) == L.ds_kv8_read(None, None) == ds.DS_ERR_INVALID_ARG
    for kw in (dict(B=0), dict(N=0, row_start=FAKE)):
        assert call("ds_kv8_write", write_params(**kw)) == ds.DS_OK
    for kw in (dict(B=0), dict(N=0)):
        assert call("ds_kv8_read", read_params(**kw)) == ds.DS_OK


def test_refusals_of_attention(L):
    def status(p):
        rc = L.ds_attn_paged8(ctypes.byref(p), None)
        assert L.ds_attn_paged8_workspace(ctypes.byref(p)) == 0
        return rc
    for kw in (dict(scale_block=0), dict(scale_block=5), dict(k_scale=None), dict(v_scale=FAKE + 2), dict(scale_stride=(8, -4, 1))):
        assert status(attn_params(**kw)) == ds.DS_ERR_INVALID_ARG, kw
    for kw in (dict(Hq=3), dict(max_q=3), dict(max_q=0), dict(window=-1), dict(sinks=-1), dict(scale=math.nan), dict(q=None), dict(out=FAKE + 4),
               dict(dtype=2), dict(cache_stride=(2048, 1024, 72)), dict(q_stride=(256, 60)), dict(table_stride=2), dict(max_len=-1), dict(lse=FAKE + 1)):
        assert status(attn_params(kw)) == ds.DS_ERR_INVALID_ARG, kw
    for kw in (dict(D=32), dict(D=256), dict(B=8193, row_start=FAKE), dict(max_pages=1 << 28, table_stride=1 << 28), dict(max_q=1 << 29, row_start=FAKE),
               dict(max_q=1 << 20, row_start=FAKE, max_pages=1 << 26, table_stride=1 << 26, Hkv=512, Hq=1024)):
        assert status(attn_params(kw)) == ds.DS_ERR_UNSUPPORTED, kw
    assert status(attn_params(dict(page_size=1 << 17), scale_block=1 << 17)) == ds.DS_ERR_UNSUPPORTED
    assert L.ds_attn_paged8(None, None) == ds.DS_ERR_INVALID_ARG and L.ds_attn_paged8_workspace(None) == 0
    assert status(attn_params(dict(B=0))) == status(attn_params(dict(N=0, row_start=FAKE))) == ds.DS_OK


def test_refusals_of_the_binding_without_a_gpu():
    cache, scale = torch.zeros(4, 2, 16, 64, dtype=torch.uint8), torch.ones(4, 2, 4)
    rows = torch.zeros(3, 2, 64)
    with pytest.raises(ValueError):
        ds.ds_kv8_write(rows, rows, cache, cache, scale, scale, torch.zeros(3, 1, dtype=torch.int32), torch.ones(3, dtype=torch.int32))

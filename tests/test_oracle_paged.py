"""Pins of the paged-cache oracle (no GPU): library routines on special cases, invariants, hand-worked values; and the
argument checks and host arithmetic of the entry points, which need no GPU either."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2601_17917_b200 as ds
from oracle import paged as oracle
from paper_2601_17917_b200 import build as ds_build
from paper_2601_17917_b200 import paged


@pytest.fixture(scope="module")
def L():
    ds_build.build()
    return ds.lib()


# ------------------------------------------------------------------------------------------------ oracle
def test_attention_over_identity_pages_is_library_attention():
    rng = np.random.default_rng(0)
    B, Hq, Hkv, D, ps, n = 2, 6, 2, 16, 4, 3
    lens = [11, 8]
    k, v = rng.standard_normal((2, 6, Hkv, ps, D))
    q = rng.standard_normal((B * n, Hq, D))
    table = np.arange(6).reshape(2, 3)
    for causal in (False, True):
        out, lse, spread, _ = oracle.attn_paged(q, k, v, table, lens, [0, n, 2 * n], 0.3, causal)
        for b in range(B):
            kk = torch.tensor(k[table[b]].transpose(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :lens[b]]).repeat_interleave(3, 0)
            vv = torch.tensor(v[table[b]].transpose(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :lens[b]]).repeat_interleave(3, 0)
            qq = torch.tensor(q[b * n:(b + 1) * n]).transpose(0, 1)
            mask = torch.ones(n, lens[b], dtype=torch.bool)
            if causal:
                mask = torch.tril(mask, diagonal=lens[b] - n)
            ref = torch.nn.functional.scaled_dot_product_attention(qq, kk, vv, attn_mask=mask, scale=0.3).transpose(0, 1)
            assert np.abs(out[b * n:(b + 1) * n] - ref.numpy()).max() < 1e-12
            z = (0.3 * qq @ kk.transpose(1, 2)).masked_fill(~mask, -math.inf)
            assert np.abs(lse[b * n:(b + 1) * n] - torch.logsumexp(z, -1).T.numpy()).max() < 1e-12
        assert (spread >= np.abs(out) - 1e-12).all()


def test_visible_rows_by_hand():
    assert oracle.visible(5, 2, 0, True, 0, 0) == [0, 1, 2, 3] and oracle.visible(5, 2, 1, True, 0, 0) == [0, 1, 2, 3, 4]
    assert oracle.visible(5, 2, 0, False, 0, 0) == [0, 1, 2, 3, 4]
    assert oracle.visible(10, 1, 0, True, 3, 2) == [0, 1, 7, 8, 9]
    assert oracle.visible(10, 2, 0, True, 3, 0) == [6, 7, 8]
    assert oracle.visible(4, 1, 0, True, 9, 2) == [0, 1, 2, 3]
    assert oracle.visible(2, 4, 0, True, 0, 0) == [] and oracle.visible(2, 4, 2, True, 0, 0) == [0]


def test_one_key_and_zero_queries():
    q, k, v = np.zeros((1, 2, 4)), np.ones((1, 1, 2, 4)), np.arange(8.0).reshape(1, 1, 2, 4)
    out, lse, _, _ = oracle.attn_paged(q, k, v, np.zeros((1, 1), int), [1], [0, 1], 1.0, True)
    assert (out == v[0, 0, 0]).all() and (lse == 0).all()
    out, lse, _, _ = oracle.attn_paged(q, k, v, np.zeros((1, 1), int), [2], [0, 1], 1.0, True)
    assert np.allclose(out, v[0, 0].mean(0)) and np.allclose(lse, math.log(2))


def test_page_update_by_hand():
    r = oracle.page_update([3, 8, 0], [2, 1, 5], [0, 1, 0], [[5, -1], [1, 2], [-1, -1]], [0, 3, 4, 9, 9, 9], 3, 4, 8)
    # pages 1 and 2 come back on top; sequence 0 crosses into a new page, 1 starts again, 2 needs two
    assert r["kv_len"].tolist() == [5, 1, 5] and r["row_start"].tolist() == [0, 2, 3, 8]
    assert r["block_table"].tolist() == [[5, 2], [1, 2], [4, 3]] and r["free_cnt"] == 1
    assert r["positions"].tolist() == [3, 4, 0, 0, 1, 2, 3, 4]
    assert r["slot_map"].tolist() == [23, 8, 4, 16, 17, 18, 19, 12] and r["refused"] == []
    assert r["free_list"].tolist() == [0, 3, 4, 1, 2, 9]
    # one free page: the first sequence takes it, the second is refused, the third needs none
    r = oracle.page_update([4, 0, 2], [1, 1, 1], None, [[0, -1], [-1, -1], [1, -1]], [2, -1], 1, 4, 3)
    assert r["refused"] == [1] and r["kv_len"].tolist() == [5, 0, 3] and r["free_cnt"] == 0
    assert r["row_start"].tolist() == [0, 1, 1, 2] and r["slot_map"].tolist() == [8, 6, -1]
    # room for two rows: the second sequence's two do not fit, nor does what follows
    r = oracle.page_update([0, 0, 0], [1, 2, 1], None, [[-1], [-1], [-1]], [0, 1, 2], 3, 4, 2)
    assert r["refused"] == [1, 2] and r["kv_len"].tolist() == [1, 0, 0] and r["free_cnt"] == 2


def test_page_update_conserves_pages():
    rng = np.random.default_rng(3)
    for _ in range(30):
        B, ps, width = int(rng.integers(1, 9)), int(rng.integers(1, 6)), 8
        n_pages = int(rng.integers(1, 40))
        perm = rng.permutation(n_pages).tolist()
        lens, table = [], np.full((B, width), -1)
        for b in range(B):
            held = min(int(rng.integers(0, 4)), len(perm))
            table[b, :held] = [perm.pop() for _ in range(held)]
            lens.append(held * ps - (int(rng.integers(0, ps)) if held else 0))
        new = [int(x) for x in rng.integers(0, 3 * ps + 1, B)]
        done = rng.integers(0, 2, B)
        r = oracle.page_update(lens, new, done, table, perm + [-7] * (n_pages - len(perm)), len(perm), ps, 40)
        held = [p for b in range(B) for p in r["block_table"][b, :-(-int(r["kv_len"][b]) // ps)]]
        assert sorted(held + r["free_list"][:r["free_cnt"]].tolist()) == sorted(
            [p for b in range(B) for p in table[b, :-(-lens[b] // ps)]] + perm)
        used = r["slot_map"][r["slot_map"] >= 0]
        assert len(set(used.tolist())) == len(used) == r["row_start"][-1]


def test_norm_rope_is_a_complex_rotation():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((5, 3, 32)), rng.standard_normal(32)
    pos = [0, 1, 7, 100, 12345]
    f, m = oracle.rope_frequencies(16, 10000.0)
    out, size = oracle.norm_rope(x, w, 1e-5, pos, f, m, True)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-5) * w
    z = (y[..., 0:16:2] + 1j * y[..., 1:16:2]) * np.exp(1j * np.outer(pos, f))[:, None]
    assert np.allclose(out[..., 0:16:2], z.real) and np.allclose(out[..., 1:16:2], z.imag)
    assert np.allclose(out[..., 16:], y[..., 16:]) and np.allclose(out[0], y[0])
    half, _ = oracle.norm_rope(x, w, 1e-5, pos, f, m, False)
    assert np.allclose((half ** 2).sum(-1), (y ** 2).sum(-1)) and not np.allclose(half[1:], out[1:])


# ------------------------------------------------------------------------------------------------ host side
@pytest.mark.parametrize("R,theta,kw", [(128, 1e6, {}), (64, 10000.0, dict(scaling="linear", factor=8.0)),
                                        (128, 500000.0, dict(scaling="ntk", factor=4.0)), (16, 2.0, {}),
                                        (256, 1e6, dict(scaling="yarn", factor=4.0, orig_len=32768)),
                                        (32, 10000.0, dict(scaling="yarn", factor=0.5, orig_len=100, beta_fast=8.0, beta_slow=2.0))])
def test_rope_table_holds_exact_phases(L, R, theta, kw):
    t = ds.RopeTable(R, theta, interleaved=True, **kw).struct
    f, m = oracle.rope_frequencies(R, theta, **kw)
    turn = np.array([x / 2.0 ** 64 for x in t.turn[:R // 2]])
    # the reference is a double: its own rounding is what the comparison can see
    assert np.abs(turn - (f / (2 * math.pi)) % 1.0).max() <= 2.0 ** -50
    assert abs(t.mscale - m) <= 2.0 ** -24 * m and t.interleaved == 1 and t.rotary_dim == R
    assert all(x == 0 for x in t.turn[R // 2:])
    # phases modulo a turn for far positions: 64 bits leave 2^31 * 2^-65 turns
    for pos in (1, 999, 1 << 20, (1 << 31) - 1):
        got = np.array([(pos * x % 2 ** 64) / 2.0 ** 64 for x in t.turn[:R // 2]])
        want = np.array([math.fmod(pos * (x / 2.0 ** 64), 1.0) for x in t.turn[:R // 2]])
        d = np.abs(got - want)
        assert np.minimum(d, 1 - d).max() <= pos * 2.0 ** -52


def test_rope_table_refusals(L):
    t = paged.RopeTableStruct()
    ok = (128, 0, 1e4, 0, 1.0, 0.0, 32.0, 1.0)
    assert L.ds_rope_table_init(ctypes.byref(t), *ok) == ds.DS_OK
    assert L.ds_rope_table_init(None, *ok) == ds.DS_ERR_INVALID_ARG
    nan, inf = float("nan"), float("inf")
    for at, values, code in ((0, (0, 1, -16, 33), 1), (0, (24, 264, 512), 2), (2, (1.0, 0.5, nan, inf), 1), (3, (-1, 4), 1)):
        for v in values:
            a = list(ok)
            a[at] = v
            assert L.ds_rope_table_init(ctypes.byref(t), *a) == code, (at, v)
    for bad in ((128, 0, 1e4, 1, 0.0, 0, 32, 1), (128, 0, 1e4, 2, -1.0, 0, 32, 1), (128, 0, 1e4, 3, nan, 100, 32, 1),
                (128, 0, 1e4, 3, 4.0, 0, 32, 1), (128, 0, 1e4, 3, 4.0, 100, 1, 1), (128, 0, 1e4, 3, 4.0, 100, 32, 0)):
        assert L.ds_rope_table_init(ctypes.byref(t), *bad) == ds.DS_ERR_INVALID_ARG, bad
    with pytest.raises(ValueError):
        ds.RopeTable(128, scaling="dynamic")
    with pytest.raises(ds.DsError):
        ds.RopeTable(40)


FAKE = 0x7f0000000000      # never dereferenced: validation fails first


def _set(p, kw):
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(p, k)[:] = v
        else:
            setattr(p, k, v)
    return p


def _pages(**kw):
    p = paged.PageParams()
    p.B, p.page_size, p.max_pages, p.n_pages, p.max_rows, p.table_stride = 4, 16, 8, 64, 32, 8
    for n in ("kv_len", "n_new", "block_table", "free_list", "free_cnt", "kv_len_out", "free_cnt_out", "row_start"):
        setattr(p, n, FAKE)
    return _set(p, kw)


def test_page_update_argument_validation(L):
    for kw in (dict(B=-1), dict(page_size=0), dict(max_pages=0), dict(n_pages=0), dict(max_rows=-1), dict(kv_len=None),
               dict(n_new=None), dict(block_table=None), dict(free_list=None), dict(free_cnt=None), dict(kv_len_out=None),
               dict(free_cnt_out=None), dict(row_start=None), dict(table_stride=7), dict(kv_len=FAKE + 2),
               dict(slot_map=FAKE + 4), dict(positions=FAKE + 1), dict(status=FAKE + 2)):
        assert L.ds_page_update(ctypes.byref(_pages(**kw)), None) == ds.DS_ERR_INVALID_ARG, kw
    assert L.ds_page_update(None, None) == ds.DS_ERR_INVALID_ARG
    for kw in (dict(B=8193), dict(page_size=1 << 29), dict(n_pages=1 << 30)):
        assert L.ds_page_update(ctypes.byref(_pages(**kw)), None) == ds.DS_ERR_UNSUPPORTED, kw


def _qk(table, **kw):
    p = paged.QkParams()
    p.N, p.Hq, p.Hkv, p.D, p.dtype, p.page_size, p.n_pages, p.eps = 4, 8, 2, 128, 1, 16, 8, 1e-6
    for n in ("q", "k", "v", "positions", "q_out", "k_cache", "v_cache", "slot_map"):
        setattr(p, n, FAKE)
    p.rope = ctypes.addressof(table)
    p.q_stride[:], p.kv_stride[:], p.q_out_stride[:] = (1536, 128), (1536, 128), (1024, 128)
    p.cache_stride[:] = (4096, 2048, 128)
    return _set(p, kw)


def test_qk_norm_rope_argument_validation(L):
    t = ds.RopeTable(128).struct
    for kw in (dict(N=-1), dict(Hq=0), dict(Hkv=0), dict(D=0), dict(dtype=2), dict(eps=-1.0), dict(eps=float("nan")),
               dict(q=None), dict(k=None), dict(v=None), dict(positions=None), dict(q_out=None), dict(rope=None),
               dict(k_out=FAKE), dict(v_cache=None), dict(slot_map=None), dict(page_size=0), dict(n_pages=0),
               dict(q=FAKE + 8), dict(q_weight=FAKE + 2), dict(slot_map=FAKE + 4), dict(q_stride=(1532, 128)),
               dict(kv_stride=(-8, 128)), dict(cache_stride=(4096, 2048, 4)), dict(n_rows=FAKE + 2)):
        assert L.ds_qk_norm_rope(ctypes.byref(_qk(t, **kw)), None) == ds.DS_ERR_INVALID_ARG, kw
    assert L.ds_qk_norm_rope(None, None) == ds.DS_ERR_INVALID_ARG
    for kw in (dict(D=272), dict(D=136), dict(D=100), dict(D=64), dict(n_pages=1 << 28)):
        assert L.ds_qk_norm_rope(ctypes.byref(_qk(t, **kw)), None) == ds.DS_ERR_UNSUPPORTED, kw
    assert L.ds_qk_norm_rope(ctypes.byref(_qk(t, N=0)), None) == ds.DS_OK


def _attn(**kw):
    p = paged.PagedParams()
    p.B, p.Hq, p.Hkv, p.D, p.dtype, p.N, p.max_q, p.max_len = 4, 8, 2, 128, 1, 4, 1, 0
    p.page_size, p.max_pages, p.n_pages, p.causal, p.scale, p.table_stride = 16, 8, 64, 1, 0.1, 8
    for n in ("kv_len", "block_table", "q", "k_cache", "v_cache", "out"):
        setattr(p, n, FAKE)
    p.q_stride[:], p.out_stride[:], p.cache_stride[:] = (1024, 128), (1024, 128), (4096, 2048, 128)
    return _set(p, kw)


def test_attn_paged_argument_validation(L):
    for kw in (dict(B=-1), dict(Hq=0), dict(Hkv=3), dict(D=0), dict(dtype=5), dict(N=-1), dict(N=3), dict(max_q=0),
               dict(max_len=-1), dict(page_size=0), dict(max_pages=0), dict(n_pages=0), dict(window=-1), dict(sinks=-1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(kv_len=None), dict(block_table=None), dict(q=None),
               dict(k_cache=None), dict(v_cache=None), dict(out=None), dict(table_stride=7), dict(q=FAKE + 8),
               dict(lse=FAKE + 2), dict(q_stride=(1020, 128)), dict(cache_stride=(4096, 2048, 100)),
               dict(out_stride=(-1024, 128)), dict(row_start=FAKE + 1)):
        assert L.ds_attn_paged(ctypes.byref(_attn(**kw)), None) == ds.DS_ERR_INVALID_ARG, kw
        assert L.ds_attn_paged_workspace(ctypes.byref(_attn(**kw))) == 0
    assert L.ds_attn_paged(None, None) == ds.DS_ERR_INVALID_ARG
    for kw in (dict(D=96), dict(D=32), dict(D=256), dict(dtype=0, D=96), dict(B=8193, N=8193), dict(page_size=1 << 29),
               dict(B=1, N=1, Hq=1, Hkv=1, max_pages=1, n_pages=1, page_size=(1 << 31) - 1)):
        assert L.ds_attn_paged(ctypes.byref(_attn(**kw)), None) == ds.DS_ERR_UNSUPPORTED, kw
    assert L.ds_attn_paged(ctypes.byref(_attn(B=0)), None) == ds.DS_OK
    assert L.ds_attn_paged(ctypes.byref(_attn(N=0, row_start=FAKE)), None) == ds.DS_OK


def test_struct_layouts_match_the_header(tmp_path):
    import subprocess
    from pathlib import Path
    root = Path(ds.__file__).resolve().parents[1]
    names = {"ds_page_params": paged.PageParams, "ds_qk_params": paged.QkParams, "ds_paged_params": paged.PagedParams,
             "ds_rope_table": paged.RopeTableStruct}
    body = "".join(f'printf("{n} %zu", sizeof({n}));' + "".join(
        f'printf(" %zu", offsetof({n}, {f[0]}));' for f in s._fields_) + 'printf("\\n");' for n, s in names.items())
    (tmp_path / "l.c").write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ds.h"\nint main(void){' + body + "return 0;}")
    subprocess.run(["gcc", "-I", str(root / "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    for line in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines():
        n, *v = line.split()
        s = names[n]
        assert [int(x) for x in v] == [ctypes.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_], n


def test_binding_refuses_host_tensors_and_wrong_shapes():
    z = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        ds.ds_attn_paged(z, z[None], z[None], i[:, None], i, 0.1)
    with pytest.raises(ValueError, match="CUDA"):
        ds.ds_qk_norm_rope(z, z, z, i, None)
    with pytest.raises(ValueError, match="CUDA"):
        ds.ds_page_update(i, i, i[:, None], i, i, 16, max_rows=4)

"""How large a call of ds_attn_paged may be.  Without a GPU: the host's checks, and the index arithmetic at sizes where a
product or a difference would leave 32 bits (the header compiled for the CPU, undefined behaviour trapped).  On a GPU: one
long prompt."""
import ctypes
import math
import subprocess
from pathlib import Path

import pytest
import torch

import paper_2601_17917_b200 as ds
from paper_2601_17917_b200 import build as ds_build
from test_oracle_paged import FAKE, _attn

CSRC = Path(__file__).resolve().parents[1] / "paper_2601_17917_b200" / "csrc"
DEV = "cuda:0"


@pytest.fixture(scope="module")
def L():
    ds_build.build()
    return ds.lib()


def call(n_q, length, Hq, Hkv, D=128, dtype=1, B=1, page_size=64, **kw):
    pages = -(-length // page_size)
    return _attn(B=B, N=B * n_q, max_q=n_q, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, page_size=page_size, max_pages=pages, table_stride=pages,
                 n_pages=min(B * pages, (1 << 31) // page_size - 1), row_start=FAKE, q_stride=(Hq * D, D), out_stride=(Hq * D, D),
                 cache_stride=(Hkv * page_size * D, page_size * D, D), **kw)


@pytest.mark.parametrize("kw", [
    dict(n_q=32768, length=32768, Hq=32, Hkv=32), dict(n_q=32768, length=32768, Hq=32, Hkv=8), dict(n_q=8192, length=131072, Hq=32, Hkv=8),
    dict(n_q=16384, length=131072, Hq=28, Hkv=4), dict(n_q=1 << 20, length=1 << 20, Hq=16, Hkv=8), dict(n_q=32768, length=131072, Hq=16, Hkv=16, D=64, dtype=0),
    dict(n_q=1024, length=1 << 24, Hq=32, Hkv=32, max_len=2000), dict(n_q=64, length=(1 << 31) - 64, Hq=4, Hkv=4, max_len=(1 << 31) - 1025)])
def test_long_prompts_are_served(L, kw):
    assert L.ds_attn_paged_workspace(ctypes.byref(call(**kw))) > 0


@pytest.mark.parametrize("kw", [
    dict(n_q=1 << 20, length=(1 << 31) - 64, Hq=128, Hkv=8, max_len=(1 << 31) - 1025), dict(n_q=(1 << 30) - 1, length=1 << 20, Hq=1, Hkv=1),
    dict(n_q=1 << 20, length=1 << 20, Hq=128, Hkv=128, D=256, dtype=0), dict(n_q=1 << 30, length=64, Hq=1, Hkv=1),
    dict(n_q=1 << 28, length=64, Hq=4, Hkv=1), dict(n_q=1, length=64, Hq=(1 << 31) - 1, Hkv=1), dict(n_q=1 << 29, length=64, Hq=4096, Hkv=4096)])
def test_what_cannot_be_counted_is_refused(L, kw):
    p = call(**kw)
    assert L.ds_attn_paged(ctypes.byref(p), None) == ds.DS_ERR_UNSUPPORTED and L.ds_attn_paged_workspace(ctypes.byref(p)) == 0


PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include "ds_paged_index.cuh"
using namespace ds;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

int main() {
  std::mt19937_64 g(4);
  auto in = [&](long long lo, long long hi) { return lo + (long long)(g() % (unsigned long long)(hi - lo + 1)); };
  int fits = 0;
  for (int round = 0; round < 400000; ++round) {
    PagedShape s;
    s.B = 1, s.G = 1, s.causal = in(0, 3) > 0;
    s.Hkv = (int)in(1, 1 << in(0, 30));
    s.bound = in(0, 1) ? (int)in(kPagedMaxLen - 300, kPagedMaxLen) : (int)in(1, 1 << in(0, 30));
    s.max_q = in(0, 1) ? (int)in(0x3fffffff - 300, 0x3fffffff) : (int)in(1, 1 << in(0, 29)), s.N = s.max_q;
    auto any = [&]() { return (int)(in(0, 2) == 0 ? in(0x7fffffff - 300, 0x7fffffff) : in(0, 1) ? in(0, 300) : in(0, s.bound)); };
    const int window = any();
    s.window = paged_window(window, s.bound), s.sinks = any();
    s.tile_log2 = (int)in(4, 7), s.row_log2 = (int)in(0, 7);
    const PagedSeq most = paged_seq(s, 0, s.max_q, s.bound);
    if (!paged_units_fit(s, most)) continue;
    ++fits;
    const int len = in(0, 1) ? s.bound - (int)in(0, s.bound < 300 ? s.bound : 300) : (int)in(0, s.bound < 300 ? s.bound : 300);
    const PagedSeq q = paged_seq(s, 0, in(0, 1) ? s.max_q : (int)in(0, s.max_q), len);
    CHECK(q.len == len && (unsigned __int128)q.row_tiles * s.Hkv * q.tiles <= 0x7fffffff);
    const int tile = 1 << s.tile_log2;
    for (int k = 0; k < 12; ++k) {
      const int x = (int)(k < 6 ? in(0, ((long long)q.tiles + 1) * tile - 1) : ((long long)q.tiles + 1) * tile - 1 - in(0, tile));
      const int t = paged_key(q, x);
      CHECK(t >= -1 && t < len);
      const int i = q.count ? (int)(in(0, 1) ? in(0, q.count - 1) : in(0, q.count < 300 ? q.count - 1 : 300)) : 0;
      const int end = s.causal ? paged_max(q.end_min + i, 0) : len;      // as the kernels have it
      const long long e = s.causal ? (long long)len - q.count + 1 + i : len;
      if (t < 0 || q.count == 0) continue;
      const bool see = t < e && (window == 0 || t < s.sinks || t >= e - window);
      CHECK(see == paged_visible(s, t, end));
      if (x + 16 <= q.tiles * (long long)tile && paged_all_visible(s, q, x, 16)) CHECK(see);
    }
  }
  CHECK(fits > 50000);
  puts("ok");
  return 0;
}
"""


@pytest.mark.timeout(300)
def test_index_arithmetic_at_the_limits(tmp_path):
    src, exe = tmp_path / "limits.cpp", tmp_path / "limits"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-x", "c++",
                    "-I", str(CSRC), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


@pytest.mark.gpu
@pytest.mark.parametrize("n_q,length,Hq,Hkv,kw", [(32768, 32768, 32, 8, {}), (32768, 32768, 32, 8, dict(window=1000, sinks=4)),
                                                  (8192, 40000, 32, 32, dict(causal=False))])
def test_a_long_prompt(n_q, length, Hq, Hkv, kw):
    """Rows picked over the whole call against 64 bits.  bf16 outputs: 2^-8 |ref|, weights (two halves 2^-16, exponential 2^-21,
    twice for their sum; scores (D + 4) u reach, twice) and sums 4 (16 + sqrt(n)) u against sum p |v|."""
    D, ps, u = 128, 64, 2.0 ** -24
    g = torch.Generator(device=DEV).manual_seed(0)
    per = -(-length // ps)
    q = torch.randn(n_q, Hq, D, generator=g, device=DEV).bfloat16()
    k, v = (torch.randn(per, Hkv, ps, D, generator=g, device=DEV).bfloat16() for _ in range(2))
    table = torch.randperm(per, generator=g, device=DEV).view(1, per).to(torch.int32)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    st, lse = i32([0]), torch.zeros(n_q, Hq, device=DEV)
    out = ds.ds_attn_paged(q, k, v, table, i32([length]), 1 / math.sqrt(D), i32([0, n_q]), max_q=n_q, lse=lse, status=st, **kw)
    assert ds.ds_read_status(st) == 0
    for j, r in enumerate(sorted({0, 1, 127, 128, n_q // 2 + 3, n_q - 129, n_q - 2, n_q - 1})):
        h = (5 * j) % Hq
        kk, vv = (x[table[0].long(), h // (Hq // Hkv)].reshape(-1, D)[:length].double() for x in (k, v))
        z = kk @ q[r, h].double() / math.sqrt(D)
        reach = (kk.abs() @ q[r, h].double().abs() / math.sqrt(D)).max()
        t = torch.arange(length, device=DEV)
        end = length - n_q + 1 + r if kw.get("causal", True) else length
        see = t < end
        if "window" in kw:
            see &= (t < kw["sinks"]) | (t >= end - kw["window"])
        z = z.masked_fill(~see, -math.inf)
        p = torch.softmax(z, 0)
        want, spread, E = p @ vv, p @ vv.abs(), (D + 4) * u * reach
        tol = 2.0 ** -8 * want.abs() + (2 * (2 * E + 2.0 ** -21 + 2.0 ** -16) + 4 * (16 + math.sqrt(length)) * u) * spread
        assert ((out[r, h].double() - want).abs() <= tol).all(), (r, h)
        want = torch.logsumexp(z, 0)
        assert (lse[r, h] - want).abs() <= E + 2.0 ** -21 + 4 * (16 + math.sqrt(length)) * u + 4 * u * want.abs(), (r, h)

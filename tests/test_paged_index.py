"""The index arithmetic of ds_attn_paged (csrc/ds_paged_index.cuh) on the CPU: the header has no CUDA in it, so a small C++
program walks it over many shapes, bad lengths, row ranges and page numbers among them, and compares with the
definitions.  Every key that a query sees is visited once, every unit of work lies in one range, the parts of a split
item are the ones its join reads, and no cache row outside the pool is named."""
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parents[1] / "paper_2601_17917_b200" / "csrc"

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <vector>
#include "ds_paged_index.cuh"
using namespace ds;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

static void divisions() {
  std::mt19937_64 g(1);
  std::vector<int> ds = {1, 2, 3, 5, 7, 16, 24, 63, 64, 65, 1000, 65535, 65536, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, 0x7fffffff};
  for (int i = 0; i < 300; ++i) ds.push_back(1 + (int)(g() % 0x7fffffff) / (1 << (g() % 30)));
  for (int d : ds) {
    const FastDiv f = make_fast_div(d);
    std::vector<long long> xs = {0, 1, 0x7fffffffLL, 0x7ffffffeLL};
    for (int i = 0; i < 200; ++i) {
      const long long q = g() % (0x80000000LL / d + 1), x = q * d;
      xs.insert(xs.end(), {x - 1, x, x + 1, (long long)(g() % 0x80000000LL)});
    }
    for (long long x : xs)
      if (x >= 0 && x <= 0x7fffffffLL) CHECK(fast_div((int)x, f) == (int)(x / d));
  }
}

static void shapes() {
  std::mt19937_64 g(2);
  auto in = [&](int lo, int hi) { return lo + (int)(g() % (unsigned long long)(hi - lo + 1)); };
  for (int round = 0; round < 3000; ++round) {
    PagedShape s;
    s.B = in(1, 6), s.G = in(1, 8), s.Hkv = in(1, 3), s.max_q = in(1, 5) * (in(0, 3) ? 1 : 9);
    s.N = in(0, s.B * s.max_q), s.bound = in(1, 500), s.causal = in(0, 1);
    s.window = in(0, 2) ? 0 : in(1, 200), s.sinks = in(0, 2) ? in(0, 30) : in(0, 600);
    s.tile_log2 = in(4, 6), s.row_log2 = in(0, 5);
    const int tile = 1 << s.tile_log2;
    const int page_size = in(1, 40), n_pages = in(1, 9);
    const FastDiv pd = make_fast_div(page_size);
    std::vector<PagedSeq> q;
    std::vector<long long> base = {0};
    int row = 0;
    for (int b = 0; b < s.B; ++b) {
      const bool bad = in(0, 9) == 0;
      const int lo = bad ? in(-5, s.N + 5) : row, hi = bad ? in(-5, s.N + 9) : paged_min(s.N, row + in(0, s.max_q));
      row = bad ? row : hi;
      const int len = in(0, 9) == 0 ? in(-9, s.bound + 50) : in(0, s.bound);
      const PagedSeq x = paged_seq(s, lo, hi, len);
      CHECK(x.first >= 0 && x.count >= 0 && x.first + x.count <= s.N && x.count <= s.max_q);
      CHECK(x.len >= 0 && x.len <= s.bound);
      CHECK(x.bad == !(lo >= 0 && lo <= s.N && hi >= lo && hi <= s.N && hi - lo <= s.max_q && len >= 0 && len <= s.bound));
      CHECK((x.tiles == 0) == (x.count == 0) && (x.row_tiles << s.row_log2) >= x.count * s.G && (x.row_tiles == 0 || ((x.row_tiles - 1) << s.row_log2) < x.count * s.G));
      // keys: each visible one once, in order, none that nobody sees beyond whole tiles
      std::map<int, int> at;
      for (int k = 0; k < x.tiles * tile; ++k) {
        const int t = paged_key(x, k);
        CHECK(t >= -1 && t < x.len);
        if (t >= 0) {
          CHECK(!at.count(t));
          at[t] = k;
        }
      }
      std::set<int> wanted;
      for (int i = 0; i < x.count; ++i) {
        const int end = s.causal ? x.len - x.count + 1 + i : x.len;
        CHECK(end <= x.end_max && (i > 0 || !s.causal || end == x.end_min));
        for (int t = 0; t < x.len; ++t) {
          const bool see = t < end && (s.window == 0 || t < s.sinks || t >= end - s.window);
          CHECK(see == paged_visible(s, t, end));
          if (see) wanted.insert(t);
        }
        CHECK(!paged_visible(s, -1, end));
      }
      for (int t : wanted) CHECK(at.count(t));
      for (int k = 0; k + 16 <= x.tiles * tile && x.count; k += 16)
        if (paged_all_visible(s, x, k, 16))
          for (int i = 0; i < x.count; ++i)
            for (int j = 0; j < 16; ++j)
              CHECK(paged_visible(s, paged_key(x, k + j), s.causal ? x.end_min + i : x.len));
      // cache rows: inside the pool whatever the table holds
      for (auto &e : at) {
        const int slot = e.first - fast_div(e.first, pd) * page_size;
        CHECK(slot >= 0 && slot < page_size);
        const int page = paged_clamp_page(in(0, 3) ? in(0, n_pages - 1) : (int)g(), n_pages);
        CHECK(page >= 0 && page < n_pages);
      }
      q.push_back(x);
      base.push_back(base.back() + paged_units(s, x));
    }
    // the ranges
    const long long total = base.back();
    const int grid = in(1, 40), min_tiles = in(1, 5);
    const long long per = paged_per_cta(total, grid, min_tiles);
    CHECK(per * grid >= total && per >= 1);
    std::map<long long, std::vector<int>> parts;      // item -> slots written, in order
    std::set<int> slots;
    std::vector<PagedJoin> joins(grid, PagedJoin{0, 0, 0, 0, 0, 0});
    std::vector<long long> join_item(grid, -1);
    std::set<long long> done;
    for (int c = 0; c < grid; ++c) {
      long long t = c * per;
      const long long t_end = t + per < total ? t + per : total;
      bool first = true;
      while (t < t_end) {
        int b = 0;
        while (t >= base[b + 1]) ++b;
        const long long u = t - base[b], item0 = t - u % q[b].tiles, end = item0 + q[b].tiles;
        const long long n = (end < t_end ? end : t_end) - t;
        if (t != item0 && first && paged_join_starts(t, per, item0)) {
          CHECK(c > 0);
          joins[c].parts = paged_join_parts(t, per, end);
          joins[c].first_slot = paged_slot(c - 1, t - per == item0);
          join_item[c] = item0;
        }
        if (t == item0 && t + n == end) CHECK(done.insert(item0).second);
        else {
          const int slot = paged_slot(c, first);
          CHECK(slot < 2 * grid && slots.insert(slot).second);
          parts[item0].push_back(slot);
        }
        first = false;
        t += n;
      }
    }
    std::set<long long> joined;
    for (int c = 0; c < grid; ++c) {
      if (!joins[c].parts) continue;
      CHECK(joined.insert(join_item[c]).second);
      const auto &want = parts[join_item[c]];
      CHECK((int)want.size() == joins[c].parts);
      for (int k = 0; k < joins[c].parts; ++k)
        CHECK(want[k] == (k == 0 ? joins[c].first_slot : 2 * (c + k - 1)));
    }
    CHECK(joined.size() == parts.size());
    long long items = 0;
    for (auto &x : q) items += (long long)x.row_tiles * s.Hkv * (x.tiles > 0);
    CHECK((long long)(done.size() + joined.size()) == items);
  }
}

// Lengths, windows and first tokens up to the largest: nothing overflows, and the keys are the definition's.
static void extremes() {
  std::mt19937_64 g(3);
  auto in = [&](long long lo, long long hi) { return lo + (long long)(g() % (unsigned long long)(hi - lo + 1)); };
  for (int round = 0; round < 200000; ++round) {
    PagedShape s;
    s.B = 1, s.G = 1, s.Hkv = 1, s.causal = in(0, 1);
    s.bound = in(0, 1) ? (int)in(kPagedMaxLen - 300, kPagedMaxLen) : (int)in(1, 1 << in(0, 30));
    const long long rows = 0x7fffffffLL / (s.bound / 16 + 2);
    s.max_q = (int)in(1, rows < 0x3fffffff ? rows : 0x3fffffff), s.N = s.max_q;
    auto any = [&]() { return (int)(in(0, 2) == 0 ? in(0x7fffffff - 300, 0x7fffffff) : in(0, 1) ? in(0, 300) : in(0, s.bound)); };
    const int window = any();
    s.window = paged_window(window, s.bound), s.sinks = any();
    s.tile_log2 = (int)in(4, 7), s.row_log2 = (int)in(0, 7);
    const int len = in(0, 1) ? s.bound - (int)in(0, s.bound < 300 ? s.bound : 300) : (int)in(0, s.bound < 300 ? s.bound : 300);
    const PagedSeq q = paged_seq(s, 0, (int)in(0, s.max_q), len);
    CHECK(q.len == len && q.sink_n >= 0 && q.sink_n <= q.sink_pad && q.body >= 0 && q.body <= len && q.tiles >= 0);
    CHECK(q.count == 0 || q.tiles <= (len >> s.tile_log2) + 2);
    const int tile = 1 << s.tile_log2;
    for (int k = 0; k < 20; ++k) {
      const int x = (int)(k < 10 ? in(0, ((long long)q.tiles + 1) * tile - 1) : ((long long)q.tiles + 1) * tile - 1 - in(0, tile));
      const int t = paged_key(q, x);
      CHECK(t >= -1 && t < len);
      const int i = q.count ? (int)in(0, q.count - 1) : 0, end = s.causal ? q.end_min + i : len;
      if (t < 0 || q.count == 0) continue;
      const bool see = t < end && (window == 0 || t < s.sinks || t >= (long long)end - window);
      CHECK(see == paged_visible(s, t, end));
      if (x + 16 <= q.tiles * (long long)tile && paged_all_visible(s, q, x, 16)) CHECK(see);
    }
  }
}

int main() {
  divisions();
  shapes();
  extremes();
  puts("ok");
  return 0;
}
"""


@pytest.mark.timeout(300)
def test_index_arithmetic(tmp_path):
    src, exe = tmp_path / "index.cpp", tmp_path / "index"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-x", "c++",
                    "-I", str(CSRC), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr

// Index arithmetic of ds_attn_paged, host and device: which keys a sequence's queries see, how the work is cut into
// equal ranges, where a row of the cache lies.  No CUDA in here, so that it can be checked on a CPU over ranges that no
// GPU test would reach.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define DS_HD __host__ __device__ __forceinline__
#else
#define DS_HD inline
#endif

namespace ds {

DS_HD int paged_min(int a, int b) { return a < b ? a : b; }
DS_HD int paged_max(int a, int b) { return a > b ? a : b; }

// x / d for 0 <= x < 2^31, 1 <= d < 2^31, as a multiplication: with l = ceil(log2 d) and m = floor(2^(31+l) / d) + 1,
// m d - 2^(31+l) lies in [1, d], so x m / 2^(31+l) exceeds x / d by less than 1 / d.
struct FastDiv {
  uint32_t d, shift;
  uint64_t mul;  // at most 2^31 + 1 .. 2^32: the product stays below 2^63
};
DS_HD FastDiv make_fast_div(int d) {
  FastDiv f;
  int l = 0;
  while (((uint64_t)1 << l) < (uint64_t)d) ++l;
  f.d = (uint32_t)d;
  f.shift = 31 + l;
  f.mul = ((uint64_t)1 << f.shift) / (uint64_t)d + 1;
  return f;
}
DS_HD int fast_div(int x, const FastDiv &f) { return (int)(((uint64_t)(uint32_t)x * f.mul) >> f.shift); }

// What the kernels need of a call's shape.
struct PagedShape {
  int B, G, Hkv, N, max_q;   // G = query heads per KV head
  int bound;                 // most cache rows of a sequence: min(max_len, max_pages * page_size)
  int causal, window, sinks; // window < bound
  int tile_log2;             // keys per unit of work (a CTA's warps take equal parts of it)
  int row_log2;              // stacked rows (query, head of the group) per unit of work
};
DS_HD int paged_ceil_shift(int x, int log2) { return (int)(((unsigned)x + (1u << log2) - 1u) >> log2); }
// Sequences may be so long: key numbers run up to two tiles beyond the last row, in 32 bits.
constexpr int kPagedMaxLen = 0x7fffffff - 1024;
// A window that no length passes hides nothing.
DS_HD int paged_window(int window, int bound) { return window >= bound ? 0 : window; }

// One sequence.  Its queries see cache rows [0, sink_n) and [body, len) between them.  The keys are numbered x: the
// first sink_n rows, padding to a whole tile, then the body.
struct PagedSeq {
  int first, count, len;
  int sink_n, sink_pad, body;
  int end_min, end_max;      // smallest and largest e_i
  int tiles, row_tiles;      // units: row_tiles * Hkv * tiles; 0 tiles when there is no query
  bool bad;
};

DS_HD PagedSeq paged_seq(const PagedShape &s, int row_lo, int row_hi, int len) {
  PagedSeq q;
  q.first = paged_min(paged_max(row_lo, 0), s.N);
  const int64_t n = (int64_t)row_hi - q.first;
  q.count = n < 0 ? 0 : paged_min(n > s.max_q ? s.max_q : (int)n, s.N - q.first);
  q.len = paged_min(paged_max(len, 0), s.bound);
  q.bad = q.first != row_lo || n != q.count || q.len != len;
  q.end_max = q.len;
  q.end_min = s.causal ? q.len - q.count + 1 : q.len;
  const int lo = s.window > 0 && q.end_min > s.window ? q.end_min - s.window : 0;
  if (lo <= s.sinks) {
    q.sink_n = q.sink_pad = q.body = 0;
  } else {
    q.sink_n = s.sinks;
    q.sink_pad = paged_ceil_shift(s.sinks, s.tile_log2) << s.tile_log2;
    q.body = lo;
  }
  q.row_tiles = paged_ceil_shift(q.count * s.G, s.row_log2);      // max_q G < 2^30
  // a sequence with queries has at least one unit, even when they see nothing: their outputs are written
  q.tiles = q.count == 0 ? 0 : paged_max(1, (q.sink_pad >> s.tile_log2) + paged_ceil_shift(q.len - q.body, s.tile_log2));
  return q;
}
DS_HD int64_t paged_units(const PagedShape &s, const PagedSeq &q) { return (int64_t)q.row_tiles * s.Hkv * q.tiles; }
// The units of a sequence within the bounds, and the products on the way there, stay below 2^31 (the kernels number them in 32
// bits).  `most`: with the most queries and the largest length; padding behind the first rows may give another one tile more.
DS_HD bool paged_units_fit(const PagedShape &s, const PagedSeq &most) {
  const int64_t items = (int64_t)most.row_tiles * s.Hkv;
  return items <= 0x7fffffffLL && items * paged_min(most.tiles + 1, (s.bound >> s.tile_log2) + 2) <= 0x7fffffffLL;
}

// Cache row of key x, -1 for padding.
DS_HD int paged_key(const PagedSeq &q, int x) {
  if (x < q.sink_pad) return x < q.sink_n ? x : -1;
  return x - q.sink_pad < q.len - q.body ? q.body + (x - q.sink_pad) : -1;
}
DS_HD bool paged_visible(const PagedShape &s, int t, int end) {
  return t >= 0 && t < end && (s.window == 0 || t < s.sinks || t >= end - s.window);
}
// Every one of the n keys from x on is there and seen by every query.
DS_HD bool paged_all_visible(const PagedShape &s, const PagedSeq &q, int x, int n) {
  if (x < q.sink_pad) return x + n <= q.sink_n;
  if (x - q.sink_pad > q.len - q.body - n) return false;
  const int t = q.body + (x - q.sink_pad);
  return t <= q.end_min - n && (s.window == 0 || t >= q.end_max - s.window);
}

// The work of a call, `total` units in the order sequence, KV head, row tile, key tile, cut into ranges of `per` units
// for the CTAs.  An item (all key tiles of a sequence, KV head and row tile) may lie in several ranges; unsplit, the
// range that an item begins in takes it whole.
DS_HD int64_t paged_per_cta(int64_t total, int n_ctas, int min_tiles) {
  const int64_t up = total + n_ctas - 1;
  const int64_t per = up >> 32 ? up / n_ctas : (int64_t)((uint32_t)up / (uint32_t)n_ctas);   // short division where it does
  return per > min_tiles ? per : min_tiles;
}

// The join of an item that several ranges share, recorded by the CTA whose range begins first inside it.
struct PagedJoin {
  int parts;                 // 0: nothing to join here
  int first_slot;            // slot of the part before this CTA's; the others are slots 2c, 2 (c + 1), ..
  int row, rows;             // stacked rows of the item
  int first, kv_head;        // its sequence's first query row, its KV head
};
// `t0`: this CTA's first unit, inside an item that begins at `item` < t0 and ends before `item_end`.
DS_HD bool paged_join_starts(int64_t t0, int64_t per, int64_t item) { return t0 - per <= item; }
DS_HD int paged_join_parts(int64_t t0, int64_t per, int64_t item_end) {
  const int64_t rest = item_end - 1 - t0;      // t0 is a multiple of per
  return 2 + (rest < per ? 0 : rest >> 32 || per >> 32 ? (int)(rest / per) : (int)((uint32_t)rest / (uint32_t)per));
}
// A CTA writes the part of the item that its range begins with to slot 2c, that of the item it ends with to 2c + 1.
DS_HD int paged_slot(int cta, bool first_segment) { return 2 * cta + (first_segment ? 0 : 1); }

// A page as the table has it -> one of the pool.
DS_HD int paged_clamp_page(int page, int n_pages) { return page < 0 ? 0 : page >= n_pages ? n_pages - 1 : page; }

}  // namespace ds

// What the kernels of ds_attn_paged and ds_attn_paged8 share: a call's parameters, the walk of a CTA over its range of the units of work, the
// output of a row, and the join of items that several ranges share.
#pragma once
#include "ds_common.cuh"
#include "ds_paged_index.cuh"
#include "ds_sm100.cuh"

namespace ds {
namespace paged {

struct Params {
  ds_paged_params p;
  PagedShape s;
  FastDiv page_div, group_div;
  int split;
  int cluster;        // CTAs of an item; 0: equal ranges
  int may_alone;      // with equal ranges: an item per CTA instead, if the lengths turn out to be even enough
  FastDiv item_div, row_div;      // by KV heads times row tiles, by row tiles (at most): with a cluster
  // The sums of weighted values hold shrink = 2^-b times them, 2^b over 512 times the most keys: a weight may be up to 256 (the
  // exponents' reference lags), and no sum then passes the largest value that it averages.  Exact down to values of 2^-126 / shrink.
  float shrink, stretch, shrink_log2;
  int part_rows;      // rows of a partial result's slot
  PagedJoin *joins;   // [gridDim.x]
  float2 *part_ml;    // [2 gridDim.x][part_rows]  maximum (base 2, scaled) and sum
  float *part_o;      // [2 gridDim.x][part_rows][D]
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool there) {
  // a chunk that is not there is filled with zeros and not read
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// Two weights as two bf16 halves each.  hi is cut off and lo is what is left of the weight (times 1 + 2^-23, so that something
// is): both are positive where the weight is, and an infinite value stays the infinity that it is by the formula.  (Rounded to
// the nearest, lo would be 0 or negative for half of the weights: infinity times that is NaN.)  16 bits of a weight are kept.
__device__ __forceinline__ void split_weights(F2 p, uint32_t &hi, uint32_t &lo) {
  const float2 w = f2_get(p);
  const uint32_t b0 = __float_as_uint(w.x), b1 = __float_as_uint(w.y);
  constexpr float kMore = 1.f + 0x1p-23f;
  hi = __byte_perm(b0, b1, 0x7632);
  lo = sm100::pack_bf16(fmaf(w.x, kMore, -__uint_as_float(b0 & 0xffff0000u)), fmaf(w.y, kMore, -__uint_as_float(b1 & 0xffff0000u)));
}
// The item a CTA works on.
struct Item {
  PagedSeq q;
  int b, g;            // sequence, KV head
  int row0, rows;      // stacked rows row0 .. row0 + rows - 1 of the sequence
};

// Stacked row -> query row of the packed arrays, head, and how much of the cache it sees.
struct Row {
  long long n;
  int h, end;
};
__device__ __forceinline__ Row row_of(const Params &a, const Item &it, int r) {
  const int rr = it.row0 + r, i = fast_div(rr, a.group_div);
  return {(long long)it.q.first + i, it.g * a.s.G + (rr - i * a.s.G), a.s.causal ? max(it.q.end_min + i, 0) : it.q.len};
}

__device__ __forceinline__ PagedSeq sequence_of(const Params &a, int b) {
  const ds_paged_params &p = a.p;
  const int lo = p.row_start ? p.row_start[b] : b * p.max_q, hi = p.row_start ? p.row_start[b + 1] : lo + p.max_q;
  return paged_seq(a.s, lo, hi, p.kv_len[b]);
}

// A CTA's range of the units, and its walk over the pieces of items in it.
struct Walk {
  long long per, t, t_end;
  Item it;
  int tile0, n_tiles, row_tile;
  bool first;      // the piece that the range begins with

  // An item to each CTA, when there are no more items than CTAs and the longest is not too far above the mean of the
  // ranges: several pieces in a range and their join cost as much as some ten tiles.  (8 x 32 heads x 1000 .. 2080 rows, 32
  // queries: 67 instead of 78 us, 24 x 8 heads x 50 .. 3000 rows in fp32: 70 instead of 49; the rule takes the better.)
  // For more than 32 sequences the block-wide form of this cost the others 1 .. 5 % and gained as little.
  __device__ bool alone(const Params &a, long long total) {
    const int lane = threadIdx.x & 31;
    PagedSeq q;
    q.tiles = q.row_tiles = 0;
    if (lane < a.p.B) q = sequence_of(a, lane);
    const int items = q.tiles > 0 ? q.row_tiles * a.s.Hkv : 0;
    int inc = items;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, off);
      if (lane >= off) inc += y;
    }
    const int n = __shfl_sync(0xffffffffu, inc, 31);
    const int longest = __reduce_max_sync(0xffffffffu, q.tiles);
    if (n > (int)gridDim.x || 10LL * longest * gridDim.x > 16 * total + 100LL * gridDim.x) return false;
    first = true;
    tile0 = n_tiles = row_tile = it.g = 0;
    per = total;
    t = t_end = 0;
    const uint32_t here = __ballot_sync(0xffffffffu, (int)blockIdx.x < inc);
    if (!here) return true;      // no item left for this CTA
    it.b = __ffs(here) - 1;
    const uint32_t item = blockIdx.x - __shfl_sync(0xffffffffu, inc - items, it.b);
    it.q = sequence_of(a, it.b);
    it.g = (int)(item / (uint32_t)it.q.row_tiles);
    row_tile = (int)(item - it.g * (uint32_t)it.q.row_tiles);
    t_end = it.q.tiles;
    return true;
  }

  // Where the range begins, from a scan of the sequences' units by the whole CTA.  scan: kThreads / 32 + 2 values of
  // shared memory, not used again before a barrier.  Flags bad lengths and row ranges.
  template <int kThreads>
  __device__ void find(const Params &a, int min_tiles, long long *scan, uint32_t &flags) {
    const ds_paged_params &p = a.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    long long total, base = 0;
    it.b = 0;
    auto range = [&]() {
      per = paged_per_cta(total, gridDim.x, min_tiles);
      t = blockIdx.x * per;
      t_end = min(total, t + per);
    };
    auto warp_scan = [&](long long inc) {
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, inc, off);
        if (lane >= off) inc += y;
      }
      return inc;
    };
    if (p.B <= 32) {      // every warp for itself
      long long mine = 0;
      if (lane < p.B) {
        const PagedSeq q = sequence_of(a, lane);
        if (q.bad) flags |= DS_DEV_INDEX;
        mine = paged_units(a.s, q);
      }
      const long long inc = warp_scan(mine);
      total = __shfl_sync(0xffffffffu, inc, 31);
      if (a.may_alone && alone(a, total)) return;
      range();
      const uint32_t here = __ballot_sync(0xffffffffu, t < inc);      // inclusive sums: the first above t
      const int src = here ? __ffs(here) - 1 : 0;
      base = __shfl_sync(0xffffffffu, inc - mine, src);
      it.b = src;
    } else {
      const int chunk = (p.B + kThreads - 1) / kThreads;
      const int b0 = min(p.B, tid * chunk), b1 = min(p.B, b0 + chunk);
      long long mine = 0;
      for (int b = b0; b < b1; ++b) {
        const PagedSeq q = sequence_of(a, b);
        if (q.bad) flags |= DS_DEV_INDEX;
        mine += paged_units(a.s, q);
      }
      const long long inc = warp_scan(mine);
      if (lane == 31) scan[warp] = inc;
      __syncthreads();
      total = 0;
      long long before = inc - mine;
      for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += scan[w];
        total += scan[w];
      }
      range();
      if (t < total && before <= t && t < before + mine) {
        for (int b = b0; b < b1; ++b) {
          const long long w = paged_units(a.s, sequence_of(a, b));
          if (t < before + w) {
            scan[kThreads / 32] = before;
            scan[kThreads / 32 + 1] = b;
            break;
          }
          before += w;
        }
      }
      __syncthreads();
      if (t < t_end) {
        base = scan[kThreads / 32];
        it.b = (int)scan[kThreads / 32 + 1];
      }
    }
    first = true;
    tile0 = n_tiles = row_tile = it.g = 0;
    if (t < t_end) {      // the one place that needs divisions: afterwards items follow one another
      it.q = sequence_of(a, it.b);
      const uint32_t u = (uint32_t)(t - base), item = u / (uint32_t)it.q.tiles;
      tile0 = (int)(u - item * (uint32_t)it.q.tiles);
      it.g = (int)(item / (uint32_t)it.q.row_tiles);
      row_tile = (int)(item - it.g * (uint32_t)it.q.row_tiles);
    }
  }
  __device__ __forceinline__ void next_item(const Params &a) {
    t += n_tiles;
    tile0 = 0;
    if (++row_tile < it.q.row_tiles) return;
    row_tile = 0;
    if (++it.g < a.s.Hkv) return;
    it.g = 0;
    if (t < t_end) do it.q = sequence_of(a, ++it.b);
      while (it.q.tiles == 0);
  }
  // The piece at t: n_tiles key tiles of `it` from tile0 on.  False at the end of the range.
  __device__ __forceinline__ bool piece(const Params &a) {
    while (t < t_end) {
      n_tiles = it.q.tiles - tile0;
      if (a.split || tile0 == 0) {
        if (a.split) n_tiles = (int)min((long long)n_tiles, t_end - t);
        it.row0 = row_tile << a.s.row_log2;
        it.rows = min(1 << a.s.row_log2, it.q.count * a.s.G - it.row0);
        return true;
      }
      next_item(a);      // unsplit, an item belongs to the range that it begins in
    }
    return false;
  }
  __device__ __forceinline__ void next(const Params &a) {
    first = false;
    next_item(a);
  }
  __device__ __forceinline__ bool whole() const { return tile0 == 0 && n_tiles == it.q.tiles; }
  // If this CTA's range is the first to begin inside the current item: what the join needs to know.
  __device__ __forceinline__ void note_join(PagedJoin &join) const {
    if (tile0 == 0 || !first || !paged_join_starts(t, per, t - tile0)) return;
    join.parts = paged_join_parts(t, per, t - tile0 + it.q.tiles);
    join.first_slot = paged_slot(blockIdx.x - 1, t - per == t - tile0);
    join.row = it.row0, join.rows = it.rows, join.first = it.q.first, join.kv_head = it.g;
  }
};

__device__ __forceinline__ void store4(float *p, const float4 &v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, const float4 &v) {
  *reinterpret_cast<uint2 *>(p) = make_uint2(sm100::pack_bf16(v.x, v.y), sm100::pack_bf16(v.z, v.w));
}

// Sums of a finished row -> output and log-sum-exp.  A row that saw nothing has sum 0; a NaN stays one.
template <typename T>
__device__ __forceinline__ void write_row4(const Params &a, const Row &row, int d, float4 v, float top, float sum) {
  const float inv = sum == 0.f ? 0.f : a.stretch / sum;
  v.x *= inv, v.y *= inv, v.z *= inv, v.w *= inv;
  store4(reinterpret_cast<T *>(a.p.out) + row.n * a.p.out_stride[0] + row.h * a.p.out_stride[1] + d, v);
  if (a.p.lse && d == 0) a.p.lse[row.n * a.p.Hq + row.h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// Joins the parts of one item: CTA = (range that begins inside the item first, stacked row).  D / 4 threads hold the
// row, the CTA's groups of so many threads take the parts in turn, eight loads in flight each, and are themselves joined
// in order: the result does not depend on timing.
constexpr int kJoinThreads = 256;
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads) attn_paged_join_kernel(const __grid_constant__ Params a) {
  constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes;
  __shared__ float4 o_s[kGroups][kLanes];
  __shared__ float sum_s[kGroups], top_s[kJoinThreads / 32];
  dependent_sync();
  const PagedJoin j = a.joins[blockIdx.x];
  const int r = blockIdx.y, tid = threadIdx.x, group = tid / kLanes, u = tid % kLanes;
  if (r >= j.rows || j.parts == 0) return;
  auto at = [&](int k) { return (long long)(k == 0 ? j.first_slot : 2 * ((int)blockIdx.x + k - 1)) * a.part_rows + r; };
  float top = -INFINITY;
  for (int k = tid; k < j.parts; k += kJoinThreads) top = fmaxf(top, a.part_ml[at(k)].x);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
  if ((tid & 31) == 0) top_s[tid >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) top = fmaxf(top, top_s[w]);
  float sum = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int k = group; k < j.parts; k += kGroups) {
    const long long s = at(k);
    const float2 ml = a.part_ml[s];
    const float4 x = *reinterpret_cast<const float4 *>(a.part_o + s * D + 4 * u);
    const float f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top);
    sum = fmaf(ml.y, f, sum);
    v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
  }
  o_s[group][u] = v;
  if (u == 0) sum_s[group] = sum;
  __syncthreads();
  if (tid >= kLanes) return;
#pragma unroll
  for (int w = 1; w < kGroups; ++w) {
    const float4 x = o_s[w][u];
    v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
  }
  sum = 0.f;
  for (int w = 0; w < kGroups; ++w) sum += sum_s[w];
  const int rr = j.row + r, i = fast_div(rr, a.group_div);
  write_row4<T>(a, {(long long)j.first + i, j.kv_head * a.s.G + (rr - i * a.s.G), 0}, 4 * u, v, top, sum);
}

// The same for items of many rows, which have few parts: CTA = (range, eight stacked rows), a warp per row.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads) attn_paged_join_rows_kernel(const __grid_constant__ Params a) {
  constexpr int E = D / 32;      // elements of a lane
  dependent_sync();
  const PagedJoin j = a.joins[blockIdx.x];
  const int r = blockIdx.y * (kJoinThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (r >= j.rows || j.parts == 0) return;
  auto at = [&](int k) { return (long long)(k == 0 ? j.first_slot : 2 * ((int)blockIdx.x + k - 1)) * a.part_rows + r; };
  float top = -INFINITY;
  for (int k = lane; k < j.parts; k += 32) top = fmaxf(top, a.part_ml[at(k)].x);
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
  float sum = 0.f, v[E] = {};
#pragma unroll 4
  for (int k = 0; k < j.parts; ++k) {
    const long long s = at(k);
    const float2 ml = a.part_ml[s];
    const float f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top);
    sum = fmaf(ml.y, f, sum);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = fmaf(a.part_o[s * D + e * 32 + lane], f, v[e]);
  }
  const int rr = j.row + r, i = fast_div(rr, a.group_div);
  const Row row = {(long long)j.first + i, j.kv_head * a.s.G + (rr - i * a.s.G), 0};
  // four neighbouring elements to every fourth lane
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float4 w = make_float4(v[e], __shfl_down_sync(0xffffffffu, v[e], 1), __shfl_down_sync(0xffffffffu, v[e], 2),
                                 __shfl_down_sync(0xffffffffu, v[e], 3));
    if ((lane & 3) == 0) write_row4<T>(a, row, e * 32 + lane, w, top, sum);
  }
}

constexpr int log2_of(int x) { return x <= 1 ? 0 : 1 + log2_of(x / 2); }
inline size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

// Sizes of a call's launch.
struct Shape {
  PagedShape s;
  int grid, tiles;      // tiles: most key tiles of an item
  int cluster, heads;   // CTAs of an item (0: equal ranges), items of a sequence
  bool may_alone;
  int part_rows, min_tiles, D;
  long long items;
  size_t bytes_joins() const { return up256(sizeof(PagedJoin) * (size_t)grid); }
  size_t bytes_ml() const { return up256(sizeof(float2) * 2 * (size_t)grid * part_rows); }
  size_t workspace() const { return bytes_joins() + bytes_ml() + sizeof(float) * 2 * (size_t)grid * part_rows * D; }
};

// The most rows that a sequence may hold, and the numbers of a call's units with tiles of so many keys and rows.
inline PagedShape units_of(const ds_paged_params &p, int tile, int rows) {
  const int cap = p.max_pages * p.page_size, bound = p.max_len > 0 && p.max_len < cap ? p.max_len : cap;
  return {p.B, p.Hq / p.Hkv, p.Hkv, p.N, p.max_q, bound, p.causal != 0, paged_window(p.window, bound), p.sinks, log2_of(tile),
          log2_of(rows)};
}
inline PagedSeq longest_of(const PagedShape &s) { return paged_seq(s, 0, s.max_q < s.N ? s.max_q : s.N, s.bound); }

// From the most that the lengths may turn out to be: resident CTAs, or fewer where the ranges would get short.
inline Shape shape_of(const ds_paged_params &p, int tile, int rows, int min_tiles, int ctas_per_sm) {
  Shape h;
  h.s = units_of(p, tile, rows);
  const PagedSeq q = longest_of(h.s);
  h.tiles = q.tiles;
  h.min_tiles = min_tiles;
  h.D = p.D;
  const long long most = (long long)q.count * h.s.G;
  h.part_rows = most < rows ? (int)(most > 0 ? most : 1) : rows;
  const long long ranges = (paged_units(h.s, q) * p.B + min_tiles - 1) / min_tiles;
  const long long resident = (long long)ctas_per_sm * sm_count();
  h.grid = (int)(ranges < resident ? (ranges > 0 ? ranges : 1) : resident);
  h.items = (long long)p.B * p.Hkv * q.row_tiles;
  h.heads = p.Hkv * q.row_tiles;
  h.cluster = 0;
  h.may_alone = false;
  return h;
}

inline Params params_of(const ds_paged_params &p, const Shape &h, size_t need) {
  Params a;
  a.p = p;
  a.s = h.s;
  a.page_div = make_fast_div(p.page_size);
  a.group_div = make_fast_div(h.s.G);
  a.split = need > 0 && p.workspace && (reinterpret_cast<uintptr_t>(p.workspace) & 255) == 0 && p.workspace_bytes >= need;
  int bits = 9;
  while ((1ll << (bits - 9)) < h.s.bound) ++bits;
  a.stretch = (float)(1ll << bits), a.shrink = 1.f / a.stretch, a.shrink_log2 = -(float)bits;
  a.part_rows = h.part_rows;
  uint8_t *ws = reinterpret_cast<uint8_t *>(p.workspace);
  a.joins = reinterpret_cast<PagedJoin *>(ws);
  a.part_ml = reinterpret_cast<float2 *>(ws + h.bytes_joins());
  a.part_o = reinterpret_cast<float *>(ws + h.bytes_joins() + h.bytes_ml());
  a.cluster = h.cluster;
  a.may_alone = h.may_alone;
  a.item_div = make_fast_div(h.heads > 0 ? h.heads : 1);
  a.row_div = make_fast_div(h.heads > 0 ? h.heads / p.Hkv : 1);
  return a;
}

// A CTA per row joins many parts quickly; with more rows the parts are few and a warp per row does.
template <typename T, int D>
int launch_join(const Params &a, const Shape &h, cudaStream_t stream) {
  constexpr int kPer = kJoinThreads / 32;
  if (h.part_rows <= kPer)
    DS_CUDA_OK(launch_kernel(attn_paged_join_kernel<T, D>, dim3(h.grid, h.part_rows), kJoinThreads, 0, 0, true, stream, a));
  else
    DS_CUDA_OK(launch_kernel(attn_paged_join_rows_kernel<T, D>, dim3(h.grid, (h.part_rows + kPer - 1) / kPer), kJoinThreads, 0, 0,
                             true, stream, a));
  note_launch(1);
  return DS_OK;
}

}  // namespace paged
}  // namespace ds

// The kernels of ds_attn_paged and ds_attn_paged8 for a few query rows per KV head, whatever engine computes a warp's rows: how
// keys stream through shared memory, how the parts of an item are joined, and how a call is divided.
//
// The (sequence, KV head, row tile, key tile) units of the whole batch are laid end to end and cut into equal ranges, one per resident
// CTA, from the lengths on the device; or few items of moderate length get a CTA or a cluster of CTAs each.  Inside a CTA the four
// warps take equal parts of every key tile and share nothing until the item ends: each has its own ring of cp.async stages.
//
// An engine (Rows) has the types T of queries and outputs, Cache of the cache's elements and Args of the kernel's parameters; D, kRows,
// kRowBytes (of a cached row), kKeys (of a stage), kQBytes, kCtas, kStages, kScaled (a scale per block of rows, two floats
// per key in every stage); and begin, step and finish.
#pragma once
#include <cooperative_groups.h>

#include "ds_attn_paged.cuh"

namespace ds {
namespace paged {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kMinTiles = 4;     // a range has at least so many key tiles
constexpr int kWholeTiles = 8;   // items of at most so many key tiles are not split
constexpr int kClusterTiles = 24;   // most key tiles of a CTA when an item has a cluster
constexpr int kManyTiles = 20;      // when there are more items than CTAs at a time
constexpr int kAloneTiles = 20;     // and when it has a CTA, whatever the others' lengths

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Transposes an 8 x 8 matrix of 16-bit values, lane 4i + q holding columns 2q and 2q + 1 of row i.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Byte offset of 16-byte chunk `c` of row `r` in a tile of rows of ROW bytes: chunks are XOR-ed with the row number
// within groups of eight, which makes ldmatrix and the float4 reads below free of bank conflicts.
// (Rows of 64 bytes have four chunks, and two rows share the banks.)
template <int ROW>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) { return r * ROW + ((c ^ (ROW == 64 ? (r >> 1) & 3 : r & 7)) << 4); }

template <class Rows>
struct Layout {
  static constexpr int kSub = Rows::kKeys * Rows::kRowBytes;        // K or V of one stage of a warp
  static constexpr int kStage = 2 * kSub + (Rows::kScaled ? 8 * Rows::kKeys : 0);
  static constexpr int kRing = Rows::kStages * kStage;                    // of one warp; holds its sums at the item's end
  static constexpr int kOffQ = kWarps * kRing;
  static constexpr int kOffMl = kOffQ + Rows::kQBytes;
  // what the ranks of a cluster write into each other's: sums, maxima and sums of weights.  Not in the rings, where the
  // receiving rank may still be loading; 32 rows leave no room for it beside them.
  static constexpr bool kClusters = Rows::kRows * Rows::D <= (Rows::kStages == 2 ? 4096 : 2048);
  static constexpr int kOffParts = kOffMl + kWarps * Rows::kRows * 8;
  static constexpr int kOffTotals = kOffParts + (kClusters ? Rows::kRows * Rows::D * 4 : 0);
  static constexpr int kOffMisc = kOffTotals + (kClusters ? 8 * Rows::kRows * 8 : 0);
  static constexpr int kBytes = kOffMisc + 64;
  static constexpr int kTile = kWarps * Rows::kKeys;
  static_assert(Rows::kRows * Rows::D * 4 <= kRing, "the ring is reused for the warp's sums");
  static_assert(Rows::kCtas * (kBytes + sizeof(Walk) + 16 + 1024) <= 228 * 1024, "shared memory of the resident CTAs");
};

// Streams key tiles tile0 .. tile0 + n_tiles - 1 of an item; afterwards (and a barrier) the rings hold the warps' sums.
template <class Rows>
__device__ __forceinline__ void stream_keys(const typename Rows::Args &a, const Item &it, int tile0, int n_tiles, uint8_t *smem, uint32_t &flags) {
  using T = typename Rows::Cache;
  using L = Layout<Rows>;
  const ds_paged_params &p = a.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t *ring = smem + warp * L::kRing;
  const float scale2 = p.scale * kLog2e;
  Rows rows;
  if constexpr (!Rows::kScaled) rows.begin(a, it, smem + L::kOffQ);
  constexpr int kStages = Rows::kStages, kChunks = Rows::kRowBytes / 16, kOps = Rows::kKeys * kChunks / 32;
  const int32_t *table = p.block_table + it.b * p.table_stride;
  const uint8_t *kbase = reinterpret_cast<const uint8_t *>(reinterpret_cast<const T *>(p.k_cache) + it.g * p.cache_stride[1]);
  const uint8_t *vbase = reinterpret_cast<const uint8_t *>(reinterpret_cast<const T *>(p.v_cache) + it.g * p.cache_stride[1]);
  const long long row_bytes = p.cache_stride[2] * (long long)sizeof(T);
  [[maybe_unused]] const float *kscale = nullptr, *vscale = nullptr;
  if constexpr (Rows::kScaled) kscale = a.k_scale + it.g * a.scale_stride[1], vscale = a.v_scale + it.g * a.scale_stride[1];
  const int x_first = tile0 * L::kTile + warp * Rows::kKeys;
  // a lane looks up the cache row of key lane % kKeys, one stage ahead of its use
  int pos = paged_key(it.q, x_first + lane % Rows::kKeys);
  int page = pos >= 0 ? table[fast_div(pos, a.page_div)] : 0;
  auto issue = [&](int i) {
    long long at = -1;
    const uint32_t dst = sm100::smem_u32(ring + (i % kStages) * L::kStage);
    [[maybe_unused]] long long scale_at = 0;
    if (pos >= 0) {
      const int ok = paged_clamp_page(page, p.n_pages);
      if (ok != page) flags |= DS_DEV_INDEX;
      const int slot = pos - fast_div(pos, a.page_div) * p.page_size;
      at = (ok * p.cache_stride[0] + slot * p.cache_stride[2]) * (long long)sizeof(T);
      if constexpr (Rows::kScaled) scale_at = ok * a.scale_stride[0] + fast_div(slot, a.scale_div) * a.scale_stride[2];
    }
    if constexpr (Rows::kScaled) {      // a lane per key; of a key that is not there, zero
      static_assert((Rows::kKeys == 32 || Rows::kKeys == 16) && kChunks <= 8, "");
      if constexpr (Rows::kKeys == 32) {
        cp_async4(dst + 2 * L::kSub + 4 * lane, kscale + scale_at, pos >= 0);
        cp_async4(dst + 2 * L::kSub + 128 + 4 * lane, vscale + scale_at, pos >= 0);
      } else {
        cp_async4(dst + 2 * L::kSub + 4 * lane, (lane < 16 ? kscale : vscale) + scale_at, pos >= 0);
      }
      // 16 keys that lie evenly (in one page) need one address
      const long long at_lo = __shfl_sync(0xffffffffu, at, 0), at_hi = __shfl_sync(0xffffffffu, at, 16);
      const uint32_t even = __ballot_sync(0xffffffffu, at >= 0 && at == (lane < 16 ? at_lo : at_hi) + (lane & 15) * row_bytes);
      const int ch = lane % kChunks;
#pragma unroll
      for (int half = 0; half < Rows::kKeys / 16; ++half) {
        if (((even >> (16 * half)) & 0xffffu) == 0xffffu) {
          long long from = (half ? at_hi : at_lo) + (lane / kChunks) * row_bytes + 16 * ch;
#pragma unroll
          for (int j = 0; j < kChunks / 2; ++j, from += (32 / kChunks) * row_bytes) {
            const uint32_t to = dst + chunk_at<Rows::kRowBytes>(16 * half + j * (32 / kChunks) + lane / kChunks, ch);
            cp_async16(to, kbase + from, true);
            cp_async16(to + L::kSub, vbase + from, true);
          }
        } else {
#pragma unroll
          for (int j = 0; j < kChunks / 2; ++j) {
            const int r = 16 * half + j * (32 / kChunks) + lane / kChunks;
            const long long off = __shfl_sync(0xffffffffu, at, r);
            const bool there = off >= 0;
            const uint32_t to = dst + chunk_at<Rows::kRowBytes>(r, ch);
            const long long from = (there ? off : 0) + 16 * ch;
            cp_async16(to, kbase + from, there);
            cp_async16(to + L::kSub, vbase + from, there);
          }
        }
      }
    } else {
      // keys that lie evenly (in one page) need one address; otherwise every row's is fetched from the lane that has it
      const long long at0 = __shfl_sync(0xffffffffu, at, 0);
      if (__all_sync(0xffffffffu, at == at0 + (lane % Rows::kKeys) * row_bytes && at0 >= 0)) {
        long long from = at0 + (lane / kChunks) * row_bytes + 16 * (lane % kChunks);
  #pragma unroll
        for (int j = 0; j < kOps; ++j) {
          const int c = j * 32 + lane;
          const uint32_t to = dst + chunk_at<Rows::kRowBytes>(c / kChunks, c % kChunks);
          cp_async16(to, kbase + from, true);
          cp_async16(to + L::kSub, vbase + from, true);
          from += kChunks >= 32 && j % (kChunks / 32 > 0 ? kChunks / 32 : 1) != kChunks / 32 - 1
                      ? 512 : kChunks >= 32 ? row_bytes - (kChunks / 32 - 1) * 512 : (32 / kChunks) * row_bytes;
        }
      } else {
  #pragma unroll
        for (int j = 0; j < kOps; ++j) {
          const int c = j * 32 + lane, r = c / kChunks, ch = c % kChunks;
          const long long off = __shfl_sync(0xffffffffu, at, r);
          const bool there = off >= 0;
          const uint32_t to = dst + chunk_at<Rows::kRowBytes>(r, ch);
          const long long from = (there ? off : 0) + 16 * ch;
          cp_async16(to, kbase + from, there);
          cp_async16(to + L::kSub, vbase + from, there);
        }
      }
    }
    if (i + 1 < n_tiles) {
      pos = paged_key(it.q, x_first + (i + 1) * L::kTile + lane % Rows::kKeys);
      page = pos >= 0 ? table[fast_div(pos, a.page_div)] : 0;
    }
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    if (i < n_tiles) issue(i);
    cp_async_commit();
  }
  if constexpr (Rows::kScaled) {      // queries through shared memory (the stage that is loaded last, or beside the ring), behind the first keys
    static_assert(Rows::kQBytes > 0 || Rows::kQSmem <= L::kStage, "");
    rows.begin(a, it, smem + (Rows::kQBytes ? L::kOffQ : (kStages - 1) * L::kStage));
  }
  for (int i = 0; i < n_tiles; ++i) {
    cp_async_wait<kStages - 2>();
    __syncwarp();      // stage i is there for the whole warp, and the warp is done with stage i - 1
    if (i + kStages - 1 < n_tiles) issue(i + kStages - 1);
    cp_async_commit();
    uint8_t *stage = ring + (i % kStages) * L::kStage;
    rows.step(a, it, stage, stage + L::kSub, x_first + i * L::kTile, scale2);
  }
  cp_async_wait<0>();
  __syncwarp();

  rows.finish(a, it, reinterpret_cast<float *>(ring), reinterpret_cast<float2 *>(smem + L::kOffMl) + warp * Rows::kRows);
  __syncthreads();
}

// The four warps' sums of elements d .. d + 3 of row r.
template <class Rows>
__device__ __forceinline__ float4 join_warps(const uint8_t *smem, int r, int d, float &top, float &sum) {
  using L = Layout<Rows>;
  const float2 *ml_all = reinterpret_cast<const float2 *>(smem + L::kOffMl);
  top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml_all[w * Rows::kRows + r].x);
  sum = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const float2 ml = ml_all[w * Rows::kRows + r];
    const float4 x = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(smem + w * L::kRing) + r * Rows::D + d);
    const float f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top);
    sum = fmaf(ml.y, f, sum);
    v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
  }
  return v;
}

// The parts of an item that the ranks of its cluster have streamed: a rank writes its sums into the other ranks' shared
// memory, an n-th of the dimensions to each, which then adds up and writes that part of the output.
template <class Rows>
__device__ __forceinline__ void cluster_join(const typename Rows::Args &a, const Item &it, int rank, uint8_t *smem) {
  namespace cg = cooperative_groups;
  using T = typename Rows::T;
  using L = Layout<Rows>;
  constexpr int D = Rows::D;
  auto cluster = cg::this_cluster();
  const int n = a.cluster, tid = threadIdx.x;
  const int quads = D / 4 / n;                   // float4 of a row that a rank adds up
  float4 *parts = reinterpret_cast<float4 *>(smem + L::kOffParts);      // [n][rows][quads]
  float2 *totals = reinterpret_cast<float2 *>(smem + L::kOffTotals);    // [n][rows]
  cluster.barrier_wait();      // every rank has started
  for (int e = tid; e < it.rows * (D / 4); e += kThreads) {
    const int r = e / (D / 4), d = e % (D / 4), to = d / quads;
    float top, sum;
    const float4 v = join_warps<Rows>(smem, r, 4 * d, top, sum);
    *cluster.map_shared_rank(parts + (rank * it.rows + r) * quads + (d - to * quads), to) = v;
    if (d == to * quads) *cluster.map_shared_rank(totals + rank * it.rows + r, to) = make_float2(top, sum);
  }
  cluster.sync();
  for (int e = tid; e < it.rows * quads; e += kThreads) {
    const int r = e / quads, d = e - r * quads;
    float top = -INFINITY, sum = 0.f;
    for (int k = 0; k < n; ++k) top = fmaxf(top, totals[k * it.rows + r].x);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < n; ++k) {
      const float2 ml = totals[k * it.rows + r];
      const float4 x = parts[(k * it.rows + r) * quads + d];
      const float f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top);
      sum = fmaf(ml.y, f, sum);
      v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
    }
    write_row4<T>(a, row_of(a, it, r), 4 * (rank * quads + d), v, top, sum);
  }
}

// An item per CTA or cluster of CTAs.
template <class Rows>
__global__ void __launch_bounds__(kThreads, Rows::kCtas) attn_paged_item_kernel(const __grid_constant__ typename Rows::Args a) {
  using T = typename Rows::T;
  using L = Layout<Rows>;
  constexpr int D = Rows::D;
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x;
  uint32_t flags = 0;
  dependent_sync();
  const int item = (int)blockIdx.x / a.cluster;
  Item it;
  it.b = fast_div(item, a.item_div);
  const int rest = item - it.b * (int)a.item_div.d;
  it.g = fast_div(rest, a.row_div);
  it.row0 = (rest - it.g * (int)a.row_div.d) << a.s.row_log2;
  it.q = sequence_of(a, it.b);
  if (it.q.bad) flags |= DS_DEV_INDEX;
  it.rows = min(Rows::kRows, it.q.count * a.s.G - it.row0);
  const int n = a.cluster, rank = blockIdx.x - item * n;
  if (it.rows > 0) {      // the whole cluster or none of it
    if constexpr (L::kClusters)
      if (n > 1) cooperative_groups::this_cluster().barrier_arrive();      // waited for in cluster_join
    const int per = n > 1 ? (it.q.tiles + n - 1) / n : it.q.tiles;         // n is at most 8
    const int tile0 = min(rank * per, it.q.tiles);
    stream_keys<Rows>(a, it, tile0, min(per, it.q.tiles - tile0), smem, flags);
    bool joined = false;
    if constexpr (L::kClusters)
      if (n > 1) {
        cluster_join<Rows>(a, it, rank, smem);
        joined = true;
      }
    for (int e = tid; !joined && e < it.rows * (D / 4); e += kThreads) {
      const int r = e / (D / 4), d = e % (D / 4) * 4;
      float top, sum;
      const float4 v = join_warps<Rows>(smem, r, d, top, sum);
      write_row4<T>(a, row_of(a, it, r), d, v, top, sum);
    }
  }
  if (flags && a.p.status) atomicOr(a.p.status, flags);
}

// Equal ranges.  The walk lives in shared memory, one thread moves it: the registers are for the rows.
template <class Rows>
__global__ void __launch_bounds__(kThreads, Rows::kCtas) attn_paged_range_kernel(const __grid_constant__ typename Rows::Args a) {
  using T = typename Rows::T;
  using L = Layout<Rows>;
  constexpr int D = Rows::D;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ Walk walk;
  __shared__ bool more;
  const int tid = threadIdx.x;
  uint32_t flags = 0;
  dependent_sync();
  {
    Walk w;
    w.find<kThreads>(a, kMinTiles, reinterpret_cast<long long *>(smem + L::kOffMisc), flags);
    if (tid == 0) {
      walk = w;
      more = walk.piece(a);
    }
  }
  PagedJoin join = {0, 0, 0, 0, 0, 0};      // thread 0's
  __syncthreads();
  while (more) {
    const Item it = walk.it;
    if (a.split && tid == 0) walk.note_join(join);
    stream_keys<Rows>(a, it, walk.tile0, walk.n_tiles, smem, flags);
    const bool whole = walk.whole();
    const int slot = paged_slot(blockIdx.x, walk.first);
    for (int e = tid; e < it.rows * (D / 4); e += kThreads) {
      const int r = e / (D / 4), d = e % (D / 4) * 4;
      float top, sum;
      const float4 v = join_warps<Rows>(smem, r, d, top, sum);
      if (whole) {
        write_row4<T>(a, row_of(a, it, r), d, v, top, sum);
      } else {
        const long long at = (long long)slot * a.part_rows + r;
        *reinterpret_cast<float4 *>(a.part_o + at * D + d) = v;
        if (d == 0) a.part_ml[at] = make_float2(top, sum);
      }
    }
    __syncthreads();
    if (tid == 0) {
      walk.next(a);
      more = walk.piece(a);
    }
    __syncthreads();
  }
  if (a.split && tid == 0) a.joins[blockIdx.x] = join;
  if (flags && a.p.status) atomicOr(a.p.status, flags);
}

template <class Rows>
Shape shape_for(const ds_paged_params &p) {
  using L = Layout<Rows>;
  Shape h = shape_of(p, L::kTile, Rows::kRows, kMinTiles, Rows::kCtas);
  // Items by themselves: a cluster per item where the items leave room for it, else a CTA, scheduled by the hardware as
  // others end.  What CTAs lose when lengths are uneven, or their number does not fill the GPU, has to stay below what
  // several pieces in a range and the second kernel cost: not with long items.  (60 x 32 heads x 0 .. 813 rows: 122 -> 68 us; from
  // 20 tiles on no gain, 32 x 32 heads x 4128 rows 320 -> 330.)
  const long long resident = (long long)Rows::kCtas * sm_count();
  if (h.items > resident) {
    if (h.tiles <= kManyTiles && h.items <= 0x7fffffff) {
      h.cluster = 1;
      h.grid = (int)h.items;
    }
  } else if (h.items > 0) {
    const bool fills = h.items * 2 > resident;
    int n = L::kClusters ? 8 : 1;
    while (n > 1 && (h.items * n > resident || n > h.tiles)) n /= 2;
    if (h.tiles <= (n > 1 ? n * kClusterTiles : fills ? kAloneTiles : kAloneTiles / 2)) {
      h.cluster = n;
      h.grid = (int)h.items * n;
    } else {
      h.may_alone = n == 1 && fills;      // the device knows the lengths
    }
  }
  return h;
}

inline size_t rows_workspace_of(const Shape &h) { return h.cluster || h.tiles <= kWholeTiles || h.grid == 1 ? 0 : h.workspace(); }

// more: sets what the engine's Args have beyond Params.
template <class Rows, class More>
int launch_rows(const ds_paged_params &p, cudaStream_t stream, More more) {
  using L = Layout<Rows>;
  const Shape h = shape_for<Rows>(p);
  typename Rows::Args a;
  static_cast<Params &>(a) = params_of(p, h, rows_workspace_of(h));
  more(a);
  static std::atomic<unsigned long long> allowed[2];
  // Set up early (8.2 -> 6.4 us for one short request) where items have CTAs of their own.  Not with equal ranges: CTAs that
  // wait in the slots that the kernel before it, often this one, leaves hold up its long CTAs (32 x 32 heads x 4128 rows back
  // to back 403 instead of 316 us).
  if (h.cluster) {
    DS_CUDA_OK(allow_smem(attn_paged_item_kernel<Rows>, L::kBytes, allowed[0]));
    DS_CUDA_OK(launch_kernel(attn_paged_item_kernel<Rows>, dim3(h.grid), kThreads, L::kBytes, h.cluster > 1 ? h.cluster : 0, true,
                             stream, a));
  } else {
    DS_CUDA_OK(allow_smem(attn_paged_range_kernel<Rows>, L::kBytes, allowed[1]));
    DS_CUDA_OK(launch_kernel(attn_paged_range_kernel<Rows>, dim3(h.grid), kThreads, L::kBytes, 0, false, stream, a));
  }
  note_launch(1);
  return a.split ? launch_join<typename Rows::T, Rows::D>(a, h, stream) : (int)DS_OK;
}

}  // namespace paged
}  // namespace ds

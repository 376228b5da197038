// ds_page_update: the bookkeeping of the paged cache, one step of it for every sequence.
//
// Latency is all there is to it.  Two scans over the sequences (pages returned, pages and rows asked for; then pages
// and rows granted) turn the rules of the header into exclusive sums kept in shared memory; after that every returned
// page, every page handed out and every new row is independent: a thread finds its sequence by bisecting the sums.
// Calls with many rows run on a cluster of CTAs: each does the scans for itself (they are short) and takes its share of
// the pages and rows; cluster barriers stand between reading what the caller may pass as input and output at
// once, returning pages, and handing them out.
#include <cooperative_groups.h>

#include "ds_common.cuh"
#include "ds_paged_index.cuh"

namespace ds {
namespace {

constexpr int kThreads = 1024;
constexpr int kCluster = 8;           // CTAs of a call with many rows
constexpr int kOneCtaRows = 4096;     // up to so many rows one CTA does it

struct Sums {
  long long back, need, rows;
};
__device__ __forceinline__ Sums operator+(const Sums &a, const Sums &b) {
  return {a.back + b.back, a.need + b.need, a.rows + b.rows};
}

// Exclusive sum of one value per thread over the CTA; `total` gets the sum of all.
__device__ Sums block_scan(const Sums &x, Sums *warp_sums, Sums &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto scan = [&](Sums inc) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Sums y = {__shfl_up_sync(0xffffffffu, inc.back, o), __shfl_up_sync(0xffffffffu, inc.need, o),
                      __shfl_up_sync(0xffffffffu, inc.rows, o)};
      if (lane >= o) inc = inc + y;
    }
    return inc;
  };
  const Sums inc = scan(x);
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  static_assert(kThreads == 1024, "one warp total per lane");
  const Sums w = warp_sums[lane], all = scan(w);
  total = {__shfl_sync(0xffffffffu, all.back, 31), __shfl_sync(0xffffffffu, all.need, 31),
           __shfl_sync(0xffffffffu, all.rows, 31)};
  const Sums ex = {all.back - w.back, all.need - w.need, all.rows - w.rows};
  const Sums before = {__shfl_sync(0xffffffffu, ex.back, warp), __shfl_sync(0xffffffffu, ex.need, warp),
                       __shfl_sync(0xffffffffu, ex.rows, warp)};
  __syncthreads();
  return {before.back + inc.back - x.back, before.need + inc.need - x.need, before.rows + inc.rows - x.rows};
}

__device__ __forceinline__ int pages_of(int rows, const FastDiv &ps) { return rows == 0 ? 0 : fast_div(rows - 1, ps) + 1; }

struct Sequence {
  int old_len, n_new, back, need;
  bool bad;
};

__device__ __forceinline__ Sequence load_sequence(const ds_page_params &p, const FastDiv &ps, int b) {
  Sequence s;
  const int cap = p.max_pages * p.page_size;
  int len = p.kv_len[b];
  s.n_new = p.n_new[b];
  const bool done = p.done && p.done[b];
  s.bad = len < 0 || len > cap || s.n_new < 0;
  len = min(max(len, 0), cap);
  const int held = pages_of(len, ps);
  s.back = done ? held : 0;
  s.old_len = done ? 0 : len;
  if (s.n_new < 0) s.n_new = 0;
  if (s.n_new > cap - s.old_len) {
    s.bad = true;
    s.n_new = 0;
  }
  s.need = pages_of(s.old_len + s.n_new, ps) - (done ? 0 : held);
  return s;
}

// The last b with sum[b] <= x, for sum[0] = 0 and x < sum[n].
__device__ __forceinline__ int owner(const int *sum, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sum[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// kVector: positions and slot_map are 16-byte aligned, four rows are written at once.
template <bool kVector>
__global__ void __launch_bounds__(kThreads) page_update_kernel(const ds_page_params p, const FastDiv ps_div) {
  namespace cg = cooperative_groups;
  extern __shared__ int smem[];
  __shared__ Sums warp_sums[kThreads / 32];
  const int n_ctas = gridDim.x;       // all in one cluster
  auto barrier = [&]() {
    if (n_ctas > 1) cg::this_cluster().sync();
    else __syncthreads();
  };
  const int B = p.B, ps = p.page_size, me = blockIdx.x * kThreads + threadIdx.x, all = n_ctas * kThreads;
  int *back_sum = smem, *page_sum = back_sum + B + 1, *row_sum = page_sum + B + 1, *old_len = row_sum + B + 1;
  uint32_t flags = 0;

  int free_cnt = *p.free_cnt;
  const int per = (B + kThreads - 1) / kThreads;
  const int b0 = min(B, (int)threadIdx.x * per), b1 = min(B, b0 + per);
  Sums mine = {0, 0, 0}, total;
  Sequence one = {0, 0, 0, 0, false};      // of b0, the only one of most threads
  for (int b = b0; b < b1; ++b) {
    const Sequence s = load_sequence(p, ps_div, b);
    if (b == b0) one = s;
    if (s.bad) flags |= DS_DEV_INDEX;
    mine = mine + Sums{s.back, s.need, s.n_new};
  }
  if (free_cnt < 0 || free_cnt > p.n_pages) {
    flags |= DS_DEV_INDEX;
    free_cnt = min(max(free_cnt, 0), p.n_pages);
  }
  Sums at = block_scan(mine, warp_sums, total);
  const int returned = (int)min(total.back, (long long)(p.n_pages - free_cnt));
  if (total.back > returned) flags |= DS_DEV_INDEX;
  const int free_now = free_cnt + returned;
  Sums granted = {0, 0, 0};
  for (int b = b0; b < b1; ++b) {
    const Sequence s = b == b0 ? one : load_sequence(p, ps_div, b);
    back_sum[b] = (int)min(at.back, (long long)returned);
    at = at + Sums{s.back, s.need, s.n_new};
    const bool ok = (s.need == 0 || at.need <= free_now) && (s.n_new == 0 || at.rows <= p.max_rows);
    if (!ok) flags |= DS_DEV_PAGES;
    // kept for the next scan: what the sequence gets
    page_sum[b] = ok ? s.need : 0;
    row_sum[b] = ok ? s.n_new : 0;
    old_len[b] = s.old_len;
    granted = granted + Sums{0, page_sum[b], row_sum[b]};
  }
  Sums run = block_scan(granted, warp_sums, total);
  for (int b = b0; b < b1; ++b) {
    const int pages = page_sum[b], rows = row_sum[b];
    page_sum[b] = (int)run.need;
    row_sum[b] = (int)run.rows;
    run = run + Sums{0, pages, rows};
  }
  const int n_alloc = (int)total.need, n_rows = (int)total.rows;
  if (threadIdx.x == 0) {
    back_sum[B] = returned;
    page_sum[B] = n_alloc;
    row_sum[B] = n_rows;
  }
  barrier();      // every CTA has read kv_len, free_cnt and the rest; from here on they may be overwritten

  if (returned > 0) {
    for (long long t = me; t < returned; t += all) {
      const int b = owner(back_sum, B, (int)t);
      const int page = p.block_table[b * p.table_stride + (t - back_sum[b])];
      if (page < 0 || page >= p.n_pages) flags |= DS_DEV_INDEX;
      p.free_list[free_cnt + t] = page;
    }
    barrier();    // the returned pages are on the list, and nobody reads old table entries of their sequences any more
  }
  for (long long t = me; t < n_alloc; t += all) {
    const int b = owner(page_sum, B, (int)t);
    const int page = p.free_list[free_now - 1 - t];
    if (page < 0 || page >= p.n_pages) flags |= DS_DEV_INDEX;
    p.block_table[b * p.table_stride + pages_of(old_len[b], ps_div) + (t - page_sum[b])] = page;
  }
  for (int b = me; b <= B; b += all) {
    p.row_start[b] = row_sum[b];
    if (b < B) p.kv_len_out[b] = old_len[b] + row_sum[b + 1] - row_sum[b];
  }
  if (me == 0) *p.free_cnt_out = free_now - n_alloc;
  if (p.positions || p.slot_map) {
    // a row's page comes from the table where it was there before this call, from the list where it is new
    constexpr int kRows = 4;
    for (long long r0 = (long long)me * kRows; r0 < p.max_rows; r0 += (long long)all * kRows) {
      int pos[kRows];
      long long slot[kRows];
      int b = r0 < n_rows ? owner(row_sum, B, (int)r0) : 0, last = -1, page = 0;
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const long long r = r0 + k;
        pos[k] = 0, slot[k] = -1;
        if (r >= n_rows) continue;
        while (row_sum[b + 1] <= r) ++b, last = -1;
        pos[k] = old_len[b] + (int)r - row_sum[b];
        const int j = fast_div(pos[k], ps_div);
        if (j != last) {
          const int have = pages_of(old_len[b], ps_div);
          page = j < have ? p.block_table[b * p.table_stride + j] : p.free_list[free_now - 1 - (page_sum[b] + j - have)];
          last = j;
        }
        if (page < 0 || page >= p.n_pages) flags |= DS_DEV_INDEX;
        else slot[k] = (long long)page * ps + (pos[k] - j * ps);
      }
      if (kVector && r0 + kRows <= p.max_rows) {
        if (p.positions) *reinterpret_cast<int4 *>(p.positions + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        if (p.slot_map) {
          *reinterpret_cast<longlong2 *>(p.slot_map + r0) = make_longlong2(slot[0], slot[1]);
          *reinterpret_cast<longlong2 *>(p.slot_map + r0 + 2) = make_longlong2(slot[2], slot[3]);
        }
      } else {
        for (int k = 0; k < kRows && r0 + k < p.max_rows; ++k) {
          if (p.positions) p.positions[r0 + k] = pos[k];
          if (p.slot_map) p.slot_map[r0 + k] = slot[k];
        }
      }
    }
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

}  // namespace

int launch_page_update(const ds_page_params &p, cudaStream_t stream) {
  const bool vec = ((reinterpret_cast<uintptr_t>(p.positions) | reinterpret_cast<uintptr_t>(p.slot_map)) & 15) == 0;
  auto kernel = vec ? page_update_kernel<true> : page_update_kernel<false>;
  DS_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.max_rows <= kOneCtaRows ? 1 : kCluster);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(int) * (4 * (size_t)p.B + 4);
  cfg.stream = stream;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = cfg.gridDim.x;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  DS_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, p, make_fast_div(p.page_size)));
  note_launch(1);
  return DS_OK;
}

}  // namespace ds

// ds_page_update: the bookkeeping of the paged cache, one step of it for every sequence.
//
// One CTA.  Two scans over the sequences (pages returned / pages and rows asked for; then pages and rows granted)
// turn the rules of the header into exclusive sums kept in shared memory; after that every returned page, every page
// handed out and every new row is independent: a thread finds its sequence by bisecting the sums.
#include "ds_common.cuh"

namespace ds {
namespace {

constexpr int kThreads = 1024;

struct Sums {
  long long back, need, rows;
};
__device__ __forceinline__ Sums operator+(const Sums &a, const Sums &b) {
  return {a.back + b.back, a.need + b.need, a.rows + b.rows};
}

// Exclusive sum of one value per thread over the CTA; `total` gets the sum of all.
__device__ Sums block_scan(const Sums &x, Sums *warp_sums, Sums &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Sums inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    Sums y = {__shfl_up_sync(0xffffffffu, inc.back, o), __shfl_up_sync(0xffffffffu, inc.need, o),
              __shfl_up_sync(0xffffffffu, inc.rows, o)};
    if (lane >= o) inc = inc + y;
  }
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  Sums before = {0, 0, 0};
  total = before;
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w == warp) before = total;
    total = total + warp_sums[w];
  }
  __syncthreads();
  return {before.back + inc.back - x.back, before.need + inc.need - x.need, before.rows + inc.rows - x.rows};
}

struct Sequence {
  int len, old_len, n_new, back, have, need;
  bool bad;
};

__device__ Sequence load_sequence(const ds_page_params &p, int b) {
  Sequence s;
  const int cap = p.max_pages * p.page_size;
  s.len = p.kv_len[b];
  s.n_new = p.n_new[b];
  s.bad = s.len < 0 || s.len > cap || s.n_new < 0;
  s.len = min(max(s.len, 0), cap);
  const bool done = p.done && p.done[b];
  const int held = (int)(((long long)s.len + p.page_size - 1) / p.page_size);
  s.back = done ? held : 0;
  s.old_len = done ? 0 : s.len;
  s.have = done ? 0 : held;
  if (s.n_new < 0) s.n_new = 0;
  if ((long long)s.old_len + s.n_new > cap) {
    s.bad = true;
    s.n_new = 0;
  }
  s.need = (int)(((long long)s.old_len + s.n_new + p.page_size - 1) / p.page_size) - s.have;
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

__global__ void __launch_bounds__(kThreads) page_update_kernel(const ds_page_params p) {
  extern __shared__ int smem[];
  __shared__ Sums warp_sums[kThreads / 32];
  const int B = p.B, ps = p.page_size;
  int *back_sum = smem, *page_sum = back_sum + B + 1, *row_sum = page_sum + B + 1, *old_len = row_sum + B + 1;
  uint32_t flags = 0;

  int free_cnt = *p.free_cnt;
  if (free_cnt < 0 || free_cnt > p.n_pages) {
    flags |= DS_DEV_INDEX;
    free_cnt = min(max(free_cnt, 0), p.n_pages);
  }
  const int per = (B + kThreads - 1) / kThreads;
  const int b0 = min(B, (int)threadIdx.x * per), b1 = min(B, b0 + per);
  Sums mine = {0, 0, 0}, total;
  for (int b = b0; b < b1; ++b) {
    const Sequence s = load_sequence(p, b);
    if (s.bad) flags |= DS_DEV_INDEX;
    mine = mine + Sums{s.back, s.need, s.n_new};
  }
  Sums at = block_scan(mine, warp_sums, total);
  const int returned = (int)min(total.back, (long long)(p.n_pages - free_cnt));
  if (total.back > returned) flags |= DS_DEV_INDEX;
  const int free_now = free_cnt + returned;
  Sums granted = {0, 0, 0};
  for (int b = b0; b < b1; ++b) {
    const Sequence s = load_sequence(p, b);
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
  __syncthreads();

  for (int t = threadIdx.x; t < returned; t += kThreads) {
    const int b = owner(back_sum, B, t);
    const int page = p.block_table[b * p.table_stride + (t - back_sum[b])];
    if (page < 0 || page >= p.n_pages) flags |= DS_DEV_INDEX;
    p.free_list[free_cnt + t] = page;
  }
  __syncthreads();
  for (int t = threadIdx.x; t < n_alloc; t += kThreads) {
    const int b = owner(page_sum, B, t);
    const int have = (int)(((long long)old_len[b] + ps - 1) / ps);
    const int page = p.free_list[free_now - 1 - t];
    if (page < 0 || page >= p.n_pages) flags |= DS_DEV_INDEX;
    p.block_table[b * p.table_stride + have + (t - page_sum[b])] = page;
  }
  for (int b = threadIdx.x; b <= B; b += kThreads) {
    p.row_start[b] = row_sum[b];
    if (b < B) p.kv_len_out[b] = old_len[b] + row_sum[b + 1] - row_sum[b];
  }
  if (threadIdx.x == 0) *p.free_cnt_out = free_now - n_alloc;
  if (p.positions || p.slot_map) {
    for (int r = threadIdx.x; r < p.max_rows; r += kThreads) {
      int pos = 0;
      long long slot = -1;
      if (r < n_rows) {
        const int b = owner(row_sum, B, r);
        const int have = (int)(((long long)old_len[b] + ps - 1) / ps);
        pos = old_len[b] + r - row_sum[b];
        const int j = pos / ps;
        const int page = j < have ? p.block_table[b * p.table_stride + j]
                                  : p.free_list[free_now - 1 - (page_sum[b] + j - have)];
        if (page < 0 || page >= p.n_pages) flags |= DS_DEV_INDEX;
        else slot = (long long)page * ps + (pos - j * ps);
      }
      if (p.positions) p.positions[r] = pos;
      if (p.slot_map) p.slot_map[r] = slot;
    }
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

}  // namespace

int launch_page_update(const ds_page_params &p, cudaStream_t stream) {
  const size_t smem = sizeof(int) * (4 * (size_t)p.B + 4);
  DS_CUDA_OK(cudaFuncSetAttribute(page_update_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024));
  page_update_kernel<<<1, kThreads, smem, stream>>>(p);
  DS_CUDA_OK(cudaGetLastError());
  note_launch(1);
  return DS_OK;
}

}  // namespace ds

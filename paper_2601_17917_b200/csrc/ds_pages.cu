// ds_page_update: the bookkeeping of the paged cache, one step of it for every sequence.
//
// Latency is all there is to it.  A scan over the sequences (pages returned, pages and rows asked for; a second one over
// what is granted when somebody is refused) turns the rules of the header into exclusive sums kept in shared memory;
// after that every returned page, every page handed out and every new row is independent: a thread finds its sequence by
// bisecting the sums.
// One CTA does a call of few rows.  Calls with many rows run on a cluster: each CTA does the scan for itself
// and takes its share of the pages; cluster barriers stand between reading what the caller may pass as input and output
// at once, returning pages, and handing them out.  The row arrays are then filled by a second kernel over the whole GPU,
// launched early and waiting for the first, from the first one's results alone (3 MB of rows through the cluster's
// eight SMs took 20 us).
#include <cooperative_groups.h>

#include "ds_common.cuh"
#include "ds_paged_index.cuh"

namespace ds {
namespace {

constexpr int kCluster = 8;           // CTAs of a call with many rows
constexpr int kOneCtaRows = 4096;     // up to so many rows one CTA does it all
constexpr int kFillThreads = 256;

struct Sums {
  long long back, need, rows;
};
__device__ __forceinline__ Sums operator+(const Sums &a, const Sums &b) {
  return {a.back + b.back, a.need + b.need, a.rows + b.rows};
}

// Exclusive sum of one value per thread over the CTA; `total` gets the sum of all.
template <int kThreads>
__device__ Sums block_scan(const Sums &x, Sums *warp_sums, Sums &total) {
  constexpr int kWarps = kThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto scan = [&](Sums inc, int lanes) {
#pragma unroll
    for (int o = 1; o < lanes; o <<= 1) {
      const Sums y = {__shfl_up_sync(0xffffffffu, inc.back, o), __shfl_up_sync(0xffffffffu, inc.need, o),
                      __shfl_up_sync(0xffffffffu, inc.rows, o)};
      if (lane >= o) inc = inc + y;
    }
    return inc;
  };
  const Sums inc = scan(x, 32);
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  const Sums w = warp_sums[lane % kWarps], all = scan(w, kWarps);
  total = {__shfl_sync(0xffffffffu, all.back, kWarps - 1), __shfl_sync(0xffffffffu, all.need, kWarps - 1),
           __shfl_sync(0xffffffffu, all.rows, kWarps - 1)};
  const Sums ex = {all.back - w.back, all.need - w.need, all.rows - w.rows};
  const Sums before = {__shfl_sync(0xffffffffu, ex.back, warp), __shfl_sync(0xffffffffu, ex.need, warp),
                       __shfl_sync(0xffffffffu, ex.rows, warp)};
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

__device__ __forceinline__ void write_rows4(const ds_page_params &p, long long r0, bool vector, const int (&pos)[4],
                                            const long long (&slot)[4]) {
  if (vector && r0 + 4 <= p.max_rows) {
    if (p.positions) *reinterpret_cast<int4 *>(p.positions + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    if (p.slot_map) {
      *reinterpret_cast<longlong2 *>(p.slot_map + r0) = make_longlong2(slot[0], slot[1]);
      *reinterpret_cast<longlong2 *>(p.slot_map + r0 + 2) = make_longlong2(slot[2], slot[3]);
    }
    return;
  }
  for (int k = 0; k < 4 && r0 + k < p.max_rows; ++k) {
    if (p.positions) p.positions[r0 + k] = pos[k];
    if (p.slot_map) p.slot_map[r0 + k] = slot[k];
  }
}

// `vector`: positions and slot_map are 16-byte aligned.
template <int kThreads>
__global__ void __launch_bounds__(kThreads) page_update_kernel(const __grid_constant__ ds_page_params p, const FastDiv ps_div,
                                                               const bool vector, const bool fill) {
  namespace cg = cooperative_groups;
  extern __shared__ int smem[];
  __shared__ Sums warp_sums[2][kThreads / 32];
  dependent_sync();
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
  Sums at = block_scan<kThreads>(mine, warp_sums[0], total);
  const int returned = (int)min(total.back, (long long)(p.n_pages - free_cnt));
  if (total.back > returned) flags |= DS_DEV_INDEX;
  const int free_now = free_cnt + returned;
  if (total.need <= free_now && total.rows <= p.max_rows) {      // everybody gets what was asked for
    for (int b = b0; b < b1; ++b) {
      const Sequence s = b == b0 ? one : load_sequence(p, ps_div, b);
      back_sum[b] = (int)min(at.back, (long long)returned);
      page_sum[b] = (int)at.need;
      row_sum[b] = (int)at.rows;
      old_len[b] = s.old_len;
      at = at + Sums{s.back, s.need, s.n_new};
    }
  } else {
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
    Sums run = block_scan<kThreads>(granted, warp_sums[1], total);
    for (int b = b0; b < b1; ++b) {
      const int pages = page_sum[b], rows = row_sum[b];
      page_sum[b] = (int)run.need;
      row_sum[b] = (int)run.rows;
      run = run + Sums{0, pages, rows};
    }
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
  if (fill) {
    // a row's page comes from the table where it was there before this call, from the list where it is new
    for (long long r0 = 4LL * me; r0 < p.max_rows; r0 += 4LL * all) {
      int pos[4];
      long long slot[4];
      int b = r0 < n_rows ? owner(row_sum, B, (int)r0) : 0, last = -1, page = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
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
      write_rows4(p, r0, vector, pos, slot);
    }
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

// The number of entries of the ascending array that are <= x, less one, by a warp: 32 probes at a time.
__device__ __forceinline__ int warp_owner(const int *sum, int n, int x) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;      // sum[lo] <= x, and x < sum[hi] or hi == n
  while (hi - lo > 1) {
    const int step = (hi - lo + 32) / 33, at = lo + (lane + 1) * step;
    const uint32_t le = __ballot_sync(0xffffffffu, at < hi && sum[at] <= x);
    const int k = __popc(le);
    lo += k * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// positions and slot_map from row_start, kv_len_out and the finished tables.
__global__ void __launch_bounds__(kFillThreads) page_rows_kernel(const __grid_constant__ ds_page_params p, const FastDiv ps_div,
                                                                 const bool vector) {
  dependent_sync();
  const int B = p.B, ps = p.page_size, warp_rows = 128;
  const long long w0 = ((long long)blockIdx.x * (kFillThreads / 32) + (threadIdx.x >> 5)) * warp_rows;
  if (w0 >= p.max_rows) return;
  const int n_rows = p.row_start[B];
  int pos[4] = {0, 0, 0, 0};
  long long slot[4] = {-1, -1, -1, -1};
  const long long r0 = w0 + 4 * (threadIdx.x & 31);
  uint32_t flags = 0;
  if (w0 < n_rows) {
    int b = warp_owner(p.row_start, B, (int)w0);
    const int b_last = warp_owner(p.row_start, B, (int)min(w0 + warp_rows, (long long)n_rows) - 1);
    if (r0 < n_rows) {
      if (b != b_last) b += owner(p.row_start + b, b_last + 1 - b, (int)r0);
      int last = -1, page = 0, start = p.row_start[b], end = p.row_start[b + 1], old = p.kv_len_out[b] - (end - start);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const long long r = r0 + k;
        if (r >= n_rows) break;
        if (r >= end) {
          do {
            start = end;
            end = p.row_start[++b + 1];
          } while (end <= r);
          old = p.kv_len_out[b] - (end - start);
          last = -1;
        }
        pos[k] = old + (int)r - start;
        const int j = fast_div(pos[k], ps_div);
        if (j != last) page = p.block_table[b * p.table_stride + j];
        last = j;
        if (page < 0 || page >= p.n_pages) flags |= DS_DEV_INDEX;
        else slot[k] = (long long)page * ps + (pos[k] - j * ps);
      }
    }
  }
  if (r0 < p.max_rows) write_rows4(p, r0, vector, pos, slot);
  if (flags && p.status) atomicOr(p.status, flags);
}

template <int kThreads>
int launch_update(const ds_page_params &p, int ctas, bool vector, bool fill, cudaStream_t stream) {
  const size_t smem = sizeof(int) * (4 * (size_t)p.B + 4);
  static std::atomic<unsigned long long> allowed{0};
  if (smem > 40 * 1024) DS_CUDA_OK(allow_smem(page_update_kernel<kThreads>, 160 * 1024, allowed));
  DS_CUDA_OK(launch_kernel(page_update_kernel<kThreads>, dim3(ctas), kThreads, smem, ctas > 1 ? ctas : 0, true, stream, p,
                           make_fast_div(p.page_size), vector, fill));
  note_launch(1);
  return DS_OK;
}

}  // namespace

int launch_page_update(const ds_page_params &p, cudaStream_t stream) {
  const bool vector = ((reinterpret_cast<uintptr_t>(p.positions) | reinterpret_cast<uintptr_t>(p.slot_map)) & 15) == 0;
  const bool rows = p.positions || p.slot_map;
  if (p.max_rows <= kOneCtaRows)
    return p.B <= 256 ? launch_update<256>(p, 1, vector, rows, stream) : launch_update<1024>(p, 1, vector, rows, stream);
  const int rc = launch_update<1024>(p, kCluster, vector, false, stream);
  if (rc != DS_OK || !rows) return rc;
  const dim3 grid((unsigned)(((long long)p.max_rows + 4 * kFillThreads - 1) / (4 * kFillThreads)));
  DS_CUDA_OK(launch_kernel(page_rows_kernel, grid, kFillThreads, 0, 0, true, stream, p, make_fast_div(p.page_size), vector));
  note_launch(1);
  return DS_OK;
}

}  // namespace ds

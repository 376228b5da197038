// ds_attn_paged for many query rows per KV head (a decoding block, grouped queries of several tokens): bf16 on the 5th
// generation tensor cores.  Small calls go to the kernel for few rows all the same.
//
// An item is up to 128 stacked rows (query, head of the group) of a sequence and KV head, the rows of a tcgen05 tile:
// S = Q K^T and O += P V in TMEM, 128 keys at a time, with the online softmax on the thread that owns the tile's row.  The
// units of work, their equal ranges over the SMs and the join of items that ranges share are those of the kernel for few
// rows.  It is bound by HBM as long as the 1536 tensor cycles of a 64 KB key tile (512 for S, 1024 for P V, below) and
// the softmax fit into the 2800 that HBM needs for it.  The softmax does not when up to 64 rows leave it to two warps (128
// keys a thread: 8 x 32 heads x 1550 rows of D = 64 with blocks of 48 take 70 us, 16 x 32/8 heads x 4000 rows of D = 128 with 10
// queries 81), so up to 64 rows stand in the tile twice (60 and 74): each copy weighs half of the keys and holds zeros for the
// others, and the copies are joined when the item ends.
//
// Warps:
//   0-3  softmax and epilogue, thread = tile row = TMEM lane
//   4    issues the products
//   5    loads the queries of the next item
//   6-9  load K and V, 32 keys each: 16-byte asynchronous copies from wherever the page table says, written in the
//        128-byte swizzle that the products read.  (A page may be as small as one row, which leaves no box for TMA.)
// K and V tiles pass through a ring of kSlots in the order in which the products need them, K0 K1 V0 K2 V1 .. V(n-1) for a
// piece of n key tiles.  The copies themselves announce a tile (an asynchronous arrival of every loading thread), so a
// loading warp waits for free slots only; the issuer of the products orders them behind the copies with a proxy fence.
// (Loading warps that wait for their copies in order to announce them keep too little in flight: 81 to 98 us.)
//
// As with few rows the weights are kept as two bf16 halves, P V = P_hi V + P_lo V, so an output is rounded once; P_hi lies
// over the first half of its own S, P_lo in columns of its own.  O is zeroed by the epilogue rather than by the first
// product, so that a row may be corrected (below) before the first product as well as between others.
//
// Every wait is bounded; on expiry the kernel raises DS_DEV_TIMEOUT, drains and frees TMEM.
#include <type_traits>

#include "ds_attn_paged.cuh"

namespace ds {
namespace {

using namespace paged;
using namespace sm100;

constexpr int kRows = 128, kKeys = 128;
constexpr int kSoftmaxWarps = 4, kMmaWarp = 4, kQueryWarp = 5, kLoadWarp = 6, kLoadWarps = 4;
constexpr int kThreads = 32 * (kLoadWarp + kLoadWarps);
constexpr int kMinTiles = 2;       // a range has at least so many key tiles
constexpr int kWholeTiles = 2;     // items of at most so many key tiles are not split
constexpr uint32_t kTmemS = 0, kTmemO = 256, kTmemLo = 384, kTmemCols = 512;      // S (2), O, P_lo (2)
constexpr int kHalfBytes = 128 * 128;      // 128 rows of 64 elements: a swizzled half of a tile of D = 128

template <int D>
struct Geo {
  static constexpr int kTile = 128 * D * 2;
  static constexpr int kSlots = D == 128 ? 5 : 10;
  static constexpr int kOffRing = kTile;      // behind the queries
  static constexpr int kOffJoin = kOffRing + kSlots * kTile;      // [128 tile rows][64] fp32: half the dimensions of O
  static constexpr int kOffMl = kOffJoin + 128 * 256;             // [128] maximum and sum
  static constexpr int kOffBar = kOffMl + 128 * 8;
  // full[kSlots], empty[kSlots], q_full, q_free, s_full[2], p_full[2], pv_done[2], o_free, vote
  static constexpr int kNumBars = 2 * kSlots + 10;
  static constexpr int kOffMisc = kOffBar + 8 * kNumBars;      // TMEM base, abort flag, vote words (2 tiles)
  static constexpr int kOffScan = (kOffMisc + 8 + 8 * kSoftmaxWarps + 7) / 8 * 8;
  static constexpr int kBytes = kOffScan + 8 * (kThreads / 32 + 2) + 1024;      // slack: the base is aligned to 1024
  static_assert(kBytes <= 227 * 1024, "shared memory");
};

// Byte offset of 16-byte chunk `c` of row `r` in a K, V or Q tile.
__device__ __forceinline__ uint32_t tile_at(int r, int c) { return (c >> 3) * kHalfBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4); }

__device__ __forceinline__ uint32_t tmem_ld1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr) : "memory");
  return r;
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, uint32_t r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(r) : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
// Arrives at the barrier when this thread's copies so far are complete.
__device__ __forceinline__ void arrive_when_copied(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// The keys of a tile that a row sees: [0, hi) without [hole, back).
struct Seen {
  int hi, hole, back;
  __device__ __forceinline__ bool operator()(int c) const { return c < hi && (c < hole || c >= back); }
  // Keys c .. c + 31 as bits.
  __device__ __forceinline__ uint32_t bits(int c) const { return below(hi - c) & (below(hole - c) | ~below(back - c)); }
  static __device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }
};
__device__ __forceinline__ Seen seen_keys(const PagedShape &s, const PagedSeq &q, int x, int end) {
  if (x < q.sink_pad) return {paged_min(q.sink_n, end) - x, kKeys, 0};
  const int t = q.body + (x - q.sink_pad);
  if (s.window == 0) return {end - t, kKeys, 0};
  return {end - t, paged_max(s.sinks - t, 0), paged_max(end - s.window, 0) - t};
}

// With copies of a row, a copy's zeros for the others' keys times an infinity in V are NaN in its sum.  So where the joined sum is
// NaN and its sum of weights is not, the n keys from x on that it is over are gone through for infinities in elements d .. d + 3
// of V: by definition one of them is the average; two of different signs, or a NaN, are NaN.
__device__ __forceinline__ float4 average_of_infinities(const Params &a, const Item &it, int x, int n, int end, int d, float4 v) {
  const ds_paged_params &p = a.p;
  const int32_t *table = p.block_table + it.b * p.table_stride;
  const __nv_bfloat16 *base = reinterpret_cast<const __nv_bfloat16 *>(p.v_cache) + it.g * p.cache_stride[1] + d;
  uint32_t pos = 0, neg = 0, nan = 0;      // by element
  const uint32_t open = (isnan(v.x) ? 1u : 0u) | (isnan(v.y) ? 2u : 0u) | (isnan(v.z) ? 4u : 0u) | (isnan(v.w) ? 8u : 0u);
#pragma unroll 1
  for (int i = 0; i < n && (open & ~(nan | (pos & neg))); ++i) {
    const int t = paged_key(it.q, x + i);
    if (!paged_visible(a.s, t, end)) continue;
    const int j = fast_div(t, a.page_div), page = paged_clamp_page(table[j], p.n_pages);
    const __nv_bfloat16 *row = base + page * p.cache_stride[0] + (t - j * p.page_size) * p.cache_stride[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y = __bfloat162float(row[e]);
      pos |= (y == INFINITY ? 1u : 0u) << e;
      neg |= (y == -INFINITY ? 1u : 0u) << e;
      nan |= (isnan(y) ? 1u : 0u) << e;
    }
  }
  auto value = [&](float y, int e) {
    const bool up = (pos >> e) & 1, down = (neg >> e) & 1;
    return !((open >> e) & 1) || ((nan >> e) & 1) || up == down ? y : up ? INFINITY : -INFINITY;
  };
  return make_float4(value(v.x, 0), value(v.y, 1), value(v.z, 2), value(v.w, 3));
}

// kCopies: how often a row stands in the tile.
template <int D, int kCopies>
__global__ void __launch_bounds__(kThreads, 1) attn_paged_tc_kernel(const __grid_constant__ Params a) {
  using G = Geo<D>;
  using T = __nv_bfloat16;
  constexpr int S = G::kSlots, kPad = kRows / kCopies, kMine = kKeys / kCopies;      // rows of a copy, keys that it weighs
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sbase = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const ds_paged_params &p = a.p;
  const uint32_t bar_full = sbase + G::kOffBar, bar_empty = bar_full + 8 * S, bar_q_full = bar_empty + 8 * S,
                 bar_q_free = bar_q_full + 8, bar_s_full = bar_q_free + 8, bar_p_full = bar_s_full + 16,
                 bar_pv_done = bar_p_full + 16, bar_o_free = bar_pv_done + 16, bar_vote = bar_o_free + 8;
  volatile uint32_t *tmem_s = reinterpret_cast<volatile uint32_t *>(smem + G::kOffMisc);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + G::kOffMisc + 4);
  volatile uint32_t *vote_s = reinterpret_cast<volatile uint32_t *>(smem + G::kOffMisc + 8);

  if (tid == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(bar_full + 8 * s, 32 * kLoadWarps);
      mbar_init(bar_empty + 8 * s, 1);
    }
    mbar_init(bar_q_full, 1);
    mbar_init(bar_q_free, 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar_s_full + 8 * s, 1);
      mbar_init(bar_p_full + 8 * s, kSoftmaxWarps);
      mbar_init(bar_pv_done + 8 * s, 1);
    }
    mbar_init(bar_o_free, kSoftmaxWarps);
    mbar_init(bar_vote, kSoftmaxWarps);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == kMmaWarp) tmem_alloc(sbase + G::kOffMisc, kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_s;
  dependent_sync();
  uint32_t flags = 0;
  Walk walk;
  walk.find<kThreads>(a, kMinTiles, reinterpret_cast<long long *>(smem + G::kOffScan), flags);
  const Item &it = walk.it;
  bool ok = true;

  if (warp >= kLoadWarp) {
    // ============================ K and V ============================
    constexpr int kChunks = D / 8, kPer = 32 / kChunks > 0 ? 32 / kChunks : 1, kOps = 16 / kPer;      // rows of an instruction
    const int first_key = 32 * (warp - kLoadWarp);
    const long long row_bytes = p.cache_stride[2] * 2;
    int f = 0;      // tiles issued
    for (; ok && walk.piece(a); walk.next(a)) {
      const int32_t *table = p.block_table + it.b * p.table_stride;
      const uint8_t *kbase = reinterpret_cast<const uint8_t *>(reinterpret_cast<const T *>(p.k_cache) + it.g * p.cache_stride[1]);
      const uint8_t *vbase = reinterpret_cast<const uint8_t *>(reinterpret_cast<const T *>(p.v_cache) + it.g * p.cache_stride[1]);
      const int x0 = walk.tile0 * kKeys + first_key + lane;
      const int ch = lane % kChunks;
      auto issue = [&](const uint8_t *base, long long at) {      // at: of key first_key + lane
        ok = __all_sync(0xffffffffu, mbar_wait(bar_empty + 8 * (f % S), ((f / S) & 1) ^ 1, abort_flag));
        if (!ok) return;
        const uint32_t dst = sbase + G::kOffRing + (f % S) * G::kTile;
        // 16 keys that lie evenly (in one page) need one address
        const long long at_lo = __shfl_sync(0xffffffffu, at, 0), at_hi = __shfl_sync(0xffffffffu, at, 16);
        const uint32_t even = __ballot_sync(0xffffffffu, at >= 0 && at == (lane < 16 ? at_lo : at_hi) + (lane & 15) * row_bytes);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (((even >> (16 * half)) & 0xffffu) == 0xffffu) {
            const uint8_t *from = base + (half ? at_hi : at_lo) + (lane / kChunks) * row_bytes + 16 * ch;
#pragma unroll
            for (int j = 0; j < kOps; ++j, from += kPer * row_bytes)
              cp_async16(dst + tile_at(first_key + 16 * half + j * kPer + lane / kChunks, ch), from, true);
          } else {
#pragma unroll
            for (int j = 0; j < kOps; ++j) {
              const int r = 16 * half + j * kPer + lane / kChunks;
              const long long off = __shfl_sync(0xffffffffu, at, r);
              cp_async16(dst + tile_at(first_key + r, ch), base + (off >= 0 ? off : 0) + 16 * ch, off >= 0);
            }
          }
        }
        arrive_when_copied(bar_full + 8 * (f % S));
        ++f;
      };
      int pos = paged_key(it.q, x0), page = pos >= 0 ? table[fast_div(pos, a.page_div)] : 0;
      long long before = -1;      // of the previous key tile
      for (int i = 0; ok && i < walk.n_tiles; ++i) {
        long long at = -1;
        if (pos >= 0) {
          const int there = paged_clamp_page(page, p.n_pages);
          if (there != page) flags |= DS_DEV_INDEX;
          const int slot = pos - fast_div(pos, a.page_div) * p.page_size;
          at = there * p.cache_stride[0] * 2 + slot * row_bytes;
        }
        if (i + 1 < walk.n_tiles) {
          pos = paged_key(it.q, x0 + (i + 1) * kKeys);
          page = pos >= 0 ? table[fast_div(pos, a.page_div)] : 0;
        }
        issue(kbase, at);
        if (ok && i > 0) issue(vbase, before);
        before = at;
      }
      if (ok) issue(vbase, before);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == kQueryWarp) {
    // ============================ queries ============================
    for (int k = 0; ok && walk.piece(a); walk.next(a), ++k) {
      if (k > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar_q_free, (k - 1) & 1, abort_flag));
      if (!ok) break;
      for (int c = lane; c < it.rows * (D / 8); c += 32) {
        const Row row = row_of(a, it, c / (D / 8));
        const T *from = reinterpret_cast<const T *>(p.q) + row.n * p.q_stride[0] + row.h * p.q_stride[1] + 8 * (c % (D / 8));
#pragma unroll
        for (int copy = 0; copy < kCopies; ++copy)
          cp_async16(sbase + tile_at(copy * kPad + c / (D / 8), c % (D / 8)), from, true);
      }
      cp_async_commit();
      cp_async_wait<0>();
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_q_full);
    }
  } else if (warp == kMmaWarp) {
    // ============================ products ============================
    constexpr uint32_t idesc_qk = instr_desc(kRows, kKeys, false, false), idesc_pv = instr_desc(kRows, D, false, true);
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t dq = smem_desc(sbase, 16, 1024);
    const uint64_t dk0 = smem_desc(sbase + G::kOffRing, 16, 1024), dv0 = smem_desc(sbase + G::kOffRing, kHalfBytes, 1024);
    int g = 0, k = 0, f = 0;      // key tiles, pieces, tiles of the ring
    bool pv_first = false;      // tile g - 1 is the first of its piece, number k_pv
    int k_pv = 0;
    auto pv = [&]() {      // P V of tile g - 1
      const int h = g - 1;
      bool w = mbar_wait2(bar_p_full + 8 * (h & 1), (h >> 1) & 1, bar_full + 8 * (f % S), (f / S) & 1, abort_flag);
      if (pv_first) w = w && mbar_wait(bar_o_free, k_pv & 1, abort_flag);
      ok = __all_sync(0xffffffffu, w);
      if (!ok) return;
      fence_proxy_async();
      tc_fence_after();
      const uint64_t dv = dv0 + (uint64_t)(((f % S) * G::kTile) >> 4);
      if (elect_one()) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int ks = 0; ks < kKeys / 16; ++ks)
            umma_ts(tm + kTmemO, tm + (part ? kTmemLo + (h & 1) * 64 : kTmemS + (h & 1) * 128) + ks * 8,
                    dv + ((ks * 2048) >> 4), idesc_pv, 1u);
        umma_commit(bar_empty + 8 * (f % S));
        umma_commit(bar_pv_done + 8 * (h & 1));
      }
      __syncwarp();
      ++f;
    };
    for (; ok && walk.piece(a); walk.next(a), ++k) {
      if (g > 0) pv();      // ends the piece before: the queries that the next product waits for may take a while
      ok = ok && __all_sync(0xffffffffu, mbar_wait(bar_q_full, k & 1, abort_flag));
      for (int i = 0; ok && i < walk.n_tiles; ++i, ++g) {
        // the tile has landed, and S[g % 2] is free: P V of tile g - 2, the last to read it, has completed
        ok = __all_sync(0xffffffffu, g < 2 ? mbar_wait(bar_full + 8 * (f % S), (f / S) & 1, abort_flag)
                                           : mbar_wait2(bar_full + 8 * (f % S), (f / S) & 1, bar_pv_done + 8 * (g & 1),
                                                        ((g - 2) >> 1) & 1, abort_flag));
        if (!ok) break;
        fence_proxy_async();
        tc_fence_after();
        const uint64_t dk = dk0 + (uint64_t)(((f % S) * G::kTile) >> 4);
        if (elect_one()) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t off = ((ks / 4) * kHalfBytes + (ks % 4) * 32) >> 4;
            umma_ss(tm + kTmemS + (g & 1) * 128, dq + off, dk + off, idesc_qk, ks > 0);
          }
          umma_commit(bar_s_full + 8 * (g & 1));
          umma_commit(bar_empty + 8 * (f % S));
          if (i == walk.n_tiles - 1) umma_commit(bar_q_free);
        }
        __syncwarp();
        ++f;
        if (i > 0) {
          pv();
          if (!ok) break;
        }
        pv_first = i == 0;
        k_pv = k;
      }
    }
    if (ok && g > 0) pv();
  } else {
    // ============================ softmax and epilogue ============================
    const uint32_t tw = tmem + ((uint32_t)(32 * warp) << 16);
    const int r = tid % kPad, copy = tid / kPad, key0 = copy * kMine;      // row of the item, keys of this copy
    // The maximum is kept of the scores as they are (negated under a negative scale) and the difference to it scaled.  Scaled
    // first, the two are fused into one operation, and what its exact product differs by from a maximum that was rounded is
    // itself a large exponent where the scores are (keys of the type's lowest values).
    const float scale2 = p.scale * kLog2e, steep = fabsf(scale2), sign = scale2 < 0.f ? -1.f : 1.f;
    PagedJoin join = {0, 0, 0, 0, 0, 0};      // thread 0's
    auto zero_o = [&]() {
      uint32_t z[32];
#pragma unroll
      for (int c = 0; c < 32; ++c) z[c] = 0;
#pragma unroll
      for (int c = 0; c < D; c += 32) tmem_st32(tw + kTmemO + c, z);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_o_free);
    };
    {
      uint32_t z[8] = {};      // P_lo of the keys of other copies stays zero
#pragma unroll
      for (int c = 0; c < 128; c += 8) tmem_st8(tw + kTmemLo + c, z);
    }
    zero_o();
    int g = 0, votes = 0, ring0 = 0;      // votes: also those of the joins; ring0: where the piece begins in the ring
    for (; ok && walk.piece(a); ring0 += 2 * walk.n_tiles, walk.next(a)) {
      if (a.split && tid == 0) walk.note_join(join);
      const bool busy = (32 * warp) % kPad < it.rows, mine = r < it.rows;
      const Row row = row_of(a, it, mine ? r : 0);
      const int end = mine ? row.end : 0;
      float m = -INFINITY, l = 0.f;
      for (int i = 0; i < walk.n_tiles; ++i, ++g) {
        const int x = (walk.tile0 + i) * kKeys;
        const bool all = paged_all_visible(a.s, it.q, x, kKeys);
        const uint32_t ts = tw + kTmemS + (g & 1) * 128, tlo = tw + kTmemLo + (g & 1) * 64;
        ok = __all_sync(0xffffffffu, mbar_wait(bar_s_full + 8 * (g & 1), (g >> 1) & 1, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const Seen seen = seen_keys(a.s, it.q, x, end);
        if (busy) {
          // ---- largest score of this copy's keys
          float top = -INFINITY;
          uint32_t s[32];
#pragma unroll 1
          for (int c = key0; c < key0 + kMine; c += 32) {
            tmem_ld32(ts + c, s);
            tmem_wait_ld();
            if (all) {
#pragma unroll
              for (int e = 0; e < 32; e += 2)
                top = fmax3(top, __uint_as_float(s[e]) * sign, __uint_as_float(s[e + 1]) * sign);
            } else {
              const uint32_t bits = seen.bits(c);
#pragma unroll
              for (int e = 0; e < 32; ++e) top = fmaxf(top, (bits >> e) & 1 ? __uint_as_float(s[e]) * sign : -INFINITY);
            }
          }
          // The reference moves only when a weight would pass 2^8: the result is the same, O is touched rarely.
          const bool over = mine && (m == -INFINITY ? top > m : (top - m) * steep > 8.f);
          if (__any_sync(0xffffffffu, over)) {
            const float keep = !over ? 1.f : m == -INFINITY ? 0.f : ex2_approx((m - top) * steep);
            if (over) m = top;
            l *= keep;
            if (i > 0) {
              ok = __all_sync(0xffffffffu, mbar_wait(bar_pv_done + 8 * ((g - 1) & 1), ((g - 1) >> 1) & 1, abort_flag));
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D; c += 32) {
                uint32_t o[32];
                tmem_ld32(tw + kTmemO + c, o);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                tmem_st32(tw + kTmemO + c, o);
              }
              tmem_wait_st();
            }
          }
          // ---- weights
          const float ref = m == -INFINITY ? 0.f : m * sign;      // nothing seen yet: exp(-inf) = 0
          // weights are scaled down in the exponent (16 x 32/8 heads x 4000 rows with 10 queries: 73.4 us, multiplied afterwards 74.3);
          // that rounds them at 2^-19, their halves do at 2^-16
          const F2 scale_2 = f2(scale2, scale2), ref_2 = f2(-ref, -ref), shrink_2 = f2(a.shrink_log2, a.shrink_log2);
          F2 l_2 = 0;
          auto weights = [&](auto every) {      // std::true_type: no key of the tile is hidden
            constexpr bool kAll = decltype(every)::value;
#pragma unroll 1
            for (int c = key0; c < key0 + kMine; c += 32) {
              uint32_t hi[16], lo[16];
              tmem_ld32(ts + c, s);
              tmem_wait_ld();
              const uint32_t bits = kAll ? 0xffffffffu : seen.bits(c);
#pragma unroll
              for (int e = 0; e < 32; e += 2) {
                float2 w = f2_get(fma2(add2(f2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), ref_2), scale_2, shrink_2));
                w.x = ex2_approx(w.x), w.y = ex2_approx(w.y);
                if (!kAll) {
                  if (!((bits >> e) & 1)) w.x = 0.f;
                  if (!((bits >> (e + 1)) & 1)) w.y = 0.f;
                }
                const F2 weight = f2(w.x, w.y);
                l_2 = add2(l_2, weight);
                split_weights(weight, hi[e / 2], lo[e / 2]);
              }
              // over scores that have been read, or are another copy's: columns c / 2 .. c / 2 + 15 <= c + 31
              tmem_st16(ts + c / 2, hi);
              tmem_st16(tlo + c / 2, lo);
            }
          };
          if (all) weights(std::true_type());
          else weights(std::false_type());
          l += f2_get(l_2).x + f2_get(l_2).y;
          if constexpr (kCopies > 1) {      // no weight for the other copies' keys
            uint32_t z[16] = {};
#pragma unroll
            for (int c = 0; c < kKeys / 2; c += 16)
              if (c < key0 / 2 || c >= (key0 + kMine) / 2) tmem_st16(ts + c, z);
          }
          tmem_wait_st();
        }
        if (!all && a.s.causal && it.q.count > 1) {
          // Keys that some rows see and others do not: a weight of zero times an infinite or NaN value would be NaN in
          // the product.  If V holds such values (rare), their terms are added to O here for the rows that see them,
          // one by one, and they are replaced by zero.
          const int f = ring0 + 2 * i + (i < walk.n_tiles - 1 ? 2 : 1);      // V of this tile in the ring
          uint8_t *v = smem + G::kOffRing + (f % S) * G::kTile;
          bool w = mbar_wait(bar_full + 8 * (f % S), (f / S) & 1, abort_flag);
          bool bad = false;
          for (int c = 0; c < D / 8; ++c) {
            const uint4 q = *reinterpret_cast<const uint4 *>(v + tile_at(tid, c));
            const uint32_t x4[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) bad |= (x4[e] & 0x7f80u) == 0x7f80u || (x4[e] & 0x7f800000u) == 0x7f800000u;
          }
          const uint32_t word = __ballot_sync(0xffffffffu, bad);
          volatile uint32_t *votes_s = vote_s + (g & 1) * kSoftmaxWarps;      // a warp may be one tile ahead of another
          if (lane == 0) {
            votes_s[warp] = word;
            mbar_arrive(bar_vote);
          }
          w = w && mbar_wait(bar_vote, votes++ & 1, abort_flag);
          ok = __all_sync(0xffffffffu, w);
          if (!ok) break;
          if (votes_s[0] | votes_s[1] | votes_s[2] | votes_s[3]) {
            if (i > 0) w = mbar_wait(bar_pv_done + 8 * ((g - 1) & 1), ((g - 1) >> 1) & 1, abort_flag);
            tc_fence_after();
            for (int key = 0; busy && key < kKeys; ++key) {
              if (key < key0 || key >= key0 + kMine || !((votes_s[key >> 5] >> (key & 31)) & 1)) continue;      // the whole warp
              const uint32_t wh = tmem_ld1(ts + key / 2), wl = tmem_ld1(tlo + key / 2);
              tmem_wait_ld();
              const float weight = key & 1 ? bf16hi_to_f32(wh) + bf16hi_to_f32(wl) : bf16lo_to_f32(wh) + bf16lo_to_f32(wl);
              for (int d = 0; d < D; ++d) {
                const float value = __bfloat162float(*reinterpret_cast<const T *>(v + tile_at(key, d / 8) + (d & 7) * 2));
                if (isfinite(value)) continue;
                float o = __uint_as_float(tmem_ld1(tw + kTmemO + d));
                tmem_wait_ld();
                if (seen(key)) o += weight * value;
                tmem_st1(tw + kTmemO + d, __float_as_uint(o));
                tmem_wait_st();
              }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_vote);      // all rows have read V
            w = w && mbar_wait(bar_vote, votes++ & 1, abort_flag);
            ok = __all_sync(0xffffffffu, w);
            if (!ok) break;
            for (int c = 0; bad && c < D / 8; ++c) {
              uint4 *at = reinterpret_cast<uint4 *>(v + tile_at(tid, c));
              uint32_t x4[4] = {at->x, at->y, at->z, at->w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((x4[e] & 0x7f80u) == 0x7f80u) x4[e] &= 0xffff0000u;
                if ((x4[e] & 0x7f800000u) == 0x7f800000u) x4[e] &= 0xffffu;
              }
              *at = make_uint4(x4[0], x4[1], x4[2], x4[3]);
            }
            fence_proxy_async();
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p_full + 8 * (g & 1));
      }
      if (!ok) break;
      // ---- the piece is done
      if (m != -INFINITY) m *= steep;
      l *= a.stretch;
      ok = __all_sync(0xffffffffu, mbar_wait(bar_pv_done + 8 * ((g - 1) & 1), ((g - 1) >> 1) & 1, abort_flag));
      if (!ok) break;
      tc_fence_after();
      const bool whole = walk.whole();
      const long long at = (long long)paged_slot(blockIdx.x, walk.first) * a.part_rows + r;
      if constexpr (kCopies == 1) {
        if (busy) {
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            tmem_ld32(tw + kTmemO + c, o);
            tmem_wait_ld();
            if (!mine) continue;
            if (whole) {
              const float inv = l == 0.f ? 0.f : a.stretch / l;
              uint4 *dst = reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.out) + row.n * p.out_stride[0] + row.h * p.out_stride[1] + c);
#pragma unroll
              for (int e = 0; e < 32; e += 8) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                  w[k] = pack_bf16(__uint_as_float(o[e + 2 * k]) * inv, __uint_as_float(o[e + 2 * k + 1]) * inv);
                dst[e / 8] = make_uint4(w[0], w[1], w[2], w[3]);
              }
            } else {
              uint4 *dst = reinterpret_cast<uint4 *>(a.part_o + at * D + c);
#pragma unroll
              for (int e = 0; e < 32; e += 4) dst[e / 4] = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
            }
          }
          if (mine && whole && p.lse) p.lse[row.n * p.Hq + row.h] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
          if (mine && !whole) a.part_ml[at] = make_float2(m, l);
        }
      } else {
        // ---- join the copies, 64 dimensions at a time; a thread adds up 64 / kCopies of them for its row
        float2 *ml_s = reinterpret_cast<float2 *>(smem + G::kOffMl);
        uint8_t *join_s = smem + G::kOffJoin;
        auto quad = [&](int tile_row, int q) { return reinterpret_cast<float4 *>(join_s + tile_row * 256 + ((q ^ (tile_row & 15)) << 4)); };
        auto meet = [&]() {
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_vote);
          ok = __all_sync(0xffffffffu, mbar_wait(bar_vote, votes++ & 1, abort_flag));
        };
        ml_s[tid] = make_float2(m, l);
#pragma unroll 1
        for (int half = 0; ok && half < D / 64; ++half) {      // code that runs once per item: kept short
          if (busy) {
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
              uint32_t o[32];
              tmem_ld32(tw + kTmemO + half * 64 + c, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; e += 4)
                *quad(tid, c / 4 + e / 4) = make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]), __uint_as_float(o[e + 2]),
                                                      __uint_as_float(o[e + 3]));
            }
          }
          meet();
          if (ok && mine) {
            float top = -INFINITY, sum = 0.f, f[kCopies];
#pragma unroll
            for (int k = 0; k < kCopies; ++k) top = fmaxf(top, ml_s[k * kPad + r].x);
#pragma unroll
            for (int k = 0; k < kCopies; ++k) {
              const float2 ml = ml_s[k * kPad + r];
              f[k] = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top);
              sum = fmaf(ml.y, f[k], sum);
            }
#pragma unroll 1
            for (int e = 0; e < 16 / kCopies; ++e) {
              const int q = copy * (16 / kCopies) + e, d = half * 64 + 4 * q;
              float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
              for (int k = 0; k < kCopies; ++k) {
                const float4 o = *quad(k * kPad + r, q);
                v.x = fmaf(o.x, f[k], v.x), v.y = fmaf(o.y, f[k], v.y), v.z = fmaf(o.z, f[k], v.z), v.w = fmaf(o.w, f[k], v.w);
              }
              if (__builtin_expect(isnan((v.x + v.y) + (v.z + v.w)) && !isnan(sum), 0))
                v = average_of_infinities(a, it, walk.tile0 * kKeys, walk.n_tiles * kKeys, end, d, v);
              if (whole) {
                write_row4<T>(a, row, d, v, top, sum);
              } else {
                *reinterpret_cast<float4 *>(a.part_o + at * D + d) = v;
                if (d == 0) a.part_ml[at] = make_float2(top, sum);
              }
            }
          }
          if (ok) meet();      // the buffer is read
        }
        if (!ok) break;
      }
      zero_o();
    }
    if (a.split && tid == 0) a.joins[blockIdx.x] = join;
  }

  if (!ok) flags |= DS_DEV_TIMEOUT;
  if (flags && p.status) atomicOr(p.status, flags);
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

size_t workspace_of(const Shape &h) { return h.tiles <= kWholeTiles || h.grid == 1 ? 0 : h.workspace(); }

// Copies of a row in the tile: two where there is room for them.  (Calls of up to 32 rows do not come here.)
int copies_for(const ds_paged_params &p) { return (long long)p.max_q * (p.Hq / p.Hkv) <= kRows / 2 ? 2 : 1; }
Shape shape_for(const ds_paged_params &p) { return shape_of(p, kKeys, kRows / copies_for(p), kMinTiles, 1); }

template <int D, int kCopies>
int launch(const ds_paged_params &p, cudaStream_t stream) {
  const Shape h = shape_for(p);
  const Params a = params_of(p, h, workspace_of(h));
  static std::atomic<unsigned long long> allowed{0};
  DS_CUDA_OK(allow_smem(attn_paged_tc_kernel<D, kCopies>, Geo<D>::kBytes, allowed));
  DS_CUDA_OK(launch_kernel(attn_paged_tc_kernel<D, kCopies>, dim3(h.grid), kThreads, Geo<D>::kBytes, 0, false, stream, a));
  note_launch(1);
  return a.split ? launch_join<__nv_bfloat16, D>(a, h, stream) : (int)DS_OK;
}

template <int D>
int launch_copies(const ds_paged_params &p, cudaStream_t stream) {
  return copies_for(p) == 2 ? launch<D, 2>(p, stream) : launch<D, 1>(p, stream);
}

}  // namespace

bool attn_paged_tc_counts_fit(const ds_paged_params &p) {
  const PagedShape s = units_of(p, kKeys, kRows / copies_for(p));
  return paged_units_fit(s, longest_of(s));
}

size_t attn_paged_tc_workspace_bytes(const ds_paged_params &p) { return workspace_of(shape_for(p)); }

int launch_attn_paged_tc(const ds_paged_params &p, cudaStream_t stream) {
  return p.D == 64 ? launch_copies<64>(p, stream) : launch_copies<128>(p, stream);
}

}  // namespace ds

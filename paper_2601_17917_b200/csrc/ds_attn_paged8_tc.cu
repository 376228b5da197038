// ds_attn_paged8 for more query rows per KV head (a decoding block, grouped queries of several tokens): bf16 queries on the 5th
// generation tensor cores.
//
// S = Q K^T takes K as it is, e4m3.  A bf16 query, scaled by a power of two so that its row's largest element lies in [2^7, 2^8), is the
// sum of an e4m3 value (rounded to the nearest 4 bits) and an e5m2 one: what is left of 8 bits is at most 8 of their units, which 3 bits
// hold.  So two products of 8-bit operands, in one accumulator, are exact in the queries down to 2^-14 of the row's largest element and
// within 2^-21 of it below.  O += P V takes fp16: four warps turn the e4m3 values of a tile into fp16, which holds them all, in the layout
// of the product; weights are fp16 with V's scale in them and a power of two for each row, as in the kernel for few rows (Weights8).  (P in 8-bit halves would drop what lies below
// 2^-22 of the largest weight, a per cent of the sum in a long cache.)
//
// Two streams of 128 tile rows each, with a warpgroup, S and O of their own, keep the tensor pipe and the exponentials busy at once:
//   kPair      rows 0 .. 127 and 128 .. 255 of an item, over the same key tiles
//   otherwise  the same rows, the even and the odd key tiles, joined when the item ends.  Up to 64 rows stand in the tile twice (kCopies):
//              each copy weighs half of the keys and has zeros for the others.
// Step u of a piece is stream u % 2, key tile u (kPair: u / 2).  A stream's products go out in the order QK0 PV0 QK2 PV2 ..; S is written
// again when the product that reads the P in its place is done (waited for: products of different kinds and shapes need not execute in the
// order of their issue; 82.5 -> 83.4 us).  The second stream starts half a step later (82 -> 80 us): its exponentials run beside the first
// one's products.
//
// Warps:
//   0-7    softmax and epilogue, thread = tile row = TMEM lane, four warps a stream
//   8-9    issue the products, a warp for each stream
//   10-11  load, every other tile each: 16-byte asynchronous copies of K (in the swizzle of the products) and V from wherever the page
//          table says, and the scales
//   12-15  at the start of a piece the queries, four threads a row; then V to fp16, 32 keys each
// (One set of four warps that loaded and converted took 5500 cycles a tile, most of them in its own instructions: 120 us where this
// took 80.)
//
// A key tile's 32 KB are 1430 cycles of an SM's share of HBM; its products 256 (e4m3, two parts) + 256 cycles and its exponentials 1024, for 128
// rows.  Measured, 16 sequences x 4 heads of 224 rows x 1500 .. 4128 keys: 84 us, where the bf16 cache takes 73 (91 with scales for every
// token); a step of a stream takes some 5000 cycles, a quarter of them for the maximum, the most for the weights of 128 keys, which is the
// latency of TMEM loads and exponentials with two softmax warps a scheduler (issue slots 32 % in use, tensor pipe 13 %, exponentials 12 % in a
// small case).  Tried and not kept: scores held in registers between the two passes and register splits between the roles (no faster), TMEM
// loads a step ahead (80.3 against 79.9 us).
//
// Every wait is bounded; on expiry the kernel raises DS_DEV_TIMEOUT, drains and frees TMEM.
#include <type_traits>

#include "ds_attn_paged.cuh"
#include "ds_e4m3.cuh"
#include "ds_paged8.cuh"

namespace ds {
namespace {

using namespace paged;
using namespace sm100;

constexpr int kKeys = 128;
constexpr int kSoftmaxWarps = 8, kMmaWarp = 8, kLoadWarp = 10, kLoadWarps = 2, kConvertWarp = 12, kConvertWarps = 4;
constexpr int kThreads = 32 * (kConvertWarp + kConvertWarps);
constexpr int kMinTiles = 2;       // a range has at least so many key tiles, where items are split
constexpr int kWholeTiles = 2;     // items of at most so many key tiles are not split
constexpr uint32_t kTmemS = 0, kTmemO = 256, kTmemCols = 512;      // S (2 x 128), O (2 x 128); P over S
constexpr int kHalfBytes = 128 * 128;      // 128 keys of 64 dimensions in fp16: a swizzled half of a tile of D = 128
constexpr int kScaleRing = 4;              // key tiles whose scales are held

template <int D, bool kPair>
struct Geo {
  static constexpr int kTile = 128 * D;      // bytes of 128 e4m3 rows
  static constexpr int kRows = kPair ? 256 : 128;
  static constexpr int kSlots = kPair ? 2 : 3;      // of the rings of K and of V
  static constexpr int kQPart = kRows * D;          // one part of the queries
  static constexpr int kOffK = 2 * kQPart;
  static constexpr int kOffV = kOffK + kSlots * kTile;
  static constexpr int kOffV16 = kOffV + kSlots * kTile;                  // [2] tiles in fp16; at the end of an item sums to be joined
  static constexpr int kOffScale = kOffV16 + 2 * 2 * kTile;               // [kScaleRing][3][128]: K's, V's, logarithms of V's where they are asked for
  static constexpr int kOffFactor = kOffScale + kScaleRing * 1536;        // [kRows]
  static constexpr int kOffMl = kOffFactor + kRows * 4;                   // [256]
  static constexpr int kOffTo = kOffMl + (kPair ? 0 : 256 * 8);           // [kRows]
  static constexpr int kOffNan = kOffTo + kRows * 8;                      // [kRows][D / 32]: outputs that V makes NaN
  static constexpr int kOffBar = kOffNan + kRows * D / 8;
  // k_full, k_empty, v_full, v_empty [kSlots], v16_full, v16_free [2], scale_ready, scale_free [kScaleRing], s_full, p_full, pv_done, o_free
  // [2], q_full, q_free, meet, joined, begun
  static constexpr int kNumBars = 4 * kSlots + 4 + 2 * kScaleRing + 8 + 5;
  static constexpr int kOffMisc = kOffBar + 8 * kNumBars;      // TMEM base, whether a wait has run out, piece with NaN in V, sizes of V's scales [kScaleRing]
  static constexpr int kOffScan = (kOffMisc + 12 + 4 * kScaleRing + 7) / 8 * 8;
  // Sums on their way out, [256][kOutDims] fp32.  Of pairs in a place of their own: a stream need not wait for the other's last products.
  static constexpr int kOutDims = kPair ? 16 : D == 128 ? 64 : 32;
  static constexpr int kOffOut = kPair ? (kOffScan + 8 * (kThreads / 32 + 2) + 127) / 128 * 128 : kOffV16;
  static constexpr int kBytes = (kPair ? kOffOut + 256 * kOutDims * 4 : kOffScan + 8 * (kThreads / 32 + 2)) + 1024;      // slack: the base is aligned to 1024
  static_assert(kBytes <= 227 * 1024, "shared memory");
  static_assert(kPair || 256 * kOutDims * 4 <= 4 * kTile, "sums to be joined");
};

// Byte offset of 16-byte chunk `c` of row `r` of e4m3 values: the 128-byte swizzle for rows of 128 bytes, the 64-byte one for 64.
template <int D>
__device__ __forceinline__ uint32_t row_at(int r, int c) { return r * D + ((c ^ (D == 64 ? (r >> 1) & 3 : r & 7)) << 4); }
// The same of a tile of fp16 values, halves of 64 dimensions.
__device__ __forceinline__ uint32_t half_at(int r, int c) { return (c >> 3) * kHalfBytes + r * 128 + (((c & 7) ^ (r & 7)) << 4); }

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t *r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
// D[tmem] (+)= A[smem] * B[smem], 8-bit operands.
__device__ __forceinline__ void umma_ss8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Descriptor of rows of `row` bytes (128 or 64) in the swizzle of that width, groups of eight rows one after the other.
__device__ __forceinline__ uint64_t rows_desc(uint32_t addr, int row) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)((8 * row) >> 4) << 32) | (1ull << 46) | ((row == 64 ? 4ull : 2ull) << 61);
}
// Instruction descriptors: fp32 accumulation; A of e5m2 or e4m3 and B of e4m3, K-major; A and B of fp16, B with its N side contiguous.
__host__ __device__ constexpr uint32_t idesc8(int n, bool a_e5m2) { return (1u << 4) | ((a_e5m2 ? 1u : 0u) << 7) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }
__host__ __device__ constexpr uint32_t idesc16(int n) { return (1u << 4) | (1u << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }

// Bounded wait in few instructions: what runs once per tile comes through the instruction caches at some four cycles each.  The word at
// `gave_up` is 0, or kSpinLimit when another role's wait has run out: then this one ends, too.
__device__ __forceinline__ bool wait_parity(uint32_t bar, uint32_t parity, uint32_t gave_up) {
  int left = kSpinLimit;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      ".reg .b32 f;\n"
      "WAIT:\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "@p bra DONE;\n\t"
      "ld.volatile.shared.u32 f, [%3];\n\t"
      "sub.s32 %0, %0, 1;\n\t"
      "sub.s32 %0, %0, f;\n\t"
      "setp.gt.s32 q, %0, 0;\n\t"
      "@q bra WAIT;\n"
      "DONE:\n\t}"
      : "+r"(left) : "r"(bar), "r"(parity), "r"(gave_up) : "memory");
  return left > 0;
}

// Arrives at the barrier when this thread's copies so far are complete.
__device__ __forceinline__ void arrive_when_copied(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
// The keys of a tile that a row sees: [0, hi) without [hole, back).
struct Seen {
  int hi, hole, back;
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

// V's NaN are zeros in the product of a tile that not every row sees whole; what they make of the rows' outputs is noted here, a bit for
// each dimension: which bytes of a chunk of 16 dimensions are NaN,
__device__ __forceinline__ uint32_t nan_bits(const uint4 &w) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) bits |= (((__vcmpeq4(x[e] & 0x7f7f7f7fu, 0x7f7f7f7fu) & 0x01010101u) * 0x01020408u) >> 24) << (4 * e);
  return bits;
}
// the rows of an item that see cache row t, which follow one another,
struct RowRange {
  int lo, hi;
};
__device__ __forceinline__ RowRange rows_that_see(const PagedShape &s, const Item &it, int t) {
  if (t < 0) return {0, 0};
  const long long last_seen = s.window > 0 && t >= s.sinks ? (long long)t + s.window : 0x7fffffffffffll;      // ends beyond t and up to this see it
  if (!s.causal) return {0, it.q.len > t && it.q.len <= last_seen ? it.rows : 0};
  auto queries = [&](long long i) { return (int)min(max(i, 0ll), (long long)it.q.count) * s.G - it.row0; };      // rows of those before i
  return {max(queries((long long)t + 1 - it.q.end_min), 0), min(queries(last_seen - it.q.end_min + 1), it.rows)};
}
// and the outputs.
__device__ __forceinline__ float4 with_nan(float4 v, uint32_t bits) {
  const float nan = __uint_as_float(0x7fffffffu);
  if (bits & 1u) v.x = nan;
  if (bits & 2u) v.y = nan;
  if (bits & 4u) v.z = nan;
  if (bits & 8u) v.w = nan;
  return v;
}

// The largest weight times scale of V, log 2, of the n keys from c on that a row sees: scores at ts, factors ks, the scales' logarithms behind
// them.  (Not inlined: the loop around it is short.)
__device__ __noinline__ float heaviest(uint32_t ts, const float *ks, int c, int n, const Seen seen, float ref, float steep) {
  float most[2] = {-INFINITY, -INFINITY};
  const F2 ref2 = f2(-ref, -ref), steep2 = f2(steep, steep);
#pragma unroll 1
  for (const int end = c + n; c < end; c += 16) {
    uint32_t z[16];
    tmem_ld16(ts + c, z);
    tmem_wait_ld();
    const uint32_t bits = seen.bits(c);
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const float4 k = *reinterpret_cast<const float4 *>(ks + c + i);
      const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(ks + 256 + c + i);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const F2 y = f2(__fmul_rn(__uint_as_float(z[i + 2 * h]), h ? k.z : k.x), __fmul_rn(__uint_as_float(z[i + 2 * h + 1]), h ? k.w : k.y));
        const float2 w = f2_get(fma2(add2(y, ref2), steep2, h ? v.y : v.x));
        most[h] = fmax3(most[h], (bits >> (i + 2 * h)) & 1 ? w.x : -INFINITY, (bits >> (i + 2 * h + 1)) & 1 ? w.y : -INFINITY);
      }
    }
  }
  return fmaxf(most[0], most[1]);
}

template <int D, bool kPair, int kCopies>
__global__ void __launch_bounds__(kThreads, 1) attn_paged8_tc_kernel(const __grid_constant__ Args8 a) {
  using G = Geo<D, kPair>;
  using T = __nv_bfloat16;
  using W = Weights8<true>;
  static_assert(!kPair || kCopies == 1, "");
  constexpr int kPad = 128 / kCopies, kMine = kKeys / kCopies;      // rows of a copy, keys that it weighs
  extern __shared__ uint8_t smem_raw[];
  // (as an offset from the array: the accesses are then known to be to shared memory, and generic ones took twice as long here)
  uint8_t *smem = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const ds_paged_params &p = a.p;
  constexpr int S = G::kSlots;
  const uint32_t bar_k_full = sbase + G::kOffBar, bar_k_empty = bar_k_full + 8 * S, bar_v_full = bar_k_empty + 8 * S, bar_v_empty = bar_v_full + 8 * S,
                 bar_v16_full = bar_v_empty + 8 * S, bar_v16_free = bar_v16_full + 16, bar_sc_ready = bar_v16_free + 16,
                 bar_sc_free = bar_sc_ready + 8 * kScaleRing, bar_s_full = bar_sc_free + 8 * kScaleRing, bar_p_full = bar_s_full + 16,
                 bar_pv_done = bar_p_full + 16, bar_o_free = bar_pv_done + 16, bar_q_full = bar_o_free + 16, bar_q_free = bar_q_full + 8,
                 bar_meet = bar_q_free + 8, bar_joined = bar_meet + 8, bar_begun = bar_joined + 8;
  volatile uint32_t *tmem_s = reinterpret_cast<volatile uint32_t *>(smem + G::kOffMisc), *gave_up = tmem_s + 1;
  volatile int *v_nan = reinterpret_cast<volatile int *>(smem + G::kOffMisc + 8);      // the last piece, from 1 on, in which kOffNan has something
  // of the largest finite scale of V of a tile, its biased exponent, rounded up; of the smallest, rounded down, times 256; kPartial: not every
  // row sees every key; kMixed: that, or some scale is below an eighth of the largest
  volatile uint32_t *vsize_s = reinterpret_cast<volatile uint32_t *>(smem + G::kOffMisc + 12);
  constexpr uint32_t kPartial = 1u << 16, kMixed = 1u << 17;
  constexpr float kShort = 3.f;      // the largest weight of a row is not to stand below 2^kShort
  float *scale_s = reinterpret_cast<float *>(smem + G::kOffScale);
  float *factor_s = reinterpret_cast<float *>(smem + G::kOffFactor);

  if (tid == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(bar_k_full + 8 * s, 32);
      mbar_init(bar_k_empty + 8 * s, kPair ? 2 : 1);
      mbar_init(bar_v_full + 8 * s, 32);
      mbar_init(bar_v_empty + 8 * s, kConvertWarps);
    }
    for (int s = 0; s < kScaleRing; ++s) {
      mbar_init(bar_sc_ready + 8 * s, 1);
      mbar_init(bar_sc_free + 8 * s, kPair ? kSoftmaxWarps : kSoftmaxWarps / 2);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar_v16_full + 8 * s, kConvertWarps);
      mbar_init(bar_v16_free + 8 * s, kPair ? 2 : 1);
      mbar_init(bar_s_full + 8 * s, 1);
      mbar_init(bar_p_full + 8 * s, kSoftmaxWarps / 2);
      mbar_init(bar_pv_done + 8 * s, 1);
      mbar_init(bar_o_free + 8 * s, kSoftmaxWarps / 2);
    }
    mbar_init(bar_q_full, kConvertWarps);
    mbar_init(bar_q_free, 2 + kSoftmaxWarps);
    mbar_init(bar_meet, kSoftmaxWarps);
    mbar_init(bar_joined, kSoftmaxWarps);
    mbar_init(bar_begun, kSoftmaxWarps / 2);
    *v_nan = 0, *gave_up = 0;
    fence_barrier_init();
  }
  uint32_t *nan_s = reinterpret_cast<uint32_t *>(smem + G::kOffNan);
  for (int i = tid; i < G::kRows * D / 32; i += kThreads) nan_s[i] = 0;
  if (warp == kMmaWarp) tmem_alloc(sbase + G::kOffMisc, kTmemCols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_s;
  dependent_sync();
  uint32_t flags = 0;
  Walk walk;
  walk.find<kThreads>(a, a.split ? kMinTiles : 1, reinterpret_cast<long long *>(smem + G::kOffScan), flags);
  const Item &it = walk.it;
  bool ok = true;
  // Every wait is the whole warp's.
  auto wait = [&](uint32_t bar, int phase) {
    const bool there = __all_sync(0xffffffffu, wait_parity(bar, phase & 1, sbase + G::kOffMisc + 4));
    if (!there) *gave_up = kSpinLimit;
    return there;
  };

  if (warp >= kConvertWarp) {
    // ============================ queries, V to fp16 ============================
    const int cw = warp - kConvertWarp, cid = tid - 32 * kConvertWarp;
    int g = 0;      // key tiles of the pieces before
    for (int k = 0; ok && walk.piece(a); g += walk.n_tiles, walk.next(a), ++k) {
      // ---- the queries, once the products and the factors of the piece before are done with; four threads a row
      if (k > 0) ok = wait(bar_q_free, k - 1);
      if (!ok) break;
      {
        constexpr int E = D / 4, kLoads = E / 8;      // elements of a thread, 16 bytes at a time
        const int u = cid & 3;
        const int r_end = (it.rows + 7) / 8 * 8;      // whole warps
        uint4 next[kLoads];
        auto load = [&](int r) {
          const Row row = row_of(a, it, r < it.rows ? r : 0);
          const T *src = reinterpret_cast<const T *>(p.q) + row.n * p.q_stride[0] + row.h * p.q_stride[1] + E * u;
#pragma unroll
          for (int i = 0; i < kLoads; ++i) next[i] = *reinterpret_cast<const uint4 *>(src + 8 * i);
        };
        if ((cid >> 2) < r_end) load(cid >> 2);
#pragma unroll 1
        for (int r = cid >> 2; r < r_end; r += 8 * kConvertWarps) {
          uint4 w[kLoads];
          const bool there = r < it.rows;
#pragma unroll
          for (int i = 0; i < kLoads; ++i) w[i] = next[i];
          if (r + 8 * kConvertWarps < r_end) load(r + 8 * kConvertWarps);
          const QueryScale q = query_scale<kLoads>(w, p.scale);
          if (there && u == 0) factor_s[r] = q.factor;
#pragma unroll
          for (int i = 0; i < kLoads; i += 2) {
            uint32_t hi[4], lo[4];
            query_parts(w + i, q.up, hi, lo);
            if (there) {
#pragma unroll
              for (int c = 0; c < kCopies; ++c) {
                uint8_t *to = smem + row_at<D>(c * kPad + r, u * (E / 16) + i / 2);
                *reinterpret_cast<uint4 *>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4 *>(to + G::kQPart) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
              }
            }
          }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_q_full);
      }
      if (!kPair && k > 0) ok = wait(bar_joined, k - 1);      // the sums of the piece before, which lie in the tiles' place
      // ---- V, tile by tile
      for (int i = 0; ok && i < walk.n_tiles; ++i) {
        const int t = g + i;
        ok = wait(bar_v_full + 8 * (t % S), t / S);
        if (!ok) break;
        if (cw == 0) {
          // the scales as the products take them, and how large V's are
          float *vs = scale_s + (t % kScaleRing) * 384 + 128 + lane;
          const bool partial = !paged_all_visible(a.s, it.q, (walk.tile0 + i) * kKeys, kKeys);
          uint32_t most = 0, least = 0x7fffffffu;
          float size[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const float v = vs[32 * c];
            const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
            most = max(most, b < 0x7f800000u ? b : 0u);
            if (!partial || paged_key(it.q, (walk.tile0 + i) * kKeys + 32 * c + lane) >= 0) least = min(least, b);
            size[c] = v;
            vs[32 * c] = v * kUnbiased, vs[32 * c - 128] *= 0x1p-24f;      // a product of queries and K is below 2^24
          }
          most = (__reduce_max_sync(0xffffffffu, most) + 0x7fffffu) >> 23, least = __reduce_min_sync(0xffffffffu, least) >> 23;
          const bool mixed = least + 3 < most || partial;
          if (mixed)
            for (int c = 0; c < 4; ++c) vs[32 * c + 128] = log_scale(size[c]);
          if (lane == 0) vsize_s[t % kScaleRing] = most | least << 8 | (partial ? kPartial : 0u) | (mixed ? kMixed : 0u);
          __syncwarp();
          if (lane == 0) mbar_arrive(bar_sc_ready + 8 * (t % kScaleRing));
        }
        ok = wait(bar_v16_free + 8 * (t & 1), t / 2 + 1);
        if (!ok) break;
        const uint8_t *from = smem + G::kOffV + (t % S) * G::kTile;
        uint8_t *to = smem + G::kOffV16 + (t & 1) * (2 * G::kTile);
        // eight rows side by side, four chunks of each; rows r and r ^ 5 next to each other meet no bank twice, in either layout
        constexpr int kOps = D / 16;
        const int r8 = 32 * cw + ((lane >> 3) ^ (lane & 4 ? 5 : 0)), c4 = lane & 3;
#pragma unroll 2
        for (int o = 0; o < kOps; ++o) {
          const int r = r8 + 8 * (o & 3), c = c4 + 4 * (o >> 2);
          const uint4 w = *reinterpret_cast<const uint4 *>(from + row_at<D>(r, c));
          *reinterpret_cast<uint4 *>(to + half_at(r, 2 * c)) = make_uint4(halves_lo(w.x), halves_hi(w.x), halves_lo(w.y), halves_hi(w.y));
          *reinterpret_cast<uint4 *>(to + half_at(r, 2 * c + 1)) = make_uint4(halves_lo(w.z), halves_hi(w.z), halves_lo(w.w), halves_hi(w.w));
        }
        if (!paged_all_visible(a.s, it.q, (walk.tile0 + i) * kKeys, kKeys)) {
          // Keys that some rows see and others do not: a weight of zero times NaN would be NaN.  NaN becomes zero here, and the outputs of
          // the rows that see it are noted.  (Where every row sees every key, the product does what it should.)
          bool nan = false;
#pragma unroll 1
          for (int o = 0; o < kOps; ++o) {
            const int r = r8 + 8 * (o & 3), c = c4 + 4 * (o >> 2);
            const uint4 w = *reinterpret_cast<const uint4 *>(from + row_at<D>(r, c));
            const uint32_t x = (((w.x & 0x7f7f7f7fu) + 0x01010101u) | ((w.y & 0x7f7f7f7fu) + 0x01010101u) | ((w.z & 0x7f7f7f7fu) + 0x01010101u) |
                                ((w.w & 0x7f7f7f7fu) + 0x01010101u)) & 0x80808080u;
            if (x == 0) continue;
            nan = true;
#pragma unroll 1
            for (int e = 0; e < 8; ++e) {
              uint32_t *h = reinterpret_cast<uint32_t *>(to + half_at(r, 2 * c + e / 4)) + (e & 3);
              const uint32_t v = *h;
              *h = v & ~(((v & 0x7c00u) == 0x7c00u ? 0xffffu : 0u) | ((v & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u));
            }
          }
          if (__any_sync(0xffffffffu, nan)) {
            if (k > 0) ok = wait(bar_o_free, k - 1) && wait(bar_o_free + 8, k - 1);      // the piece before is written out
            if (!ok) break;
#pragma unroll 1
            for (int o = 0; o < kOps; ++o) {
              const int r = r8 + 8 * (o & 3), c = c4 + 4 * (o >> 2);
              const uint32_t bits = nan_bits(*reinterpret_cast<const uint4 *>(from + row_at<D>(r, c)));
              if (bits == 0) continue;
              const RowRange rows = rows_that_see(a.s, it, paged_key(it.q, (walk.tile0 + i) * kKeys + r));
#pragma unroll 1
              for (int row = rows.lo; row < rows.hi; ++row) atomicOr(nan_s + row * (D / 32) + c / 2, bits << (16 * (c & 1)));
            }
            *v_nan = k + 1;
            __syncwarp();
          }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar_v16_full + 8 * (t & 1));
          mbar_arrive(bar_v_empty + 8 * (t % S));
        }
      }
    }
  } else if (warp >= kMmaWarp) {
   if (warp >= kLoadWarp) {
    // ============================ K, V, scales ============================
    constexpr int kChunks = D / 16, kPer = 32 / kChunks, kOps = 16 / kPer;      // chunks of a row, rows of an instruction
    const int lw = warp - kLoadWarp, ch = lane % kChunks;
    const long long row_bytes = p.cache_stride[2];
    int g = 0;      // key tiles of the pieces before
    for (; ok && walk.piece(a); g += walk.n_tiles, walk.next(a)) {
      const int32_t *table = p.block_table + it.b * p.table_stride;
      const uint8_t *kbase = reinterpret_cast<const uint8_t *>(p.k_cache) + it.g * p.cache_stride[1];
      const uint8_t *vbase = reinterpret_cast<const uint8_t *>(p.v_cache) + it.g * p.cache_stride[1];
      const float *kscale = a.k_scale + it.g * a.scale_stride[1], *vscale = a.v_scale + it.g * a.scale_stride[1];
      int i = (lw ^ g) & 1;      // this warp's first tile of the piece
      int pos[4], page[4];               // of keys lane + 32 j
      auto look_up = [&]() {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          pos[j] = i < walk.n_tiles ? paged_key(it.q, (walk.tile0 + i) * kKeys + 32 * j + lane) : -1;
          page[j] = pos[j] >= 0 ? table[fast_div(pos[j], a.page_div)] : 0;
        }
      };
      look_up();
      for (; i < walk.n_tiles; i += kLoadWarps) {
        const int t = g + i, slot_of_t = t % S;
        // Code that runs for every tile is kept short: five roles share the instruction caches, and with all loops of these copies
        // unrolled (24 KB) every role waited for its instructions (123 us, 93 with short loops).
        long long at[4], scale_at[4];
        uint32_t even = 0;      // bit 2 j + half: 16 keys that lie evenly (in one page) need one address
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          at[j] = -1, scale_at[j] = -1;
          if (pos[j] >= 0) {
            const int there = paged_clamp_page(page[j], p.n_pages);
            if (there != page[j]) flags |= DS_DEV_INDEX;
            const int slot = pos[j] - fast_div(pos[j], a.page_div) * p.page_size;
            at[j] = there * p.cache_stride[0] + slot * row_bytes;
            scale_at[j] = there * a.scale_stride[0] + fast_div(slot, a.scale_div) * a.scale_stride[2];
          }
          const long long first = __shfl_sync(0xffffffffu, at[j], lane & 16);
          const uint32_t b = __ballot_sync(0xffffffffu, at[j] >= 0 && at[j] == first + (lane & 15) * row_bytes);
          even |= ((b & 0xffffu) == 0xffffu ? 1u : 0u) << (2 * j) | (b >> 16 == 0xffffu ? 2u : 0u) << (2 * j);
        }
#pragma unroll 1
        for (int v = 0; ok && v < 2; ++v) {
          ok = wait((v ? bar_v_empty : bar_k_empty) + 8 * slot_of_t, t / S + 1);
          if (!ok) break;
          const uint8_t *base = (v ? vbase : kbase) + 16 * ch;
          const uint32_t dst = sbase + (v ? G::kOffV : G::kOffK) + slot_of_t * G::kTile;
#pragma unroll 1
          for (int jh = 0; jh < 8; ++jh) {
            const long long mine = jh < 4 ? (jh < 2 ? at[0] : at[1]) : jh < 6 ? at[2] : at[3];
            const int r0 = 16 * jh + lane / kChunks, src = 16 * (jh & 1);
            if ((even >> jh) & 1) {
              const uint8_t *from = base + __shfl_sync(0xffffffffu, mine, src) + (lane / kChunks) * row_bytes;
#pragma unroll
              for (int o = 0; o < kOps; ++o, from += kPer * row_bytes) cp_async16(dst + row_at<D>(r0 + o * kPer, ch), from, true);
            } else {
#pragma unroll
              for (int o = 0; o < kOps; ++o) {
                const long long off = __shfl_sync(0xffffffffu, mine, src + o * kPer + lane / kChunks);
                cp_async16(dst + row_at<D>(r0 + o * kPer, ch), base + (off >= 0 ? off : 0), off >= 0);
              }
            }
          }
          arrive_when_copied((v ? bar_v_full : bar_k_full) + 8 * slot_of_t);
          if (v == 0) {
            ok = wait(bar_sc_free + 8 * (t % kScaleRing), t / kScaleRing + 1);
            if (!ok) break;
            const uint32_t sc = sbase + G::kOffScale + (t % kScaleRing) * 1536 + 4 * lane;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              cp_async4(sc + 128 * j, kscale + (scale_at[j] >= 0 ? scale_at[j] : 0), scale_at[j] >= 0);
              cp_async4(sc + 512 + 128 * j, vscale + (scale_at[j] >= 0 ? scale_at[j] : 0), scale_at[j] >= 0);
            }
          }
        }
        i += kLoadWarps;
        look_up();      // of this warp's next tile
        i -= kLoadWarps;
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
   } else {
    // ============================ products, a warp for each stream ============================
    const int s = warp - kMmaWarp;
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), ts = tm + kTmemS + s * 128, to = tm + kTmemO + s * 128;
    const uint64_t dq = rows_desc(sbase + (kPair ? s * 128 * D : 0), D), dk0 = rows_desc(sbase + G::kOffK, D), dv0 = smem_desc(sbase + G::kOffV16, kHalfBytes, 1024);
    int g = 0, n = 0;      // key tiles of the pieces before; steps of this stream
    for (int k = 0; ok && walk.piece(a); g += walk.n_tiles, walk.next(a), ++k) {
      const int steps = kPair ? 2 * walk.n_tiles : walk.n_tiles;
      ok = wait(bar_q_full, k);
      if (s >= steps && lane == 0) mbar_arrive(bar_q_free);      // nothing for this stream
      // Half a step apart: the exponentials of one stream beside the products of the other.  (In step, they wait for each other's pipes.)
      // bar_begun, a phase a piece, as the first stream's steps may pass two while this warp waits for one: the next piece's phase needs its
      // bar_q_free, which this warp's last product arrives at.
      if (ok && s == 1 && s < steps) ok = wait(bar_begun, k);
#pragma unroll 1
      for (int u = s - 2; ok && u < steps; u += 2) {
        if (u >= 0) {
          const int t = g + (kPair ? u >> 1 : u);
          ok = wait(bar_p_full + 8 * s, n) && wait(bar_v16_full + 8 * (t & 1), t / 2);
          if (ok && u < 2 && k > 0) ok = wait(bar_o_free + 8 * s, k - 1);
          if (!ok) break;
          ++n;
          tc_fence_after();
          if (elect_one()) {
            uint64_t dv = dv0 + (uint64_t)(((t & 1) * 2 * G::kTile) >> 4);
#pragma unroll 4
            for (int ks = 0; ks < kKeys / 16; ++ks, dv += 2048 >> 4) umma_ts(to, ts + ks * 8, dv, idesc16(D), u >= 2 || ks > 0);
            umma_commit(bar_v16_free + 8 * (t & 1));
            umma_commit(bar_pv_done + 8 * s);
          }
          __syncwarp();
        }
        if (u + 2 < steps) {
          const int t = g + (kPair ? (u + 2) >> 1 : u + 2);
          ok = wait(bar_k_full + 8 * (t % S), t / S) && (u < 0 || wait(bar_pv_done + 8 * s, n - 1));
          if (!ok) break;
          fence_proxy_async();
          tc_fence_after();
          if (elect_one()) {
            const uint64_t dk = dk0 + (uint64_t)(((t % S) * G::kTile) >> 4);
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
              for (int ks = 0; ks < D / 32; ++ks)
                umma_ss8(ts, dq + ((part * G::kQPart + ks * 32) >> 4), dk + ((ks * 32) >> 4), idesc8(kKeys, part == 1), part > 0 || ks > 0);
            umma_commit(bar_s_full + 8 * s);
            umma_commit(bar_k_empty + 8 * (t % S));
            if (u + 4 >= steps) umma_commit(bar_q_free);
          }
          __syncwarp();
        }
      }
    }
   }
  } else {
    // ============================ softmax and epilogue ============================
    const int s = warp >> 2, tr = tid & 127;      // stream, tile row
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t ts = tmem + lanes + kTmemS + s * 128, to = tmem + lanes + kTmemO + s * 128;
    const int copy = tr / kPad, key0 = copy * kMine, r = kPair ? tid : tr % kPad;      // row of the item
    PagedJoin join = {0, 0, 0, 0, 0, 0};      // thread 0's
    int g = 0, n = 0, meets = 0;      // key tiles of the pieces before, steps of this stream
    for (int k = 0; ok && walk.piece(a); g += walk.n_tiles, walk.next(a), ++k) {
      if (a.split && tid == 0) walk.note_join(join);
      const bool mine = r < it.rows, busy = (kPair ? 32 * warp : (32 * (warp & 3)) % kPad) < it.rows;
      const Row row = row_of(a, it, mine ? r : 0);
      const int end = mine ? row.end : 0;
      ok = wait(bar_q_full, k);
      if (!ok) break;
      const float steep = mine ? fminf(factor_s[r] * 0x1p24f, 0x1p126f) : 1.f;      // K's scales are 2^-24 of themselves
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_q_free);
      float m = -INFINITY, l = 0.f;      // m: the largest score before its factor
      float e = 0.f;                     // of the row's weights
      const int steps = kPair ? 2 * walk.n_tiles : walk.n_tiles;
      int done = 0;
      for (int u = s; u < steps; u += 2, ++n, ++done) {
        const int i = kPair ? u >> 1 : u, t = g + i, x = (walk.tile0 + i) * kKeys;
        const bool all = paged_all_visible(a.s, it.q, x, kKeys);
        ok = wait(bar_sc_ready + 8 * (t % kScaleRing), t / kScaleRing) && wait(bar_s_full + 8 * s, n);
        if (!ok) break;
        tc_fence_after();
        if (busy) {
          const float *ks = scale_s + (t % kScaleRing) * 384, *vs = ks + 128;
          const Seen seen = seen_keys(a.s, it.q, x, end);
          // ---- largest score of this copy's keys, 16 at a time in a short loop
          float top = -INFINITY, top1 = -INFINITY;
          uint32_t z[16];
          float y[16];
          auto scores = [&](int c) {      // rounded before the reference is taken off: equal keys stay equal
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const float4 f = *reinterpret_cast<const float4 *>(ks + c + i);
              y[i] = __fmul_rn(__uint_as_float(z[i]), f.x), y[i + 1] = __fmul_rn(__uint_as_float(z[i + 1]), f.y);
              y[i + 2] = __fmul_rn(__uint_as_float(z[i + 2]), f.z), y[i + 3] = __fmul_rn(__uint_as_float(z[i + 3]), f.w);
            }
          };
          auto hide = [&](int c, float what) {
            const uint32_t bits = seen.bits(c);
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = (bits >> e) & 1 ? y[e] : what;
          };
#pragma unroll 1
          for (int c = key0; c < key0 + kMine; c += 16) {
            tmem_ld16(ts + c, z);
            tmem_wait_ld();
            scores(c);
            if (!all) hide(c, -INFINITY);
#pragma unroll
            for (int e = 0; e < 16; e += 4) top = fmax3(top, y[e], y[e + 1]), top1 = fmax3(top1, y[e + 2], y[e + 3]);
          }
          top = fmaxf(top, top1);
          // The references of the row's scores and weights move only when one would pass its limit, and O with them: rarely.
          const uint32_t size = vsize_s[t % kScaleRing];
          const float v_most = (float)((int)(size & 255u) - 127), v_least = (float)((int)(size >> 8 & 255u) - 127);
          const bool first = m == -INFINITY;
          const float rise = (top - m) * steep;
          // the reference of the scores moves with the largest weight, too, where that is the row's own whatever the key
          const float now = mine && (first ? top > m : rise > W::kLag || (!(size & kPartial) && rise > 0.f && rise + (e + v_most) > W::kTop)) ? top : m;
          const float start = first ? W::kMost : e;
          // the largest weight: at most this, with the tile's largest scale, whoever sees it
          float most = mine ? (top - now) * steep + (start + v_most) : -INFINITY;
          const bool over = now != m || most > W::kTop;
          if (__any_sync(0xffffffffu, over)) {
            // Where that and the smallest scale do not settle it, and the tile is mixed, the row's own keys are gone through.
            const bool settled = !(most > W::kTop) && (now == m || (!first && e + v_least >= kShort));
            if ((size & kMixed) && __any_sync(0xffffffffu, !settled)) {
              const float exact = start + heaviest(ts, ks, key0, kMine, seen, now, steep);
              if (!settled) most = exact;
            }
            const float fall = now == m ? 0.f : first ? -INFINITY : (m - now) * steep;      // of sums under an unchanged e
            float fresh = e;
            if (most > W::kTop || (now != m && (first || most < kShort)))
              fresh = fmaxf(floorf(fminf(start + (W::kLog2 - most), fminf(e - fall, W::kMost))), W::kLeast);
            if (now != m) l *= ex2_approx(fall);
            const float keep = ex2_approx(fall + (fresh - e));
            m = now, e = fresh;
            if (done > 0 && __any_sync(0xffffffffu, keep != 1.f)) {
              ok = wait(bar_pv_done + 8 * s, n - 1);
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                tmem_ld16(to + c, z);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] = __float_as_uint(__uint_as_float(z[i]) * keep);
                tmem_st16(to + c, z);
              }
            }
          }
          // ---- weights
          const float ref = m == -INFINITY ? 0.f : m;      // nothing seen yet: exp(-inf) = 0
          const F2 ref2 = f2(-ref, -ref), steep2 = f2(steep, steep);
          const float up = power_of_two(e + W::kBias);
          const F2 up2 = f2(up, up);
          F2 l2[2] = {0, 0};
#pragma unroll 1
          for (int c = key0; c < key0 + kMine; c += 16) {
            tmem_ld16(ts + c, z);
            tmem_wait_ld();
            scores(c);
            if (!all) hide(c, -INFINITY);
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              const ulonglong2 v = *reinterpret_cast<const ulonglong2 *>(vs + c + e);
#pragma unroll
              for (int h = 0; h < 4; h += 2) {
                float2 q = f2_get(mul2(add2(f2(y[e + h], y[e + h + 1]), ref2), steep2));
                q.x = ex2_approx(q.x), q.y = ex2_approx(q.y);
                const F2 weight = f2(q.x, q.y);
                l2[h / 2] = add2(l2[h / 2], weight);
                const float2 b = f2_get(mul2(mul2(weight, up2), h ? v.y : v.x));
                y[e + h] = b.x, y[e + h + 1] = b.y;
              }
            }
            if (!all) hide(c, 0.f);      // zero times a scale that is not finite
            uint32_t w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = pack_half(y[2 * e], y[2 * e + 1]);
            // over scores that have been read, or are another copy's: columns c / 2 .. c / 2 + 7 <= c + 15
            tmem_st8(ts + c / 2, w);
          }
          const float2 sum2 = f2_get(add2(l2[0], l2[1]));
          l += sum2.x + sum2.y;
          if constexpr (kCopies > 1) {      // no weight for the other copies' keys
            uint32_t z[16] = {};
#pragma unroll
            for (int c = 0; c < kKeys / 2; c += 16)
              if (c < key0 / 2 || c >= (key0 + kMine) / 2) tmem_st16(ts + c, z);
          }
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar_p_full + 8 * s);
          if (u == 0) mbar_arrive(bar_begun);
          mbar_arrive(bar_sc_free + 8 * (t % kScaleRing));
        }
      }
      if (!ok) break;
      // ---- the piece is done
      if (m != -INFINITY) m *= steep;
      if (done > 0) {
        ok = wait(bar_pv_done + 8 * s, n - 1);
        if (!ok) break;
        tc_fence_after();
      }
      const bool whole = walk.whole();
      const long long slot = (long long)paged_slot(blockIdx.x, walk.first) * a.part_rows;
      const float down = power_of_two(-e);
      // O times this, and down, is a share of the output, or of the part's sums: over the sum of weights or shrunk
      auto share = [&](float sum) { return whole ? (sum == 0.f ? 0.f : 1.f / sum) : a.shrink; };
      bool nan = false;      // known when the stream's products are done (all of the piece, where a row has two): their tiles have been looked through
      auto finish_row = [&](const Row &row, int r, float top, float sum) {
        if (!whole) a.part_ml[slot + r] = make_float2(top, sum);
        else if (p.lse) p.lse[row.n * p.Hq + row.h] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
      };
      constexpr int J = G::kOutDims, kQuads = J / 4;
      auto quad = [&](int i, int q) { return reinterpret_cast<float4 *>(smem + G::kOffOut + i * (4 * J)) + (q ^ (kQuads == 4 ? (i >> 1) & 3 : i & 7)); };
      auto meet = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_meet);
        ok = wait(bar_meet, meets++);
      };
      // O times `by` of dimensions c .. to shared memory
      auto put_down = [&](int c, float by) {
#pragma unroll 1
        for (int c2 = 0; c2 < J; c2 += 16) {
          uint32_t o[16];
          tmem_ld16(to + c + c2, o);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            *quad(tid, (c2 + e) / 4) = make_float4(__uint_as_float(o[e]) * by, __uint_as_float(o[e + 1]) * by, __uint_as_float(o[e + 2]) * by,
                                                  __uint_as_float(o[e + 3]) * by);
        }
      };
      // Where the elements of a row go: looked up, as working it out for every four of them was half of the epilogue.
      long long *to_s = reinterpret_cast<long long *>(smem + G::kOffTo);
      if (mine && (kPair || (s == 0 && copy == 0)))      // (the piece before is written out: its sums were, before this one's products)
        to_s[r] = whole ? row.n * p.out_stride[0] + row.h * p.out_stride[1] : (slot + r) * D;
      auto put_out = [&](int r, int d, float4 v) {
        if (__builtin_expect(nan, 0)) v = with_nan(v, nan_s[r * (D / 32) + d / 32] >> (d & 31));
        if (whole) store4(reinterpret_cast<T *>(p.out) + to_s[r] + d, v);
        else *reinterpret_cast<float4 *>(a.part_o + to_s[r] + d) = v;
      };
      if constexpr (kPair) {
        // rows are a warp's own; through shared memory, so that neighbouring lanes write neighbouring elements (a row to a thread took 8000
        // cycles)
        nan = *v_nan == k + 1;
        if (busy) {
          const float by = share(l) * down;
          if (mine) finish_row(row, r, m, l);
#pragma unroll 1
          for (int c = 0; c < D; c += J) {
            put_down(c, by);
            __syncwarp();
#pragma unroll 1
            for (int e = lane; e < 32 * kQuads; e += 128) {
              float4 v[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) v[j] = *quad(32 * warp + (e + 32 * j) / kQuads, e % kQuads);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int i = 32 * warp + (e + 32 * j) / kQuads;
                if (i < it.rows) put_out(i, c + 4 * (e % kQuads), v[j]);
              }
            }
            __syncwarp();
          }
          if (__builtin_expect(nan, 0)) {
            for (int i = 0; i < D / 32; ++i) nan_s[(32 * warp + lane) * (D / 32) + i] = 0;
          }
        }
      } else {
        // ---- join the streams and copies of a row: each brings its O to the row's reference and writes it down, and they are added up
        float2 *ml_s = reinterpret_cast<float2 *>(smem + G::kOffMl);
        ml_s[tid] = make_float2(m, l);
        meet();      // all products have been waited for, too: V's tiles are free
        if (!ok) break;
        nan = *v_nan == k + 1;
        const int rr = tr % kPad;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int j = 0; j < 2 * kCopies; ++j) top = fmaxf(top, ml_s[j * kPad + rr].x);
#pragma unroll
        for (int j = 0; j < 2 * kCopies; ++j) {
          const float2 ml = ml_s[j * kPad + rr];
          sum = fmaf(ml.y, ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top), sum);
        }
        const float by = (m == -INFINITY ? 0.f : ex2_approx(m - top)) * share(sum) * down;
        if (s == 0 && copy == 0 && mine) finish_row(row, r, top, sum);
#pragma unroll 1
        for (int c = 0; ok && c < D; c += J) {
          if (busy && done > 0) {
            put_down(c, by);
          } else if (busy) {      // a stream without a tile has nothing in O
#pragma unroll 1
            for (int q = 0; q < kQuads; ++q) *quad(tid, q) = make_float4(0.f, 0.f, 0.f, 0.f);
          }
          meet();
          if (!ok) break;
#pragma unroll 1
          for (int e = tid; e < it.rows * kQuads; e += 32 * kSoftmaxWarps) {
            const int i = e / kQuads, q = e % kQuads;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int j = 0; j < 2 * kCopies; ++j) {
              const float4 o = *quad(j * kPad + i, q);
              v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
            }
            put_out(i, c + 4 * q, v);
          }
          if (c + J < D) meet();      // the buffer is read
        }
        if (!ok) break;
        if (__builtin_expect(nan, 0)) {
          meet();      // every row is written
          if (!ok) break;
          for (int i = tid; i < G::kRows * D / 32; i += 32 * kSoftmaxWarps) nan_s[i] = 0;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_joined);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_o_free + 8 * s);
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

long long rows_per_head(const ds_paged_params &p) { return (long long)p.max_q * (p.Hq / p.Hkv); }
int tile_rows(const ds_paged_params &p) {
  const long long rows = rows_per_head(p);
  return rows <= 64 ? 64 : rows <= 128 ? 128 : 256;      // (fewer than 33 are the other kernel's)
}
Shape shape_for(const ds_paged_params &p) {
  const int rows = tile_rows(p);
  return shape_of(p, kKeys, rows, longest_of(units_of(p, kKeys, rows)).tiles <= kWholeTiles ? 1 : kMinTiles, 1);
}

template <int D, bool kPair, int kCopies>
int launch(const ds_paged8_params &p, cudaStream_t stream) {
  using G = Geo<D, kPair>;
  const Shape h = shape_for(p.a);
  const Args8 a = args8_of(p, h, workspace_of(h));
  static std::atomic<unsigned long long> allowed{0};
  DS_CUDA_OK(allow_smem(attn_paged8_tc_kernel<D, kPair, kCopies>, G::kBytes, allowed));
  DS_CUDA_OK(launch_kernel(attn_paged8_tc_kernel<D, kPair, kCopies>, dim3(h.grid), kThreads, G::kBytes, 0, false, stream, a));
  note_launch(1);
  return a.split ? launch_join<__nv_bfloat16, D>(a, h, stream) : (int)DS_OK;
}

template <int D>
int launch_rows_of(const ds_paged8_params &p, cudaStream_t stream) {
  switch (tile_rows(p.a)) {
    case 64: return launch<D, false, 2>(p, stream);
    case 128: return launch<D, false, 1>(p, stream);
    default: return launch<D, true, 1>(p, stream);
  }
}

}  // namespace

bool attn_paged8_tc_counts_fit(const ds_paged_params &p) {
  const PagedShape s = units_of(p, kKeys, tile_rows(p));
  return paged_units_fit(s, longest_of(s));
}

size_t attn_paged8_tc_workspace_bytes(const ds_paged_params &p) { return workspace_of(shape_for(p)); }

int launch_attn_paged8_tc(const ds_paged8_params &p, cudaStream_t stream) {
  return p.a.D == 64 ? launch_rows_of<64>(p, stream) : launch_rows_of<128>(p, stream);
}

}  // namespace ds

// ds_attn_paged: attention of the new rows of every sequence over its pages.
//
// With one or a few query rows per KV head this is a stream over the cache: every byte of K and V is used for
// G n_b rows at most, so the kernel is built to keep loads in flight.  The (sequence, KV head, row tile, key tile)
// units of the whole batch are laid end to end and cut into equal ranges, one per resident CTA, from the lengths on the
// device: uneven lengths cost nothing and one long sequence spreads over the whole GPU.  An item that crosses a range
// boundary leaves partial results (unnormalised sums with their maximum) in the workspace; a second, small
// kernel, launched early and waiting for the first, joins them in a fixed order.
// Few items of moderate length (a small batch) are instead given a CTA each, or a cluster of CTAs that join through
// distributed shared memory: no second launch, no workspace, no search for the range's first item.
//
// Inside a CTA the four warps take equal parts of every key tile and share nothing until the item ends: each has its own
// ring of cp.async stages in shared memory (16-byte chunks, XOR swizzle), its own running maximum, sum and output, so
// the loop has no CTA-wide barrier.  At the end of an item the four results are joined through shared memory.
//
// bf16: mma.sync m16n8k16.  The few rows leave tcgen05's 128-row tile nearly empty and the stream, not the products,
// bounds the kernel.  The weights enter the second product as two bf16
// halves (hi + lo), which keeps 16 bits of them: the product is free here, and an output is then rounded once.
// fp32: CUDA cores.
#include <cooperative_groups.h>

#include <type_traits>

#include "ds_attn_paged.cuh"

namespace ds {
namespace {

using namespace paged;

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
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Transposes an 8 x 8 matrix of 16-bit values, lane 4i + q holding columns 2q and 2q + 1 of row i.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// Byte offset of 16-byte chunk `c` of row `r` in a tile of rows of ROW bytes: chunks are XOR-ed with the row number
// within groups of eight, which makes ldmatrix and the float4 reads below free of bank conflicts.
template <int ROW>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) { return r * ROW + ((c ^ (r & 7)) << 4); }

// ---------------------------------------------------------------------------------------------------------------
// A warp's share of an item in bf16: NB blocks of 8 rows against 16 keys at a time, with the keys as the products' 16-wide
// side, S^T = K Q^T and O^T = V^T P^T, so that a block of 8 rows (a single token of most grouped-query models) costs
// half of what 16 rows would.  Lane 4i + q holds, of S^T, keys i and i + 8 of rows 2q and 2q + 1 of every block; movmatrix
// turns the weights into the second product's fragments.
template <int D_, int NB, int kStages_ = D_ == 128 && NB == 1 ? 2 : 3>
struct TensorRows {
  using T = __nv_bfloat16;
  static constexpr int D = D_, kRows = 8 * NB, kRowBytes = 2 * D, kKeys = 16;
  static constexpr bool kQRegs = NB <= 2;      // more rows read their queries' fragments from shared memory
  static constexpr int kQBytes = kQRegs ? 0 : kRows * kRowBytes;
  // CTAs per SM and stages of a ring: what registers and shared memory hold.  For one block of rows three CTAs with two
  // stages beat two with three (32 x 32 heads x 4128 rows, D = 128: 316 against 330 us).
  static constexpr int kCtas = D == 64 && NB == 1 ? 4 : NB == 1 || (D == 64 && NB == 2) ? 3 : 2, kStages = kStages_;
  float o[NB][D / 16][4];        // dimensions 16 j + lane / 4 (+ 8), rows 2q, 2q + 1
  float m[NB][2], l[NB][2];
  int end[NB][2];
  uint32_t qf[kQRegs ? NB : 1][kQRegs ? D / 16 : 1][2];
  uint32_t q_smem;

  __device__ void begin(const Params &a, const Item &it, uint8_t *q_buf) {
    const int lane = threadIdx.x & 31;
    q_smem = sm100::smem_u32(q_buf);
    const T *q = reinterpret_cast<const T *>(a.p.q);
    if constexpr (kQRegs) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int r = 8 * nb + (lane >> 2);
        const bool there = r < it.rows;
        const Row row = row_of(a, it, there ? r : 0);
        const T *src = q + row.n * a.p.q_stride[0] + row.h * a.p.q_stride[1] + (lane & 3) * 2;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            qf[nb][k][h] = there ? *reinterpret_cast<const uint32_t *>(src + 16 * k + 8 * h) : 0u;
      }
    } else {
      for (int c = threadIdx.x; c < kRows * (kRowBytes / 16); c += kThreads) {
        const int r = c / (kRowBytes / 16), ch = c % (kRowBytes / 16);
        uint4 w = make_uint4(0, 0, 0, 0);
        if (r < it.rows) {
          const Row row = row_of(a, it, r);
          w = *reinterpret_cast<const uint4 *>(q + row.n * a.p.q_stride[0] + row.h * a.p.q_stride[1] + 8 * ch);
        }
        *reinterpret_cast<uint4 *>(q_buf + chunk_at<kRowBytes>(r, ch)) = w;
      }
      __syncthreads();
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nb][j][e] = 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[nb][e] = -INFINITY, l[nb][e] = 0.f;
        const int r = 8 * nb + 2 * (lane & 3) + e;
        end[nb][e] = r < it.rows ? row_of(a, it, r).end : 0;
      }
    }
  }

  // 16 keys from x on; K and V as loaded, V is scratch afterwards.
  __device__ __forceinline__ void step(const Params &a, const Item &it, uint8_t *kbuf, uint8_t *vbuf, int x, float scale2) {
    const int lane = threadIdx.x & 31;
    const uint32_t ks = sm100::smem_u32(kbuf), vs = sm100::smem_u32(vbuf);
    // even and odd 16s of the dimensions in accumulators of their own, all fragments of K first
    float s[NB][4], odd[NB][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nb][e] = odd[nb][e] = 0.f;
    {
      uint32_t kf[D / 16][4];
#pragma unroll
      for (int k = 0; k < D / 16; ++k) ldmatrix4(ks + chunk_at<kRowBytes>(lane & 15, 2 * k + (lane >> 4)), kf[k]);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        if constexpr (kQRegs) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma16816(k & 1 ? odd[nb] : s[nb], kf[k], qf[nb][k][0], qf[nb][k][1]);
        } else {
#pragma unroll
          for (int nb = 0; nb < NB; nb += 2) {
            uint32_t bf[4];      // rows 8 nb .. + 7: two halves of the 16 dimensions, then the next block's
            ldmatrix4(q_smem + chunk_at<kRowBytes>(8 * nb + (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)), bf);
            mma16816(k & 1 ? odd[nb] : s[nb], kf[k], bf[0], bf[1]);
            mma16816(k & 1 ? odd[nb + 1] : s[nb + 1], kf[k], bf[2], bf[3]);
          }
        }
      }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[nb][e] = __fmul_rn(s[nb][e] + odd[nb][e], scale2);      // not to be fused with the subtraction
    const bool partial = !paged_all_visible(a.s, it.q, x, kKeys);
    uint32_t seen[NB] = {};      // only with partial: bit 2h + e: key lane / 4 + 8h, row 2q + e
    if (partial) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int pos = paged_key(it.q, x + 8 * h + (lane >> 2));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (paged_visible(a.s, pos, end[nb][e])) seen[nb] |= 1u << (2 * h + e);
            else s[nb][2 * h + e] = -INFINITY;
          }
      }
    }
    // The reference of the exponents moves only when a weight would pass 2^8 (the result is the same): no maximum is
    // exchanged until some lane finds such a score.
    bool over = false;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) over |= fmaxf(s[nb][e], s[nb][2 + e]) > m[nb][e] + 8.f;
    if (__any_sync(0xffffffffu, over)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = fmaxf(m[nb][e], fmaxf(s[nb][e], s[nb][2 + e]));
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
          const float keep = m[nb][e] == top ? 1.f : ex2_approx(m[nb][e] - top);
          m[nb][e] = top;
          l[nb][e] *= keep;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) o[nb][j][e] *= keep, o[nb][j][2 + e] *= keep;
        }
    }
    uint32_t hi[NB][2], lo[NB][2];      // keys 0-7, 8-15: the weights' halves, rows 2q and 2q + 1
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      // nothing seen yet: weights exp(-inf) = 0
      const float ref0 = m[nb][0] == -INFINITY ? 0.f : m[nb][0], ref1 = m[nb][1] == -INFINITY ? 0.f : m[nb][1];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float p0 = ex2_approx(s[nb][2 * h] - ref0), p1 = ex2_approx(s[nb][2 * h + 1] - ref1);
        l[nb][0] += p0;
        l[nb][1] += p1;
        split_weights(mul2(f2(p0, p1), f2(a.shrink, a.shrink)), hi[nb][h], lo[nb][h]);
      }
    }
    if (partial) keep_hidden_values_out(vbuf, hi, lo, seen);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int h = 0; h < 2; ++h) hi[nb][h] = transpose8(hi[nb][h]), lo[nb][h] = transpose8(lo[nb][h]);
    constexpr int kSet = 4;      // fragments of V at a time, the low halves after the high ones of all four
#pragma unroll
    for (int j0 = 0; j0 < D / 16; j0 += kSet) {
      uint32_t vf[kSet][4];
#pragma unroll
      for (int j = 0; j < kSet; ++j)
        ldmatrix4_trans(vs + chunk_at<kRowBytes>((lane & 7) + ((lane >> 4) << 3), 2 * (j0 + j) + ((lane >> 3) & 1)), vf[j]);
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int j = 0; j < kSet; ++j)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            mma16816(o[nb][j0 + j], vf[j], part ? lo[nb][0] : hi[nb][0], part ? lo[nb][1] : hi[nb][1]);
    }
  }

  // Keys that some rows see and others do not (or that are padding): a weight of zero times an infinite or NaN value
  // would be NaN in the product.  If V holds such values (rare), their terms are added here for the rows that
  // see them, one by one, and they are replaced by zero.
  __device__ __forceinline__ void keep_hidden_values_out(uint8_t *vbuf, const uint32_t (&hi)[NB][2], const uint32_t (&lo)[NB][2],
                                                         const uint32_t (&seen)[NB]) {
    const int lane = threadIdx.x & 31;
    constexpr int kWords = kKeys * kRowBytes / 4;
    uint32_t *words = reinterpret_cast<uint32_t *>(vbuf);
    bool bad = false;
    for (int w = lane; w < kWords; w += 32) {
      const uint32_t v = words[w];
      bad |= (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
    }
    if (!__any_sync(0xffffffffu, bad)) return;
#pragma unroll 1
    for (int key = 0; key < kKeys; ++key) {
      const int src = (key & 7) * 4 + (lane & 3), h = key >> 3;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const uint32_t wh = __shfl_sync(0xffffffffu, h ? hi[nb][1] : hi[nb][0], src);
        const uint32_t wl = __shfl_sync(0xffffffffu, h ? lo[nb][1] : lo[nb][0], src);
        const uint32_t vis = __shfl_sync(0xffffffffu, seen[nb], src) >> (2 * h);
        const float w0 = bf16lo_to_f32(wh) + bf16lo_to_f32(wl), w1 = bf16hi_to_f32(wh) + bf16hi_to_f32(wl);
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const float v = __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(
                vbuf + chunk_at<kRowBytes>(key, 2 * j + half) + (lane >> 2) * 2));
            if (isfinite(v)) continue;
            if (vis & 1) o[nb][j][2 * half] += w0 * v;
            if (vis & 2) o[nb][j][2 * half + 1] += w1 * v;
          }
      }
    }
    __syncwarp();
    for (int w = lane; w < kWords; w += 32) {
      uint32_t v = words[w];
      if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
      if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
      words[w] = v;
    }
    __syncwarp();
  }

  // The warp's sums to shared memory: out[kRows][D], ml[kRows].
  __device__ void finish(const Item &it, float *out, float2 *ml) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * nb + 2 * (lane & 3) + e;
        float sum = l[nb][e];
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (r >= it.rows) continue;
        if (lane < 4) ml[r] = make_float2(m[nb][e], sum);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          out[r * D + 16 * j + (lane >> 2)] = o[nb][j][e];
          out[r * D + 16 * j + 8 + (lane >> 2)] = o[nb][j][2 + e];
        }
      }
  }
};

// ---------------------------------------------------------------------------------------------------------------
// A warp's share of an item in fp32: R rows against kKeys keys at a time, on the CUDA cores.  First product: lane = key and
// a part of the dimensions, so that a score needs log2(kParts) shuffles and each lane weighs keys of its own; the queries
// come from shared memory, the same word for a whole part.  Second product: lane = dimensions, the weights from
// shared memory.  Products are two wide (fma.rn.f32x2), over dimensions and over pairs of rows.
// (With 8 lanes per key, each computing every weight of it, 24 x 8 heads x 1007 rows of D = 64 with 8 rows took 62 us, now 27.)
template <int D_, int R>
struct ScalarRows {
  using T = float;
  static constexpr int D = D_, kRows = R, kRowBytes = 4 * D, kKeys = kRowBytes >= 512 ? 4096 / kRowBytes : 16;
  static constexpr int kParts = 32 / kKeys, kDims = D / kParts, E = D / 32;      // dimensions of a lane in either product
  static constexpr int kPartStride = R * kDims + 4;                              // floats; 4: parts in banks of their own
  static constexpr int kOffP = kParts * kPartStride * 4;
  static constexpr int kQBytes = (kOffP + kWarps * kKeys * R * 4 + 15) / 16 * 16;      // queries; weights of each warp
  // Three CTAs with two stages beat two with three: 24 x 8 heads x 1007 rows of D = 64 with 8 rows 27 against 32 us, 64 x 8 heads
  // x 1250 rows of D = 128 with one row 106 against 109; but one long sequence with 8 rows of D = 64 27 against 25 (more parts),
  // which a second instance of the kernel for such calls would not be worth.
  static constexpr int kCtas = R == 1 ? (D == 32 ? 4 : 3) : D <= 64 ? 3 : 2;
  static constexpr int kStages = (R == 1 && D == 32) || (R == 8 && D == 128) ? 3 : 2;
  static constexpr int kMine = R >= kParts ? R / kParts : 1;      // rows whose weights a lane computes for its key
  F2 o[(R + 1) / 2][E];                                            // pairs of rows (R = 1: the second is unused)
  float m[R], l[kMine];
  int end[R];
  float *q_s, *p_s;

  __device__ void begin(const Params &a, const Item &it, uint8_t *buf) {
    q_s = reinterpret_cast<float *>(buf);
    p_s = reinterpret_cast<float *>(buf + kOffP) + (threadIdx.x >> 5) * kKeys * R;
    for (int c = threadIdx.x; c < R * (D / 4); c += kThreads) {
      const int r = c / (D / 4), d = c % (D / 4) * 4;
      float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < it.rows) {
        const Row row = row_of(a, it, r);
        w = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(a.p.q) + row.n * a.p.q_stride[0] + row.h * a.p.q_stride[1] + d);
      }
      *reinterpret_cast<float4 *>(q_s + d / kDims * kPartStride + r * kDims + d % kDims) = w;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      m[r] = -INFINITY;
      end[r] = r < it.rows ? row_of(a, it, r).end : 0;
    }
#pragma unroll
    for (int i = 0; i < kMine; ++i) l[i] = 0.f;
#pragma unroll
    for (int i = 0; i < (R + 1) / 2; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) o[i][e] = 0;
    __syncthreads();
  }

  __device__ __forceinline__ void step(const Params &a, const Item &it, uint8_t *kbuf, uint8_t *vbuf, int x, float scale2) {
    const int lane = threadIdx.x & 31, key = lane % kKeys, part = lane / kKeys;
    const bool partial = !paged_all_visible(a.s, it.q, x, kKeys);
    float z[R];
    {
      F2 z2[R];
#pragma unroll
      for (int r = 0; r < R; ++r) z2[r] = 0;
      const float *q = q_s + part * kPartStride;
#pragma unroll
      for (int c = 0; c < kDims / 4; ++c) {
        const ulonglong2 k = *reinterpret_cast<const ulonglong2 *>(kbuf + chunk_at<kRowBytes>(key, part * (kDims / 4) + c));
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const ulonglong2 w = *reinterpret_cast<const ulonglong2 *>(q + r * kDims + 4 * c);
          z2[r] = fma2(w.y, k.y, fma2(w.x, k.x, z2[r]));
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float2 t = f2_get(z2[r]);
        z[r] = t.x + t.y;
#pragma unroll
        for (int off = kKeys; off < 32; off <<= 1) z[r] += __shfl_xor_sync(0xffffffffu, z[r], off);
        z[r] = __fmul_rn(z[r], scale2);      // not to be fused with the subtraction of the maximum
      }
    }
    uint32_t hidden = 0;      // bit r: the row does not see this lane's key
    if (partial) {
      const int pos = paged_key(it.q, x + key);
#pragma unroll
      for (int r = 0; r < R; ++r)
        if (!paged_visible(a.s, pos, end[r])) {
          z[r] = -INFINITY;
          hidden |= 1u << r;
        }
    }
    // The reference moves only when a weight would pass 2^8 (the result is the same).
    bool over = false;
#pragma unroll
    for (int r = 0; r < R; ++r) over |= z[r] > m[r] + 8.f;
    if (__any_sync(0xffffffffu, over)) {
      float keep[R + 1];
      keep[R] = 1.f;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float top = fmaxf(m[r], z[r]);
#pragma unroll
        for (int off = 1; off < kKeys; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        keep[r] = m[r] == top ? 1.f : ex2_approx(m[r] - top);
        m[r] = top;
      }
#pragma unroll
      for (int i = 0; i < (R + 1) / 2; ++i) {
        const F2 k2 = f2(keep[2 * i], keep[2 * i + 1]);
#pragma unroll
        for (int e = 0; e < E; ++e) o[i][e] = mul2(o[i][e], k2);
      }
#pragma unroll
      for (int i = 0; i < kMine; ++i) l[i] *= mine(keep, i, part);
    }
    // ---- this lane's weights
    float p[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const float ref = mine(m, i, part);
      p[i] = ex2_approx(mine(z, i, part) - (ref == -INFINITY ? 0.f : ref));      // nothing seen yet: exp(-inf) = 0
      l[i] += p[i];
      p[i] *= a.shrink;
    }
    float *to = p_s + key * R + part * kMine;
    if constexpr (kMine == 4) *reinterpret_cast<float4 *>(to) = make_float4(p[0], p[1], p[2], p[3]);
    else if constexpr (kMine == 2) *reinterpret_cast<float2 *>(to) = make_float2(p[0], p[1]);
    else if (part < R) *to = p[0];
    __syncwarp();
    if (partial && odd_values(vbuf)) {
      // keys that some rows see and others do not, and V holds infinities or NaN (rare): zero times those is not zero
      for (int k = 0; k < kKeys; ++k) {
        const uint32_t hide = __shfl_sync(0xffffffffu, hidden, k);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float v = value(vbuf, k, e);
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (!((hide >> r) & 1)) {
              const float2 t = f2_get(o[r / 2][e]);
              const float sum = fmaf(p_s[k * R + r], v, r & 1 ? t.y : t.x);
              o[r / 2][e] = r & 1 ? f2(t.x, sum) : f2(sum, t.y);
            }
        }
      }
      return;
    }
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
      float v[E];
      if constexpr (E == 1) {
        v[0] = value(vbuf, k, 0);
      } else {
#pragma unroll
        for (int e = 0; e < E; e += E < 4 ? 2 : 4) {
          const uint8_t *at = vbuf + chunk_at<kRowBytes>(k, (lane * E + e) / 4) + (lane * E + e) % 4 * 4;
          if constexpr (E == 2) {
            const float2 t = *reinterpret_cast<const float2 *>(at);
            v[e] = t.x, v[e + 1] = t.y;
          } else {
            const float4 t = *reinterpret_cast<const float4 *>(at);
            v[e] = t.x, v[e + 1] = t.y, v[e + 2] = t.z, v[e + 3] = t.w;
          }
        }
      }
      F2 w[(R + 1) / 2];
      if constexpr (R == 1) {
        w[0] = f2(p_s[k], 0.f);
      } else {
#pragma unroll
        for (int i = 0; i < R / 2; i += 2) {
          const ulonglong2 t = *reinterpret_cast<const ulonglong2 *>(p_s + k * R + 2 * i);
          w[i] = t.x, w[i + 1] = t.y;
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const F2 v2 = f2(v[e], v[e]);
#pragma unroll
        for (int i = 0; i < (R + 1) / 2; ++i) o[i][e] = fma2(w[i], v2, o[i][e]);
      }
    }
  }

  // Element i of this lane's rows, without indexing registers by `part`.
  template <int N>
  static __device__ __forceinline__ float mine(const float (&x)[N], int i, int part) {
    float y = x[i];
#pragma unroll
    for (int j = 1; j < kParts; ++j)
      if (j * kMine + i < R && part == j) y = x[j * kMine + i];
    return y;
  }
  static __device__ __forceinline__ float value(const uint8_t *vbuf, int k, int e) {
    const int d = (threadIdx.x & 31) * E + e;
    return *reinterpret_cast<const float *>(vbuf + chunk_at<kRowBytes>(k, d / 4) + d % 4 * 4);
  }
  static __device__ __forceinline__ bool odd_values(const uint8_t *vbuf) {
    bool odd = false;
    for (int w = threadIdx.x & 31; w < kKeys * D; w += 32)
      odd |= (reinterpret_cast<const uint32_t *>(vbuf)[w] & 0x7f800000u) == 0x7f800000u;
    return __any_sync(0xffffffffu, odd);
  }

  __device__ void finish(const Item &it, float *out, float2 *ml) {
    const int lane = threadIdx.x & 31, part = lane / kKeys;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
#pragma unroll
      for (int off = 1; off < kKeys; off <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
      const int r = part * kMine + i;
      if (lane % kKeys == 0 && r < it.rows) ml[r] = make_float2(mine(m, i, part), l[i]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r >= it.rows) break;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 t = f2_get(o[r / 2][e]);
        out[r * D + lane * E + e] = r & 1 ? t.y : t.x;
      }
    }
  }
};

template <class Rows>
struct Layout {
  static constexpr int kSub = Rows::kKeys * Rows::kRowBytes;        // K or V of one stage of a warp
  static constexpr int kRing = Rows::kStages * 2 * kSub;                  // of one warp; holds its sums at the item's end
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
__device__ __forceinline__ void stream_keys(const Params &a, const Item &it, int tile0, int n_tiles, uint8_t *smem, uint32_t &flags) {
  using T = typename Rows::T;
  using L = Layout<Rows>;
  const ds_paged_params &p = a.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t *ring = smem + warp * L::kRing;
  const float scale2 = p.scale * kLog2e;
  Rows rows;
  rows.begin(a, it, smem + L::kOffQ);
  constexpr int kStages = Rows::kStages, kChunks = Rows::kRowBytes / 16, kOps = Rows::kKeys * kChunks / 32;
  const int32_t *table = p.block_table + it.b * p.table_stride;
  const uint8_t *kbase = reinterpret_cast<const uint8_t *>(reinterpret_cast<const T *>(p.k_cache) + it.g * p.cache_stride[1]);
  const uint8_t *vbase = reinterpret_cast<const uint8_t *>(reinterpret_cast<const T *>(p.v_cache) + it.g * p.cache_stride[1]);
  const long long row_bytes = p.cache_stride[2] * (long long)sizeof(T);
  const int x_first = tile0 * L::kTile + warp * Rows::kKeys;
  // a lane looks up the cache row of key lane % kKeys, one stage ahead of its use
  int pos = paged_key(it.q, x_first + lane % Rows::kKeys);
  int page = pos >= 0 ? table[fast_div(pos, a.page_div)] : 0;
  auto issue = [&](int i) {
    long long at = -1;
    if (pos >= 0) {
      const int ok = paged_clamp_page(page, p.n_pages);
      if (ok != page) flags |= DS_DEV_INDEX;
      const int slot = pos - fast_div(pos, a.page_div) * p.page_size;
      at = (ok * p.cache_stride[0] + slot * p.cache_stride[2]) * (long long)sizeof(T);
    }
    const uint32_t dst = sm100::smem_u32(ring + (i % kStages) * 2 * L::kSub);
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
  for (int i = 0; i < n_tiles; ++i) {
    cp_async_wait<kStages - 2>();
    __syncwarp();      // stage i is there for the whole warp, and the warp is done with stage i - 1
    if (i + kStages - 1 < n_tiles) issue(i + kStages - 1);
    cp_async_commit();
    uint8_t *stage = ring + (i % kStages) * 2 * L::kSub;
    rows.step(a, it, stage, stage + L::kSub, x_first + i * L::kTile, scale2);
  }
  cp_async_wait<0>();
  __syncwarp();

  rows.finish(it, reinterpret_cast<float *>(ring), reinterpret_cast<float2 *>(smem + L::kOffMl) + warp * Rows::kRows);
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
__device__ __forceinline__ void cluster_join(const Params &a, const Item &it, int rank, uint8_t *smem) {
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
__global__ void __launch_bounds__(kThreads, Rows::kCtas) attn_paged_item_kernel(const __grid_constant__ Params a) {
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
__global__ void __launch_bounds__(kThreads, Rows::kCtas) attn_paged_range_kernel(const __grid_constant__ Params a) {
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

size_t workspace_of(const Shape &h) { return h.cluster || h.tiles <= kWholeTiles || h.grid == 1 ? 0 : h.workspace(); }

template <class Rows>
int launch_rows(const ds_paged_params &p, cudaStream_t stream) {
  using L = Layout<Rows>;
  const Shape h = shape_for<Rows>(p);
  const Params a = params_of(p, h, workspace_of(h));
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

// Calls f with the row engine for the call's type, head dimension and rows per KV head.  More rows than an engine holds (32
// in bf16, 8 in fp32) are several items, each of which streams K and V again.
template <class F>
auto with_rows(const ds_paged_params &p, F f) {
  const long long rows = (long long)p.max_q * (p.Hq / p.Hkv);
  if (p.dtype == DS_BF16) {
    if (p.D == 64) return rows <= 8 ? f(TensorRows<64, 1>()) : rows <= 16 ? f(TensorRows<64, 2>()) : f(TensorRows<64, 4>());
    if (rows <= 16) return rows <= 8 ? f(TensorRows<128, 1>()) : f(TensorRows<128, 2>());
    // two stages leave room for the cluster's buffers (2 x 8 heads x 375 .. 1127 rows: 25 -> 14 us), three are a little faster
    return shape_for<TensorRows<128, 4, 2>>(p).cluster > 1 ? f(TensorRows<128, 4, 2>()) : f(TensorRows<128, 4, 3>());
  }
  switch (p.D) {
    case 32: return rows == 1 ? f(ScalarRows<32, 1>()) : f(ScalarRows<32, 8>());
    case 64: return rows == 1 ? f(ScalarRows<64, 1>()) : f(ScalarRows<64, 8>());
    case 128: return rows == 1 ? f(ScalarRows<128, 1>()) : f(ScalarRows<128, 8>());
    default: return rows == 1 ? f(ScalarRows<256, 1>()) : f(ScalarRows<256, 8>());
  }
}

// Rows per KV head from which the kernel with tcgen05 tiles takes over.  Up to 32 rows one pass of this kernel is no slower
// (8 x 32 heads x 1550 rows each, 32 queries: 59 us, and 72 with a form of the other that held every row four times; 32 x 28/4
// heads x 4000 rows, 4 queries: 67 against 69); from 33 on it needs a second.  That pays while one wave of clusters does it with short pieces: a small call takes the other
// kernel 14 .. 25 us whatever its size.  (2 x 8 heads, 33 queries: 800 rows 15 against 23 us, 2400 rows 20 against 26, 8000 rows,
// 16 tiles a CTA, 38 against 32; 28/4 heads, 32 queries, 224 rows per KV head: 13 against 25, 18 against 28, 36 against 37.)
constexpr int kTensorTileRows = 33, kFewTiles = 12;
bool wide(const ds_paged_params &p) {
  if (p.dtype != DS_BF16 || (long long)p.max_q * (p.Hq / p.Hkv) < kTensorTileRows) return false;
  using Rows = TensorRows<128, 4, 2>;      // resident CTAs and tiles are those of D = 64, too
  const Shape h = shape_for<Rows>(p);
  return h.cluster == 0 || h.items > (long long)Rows::kCtas * sm_count() || h.tiles > kFewTiles * h.cluster;
}

}  // namespace

// The numbers of units of the kernel that the call goes to.  (Of 33 rows and more this file's kernels take small calls only.)
bool attn_paged_counts_fit(const ds_paged_params &p) {
  const long long rows = (long long)p.max_q * (p.Hq / p.Hkv);
  if (p.dtype == DS_BF16 && rows >= kTensorTileRows) return attn_paged_tc_counts_fit(p);
  return with_rows(p, [&](auto engine) {
    using Rows = decltype(engine);
    const PagedShape s = units_of(p, Layout<Rows>::kTile, Rows::kRows);
    return paged_units_fit(s, longest_of(s));
  });
}

size_t attn_paged_workspace_bytes(const ds_paged_params &p) {
  if (p.B == 0 || p.N == 0) return 0;
  if (wide(p)) return attn_paged_tc_workspace_bytes(p);
  return with_rows(p, [&](auto rows) { return workspace_of(shape_for<decltype(rows)>(p)); });
}

int launch_attn_paged(const ds_paged_params &p, cudaStream_t stream) {
  if (wide(p)) return launch_attn_paged_tc(p, stream);
  return with_rows(p, [&](auto rows) { return launch_rows<decltype(rows)>(p, stream); });
}

}  // namespace ds

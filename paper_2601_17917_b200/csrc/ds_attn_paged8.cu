// ds_attn_paged8: ds_attn_paged over a cache of e4m3 values with a scale for every block of rows and KV head.
//
// The stream is half as long as bf16's, so a key has half the time.  As with bf16 the keys are the 16-wide side of the products
// (mma.sync m16n8k16), S^T = K Q^T and O^T = V^T P^T, blocks of 8 rows the other; K and V become fp16 in registers, two values an
// instruction, which holds every e4m3 value.
//
// K: a lane's four bytes of an ldmatrix are four neighbouring dimensions of a key, two and two of which stand where the
// product has dimensions 2q, 2q + 1 and 2q + 8, 2q + 9: the queries are laid out in the same order.  V: transposed as bytes, a lane's four
// are four neighbouring keys of a dimension, two and two of which stand where the product has keys 2q, 2q + 1 and 2q + 8, 2q + 9; K's rows
// are taken in the order that puts the weights of these keys there.
//
// Queries enter as fp16 too: a row is scaled by a power of two that puts its largest element into [2^14, 2^15), and 11 bits hold bf16's 8
// down to 2^-31 of that.  fp32 queries are two such parts (22 bits).  The scale of K and the row's factor multiply the score, the scale of V
// the weight, with a power of two for each row (Weights8): the largest weight that the row sees stands at 2^6 .. 2^15, which keeps 11 bits down
// to 2^-20 of it and drops what is below 2^-31: a weight's rounding, 2^-11, is an eighth of the output's in bf16.  For fp32 outputs it stands
// at 2^10 .. 2^15 and the weights are two such parts, the second times 2^11 against V 2^-11: fp16's smallest steps would otherwise end it
// at 2^-12 of the largest.  22 bits down to 2^-24 of the largest, nothing below 2^-46.
//
// Measured: 32 x 32 heads at length, 1.08 GB, 176 - 189 us by box (5.7 to 6.2 TB/s, nine tenths of a plain copy; 2 us more with V transposed
// in pairs and permuted); the issue slots are half in use, a third of them for conversions.  8 x 32 heads of 32 rows x 1024 .. 2080 keys 66 us, which is the
// chain score -> weight -> product in eight warps an SM (issue slots 40 %, tensor pipe 24 %); equal ranges, 16 rows to an item with 12 warps and
// tcgen05 tiles, three quarters empty, were slower (75, 65 and 68 when this took 61).  Products of e4m3 (m16n8k32) for the scores, twice the rate, need two of them for the
// queries' bits and as many conversions of V: 189 -> 206 us.
#include <type_traits>

#include "ds_attn_paged_rows.cuh"
#include "ds_e4m3.cuh"
#include "ds_paged8.cuh"

namespace ds {
namespace {

using namespace paged;

__device__ __forceinline__ void mma_half(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two 16 x 16 matrices of bytes, transposed: lane 4i + q gets rows 4q .. 4q + 3 of column i and of column i + 8, of either.
__device__ __forceinline__ void ldmatrix2_trans_bytes(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

template <typename T_, int D_, int NB, int kKeys_ = 32>
struct ByteRows {
  using T = T_;
  using Cache = uint8_t;
  using Args = Args8;
  static constexpr bool kScaled = true;
  using W = Weights8<!std::is_same<T, float>::value>;
  static constexpr int D = D_, kRows = 8 * NB, kRowBytes = D, kKeys = kKeys_;
  static constexpr int kParts = std::is_same<T, float>::value ? 2 : 1;      // of a query, of a weight
  static constexpr int kBlocks = kParts * NB;                                // of 8 rows of queries
  static constexpr bool kQRegs = kBlocks <= 2;
  static constexpr int kQRowBytes = 2 * D;
  static constexpr int kOffFactor = kBlocks * 8 * kQRowBytes;
  static constexpr int kQSmem = kOffFactor + kRows * 4, kQBytes = kQRegs ? 0 : kQSmem;      // for a moment in the ring, or beside it
  static constexpr int kGroups = NB * kParts <= 2 && kKeys == 32 ? 2 : 1;      // 16s of keys at a time
  static constexpr int kCtas = NB == 1 ? (D == 64 || kKeys == 16 ? 4 : 3) : 2, kStages = kKeys == 16 ? 3 : 2;
  float o[NB][D / 16][4];      // dimensions 16 j + lane / 4 (+ 8), rows 2q, 2q + 1
  float m[NB][2], l[NB][2], e[NB][2], factor[kQRegs ? NB : 1][2];      // (more factors stay where the queries are)
  int end[NB][2];
  uint32_t qf[kQRegs ? kBlocks : 1][kQRegs ? D / 16 : 1][2];
  uint32_t q_smem;

  __device__ void begin(const Args8 &a, const Item &it, uint8_t *q_buf) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    q_smem = sm100::smem_u32(q_buf);
    float *factor_s = reinterpret_cast<float *>(q_buf + kOffFactor);
    constexpr int kLanes = D / 4, kPer = 32 / kLanes;      // lanes of a row, four elements each; rows of a warp at a time
    const int u = lane % kLanes;
#pragma unroll 1
    for (int r0 = warp * kPer; r0 < kRows; r0 += kWarps * kPer) {
      const int r = r0 + lane / kLanes;
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (r < it.rows) {
        const Row row = row_of(a, it, r);
        const T *src = reinterpret_cast<const T *>(a.p.q) + row.n * a.p.q_stride[0] + row.h * a.p.q_stride[1] + 4 * u;
        if constexpr (kParts == 2) {
          const float4 w = *reinterpret_cast<const float4 *>(src);
          x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w;
        } else {
          const uint2 w = *reinterpret_cast<const uint2 *>(src);
          x[0] = bf16lo_to_f32(w.x), x[1] = bf16hi_to_f32(w.x), x[2] = bf16lo_to_f32(w.y), x[3] = bf16hi_to_f32(w.y);
        }
      }
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t b = __float_as_uint(x[e]) & 0x7fffffffu;
        top = max(top, b < 0x7f800000u ? b : 0u);
      }
#pragma unroll
      for (int off = 1; off < kLanes; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
      const int shift = min(100, 14 + 127 - (int)(top >> 23));
      const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
      if (u == 0) factor_s[r] = __uint_as_float((uint32_t)(127 - shift) << 23) * (a.p.scale * kLog2e);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = isfinite(x[e]) ? x[e] * up : __uint_as_float(0x7fffffffu);
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
        // dimensions 4q, 4q + 1 of 16 stand at 2q, 2q + 1, dimensions 4q + 2, 4q + 3 at 2q + 8, 2q + 9
        const uint32_t first = pack_half(x[0], x[1]), second = pack_half(x[2], x[3]);
        uint8_t *to = q_buf + (u & 3) * 4;
        *reinterpret_cast<uint32_t *>(to + chunk_at<kQRowBytes>(part * kRows + r, 2 * (u >> 2))) = first;
        *reinterpret_cast<uint32_t *>(to + chunk_at<kQRowBytes>(part * kRows + r, 2 * (u >> 2) + 1)) = second;
        if constexpr (kParts == 2) {      // what is left
          const float2 f = halves_f32(first), s = halves_f32(second);
          x[0] -= f.x, x[1] -= f.y, x[2] -= s.x, x[3] -= s.y;
        }
      }
    }
    __syncthreads();
    if constexpr (kQRegs) {
#pragma unroll
      for (int t = 0; t < kBlocks; ++t)
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            qf[t][k][h] = *reinterpret_cast<const uint32_t *>(q_buf + chunk_at<kQRowBytes>(8 * t + (lane >> 2), 2 * k + h) + (lane & 3) * 4);
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nb][j][e] = 0.f;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int r = 8 * nb + 2 * (lane & 3) + y;
        m[nb][y] = -INFINITY, l[nb][y] = 0.f, e[nb][y] = 0.f;
        if constexpr (kQRegs) factor[nb][y] = factor_s[r];
        end[nb][y] = r < it.rows ? row_of(a, it, r).end : 0;
      }
    }
    if constexpr (kQRegs) __syncthreads();      // warp 0 loads keys there next
  }

  // Of this lane's rows.
  __device__ __forceinline__ float2 factors(int nb) const {
    if constexpr (kQRegs) return make_float2(factor[nb][0], factor[nb][1]);
    float2 f;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(f.x), "=f"(f.y) : "r"(q_smem + kOffFactor + (8 * nb + 2 * (threadIdx.x & 3)) * 4) : "memory");
    return f;
  }

  // The key of 16 that stands in row i of half h of a product: a lane of the second product has four neighbouring keys of V.
  static __device__ __forceinline__ int key_at(int i, int h) { return 4 * (i >> 1) + (i & 1) + 2 * h; }

  // kKeys keys from x on; K, V and their scales (behind V: of K, of V) as loaded, V is scratch afterwards.
  __device__ __forceinline__ void step(const Args8 &a, const Item &it, uint8_t *kbuf, uint8_t *vbuf, int x, float) {
    const float *scales = reinterpret_cast<const float *>(vbuf + kKeys * kRowBytes);
#pragma unroll 1
    for (int g = 0; g < kKeys / 16; g += kGroups) keys16(a, it, kbuf, vbuf, scales, x, g);
  }

  // The rows' references to the largest score so far, if `scores`, and the exponents of their weights.  s, top and vscale: scores of this
  // lane's keys, the largest of them, their scales of V.  (Short rather than quick: it is run a few times in an item, and instructions that
  // are fetched for the first time cost most of it.)
  __device__ __forceinline__ void move_references(bool scores, const float (&s)[NB][kGroups][4], const float (&top)[NB][2], const float (&vscale)[kGroups][2]) {
    float lv[kGroups][2];
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
      for (int h = 0; h < 2; ++h) lv[g][h] = log_scale(vscale[g][h]);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const float old = m[nb][y];
        float t = scores ? fmaxf(old, top[nb][y]) : old;
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, off));
        const float moved = old == t ? e[nb][y] : e[nb][y] + (t - old), start = fminf(moved, W::kMost);
        l[nb][y] *= old == t ? 1.f : ex2_approx(old - t);
        float most = -INFINITY;
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
          for (int h = 0; h < 2; ++h) most = fmaxf(most, (s[nb][g][2 * h + y] - t) + (start + lv[g][h]));
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
        const float fresh = exponent_of_weights<W>(start, most, old != t), keep = ex2_approx(fresh - moved);
        m[nb][y] = t, e[nb][y] = fresh;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) o[nb][j][y] *= keep, o[nb][j][2 + y] *= keep;
      }
  }

  // Groups g .. g + kGroups - 1 of 16 keys.
  __device__ __forceinline__ void keys16(const Args8 &a, const Item &it, const uint8_t *kbuf, uint8_t *vbuf, const float *scales, int x, int g0) {
    const int lane = threadIdx.x & 31;
    const uint32_t ks = sm100::smem_u32(kbuf), vs = sm100::smem_u32(vbuf);
    float s[NB][kGroups][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nb][g][e] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      uint32_t qs[kQRegs ? 1 : 2][kQRegs ? 1 : kBlocks][2];
      if constexpr (!kQRegs) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int t = 0; t < kBlocks; t += 2) {
            uint32_t w[4];
            ldmatrix4(q_smem + chunk_at<kQRowBytes>(8 * t + (lane & 7) + ((lane >> 4) << 3), 2 * (2 * c + k) + ((lane >> 3) & 1)), w);
            qs[k][t][0] = w[0], qs[k][t][1] = w[1], qs[k][t + 1][0] = w[2], qs[k][t + 1][1] = w[3];
          }
      }
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        uint32_t w[4];      // keys key_at(.., 0) and key_at(.., 1) of dimensions 32 c .. + 15, the same of + 16 .. + 31
        ldmatrix4(ks + chunk_at<kRowBytes>(16 * (g0 + g) + key_at(lane & 7, (lane >> 3) & 1), 2 * c + (lane >> 4)), w);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t a0 = halves_lo(w[2 * k]), a1 = halves_lo(w[2 * k + 1]), a2 = halves_hi(w[2 * k]), a3 = halves_hi(w[2 * k + 1]);
#pragma unroll
          for (int t = 0; t < kBlocks; ++t) {
            const uint32_t b0 = kQRegs ? qf[kQRegs ? t : 0][kQRegs ? 2 * c + k : 0][0] : qs[kQRegs ? 0 : k][kQRegs ? 0 : t][0];
            const uint32_t b1 = kQRegs ? qf[kQRegs ? t : 0][kQRegs ? 2 * c + k : 0][1] : qs[kQRegs ? 0 : k][kQRegs ? 0 : t][1];
            mma_half(s[t % NB][g], a0, a1, a2, a3, b0, b1);
          }
        }
      }
    }
    float vscale[kGroups][2], vmost = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int key = 16 * (g0 + g) + key_at(lane >> 2, h);
        const float kscale = scales[key];
        vscale[g][h] = scales[kKeys + key];
        vmost = fmaxf(vmost, fabsf(vscale[g][h]));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const float2 f = factors(nb);
          s[nb][g][2 * h] = __fmul_rn(s[nb][g][2 * h], f.x * kscale);
          s[nb][g][2 * h + 1] = __fmul_rn(s[nb][g][2 * h + 1], f.y * kscale);
        }
      }
    const bool partial = !paged_all_visible(a.s, it.q, x + 16 * g0, 16 * kGroups);
    uint32_t seen[NB] = {};      // only with partial: bit 4g + 2h + e: key 16g + key_at(lane / 4, h), row 2q + e
    if (partial) {
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int pos = paged_key(it.q, x + 16 * (g0 + g) + key_at(lane >> 2, h));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              if (paged_visible(a.s, pos, end[nb][e])) seen[nb] |= 1u << (4 * g + 2 * h + e);
              else s[nb][g][2 * h + e] = -INFINITY;
            }
        }
    }
    // The references move only when a weight would pass 2^kTop (the result is the same): no maximum is exchanged until some lane finds
    // such a score, or that its largest score with the largest scale of its keys might be one.
    bool over = false, heavy = false;
    float top[NB][2];
    const float lmost = lg2_approx(vmost);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        top[nb][y] = fmaxf(s[nb][0][y], s[nb][0][2 + y]);
#pragma unroll
        for (int g = 1; g < kGroups; ++g) top[nb][y] = fmaxf(top[nb][y], fmaxf(s[nb][g][y], s[nb][g][2 + y]));
        const float rise = top[nb][y] - m[nb][y];
        over |= rise > W::kLag, heavy |= rise + (e[nb][y] + lmost) > W::kTop;
      }
    if (__any_sync(0xffffffffu, over || heavy)) move_references(__any_sync(0xffffffffu, over), s, top, vscale);
    uint32_t w[NB][kGroups][kParts][2];      // keys key_at(.., 0 and 1): the weights (their parts), rows 2q and 2q + 1
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      // nothing seen yet: weights exp(-inf) = 0
      const float ref0 = m[nb][0] == -INFINITY ? 0.f : m[nb][0], ref1 = m[nb][1] == -INFINITY ? 0.f : m[nb][1];
      const float up0 = power_of_two(e[nb][0] + W::kBias), up1 = power_of_two(e[nb][1] + W::kBias);
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float p0 = ex2_approx(s[nb][g][2 * h] - ref0), p1 = ex2_approx(s[nb][g][2 * h + 1] - ref1);
          l[nb][0] += p0;
          l[nb][1] += p1;
          float w0 = (p0 * up0) * (vscale[g][h] * kUnbiased), w1 = (p1 * up1) * (vscale[g][h] * kUnbiased);
          if (partial) {      // zero times a scale that is not finite
            if (!((seen[nb] >> (4 * g + 2 * h)) & 1)) w0 = 0.f;
            if (!((seen[nb] >> (4 * g + 2 * h + 1)) & 1)) w1 = 0.f;
          }
          w[nb][g][0][h] = pack_half(w0, w1);
          if constexpr (kParts == 2) {
            const float2 f = halves_f32(w[nb][g][0][h]);
            w[nb][g][1][h] = pack_half(isfinite(f.x) ? (w0 - f.x) * 0x1p11f : 0.f, isfinite(f.y) ? (w1 - f.y) * 0x1p11f : 0.f);
          }
        }
    }
    if (partial) keep_hidden_values_out(vbuf, g0, seen);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
          for (int h = 0; h < 2; ++h) w[nb][g][part][h] = transpose8(w[nb][g][part][h]);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        uint32_t v[4];      // keys 4q .. 4q + 3 of dimensions 32 c + lane / 4, + 8, + 16, + 24
        ldmatrix2_trans_bytes(vs + chunk_at<kRowBytes>(16 * (g0 + g) + (lane & 15), 2 * c + (lane >> 4)), v);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t a0 = halves_lo(v[2 * k]), a1 = halves_lo(v[2 * k + 1]), a2 = halves_hi(v[2 * k]), a3 = halves_hi(v[2 * k + 1]);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) mma_half(o[nb][2 * c + k], a0, a1, a2, a3, w[nb][g][0][0], w[nb][g][0][1]);
          if constexpr (kParts == 2) {      // V 2^-11, which fp16 holds too: e4m3 values are multiples of 2^-9
            const uint32_t s0 = mul_halves(a0, 0x10001000u), s1 = mul_halves(a1, 0x10001000u), s2 = mul_halves(a2, 0x10001000u), s3 = mul_halves(a3, 0x10001000u);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma_half(o[nb][2 * c + k], s0, s1, s2, s3, w[nb][g][1][0], w[nb][g][1][1]);
          }
        }
      }
  }

  // Keys that some rows see and others do not (or that are padding): a weight of zero times NaN would be NaN in the product.  If V
  // holds NaN there (rare), the rows that see it get it here, and it is replaced by zero.
  __device__ __forceinline__ void keep_hidden_values_out(uint8_t *vbuf, int g0, const uint32_t (&seen)[NB]) {
    const int lane = threadIdx.x & 31;
    constexpr int kWords = 16 * kGroups * kRowBytes / 4;
    uint32_t *words = reinterpret_cast<uint32_t *>(vbuf + 16 * g0 * kRowBytes);
    bool bad = false;
    for (int i = lane; i < kWords; i += 32) bad |= any_nan_e4m3(words[i]);
    if (!__any_sync(0xffffffffu, bad)) return;
#pragma unroll 1
    for (int key = 0; key < 16 * kGroups; ++key) {
      // key_at(i, h) is this key
      const int src = (((key >> 2) & 3) * 2 + (key & 1)) * 4 + (lane & 3), at = 4 * (key >> 4) + 2 * ((key >> 1) & 1);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const uint32_t vis = __shfl_sync(0xffffffffu, seen[nb], src) >> at;
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
          for (int odd = 0; odd < 2; ++odd) {
            const uint8_t b = vbuf[chunk_at<kRowBytes>(16 * g0 + key, j) + (lane >> 2) + 8 * odd];
            if ((b & 0x7f) != 0x7f) continue;
            if (vis & 1) o[nb][j][2 * odd] = __uint_as_float(0x7fffffffu);
            if (vis & 2) o[nb][j][2 * odd + 1] = __uint_as_float(0x7fffffffu);
          }
      }
    }
    __syncwarp();
    for (int i = lane; i < kWords; i += 32) words[i] &= ~__vcmpeq4(words[i] & 0x7f7f7f7fu, 0x7f7f7f7fu);
    __syncwarp();
  }

  // The warp's sums to shared memory: out[kRows][D], ml[kRows].
  __device__ void finish(const Args8 &a, const Item &it, float *out, float2 *ml) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int r = 8 * nb + 2 * (lane & 3) + y;
        float sum = l[nb][y];
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (r >= it.rows) continue;
        if (lane < 4) ml[r] = make_float2(m[nb][y], sum);
        const float down = power_of_two(-e[nb][y]);
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
          out[r * D + 16 * j + (lane >> 2)] = o[nb][j][y] * a.shrink * down, out[r * D + 16 * j + 8 + (lane >> 2)] = o[nb][j][2 + y] * a.shrink * down;
      }
  }
};

// Calls f with the row engine for the call's type, head dimension and rows per KV head; more rows are several items.
template <class F>
auto with_rows(const ds_paged_params &p, F f) {
  const long long rows = (long long)p.max_q * (p.Hq / p.Hkv);
  if (p.dtype == DS_BF16) {
    using T = __nv_bfloat16;
    if (p.D == 64) return rows <= 8 ? f(ByteRows<T, 64, 1>()) : rows <= 16 ? f(ByteRows<T, 64, 2>()) : f(ByteRows<T, 64, 4>());
    return rows <= 8 ? f(ByteRows<T, 128, 1>()) : rows <= 16 ? f(ByteRows<T, 128, 2>()) : f(ByteRows<T, 128, 4>());
  }
  if (p.D == 64) return rows <= 8 ? f(ByteRows<float, 64, 1>()) : f(ByteRows<float, 64, 2>());
  return rows <= 8 ? f(ByteRows<float, 128, 1>()) : f(ByteRows<float, 128, 2>());
}

// As with_rows; with 8 rows of 128 dimensions, items that get CTAs or clusters of their own load 16 keys a stage and run four CTAs
// an SM: they are short, and start sooner (7.7 -> 7.3 us for one request, 19.4 -> 18.0 for 16 of 8 heads).  Ranges are better off
// with 32 (186 against 205 us for 32 x 32 heads, 39 against 42 for one request of 131072 rows).
template <class F>
auto with_rows_at_length(const ds_paged_params &p, F f) {
  using Short = ByteRows<__nv_bfloat16, 128, 1, 16>;
  if (p.dtype == DS_BF16 && p.D == 128 && (long long)p.max_q * (p.Hq / p.Hkv) <= 8 && shape_for<Short>(p).cluster) return f(Short());
  return with_rows(p, f);
}

// Rows per KV head from which the kernel with tcgen05 tiles takes over (27 rows: 70 against 90 us; 40: 127 against 93, both 8 x 32 heads
// x 2000 keys).
constexpr int kTensorTileRows = 33;
bool many_rows(const ds_paged_params &p) { return p.dtype == DS_BF16 && (long long)p.max_q * (p.Hq / p.Hkv) >= kTensorTileRows; }
// But not for a few short items, which the clusters of the other are done with before a CTA of 200 KB is under way (4 KV heads of 224
// rows x 1000 keys: 23 against 33 us; at four tiles of 128 keys to a CTA the two are level).
bool wide(const ds_paged_params &p) {
  if (!many_rows(p)) return false;
  using T = __nv_bfloat16;
  const Shape h = p.D == 64 ? shape_for<ByteRows<T, 64, 4>>(p) : shape_for<ByteRows<T, 128, 4>>(p);
  return !(h.cluster && 4 * h.items <= 2 * sm_count() && h.tiles <= 3 * h.cluster);
}

}  // namespace

bool attn_paged8_counts_fit(const ds_paged8_params &p) {
  if (many_rows(p.a)) return attn_paged8_tc_counts_fit(p.a);
  return with_rows(p.a, [&](auto engine) {
    using Rows = decltype(engine);
    const PagedShape s = units_of(p.a, Layout<Rows>::kTile, Rows::kRows);
    return paged_units_fit(s, longest_of(s));
  });
}

size_t attn_paged8_workspace_bytes(const ds_paged8_params &p) {
  if (p.a.B == 0 || p.a.N == 0) return 0;
  if (wide(p.a)) return attn_paged8_tc_workspace_bytes(p.a);
  return with_rows_at_length(p.a, [&](auto rows) { return rows_workspace_of(shape_for<decltype(rows)>(p.a)); });
}

int launch_attn_paged8(const ds_paged8_params &p, cudaStream_t stream) {
  if (wide(p.a)) return launch_attn_paged8_tc(p, stream);
  return with_rows_at_length(p.a, [&](auto rows) {
    return launch_rows<decltype(rows)>(p.a, stream, [&](Args8 &a) { set_scales(p, a); });
  });
}

}  // namespace ds

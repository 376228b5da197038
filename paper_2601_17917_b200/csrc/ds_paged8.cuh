// What the kernels of ds_attn_paged8 share.
#pragma once
#include "ds_attn_paged.cuh"
#include "ds_e4m3.cuh"

namespace ds {
namespace paged {

struct Args8 : Params {
  const float *k_scale, *v_scale;
  long long scale_stride[3];
  FastDiv scale_div;      // by rows of a block
};

// Weights in fp16.  A weight is p |vs| 2^e: p = exp(score - reference), vs the scale of V, and e, a whole number for each query row, such
// that the largest p |vs| of the keys that the row sees stands near 2^kLog2.  The reference moves when p would pass 2^kLag, e with it or when a
// weight would pass 2^kTop: by the scales that the row itself sees, whatever is hidden from it.  What falls below 2^-25 is dropped.  bf16
// outputs take a wide range for the lag: moving either costs the tcgen05 kernel as much as a tile.
// p 2^e stays a normal number for every vs of 2^-96 .. 2^128 with 2^kBias taken out of vs; e is at most kMost, and at least kLeast, which no
// finite vs passes 2^kTop with.
template <bool kBf16>
struct Weights8 {
  static constexpr float kLog2 = kBf16 ? 7.f : 11.f, kTop = 15.f, kLag = kTop - kLog2;
  static constexpr float kMost = 102.f, kLeast = -126.f;
  static constexpr int kBias = 16;
};
constexpr float kUnbiased = 0x1p-16f;      // 2^-kBias
// The exponent of a row's weights, from the one that would leave its sums as they are and the largest weight, log 2, under that; with room for
// more where the row's reference has moved.
template <class W>
__device__ __forceinline__ float exponent_of_weights(float e, float largest, bool moved) {
  return fmaxf(floorf(largest > (moved ? W::kLog2 : W::kTop) ? e + (W::kLog2 - largest) : e), W::kLeast);
}
// 2^e of a whole number, from the low bits of a sum.
__device__ __forceinline__ float power_of_two(float e) { return __uint_as_float(__float_as_uint(e + (0x1p23f + 127.f)) << 23); }
__device__ __forceinline__ float lg2_approx(float x) {
  float y;
  asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// log2 |vs|, of what is not finite that of zero: it is NaN in the output whatever e is.
__device__ __forceinline__ float log_scale(float vs) {
  const float x = fabsf(vs);
  return x < INFINITY ? lg2_approx(x) : -INFINITY;
}

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ uint32_t e4m3_of_halves(uint32_t h) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(h));
  return r;
}
__device__ __forceinline__ uint32_t e5m2_of_halves(uint32_t h) {
  uint16_t r;
  asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(r) : "r"(h));
  return r;
}
__device__ __forceinline__ uint32_t mul_halves(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t sub_halves(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// The larger of two bf16 each, NaN if one is.
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// A bf16 query row, scaled by a power of two (and the sign of the score's factor) so that its largest element lies in [2^7, 2^8), as the sum of
// an e4m3 value, rounded to the nearest 4 bits, and an e5m2 one: of bf16's 8 bits at most 8 units are left, which 3 bits hold.  Exact
// down to 2^-14 of the row's largest element, within 2^-21 of that below.  A row that is not finite becomes NaN.
// Four neighbouring lanes hold a row, each kLoads times 8 elements.
struct QueryScale {
  float up, factor;      // of the elements; of the scores, times log2 e
};
template <int kLoads>
__device__ __forceinline__ QueryScale query_scale(const uint4 *w, float scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const uint32_t y[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max_nan_bf16x2(top, y[e] & 0x7fff7fffu);
  }
  top = max_nan_bf16x2(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max_nan_bf16x2(top, __shfl_xor_sync(0xffffffffu, top, 2));
  top = max_nan_bf16x2(top, top >> 16) & 0xffffu;
  const int shift = min(100, 7 + 127 - (int)(top >> 7));
  const float up = top >= 0x7f80u ? __uint_as_float(0x7fffffffu) : __uint_as_float((uint32_t)(127 + shift) << 23);
  // a scale of 0: scores of 0
  return {scale < 0.f ? -up : scale > 0.f ? up : up * 0.f,
          scale == 0.f ? 1.f : fmaxf(__uint_as_float((uint32_t)(127 - shift) << 23) * (fabsf(scale) * kLog2e), 0x1p-126f)};
}
// 16 elements.
__device__ __forceinline__ void query_parts(const uint4 *w, float up, uint32_t (&hi)[4], uint32_t (&lo)[4]) {
  const F2 up2 = f2(up, up);
  const uint32_t y[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    uint32_t h[2], l[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const float2 x = f2_get(mul2(f2(bf16lo_to_f32(y[2 * e + z]), bf16hi_to_f32(y[2 * e + z])), up2));
      const uint32_t f = pack_half(x.x, x.y);      // exact but for what is below 2^-32 of the largest
      h[z] = e4m3_of_halves(f);
      l[z] = e5m2_of_halves(sub_halves(f, halves_lo(h[z])));
    }
    hi[e] = h[0] | (h[1] << 16), lo[e] = l[0] | (l[1] << 16);
  }
}

inline void set_scales(const ds_paged8_params &p, Args8 &a) {
  a.k_scale = p.k_scale, a.v_scale = p.v_scale;
  for (int d = 0; d < 3; ++d) a.scale_stride[d] = p.scale_stride[d];
  a.scale_div = make_fast_div(p.scale_block);
}
inline Args8 args8_of(const ds_paged8_params &p, const Shape &h, size_t need) {
  Args8 a;
  static_cast<Params &>(a) = params_of(p.a, h, need);
  set_scales(p, a);
  return a;
}

}  // namespace paged
}  // namespace ds

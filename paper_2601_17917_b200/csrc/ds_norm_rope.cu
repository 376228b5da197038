// ds_qk_norm_rope: RMS norm of every query and key head, rotary position, and the write of K and V into the pages,
// in one pass over the projection's output.
//
// Bound by HBM, and close to being bound by instructions: every element is read once and written once, 4 bytes in bf16
// for some 25 instructions per 8 elements.  A warp owns one row and walks over its heads (a share of them when there are
// few rows), W = 8, 16 or 32 lanes per head.  Lane u of a head holds eight elements in two chunks of four, chosen so that
// both members of its rotary pairs 4u .. 4u + 3 are its own: d and d + R/2 in the half layout, 8u .. 8u + 7 when
// interleaved.  The rotation then needs no exchange and the norm a few shuffles.  Weight, sine and cosine are
// multiplied once per row into two factors per element, out = r (x P + partner Q), which serve all its heads; the
// products are two wide (fma.rn.f32x2).  The loads of four steps are in flight at once.
// The phase of a pair is position * turn in integers modulo 2^64: exact for every position, and its top 32 bits are an
// angle in [-1/2, 1/2) turns, which sincospif takes without a range reduction.
#include <type_traits>

#include "ds_common.cuh"
#include "ds_paged_index.cuh"

namespace ds {
namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;
constexpr int kBatch = 4;   // steps (a head per lane group) whose loads are in flight together

// Four elements as they lie in memory.
template <typename T>
struct Raw4;
template <>
struct Raw4<float> {
  using type = float4;
};
template <>
struct Raw4<__nv_bfloat16> {
  using type = uint2;
};
// Two fp32 values side by side.
using F2 = unsigned long long;
__device__ __forceinline__ F2 f2(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 f2_get(F2 x) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
  return r;
}
__device__ __forceinline__ F2 f2_swap(F2 x) {
  const float2 v = f2_get(x);
  return f2(v.y, v.x);
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ void unpack4(const float4 &w, F2 *f) { f[0] = f2(w.x, w.y), f[1] = f2(w.z, w.w); }
__device__ __forceinline__ void unpack4(const uint2 &w, F2 *f) {
  f[0] = f2(bf16lo_to_f32(w.x), bf16hi_to_f32(w.x)), f[1] = f2(bf16lo_to_f32(w.y), bf16hi_to_f32(w.y));
}
__device__ __forceinline__ uint32_t pack2(F2 x) {
  const float2 f = f2_get(x);
  const __nv_bfloat162 v = __floats2bfloat162_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ void pack4(const F2 *f, float4 &w) {
  const float2 a = f2_get(f[0]), b = f2_get(f[1]);
  w = make_float4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void pack4(const F2 *f, uint2 &w) { w = make_uint2(pack2(f[0]), pack2(f[1])); }

struct Launch {
  int chunks, heads_per_warp;   // units of a row, heads of a unit (a multiple of 32 / W)
  FastDiv chunk_div, page_div;
  float inv_d;
};

template <typename T, int W, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const __grid_constant__ ds_qk_params p,
                                                             const __grid_constant__ ds_rope_table rope,
                                                             const __grid_constant__ Launch launch) {
  using Raw = typename Raw4<T>::type;
  constexpr int kGroups = 32 / W;   // heads side by side
  const int lane = threadIdx.x & 31, u = lane % W, group = lane / W;
  const long long unit = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int n_rows = p.n_rows ? min(max(*p.n_rows, 0), p.N) : p.N;
  if (unit >= (long long)n_rows * launch.chunks) return;
  const int n = fast_div((int)unit, launch.chunk_div), heads = p.Hq + 2 * p.Hkv;
  const int h_begin = ((int)unit - n * launch.chunks) * launch.heads_per_warp;
  const int h_end = min(heads, h_begin + launch.heads_per_warp);

  const int R = rope.rotary_dim, D = p.D;
  const bool live = 8 * u < D, rotated = 8 * u < R;
  const int da = !kInterleaved && rotated ? 4 * u : 8 * u, db = !kInterleaved && rotated ? (R >> 1) + 4 * u : 8 * u + 4;

  float cs[4], sn[4];
  if (h_begin < p.Hq + p.Hkv) {
    const long long pos = p.positions[n];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      cs[i] = 1.f, sn[i] = 0.f;
      if (rotated) {
        const unsigned long long phase = (unsigned long long)pos * rope.turn[4 * u + i];
        sincospif((float)(int)(phase >> 32) * 0x1p-31f, &sn[i], &cs[i]);   // half turns in [-1, 1)
        cs[i] *= rope.mscale, sn[i] *= rope.mscale;
      }
    }
  }
  long long at = -1;      // the row's place in the caches
  if (p.k_cache && h_end > p.Hq) {
    const long long slot = p.slot_map[n];
    if (slot >= 0 && slot < (long long)p.n_pages * p.page_size) {
      const int page = fast_div((int)slot, launch.page_div);
      at = page * p.cache_stride[0] + (slot - (long long)page * p.page_size) * p.cache_stride[2];
    } else if (slot != -1 && p.status && lane == 0) {
      atomicOr(p.status, DS_DEV_INDEX);
    }
  }

  // Heads lo .. hi - 1 of one of the three tensors.
  enum { kQ, kK, kV };
  auto walk = [&](auto kind, int lo, int hi, const T *src, long long src_step, const T *weight, T *dst, long long dst_step, T *dst2,
                  long long dst2_step) {
    constexpr int kKind = decltype(kind)::value;
    if (lo >= hi) return;
    F2 P[4], Q[4];
    if (kKind != kV && live) {
      float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
      if (weight) {
        F2 x[4];
        unpack4(*reinterpret_cast<const Raw *>(weight + da), x);
        unpack4(*reinterpret_cast<const Raw *>(weight + db), x + 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 v = f2_get(x[j]);
          w[2 * j] = v.x, w[2 * j + 1] = v.y;
        }
      }
      float pf[8], qf[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int l = kInterleaved ? 2 * i : i, h = kInterleaved ? 2 * i + 1 : i + 4;
        pf[l] = w[l] * cs[i], qf[l] = -w[h] * sn[i];
        pf[h] = w[h] * cs[i], qf[h] = w[l] * sn[i];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) P[j] = f2(pf[2 * j], pf[2 * j + 1]), Q[j] = f2(qf[2 * j], qf[2 * j + 1]);
    }
    src += (long long)(lo + group) * src_step;
    if (dst) dst += (long long)(lo + group) * dst_step;
    if (dst2) dst2 += (long long)(lo + group) * dst2_step;
    int left = hi - lo - group;      // of this lane group, in heads: > 0 while it has one
    if (!live) left = 0;
    for (int h0 = lo; h0 < hi; h0 += kBatch * kGroups) {
      Raw a[kBatch], b[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        a[i] = Raw{}, b[i] = Raw{};
        if (i * kGroups < left) {
          a[i] = *reinterpret_cast<const Raw *>(src + i * kGroups * src_step + da);
          b[i] = *reinterpret_cast<const Raw *>(src + i * kGroups * src_step + db);
        }
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (h0 + i * kGroups >= hi) break;      // the whole warp
        Raw oa = a[i], ob = b[i];               // V: bits as they are
        if constexpr (kKind != kV) {
          F2 x[4];
          unpack4(oa, x);
          unpack4(ob, x + 2);
          if (weight) {
            const float2 t = f2_get(fma2(x[3], x[3], fma2(x[2], x[2], fma2(x[1], x[1], mul2(x[0], x[0])))));
            float ss = t.x + t.y;
#pragma unroll
            for (int o = W / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            const float r = rsqrtf(fmaf(ss, launch.inv_d, p.eps));
            const F2 r2 = f2(r, r);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = mul2(x[j], r2);
          }
          F2 y[4];
          if (rotated) {
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = fma2(x[j], P[j], mul2(kInterleaved ? f2_swap(x[j]) : x[j ^ 2], Q[j]));
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = mul2(x[j], P[j]);
          }
          pack4(y, oa);
          pack4(y + 2, ob);
        }
        if (i * kGroups < left) {
          if (kKind == kQ || dst) {
            *reinterpret_cast<Raw *>(dst + i * kGroups * dst_step + da) = oa;
            *reinterpret_cast<Raw *>(dst + i * kGroups * dst_step + db) = ob;
          }
          if (kKind != kQ && dst2) {
            *reinterpret_cast<Raw *>(dst2 + i * kGroups * dst2_step + da) = oa;
            *reinterpret_cast<Raw *>(dst2 + i * kGroups * dst2_step + db) = ob;
          }
        }
      }
      constexpr int kStep = kBatch * kGroups;
      src += kStep * src_step, left -= kStep;
      if (kKind == kQ || dst) dst += kStep * dst_step;
      if (kKind != kQ && dst2) dst2 += kStep * dst2_step;
    }
  };
  auto in = [&](const void *t, long long off) { return reinterpret_cast<const T *>(t) + off; };
  auto out = [&](void *t, long long off) { return t && off >= 0 ? reinterpret_cast<T *>(t) + off : nullptr; };
  walk(std::integral_constant<int, kQ>(), h_begin, min(h_end, p.Hq), in(p.q, n * p.q_stride[0]), p.q_stride[1],
       reinterpret_cast<const T *>(p.q_weight), out(p.q_out, n * p.q_out_stride[0]), p.q_out_stride[1], nullptr, 0);
  walk(std::integral_constant<int, kK>(), max(h_begin - p.Hq, 0), min(h_end - p.Hq, p.Hkv), in(p.k, n * p.kv_stride[0]),
       p.kv_stride[1], reinterpret_cast<const T *>(p.k_weight), out(p.k_out, n * p.kv_out_stride[0]), p.kv_out_stride[1],
       out(p.k_cache, at), p.cache_stride[1]);
  walk(std::integral_constant<int, kV>(), max(h_begin - p.Hq - p.Hkv, 0), h_end - p.Hq - p.Hkv, in(p.v, n * p.kv_stride[0]),
       p.kv_stride[1], nullptr, out(p.v_out, n * p.kv_out_stride[0]), p.kv_out_stride[1], out(p.v_cache, at), p.cache_stride[1]);
}

template <typename T, int W>
int launch_width(const ds_qk_params &p, cudaStream_t stream) {
  constexpr int kGroups = 32 / W;
  const int heads = p.Hq + 2 * p.Hkv, steps = (heads + kGroups - 1) / kGroups;
  // few rows: their heads are shared out until the GPU has 32 warps per SM
  const long long want = 32LL * sm_count();
  long long chunks = p.N >= want ? 1 : (want + p.N - 1) / p.N;
  if (chunks > steps) chunks = steps;
  Launch l;
  l.heads_per_warp = (int)((steps + chunks - 1) / chunks) * kGroups;
  l.chunks = (heads + l.heads_per_warp - 1) / l.heads_per_warp;
  l.chunk_div = make_fast_div(l.chunks);
  l.inv_d = 1.f / (float)p.D;
  l.page_div = make_fast_div(p.page_size > 0 ? p.page_size : 1);
  if ((long long)p.N * l.chunks > 0x7fffffffLL) return DS_ERR_UNSUPPORTED;      // needs more than 400000 heads
  const long long blocks = ((long long)p.N * l.chunks + kWarps - 1) / kWarps;
  if (p.rope->interleaved) norm_rope_kernel<T, W, true><<<(unsigned)blocks, kThreads, 0, stream>>>(p, *p.rope, l);
  else norm_rope_kernel<T, W, false><<<(unsigned)blocks, kThreads, 0, stream>>>(p, *p.rope, l);
  DS_CUDA_OK(cudaGetLastError());
  note_launch(1);
  return DS_OK;
}

template <typename T>
int launch_typed(const ds_qk_params &p, cudaStream_t stream) {
  // lanes of a head: the power of two that holds D / 8
  return p.D <= 64 ? launch_width<T, 8>(p, stream) : p.D <= 128 ? launch_width<T, 16>(p, stream) : launch_width<T, 32>(p, stream);
}

}  // namespace

int launch_qk_norm_rope(const ds_qk_params &p, cudaStream_t stream) {
  return p.dtype == DS_BF16 ? launch_typed<__nv_bfloat16>(p, stream) : launch_typed<float>(p, stream);
}

}  // namespace ds

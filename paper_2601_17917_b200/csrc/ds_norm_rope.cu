// ds_qk_norm_rope: RMS norm of every query and key head, rotary position, and the write of K and V into the pages,
// in one pass over the projection's output.
//
// Bound by HBM: every element is read once and written once.  A warp owns one row and walks over its heads (a share of
// them when there are few rows), W = 8, 16 or 32 lanes per head.  Lane u of a head holds eight elements in two
// chunks of four, chosen so that both members of its rotary pairs 4u .. 4u + 3 are its own: d and d + R/2 in the half
// layout, 8u .. 8u + 7 when interleaved.  The rotation then needs no exchange, the norm a few shuffles, and the four
// sines and cosines of a lane serve all heads of the row.  The loads of four heads are in flight at once.
// The phase of a pair is position * turn in integers modulo 2^64: exact for every position, and its top 32 bits are an
// angle in [-1/2, 1/2) turns, which sincospif takes without a range reduction.
#include "ds_common.cuh"
#include "ds_paged_index.cuh"

namespace ds {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBatch = 4;   // heads per lane group whose loads are in flight together

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
__device__ __forceinline__ void unpack4(const float4 &w, float *f) { f[0] = w.x, f[1] = w.y, f[2] = w.z, f[3] = w.w; }
__device__ __forceinline__ void unpack4(const uint2 &w, float *f) {
  f[0] = bf16lo_to_f32(w.x), f[1] = bf16hi_to_f32(w.x), f[2] = bf16lo_to_f32(w.y), f[3] = bf16hi_to_f32(w.y);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ void pack4(const float *f, float4 &w) { w = make_float4(f[0], f[1], f[2], f[3]); }
__device__ __forceinline__ void pack4(const float *f, uint2 &w) { w = make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3])); }

struct Launch {
  int chunks, heads_per_warp;   // units of a row, heads of a unit (a multiple of 32 / W)
  FastDiv chunk_div, page_div;
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

  for (int h0 = h_begin; h0 < h_end; h0 += kBatch * kGroups) {
    Raw a[kBatch], b[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int hh = h0 + i * kGroups + group;
      if (hh < h_end && live) {
        const bool is_q = hh < p.Hq, is_v = hh >= p.Hq + p.Hkv;
        const int h = is_q ? hh : hh - p.Hq - (is_v ? p.Hkv : 0);
        const T *src = reinterpret_cast<const T *>(is_q ? p.q : is_v ? p.v : p.k) +
                       (is_q ? n * p.q_stride[0] + h * p.q_stride[1] : n * p.kv_stride[0] + h * p.kv_stride[1]);
        a[i] = *reinterpret_cast<const Raw *>(src + da);
        b[i] = *reinterpret_cast<const Raw *>(src + db);
      } else {
        a[i] = Raw{}, b[i] = Raw{};
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int hh = h0 + i * kGroups + group;
      if (h0 + i * kGroups >= h_end) break;      // the whole warp
      const bool is_q = hh < p.Hq, is_v = hh >= p.Hq + p.Hkv;
      const int h = is_q ? hh : hh - p.Hq - (is_v ? p.Hkv : 0);
      const T *weight = is_v ? nullptr : reinterpret_cast<const T *>(is_q ? p.q_weight : p.k_weight);
      float x[8];
      unpack4(a[i], x);
      unpack4(b[i], x + 4);
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) ss = fmaf(x[k], x[k], ss);
#pragma unroll
      for (int o = W / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (hh >= h_end || !live) continue;
      if (!is_v) {
        if (weight) {
          const float r = rsqrtf(ss / (float)D + p.eps);
          float w[8];
          unpack4(*reinterpret_cast<const Raw *>(weight + da), w);
          unpack4(*reinterpret_cast<const Raw *>(weight + db), w + 4);
#pragma unroll
          for (int k = 0; k < 8; ++k) x[k] = x[k] * r * w[k];
        }
        if (rotated) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float &lo = kInterleaved ? x[2 * k] : x[k], &hi = kInterleaved ? x[2 * k + 1] : x[k + 4];
            const float y = fmaf(hi, cs[k], lo * sn[k]);
            lo = fmaf(lo, cs[k], -hi * sn[k]);
            hi = y;
          }
        }
      }
      Raw oa, ob;
      if (is_v) oa = a[i], ob = b[i];      // bits as they are
      else pack4(x, oa), pack4(x + 4, ob);
      if (is_q) {
        T *dst = reinterpret_cast<T *>(p.q_out) + n * p.q_out_stride[0] + h * p.q_out_stride[1];
        *reinterpret_cast<Raw *>(dst + da) = oa;
        *reinterpret_cast<Raw *>(dst + db) = ob;
        continue;
      }
      if (p.k_out) {
        T *dst = reinterpret_cast<T *>(is_v ? p.v_out : p.k_out) + n * p.kv_out_stride[0] + h * p.kv_out_stride[1];
        *reinterpret_cast<Raw *>(dst + da) = oa;
        *reinterpret_cast<Raw *>(dst + db) = ob;
      }
      if (at >= 0) {
        T *dst = reinterpret_cast<T *>(is_v ? p.v_cache : p.k_cache) + at + h * p.cache_stride[1];
        *reinterpret_cast<Raw *>(dst + da) = oa;
        *reinterpret_cast<Raw *>(dst + db) = ob;
      }
    }
  }
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

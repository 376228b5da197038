// ds_attn_paged: attention of the new rows of every sequence over its pages.
//
// One warp owns one query row and head; the lanes split the head dimension, and the keys that the row sees are visited
// in order with an online softmax in fp32 (base 2).
#include "ds_common.cuh"

namespace ds {
namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float x, float &y) { y = x; }
__device__ __forceinline__ void from_f32(float x, __nv_bfloat16 &y) { y = __float2bfloat16_rn(x); }

template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32) attn_paged_row_kernel(const ds_paged_params p) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31, b = blockIdx.y;
  const long long idx = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int i = (int)(idx / p.Hq), h = (int)(idx % p.Hq), g = h / (p.Hq / p.Hkv);
  uint32_t flags = 0;
  int first = b * p.max_q, count = p.max_q;
  if (p.row_start) {
    const int lo = p.row_start[b], hi = p.row_start[b + 1];
    first = min(max(lo, 0), p.N);
    count = min(max(hi - first, 0), min(p.max_q, p.N - first));
    if (first != lo || hi - lo != count) flags |= DS_DEV_INDEX;
  }
  const int cap = p.max_pages * p.page_size;
  const int bound = p.max_len > 0 ? min(p.max_len, cap) : cap;
  int len = p.kv_len[b];
  if (len < 0 || len > bound) flags |= DS_DEV_INDEX;
  len = min(max(len, 0), bound);
  if (i < count) {
    const long long row = first + i;
    const int end = p.causal ? len - count + 1 + i : len;
    float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[e] = to_f32(reinterpret_cast<const T *>(p.q)[row * p.q_stride[0] + h * p.q_stride[1] + e * 32 + lane]);
      o[e] = 0.f;
    }
    const float scale2 = p.scale * kLog2e;
    const int lo = p.window ? max(end - p.window, min(p.sinks, end)) : 0;
    for (int t = 0; t < end; ++t) {
      if (t < lo && t >= p.sinks) t = lo;
      int page = p.block_table[b * p.table_stride + t / p.page_size];
      if (page < 0 || page >= p.n_pages) {
        flags |= DS_DEV_INDEX;
        page = page < 0 ? 0 : p.n_pages - 1;
      }
      const long long at = page * p.cache_stride[0] + g * p.cache_stride[1] + (long long)(t % p.page_size) * p.cache_stride[2];
      float z = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) z = fmaf(q[e], to_f32(reinterpret_cast<const T *>(p.k_cache)[at + e * 32 + lane]), z);
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) z += __shfl_xor_sync(0xffffffffu, z, x);
      z *= scale2;
      const float nm = fmaxf(m, z);
      // a score of -inf has no weight, also while nothing else has been seen (-inf - -inf would be NaN)
      const float keep = m == -INFINITY ? 0.f : ex2_approx(m - nm), w = z == -INFINITY ? 0.f : ex2_approx(z - nm);
      m = nm;
      l = fmaf(l, keep, w);
#pragma unroll
      for (int e = 0; e < E; ++e)
        o[e] = fmaf(o[e], keep, w * to_f32(reinterpret_cast<const T *>(p.v_cache)[at + e * 32 + lane]));
    }
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
#pragma unroll
    for (int e = 0; e < E; ++e)
      from_f32(o[e] * inv, reinterpret_cast<T *>(p.out)[row * p.out_stride[0] + h * p.out_stride[1] + e * 32 + lane]);
    if (p.lse && lane == 0) p.lse[row * p.Hq + h] = l > 0.f ? (m + log2f(l)) * kLn2 : (l == 0.f ? -INFINITY : l);
  }
  if (flags && p.status && lane == 0) atomicOr(p.status, flags);
}

template <typename T, int D>
int launch_rows(const ds_paged_params &p, cudaStream_t stream) {
  const long long blocks = ((long long)p.max_q * p.Hq + kWarps - 1) / kWarps;
  if (blocks > 0x7fffffffLL) return DS_ERR_UNSUPPORTED;
  attn_paged_row_kernel<T, D><<<dim3((unsigned)blocks, p.B), kWarps * 32, 0, stream>>>(p);
  DS_CUDA_OK(cudaGetLastError());
  note_launch(1);
  return DS_OK;
}

}  // namespace

size_t attn_paged_workspace_bytes(const ds_paged_params &) { return 0; }

int launch_attn_paged(const ds_paged_params &p, cudaStream_t stream) {
  if (p.dtype == DS_BF16)
    return p.D == 64 ? launch_rows<__nv_bfloat16, 64>(p, stream) : launch_rows<__nv_bfloat16, 128>(p, stream);
  switch (p.D) {
    case 32: return launch_rows<float, 32>(p, stream);
    case 64: return launch_rows<float, 64>(p, stream);
    case 128: return launch_rows<float, 128>(p, stream);
    default: return launch_rows<float, 256>(p, stream);
  }
}

}  // namespace ds

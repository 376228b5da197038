// ds_qk_norm_rope: RMS norm of every query and key head, rotary position, and the write of K and V into the pages,
// in one pass over the projection's output.
//
// One group of lanes owns one head of one row: lane u holds elements 8u .. 8u + 7 (one 16-byte load in bf16, two in
// fp32), so the mean square is a few shuffles and the partner of a half-layout pair, rotary_dim / 2 elements away, is
// held by lane u +- rotary_dim / 16 of the same group (interleaved pairs are in the lane).  The phase of a pair is
// position * turn in integers modulo 2^64: exact for every position, and its top 32 bits are an angle in
// [-1/2, 1/2) turns, which sincospif takes without a range reduction.
#include "ds_common.cuh"

namespace ds {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float (&f)[8]) {
  const uint4 w = *reinterpret_cast<const uint4 *>(p);
  f[0] = bf16lo_to_f32(w.x), f[1] = bf16hi_to_f32(w.x), f[2] = bf16lo_to_f32(w.y), f[3] = bf16hi_to_f32(w.y);
  f[4] = bf16lo_to_f32(w.z), f[5] = bf16hi_to_f32(w.z), f[6] = bf16lo_to_f32(w.w), f[7] = bf16hi_to_f32(w.w);
}
__device__ __forceinline__ void load8(const float *p, float (&f)[8]) {
  const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
  f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&f)[8]) {
  *reinterpret_cast<uint4 *>(p) = make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]));
}
__device__ __forceinline__ void store8(float *p, const float (&f)[8]) {
  *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4 *>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}

// T: element type; W: lanes of a group, the power of two >= D / 8.
template <typename T, int W>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const ds_qk_params p, const __grid_constant__ ds_rope_table rope) {
  const int heads = p.Hq + 2 * p.Hkv;
  const long long unit = ((long long)blockIdx.x * kThreads + threadIdx.x) / W;
  const int u = threadIdx.x % W, d0 = u * 8;
  const int n_rows = p.n_rows ? min(max(*p.n_rows, 0), p.N) : p.N;
  // whole groups leave together; the shuffles below name the group's lanes only
  if (unit >= (long long)n_rows * heads) return;
  const uint32_t group = W == 32 ? 0xffffffffu : ((1u << W) - 1u) << ((threadIdx.x & 31) / W * W);
  const int n = (int)(unit / heads), hh = (int)(unit % heads);
  const bool live = d0 < p.D;
  const bool is_q = hh < p.Hq, is_v = hh >= p.Hq + p.Hkv;
  const int h = is_q ? hh : hh - p.Hq - (is_v ? p.Hkv : 0);
  const T *src = reinterpret_cast<const T *>(is_q ? p.q : is_v ? p.v : p.k) +
                 n * (is_q ? p.q_stride[0] : p.kv_stride[0]) + h * (is_q ? p.q_stride[1] : p.kv_stride[1]);
  float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (live) load8(src + d0, x);
  if (!is_v) {
    const T *weight = reinterpret_cast<const T *>(is_q ? p.q_weight : p.k_weight);
    if (weight) {
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) ss = fmaf(x[k], x[k], ss);
#pragma unroll
      for (int o = W / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(group, ss, o, W);
      const float r = 1.f / sqrtf(ss / (float)p.D + p.eps);
      float w[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (live) load8(weight + d0, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = x[k] * r * w[k];
    }
    const int R = rope.rotary_dim, half = R >> 1;
    const long long pos = p.positions[n];
    const bool rotated = d0 < R, upper = !rope.interleaved && d0 >= half;
    float y[8];
    if (rope.interleaved) {
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = x[k ^ 1];
    } else {
      const int other = rotated ? (upper ? u - half / 8 : u + half / 8) : u;
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = __shfl_sync(group, x[k], other, W);
    }
    if (rotated) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int pair = rope.interleaved ? (d0 + k) >> 1 : (upper ? d0 - half : d0) + k;
        const bool second = rope.interleaved ? (k & 1) : upper;
        const unsigned long long phase = (unsigned long long)pos * rope.turn[pair];
        const float a = (float)(int)(phase >> 32) * 0x1p-31f;  // half turns in [-1, 1)
        float sn, cs;
        sincospif(a, &sn, &cs);
        x[k] = (second ? fmaf(x[k], cs, y[k] * sn) : fmaf(x[k], cs, -y[k] * sn)) * rope.mscale;
      }
    }
  }
  if (!live) return;
  if (is_q) {
    store8(reinterpret_cast<T *>(p.q_out) + n * p.q_out_stride[0] + h * p.q_out_stride[1] + d0, x);
    return;
  }
  if (p.k_out)
    store8(reinterpret_cast<T *>(is_v ? p.v_out : p.k_out) + n * p.kv_out_stride[0] + h * p.kv_out_stride[1] + d0, x);
  if (p.k_cache) {
    const long long slot = p.slot_map[n];
    if (slot >= 0 && slot < (long long)p.n_pages * p.page_size) {
      const long long page = slot / p.page_size, row = slot % p.page_size;
      store8(reinterpret_cast<T *>(is_v ? p.v_cache : p.k_cache) + page * p.cache_stride[0] + h * p.cache_stride[1] +
                 row * p.cache_stride[2] + d0, x);
    } else if (slot != -1 && p.status) {
      atomicOr(p.status, DS_DEV_INDEX);
    }
  }
}

template <typename T>
int launch_typed(const ds_qk_params &p, cudaStream_t stream) {
  const int lanes = p.D / 8;
  const int W = lanes <= 4 ? 4 : lanes <= 8 ? 8 : lanes <= 16 ? 16 : 32;
  const long long units = (long long)p.N * (p.Hq + 2 * p.Hkv);
  const long long blocks = (units * W + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffffLL) return DS_ERR_UNSUPPORTED;
  switch (W) {
    case 4: norm_rope_kernel<T, 4><<<(unsigned)blocks, kThreads, 0, stream>>>(p, *p.rope); break;
    case 8: norm_rope_kernel<T, 8><<<(unsigned)blocks, kThreads, 0, stream>>>(p, *p.rope); break;
    case 16: norm_rope_kernel<T, 16><<<(unsigned)blocks, kThreads, 0, stream>>>(p, *p.rope); break;
    default: norm_rope_kernel<T, 32><<<(unsigned)blocks, kThreads, 0, stream>>>(p, *p.rope); break;
  }
  DS_CUDA_OK(cudaGetLastError());
  note_launch(1);
  return DS_OK;
}

}  // namespace

int launch_qk_norm_rope(const ds_qk_params &p, cudaStream_t stream) {
  return p.dtype == DS_BF16 ? launch_typed<__nv_bfloat16>(p, stream) : launch_typed<float>(p, stream);
}

}  // namespace ds

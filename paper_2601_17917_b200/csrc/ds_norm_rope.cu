// ds_qk_norm_rope: RMS norm of every query and key head, rotary position, and the write of K and V into the pages,
// in one pass over the projection's output.
//
// Bound by HBM, with few instructions to spare: every element is read once and written once.  A warp owns one row and
// walks over its heads (a share of them when there are few rows), W lanes per head.  Lane u of a head holds two chunks of
// 16 bytes, E elements each, contiguous across lanes and chosen so that both members of a rotary pair are the lane's
// own: E u and R/2 + E u in the half layout (what lies behind R is halved among the other lanes), E u and D/2 + E u when
// interleaved.  The rotation then needs no exchange and the norm a few shuffles.  Weight, sine and cosine are
// multiplied once per row into two factors per element, out = r (x P + partner Q), which serve all its heads; the
// products are two wide (fma.rn.f32x2).
// Loads are asynchronous copies to shared memory, some steps ahead through the heads of q, k and v alike; a lane
// reads back what it copied, so nothing is synchronised.  (16384 rows of 36 x 128 bf16: with the loads of four steps
// held in registers 74 us, waiting for them; with copies of 8 bytes, twice the steps, 58 us and 79 % of the issue slots;
// as it is 57 .. 59 us, 5.1 .. 5.3 TB/s.  Eight steps ahead 64 us, two 60; CTAs of 128 threads 57, of 256 62; resident warps
// that load their next row's heads ahead of the row's end 62.)
// The phase of a pair is position * turn in integers modulo 2^64: exact for every position, and its top 32 bits are an
// angle in [-1/2, 1/2) turns, which sincospif takes without a range reduction.
#include <type_traits>

#include "ds_common.cuh"
#include "ds_paged_index.cuh"

namespace ds {
namespace {

constexpr int kThreads = 64, kWarps = kThreads / 32;
constexpr int kAhead = 4;   // steps (a head per lane group) whose loads are in flight
constexpr int kMaxPairs = 128;

// A chunk of 16 bytes as pairs of fp32 and back.
template <typename T>
struct Chunk;
template <>
struct Chunk<float> {
  static constexpr int kElems = 4;
  static __device__ __forceinline__ void unpack(const uint4 &w, F2 *f) {
    f[0] = f2(__uint_as_float(w.x), __uint_as_float(w.y)), f[1] = f2(__uint_as_float(w.z), __uint_as_float(w.w));
  }
  static __device__ __forceinline__ uint4 pack(const F2 *f) {
    const float2 a = f2_get(f[0]), b = f2_get(f[1]);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
};
template <>
struct Chunk<__nv_bfloat16> {
  static constexpr int kElems = 8;
  static __device__ __forceinline__ F2 wide(uint32_t w) { return f2(bf16lo_to_f32(w), bf16hi_to_f32(w)); }
  static __device__ __forceinline__ uint32_t narrow(F2 x) {
    const float2 f = f2_get(x);
    const __nv_bfloat162 v = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t *>(&v);
  }
  static __device__ __forceinline__ void unpack(const uint4 &w, F2 *f) {
    f[0] = wide(w.x), f[1] = wide(w.y), f[2] = wide(w.z), f[3] = wide(w.w);
  }
  static __device__ __forceinline__ uint4 pack(const F2 *f) {
    return make_uint4(narrow(f[0]), narrow(f[1]), narrow(f[2]), narrow(f[3]));
  }
};

struct Launch {
  int chunks, heads_per_warp;   // units of a row, heads of a unit (a multiple of 32 / W)
  FastDiv chunk_div, page_div;
  float inv_d;
};

template <typename T, int W, bool kInterleaved>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const __grid_constant__ ds_qk_params p,
                                                             const __grid_constant__ ds_rope_table rope,
                                                             const __grid_constant__ Launch launch) {
  using C = Chunk<T>;
  constexpr int kGroups = 32 / W;   // heads side by side
  constexpr int E = C::kElems, H = E / 2;      // elements and pairs of fp32 of a chunk
  __shared__ __align__(16) uint4 ring_s[kWarps][kAhead][2][32];
  __shared__ __align__(16) float2 turn_s[kWarps][kMaxPairs];
  dependent_sync();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, u = lane % W, group = lane / W;
  const long long unit = (long long)blockIdx.x * kWarps + warp;
  const int n_rows = p.n_rows ? min(max(*p.n_rows, 0), p.N) : p.N;
  if (unit >= (long long)n_rows * launch.chunks) return;
  const int n = fast_div((int)unit, launch.chunk_div), heads = p.Hq + 2 * p.Hkv;
  const int h_begin = ((int)unit - n * launch.chunks) * launch.heads_per_warp;
  const int h_end = min(heads, h_begin + launch.heads_per_warp);

  const int R = rope.rotary_dim, D = p.D;
  const bool live = 2 * E * u < D;
  int da = E * u, db = (D >> 1) + E * u;
  if (!kInterleaved) {
    if (2 * E * u < R) db = (R >> 1) + E * u;
    else da = R + E * (u - R / (2 * E)), db = da + ((D - R) >> 1);
  }
  const bool rot_a = da < R, rot_b = db < R;      // equal in the half layout

  // ---- the steps' loads: this warp's heads of q, then of k, then of v
  enum { kQ, kK, kV };
  const int lo_q = h_begin, hi_q = min(h_end, p.Hq);
  const int lo_k = max(h_begin - p.Hq, 0), hi_k = min(h_end - p.Hq, p.Hkv);
  const int lo_v = max(h_begin - p.Hq - p.Hkv, 0), hi_v = h_end - p.Hq - p.Hkv;
  int todo = kQ, ahead_left = hi_q - lo_q, ahead_slot = 0;      // the tensor that loads are issued for, its heads to go
  const T *ahead = reinterpret_cast<const T *>(p.q) + n * p.q_stride[0] + (lo_q + group) * p.q_stride[1];
  long long ahead_step = kGroups * p.q_stride[1];
  const uint32_t ring_u = (uint32_t)__cvta_generic_to_shared(&ring_s[warp][0][0][lane]);
  auto issue = [&]() {
    while (ahead_left <= 0 && todo < kV) {
      ++todo;
      ahead_left = todo == kK ? hi_k - lo_k : hi_v - lo_v;
      ahead = reinterpret_cast<const T *>(todo == kK ? p.k : p.v) + n * p.kv_stride[0] +
              ((todo == kK ? lo_k : lo_v) + group) * p.kv_stride[1];
      ahead_step = kGroups * p.kv_stride[1];
    }
    if (group < ahead_left && live) {
      const uint32_t to = ring_u + ahead_slot * 1024;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(ahead + da) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 512), "l"(ahead + db) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ahead += ahead_step;
    ahead_left -= kGroups;
    ahead_slot = (ahead_slot + 1) % kAhead;
  };
#pragma unroll 1
  for (int i = 0; i < kAhead; ++i) issue();

  if (h_begin < p.Hq + p.Hkv) {
    const long long pos = p.positions[n];
    for (int i = lane; i < R >> 1; i += 32) {
      const unsigned long long phase = (unsigned long long)pos * rope.turn[i];
      float sn, cs;
      sincospif((float)(int)(phase >> 32) * 0x1p-31f, &sn, &cs);   // half turns in [-1, 1)
      turn_s[warp][i] = make_float2(cs * rope.mscale, sn * rope.mscale);
    }
    __syncwarp();
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

  int slot = 0;
  auto walk = [&](auto kind, int lo, int hi, const T *weight, T *dst, long long dst_step, T *dst2, long long dst2_step) {
    constexpr int kKind = decltype(kind)::value;
    if (lo >= hi) return;
    F2 P[2 * H], Q[2 * H];      // chunk a, chunk b
    if (kKind != kV && live) {
      float w[2 * E];
#pragma unroll
      for (int i = 0; i < 2 * E; ++i) w[i] = 1.f;
      if (weight) {
        F2 x[2 * H];
        C::unpack(*reinterpret_cast<const uint4 *>(weight + da), x);
        C::unpack(*reinterpret_cast<const uint4 *>(weight + db), x + H);
#pragma unroll
        for (int j = 0; j < 2 * H; ++j) {
          const float2 v = f2_get(x[j]);
          w[2 * j] = v.x, w[2 * j + 1] = v.y;
        }
      }
      float pf[2 * E], qf[2 * E];
#pragma unroll
      for (int i = 0; i < E; ++i) {      // the lane's pairs
        const bool second = kInterleaved && i >= H;
        const int l = kInterleaved ? 2 * i : i, h = kInterleaved ? 2 * i + 1 : i + E;
        const int pair = kInterleaved ? ((second ? db : da) >> 1) + i % H : da + i;
        const float2 t = (second ? rot_b : rot_a) ? turn_s[warp][pair] : make_float2(1.f, 0.f);
        pf[l] = w[l] * t.x, qf[l] = -w[h] * t.y;
        pf[h] = w[h] * t.x, qf[h] = w[l] * t.y;
      }
#pragma unroll
      for (int j = 0; j < 2 * H; ++j) P[j] = f2(pf[2 * j], pf[2 * j + 1]), Q[j] = f2(qf[2 * j], qf[2 * j + 1]);
    }
    if (dst) dst += (long long)(lo + group) * dst_step;
    if (dst2) dst2 += (long long)(lo + group) * dst2_step;
#pragma unroll 1
    for (int left = hi - lo; left > 0; left -= kGroups) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
      uint4 oa = make_uint4(0, 0, 0, 0), ob = oa;
      const bool mine = group < left && live;
      if (mine) oa = ring_s[warp][slot][0][lane], ob = ring_s[warp][slot][1][lane];      // V: bits as they are
      slot = (slot + 1) % kAhead;
      issue();
      if constexpr (kKind != kV) {
        F2 x[2 * H];
        C::unpack(oa, x);
        C::unpack(ob, x + H);
        if (weight) {
          F2 t = mul2(x[0], x[0]);
#pragma unroll
          for (int j = 1; j < 2 * H; ++j) t = fma2(x[j], x[j], t);
          float ss = f2_get(t).x + f2_get(t).y;
#pragma unroll
          for (int o = W / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
          const float r = rsqrtf(fmaf(ss, launch.inv_d, p.eps));
          const F2 r2 = f2(r, r);
#pragma unroll
          for (int j = 0; j < 2 * H; ++j) x[j] = mul2(x[j], r2);
        }
        F2 y[2 * H];
#pragma unroll
        for (int j = 0; j < 2 * H; ++j) y[j] = mul2(x[j], P[j]);      // all of it where nothing is rotated:
        if constexpr (kInterleaved) {                                   // the partner may be infinite there
          if (rot_a)
#pragma unroll
            for (int j = 0; j < H; ++j) y[j] = fma2(f2_swap(x[j]), Q[j], y[j]);
          if (rot_b)
#pragma unroll
            for (int j = H; j < 2 * H; ++j) y[j] = fma2(f2_swap(x[j]), Q[j], y[j]);
        } else if (rot_a) {
#pragma unroll
          for (int j = 0; j < 2 * H; ++j) y[j] = fma2(x[j < H ? j + H : j - H], Q[j], y[j]);
        }
        oa = C::pack(y);
        ob = C::pack(y + H);
      }
      if (mine) {
        if (kKind == kQ || dst) {
          *reinterpret_cast<uint4 *>(dst + da) = oa;
          *reinterpret_cast<uint4 *>(dst + db) = ob;
        }
        if (kKind != kQ && dst2) {
          *reinterpret_cast<uint4 *>(dst2 + da) = oa;
          *reinterpret_cast<uint4 *>(dst2 + db) = ob;
        }
      }
      if (kKind == kQ || dst) dst += kGroups * dst_step;
      if (kKind != kQ && dst2) dst2 += kGroups * dst2_step;
    }
  };
  auto out = [&](void *t, long long off) { return t && off >= 0 ? reinterpret_cast<T *>(t) + off : nullptr; };
  walk(std::integral_constant<int, kQ>(), lo_q, hi_q, reinterpret_cast<const T *>(p.q_weight),
       out(p.q_out, n * p.q_out_stride[0]), p.q_out_stride[1], nullptr, 0);
  walk(std::integral_constant<int, kK>(), lo_k, hi_k, reinterpret_cast<const T *>(p.k_weight),
       out(p.k_out, n * p.kv_out_stride[0]), p.kv_out_stride[1], out(p.k_cache, at), p.cache_stride[1]);
  walk(std::integral_constant<int, kV>(), lo_v, hi_v, nullptr, out(p.v_out, n * p.kv_out_stride[0]), p.kv_out_stride[1],
       out(p.v_cache, at), p.cache_stride[1]);
}

template <typename T, int W>
int launch_width(const ds_qk_params &p, cudaStream_t stream) {
  constexpr int kGroups = 32 / W;
  const int heads = p.Hq + 2 * p.Hkv, steps = (heads + kGroups - 1) / kGroups;
  // few rows: their heads are shared out until the GPU has 16 warps per SM
  const long long want = 16LL * sm_count();
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
  DS_CUDA_OK(launch_kernel(p.rope->interleaved ? norm_rope_kernel<T, W, true> : norm_rope_kernel<T, W, false>,
                           dim3((unsigned)blocks), kThreads, 0, 0, true, stream, p, *p.rope, l));
  note_launch(1);
  return DS_OK;
}

template <typename T>
int launch_typed(const ds_qk_params &p, cudaStream_t stream) {
  // lanes of a head: the power of two that holds its chunk pairs
  const int lanes = p.D / (2 * Chunk<T>::kElems);
  if (lanes <= 4) return launch_width<T, 4>(p, stream);
  if (lanes <= 8) return launch_width<T, 8>(p, stream);
  if (lanes <= 16) return launch_width<T, 16>(p, stream);
  if constexpr (sizeof(T) == 4) return launch_width<T, 32>(p, stream);
  return DS_ERR_UNSUPPORTED;      // D > 256
}

}  // namespace

int launch_qk_norm_rope(const ds_qk_params &p, cudaStream_t stream) {
  return p.dtype == DS_BF16 ? launch_typed<__nv_bfloat16>(p, stream) : launch_typed<float>(p, stream);
}

}  // namespace ds

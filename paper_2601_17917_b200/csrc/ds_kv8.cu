// ds_kv8_write and ds_kv8_read: rows of K and V quantised into the pages of an 8-bit cache, and back.
//
// Both are bound by HBM; with few rows by launch and a chain of dependent loads (row starts, length, table, rows).
//
// Writing.  The rows of a call that fall into one block of a page are neighbours among the packed rows, a run; its first row is
// that of a sequence or of a block.  A CTA looks for the first rows of runs among its share of the packed rows.  An item is a run in one head
// of K or V and belongs to L lanes: they find the largest magnitude of the run, settle the exponent, and quantise; the run is read a
// second time (from the caches close by) where it is longer than the lanes' registers hold.
//
// The power of two is found in the exponent bits: the smallest 2^e with a <= 448 2^e = 1.75 2^(e + 8) has a's exponent less 8, one
// more if a's fraction is above 1.75, which an addition carries into the exponent.
#include <type_traits>

#include "ds_common.cuh"
#include "ds_e4m3.cuh"
#include "ds_paged_index.cuh"

namespace ds {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// How many of the n values do not exceed r, by the whole warp: 32 probes at a time.  The values ascend; if they do not, some
// number between 0 and n.
__device__ __forceinline__ int count_up_to(const int32_t *values, int n, int r) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step - 1;
    const uint32_t past = ~__ballot_sync(0xffffffffu, at < hi && values[at < hi ? at : hi - 1] <= r);
    const int c = past ? __ffs(past) - 1 : 32;
    const int stop = lo + (c + 1) * step - 1;
    lo = min(hi, lo + c * step);
    if (c < 32 && stop < hi) hi = stop;
  }
  return lo;
}

template <typename T>
struct Chunk;      // 16 bytes of K or V
template <>
struct Chunk<float> {
  static constexpr int kElems = 4;
  static __device__ __forceinline__ void wide(const uint4 &w, float *f) {
    f[0] = __uint_as_float(w.x), f[1] = __uint_as_float(w.y), f[2] = __uint_as_float(w.z), f[3] = __uint_as_float(w.w);
  }
};
template <>
struct Chunk<__nv_bfloat16> {
  static constexpr int kElems = 8;
  static __device__ __forceinline__ void wide(const uint4 &w, float *f) {
    f[0] = bf16lo_to_f32(w.x), f[1] = bf16hi_to_f32(w.x), f[2] = bf16lo_to_f32(w.y), f[3] = bf16hi_to_f32(w.y);
    f[4] = bf16lo_to_f32(w.z), f[5] = bf16hi_to_f32(w.z), f[6] = bf16lo_to_f32(w.w), f[7] = bf16hi_to_f32(w.w);
  }
};

constexpr uint32_t kInfBits = 0x7f800000u, kMostBits = 0x7f700000u;      // 1.875 * 2^127

// The value times a power of two, as it is quantised.
__device__ __forceinline__ float scaled(float x, float by) {
  const float most = __uint_as_float(kMostBits);
  const float y = fminf(fmaxf(x, -most), most) * by;
  return (__float_as_uint(x) & 0x7fffffffu) < kInfBits ? y : __uint_as_float(0x7fffffffu);
}

struct WriteLaunch {
  int rows;               // of the packed rows, per CTA
  int items, per_cta;     // K and V of every head; of a CTA
  int bound;              // most rows of a sequence
  FastDiv page_div, block_div, chunk_div;
};

struct NewRows {
  int lo, n, len;
  bool ok;
};
__device__ __forceinline__ NewRows new_rows(const ds_kv8_write_params &p, int bound, int b) {
  const int lo = p.row_start ? p.row_start[b] : b * p.max_q, hi = p.row_start ? p.row_start[b + 1] : lo + p.max_q;
  const int len = p.kv_len[b];
  const long long n = (long long)hi - lo;
  return {lo, (int)n, len, lo >= 0 && n >= 0 && hi <= p.N && n <= p.max_q && len <= bound && n <= len};
}

// One run in one head of K or V by L lanes (u: the lane's number): `count` rows from `src` on, into rows from `code` on; `held` rows
// before them in the block, at `before`.  Every lane of the warp comes here; those without an item have count 0.
template <typename T, int L>
__device__ __forceinline__ void write_run(const T *src, long long src_row, int count, uint8_t *code, long long code_row, uint8_t *before,
                                          int held, float *scale, int D, const FastDiv &chunk_div, int u) {
  using C = Chunk<T>;
  constexpr int E = C::kElems, kKeep = 8;      // chunks of a lane that stay in registers
  const int chunks = (int)chunk_div.d, total = count * chunks;
  uint4 keep[kKeep];
  uint32_t top = 0;
  auto load = [&](int c) {
    const int row = fast_div(c, chunk_div);
    return *reinterpret_cast<const uint4 *>(src + row * src_row + (c - row * chunks) * E);
  };
  auto peak = [&](const uint4 &w) {
    float f[E];
    C::wide(w, f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t b = __float_as_uint(f[e]) & 0x7fffffffu;
      top = max(top, b < kInfBits ? b : 0u);
    }
  };
  const float s0 = held > 0 ? *scale : 0.f;
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
    if (u + i * L < total) keep[i] = load(u + i * L);
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
    if (u + i * L < total) peak(keep[i]);
#pragma unroll 4
  for (int c = u + kKeep * L; c < total; c += L) peak(load(c));
#pragma unroll
  for (int off = 1; off < L; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
  // biased exponents
  int e = (int)((min(top, kMostBits) + 0x1fffffu) >> 23) - 8;
  const uint32_t b0 = __float_as_uint(s0) & 0x7fffffffu;
  if (b0 <= 0x7f000000u) e = max(e, (int)((b0 + 0x7fffffu) >> 23));
  e = max(e, 1);
  const uint32_t to_bits = (uint32_t)e << 23;
  const float by = __uint_as_float(e == 254 ? 0x00400000u : (uint32_t)(254 - e) << 23);      // 2^-e, exactly
  auto store = [&](int c, const uint4 &w) {
    float f[E];
    C::wide(w, f);
#pragma unroll
    for (int k = 0; k < E; ++k) f[k] = scaled(f[k], by);
    const int row = fast_div(c, chunk_div);
    uint8_t *to = code + row * code_row + (c - row * chunks) * E;
    if constexpr (E == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(pack_e4m3x4(f[0], f[1], f[2], f[3]), pack_e4m3x4(f[4], f[5], f[6], f[7]));
    else *reinterpret_cast<uint32_t *>(to) = pack_e4m3x4(f[0], f[1], f[2], f[3]);
  };
#pragma unroll
  for (int i = 0; i < kKeep; ++i)
    if (u + i * L < total) store(u + i * L, keep[i]);
#pragma unroll 4
  for (int c = u + kKeep * L; c < total; c += L) store(c, load(c));
  if (count == 0) return;
  if (held > 0 && __float_as_uint(s0) != to_bits) {
    const float f = s0 * by;
    for (int c = u; c < held * (D / 16); c += L) {
      uint4 *at = reinterpret_cast<uint4 *>(before + c / (D / 16) * code_row + c % (D / 16) * 16);
      const uint4 w = *at;
      uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 lo = halves_f32(halves_lo(x[k])), hi = halves_f32(halves_hi(x[k]));
        x[k] = pack_e4m3x4(scaled(lo.x * f, 1.f), scaled(lo.y * f, 1.f), scaled(hi.x * f, 1.f), scaled(hi.y * f, 1.f));
      }
      *at = make_uint4(x[0], x[1], x[2], x[3]);
    }
  }
  if (u == 0 && !(held > 0 && __float_as_uint(s0) == to_bits)) *scale = __uint_as_float(to_bits);
}

template <typename T, int L>
__global__ void __launch_bounds__(kThreads) kv8_write_kernel(const __grid_constant__ ds_kv8_write_params p,
                                                             const __grid_constant__ WriteLaunch launch) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, u = lane % L;
  constexpr int kGroups = 32 / L;
  uint32_t flags = 0;
  dependent_sync();
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int b = threadIdx.x; b < p.B; b += kThreads)
      if (!new_rows(p, launch.bound, b).ok) flags |= DS_DEV_INDEX;
  int r = blockIdx.x * launch.rows;
  const int r_end = r + min(launch.rows, p.N - r);
  const int item_end = min(launch.items, (int)(blockIdx.y + 1) * launch.per_cta);
  while (r < r_end) {
    const int b = p.row_start ? count_up_to(p.row_start + 1, p.B, r) : r / p.max_q;
    if (b >= p.B) break;
    const NewRows q = new_rows(p, launch.bound, b);
    if (r < q.lo) {
      r = q.lo;
      continue;
    }
    const int hi = (int)min((long long)p.N, (long long)q.lo + max(q.n, 0));
    if (!q.ok || r >= hi) {
      r = max(r + 1, hi);
      continue;
    }
    const int pos = q.len - q.n + (r - q.lo), block = fast_div(pos, launch.block_div), in_block = pos - block * p.scale_block;
    const int next = (int)min((long long)hi, (long long)r + p.scale_block - in_block);
    if (r == q.lo || in_block == 0) {
      const int j = fast_div(pos, launch.page_div), slot = pos - j * p.page_size;
      const int page = p.block_table[b * p.table_stride + j];
      if (page < 0 || page >= p.n_pages) {
        flags |= DS_DEV_INDEX;
      } else {
        const long long cache = page * p.cache_stride[0], at_scale = page * p.scale_stride[0] + fast_div(slot, launch.block_div) * p.scale_stride[2];
        for (int first = blockIdx.y * launch.per_cta + warp * kGroups; first < item_end; first += kWarps * kGroups) {
          const int item = first + lane / L, h = item >> 1;
          const bool mine = item < item_end, value = item & 1;
          const T *src = reinterpret_cast<const T *>(value ? p.v : p.k) + r * p.kv_stride[0] + h * p.kv_stride[1];
          uint8_t *code = reinterpret_cast<uint8_t *>(value ? p.v_cache : p.k_cache) + cache + h * p.cache_stride[1] + slot * p.cache_stride[2];
          float *scale = (value ? p.v_scale : p.k_scale) + at_scale + h * p.scale_stride[1];
          const int held = mine && r == q.lo ? in_block : 0;
          write_run<T, L>(src, p.kv_stride[0], mine ? next - r : 0, code, p.cache_stride[2], code - held * p.cache_stride[2], held, scale, p.D,
                          launch.chunk_div, u);
        }
      }
    }
    r = next;
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

// ---------------------------------------------------------------------------------------------------------------
struct ReadLaunch {
  int rows;      // of the output, per CTA; of one sequence when dense
  int per_seq;   // dense: CTAs of a sequence
  int items, per_cta;
  FastDiv page_div, block_div, chunk_div, seq_div;
};
constexpr int kReadRows = 32;

template <typename T>
__global__ void __launch_bounds__(kThreads) kv8_read_kernel(const __grid_constant__ ds_kv8_read_params p,
                                                            const __grid_constant__ ReadLaunch launch) {
  __shared__ long long code_s[kReadRows], scale_s[kReadRows], out_s[kReadRows];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t flags = 0;
  dependent_sync();
  const int bound = p.max_pages * p.page_size;
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int b = tid; b < p.B; b += kThreads) {
      const int len = p.kv_len[b];
      if (len < 0 || len > bound || (p.first && p.first[b] < 0)) flags |= DS_DEV_INDEX;
      if (p.out_start) {
        const int lo = p.out_start[b], hi = p.out_start[b + 1];
        if (lo < 0 || hi < lo || hi > p.N) flags |= DS_DEV_INDEX;
      }
    }
  const int seq = p.out_start ? 0 : fast_div(blockIdx.x, launch.seq_div);
  const int r0 = (p.out_start ? (int)blockIdx.x : (int)blockIdx.x - seq * launch.per_seq) * launch.rows;
  const int n = min(launch.rows, p.N - r0);
  for (int i = warp; i < n; i += kWarps) {      // a warp per row
    const int r = r0 + i, b = p.out_start ? count_up_to(p.out_start + 1, p.B, r) : seq;
    if (lane != 0) continue;
    long long code = -1, scale = 0, out = 0;
    if (b < p.B) {
      const int lo = p.out_start ? p.out_start[b] : 0, hi = p.out_start ? min(p.out_start[b + 1], p.N) : p.N;
      const int len = p.kv_len[b], first = p.first ? p.first[b] : 0;
      const long long pos = (long long)first + (r - lo);
      if (lo >= 0 && r >= lo && r < hi && first >= 0 && len >= 0 && len <= bound) {
        if (pos < len) {
          const int j = fast_div((int)pos, launch.page_div), slot = (int)pos - j * p.page_size;
          const int page = p.block_table[b * p.table_stride + j];
          if (page < 0 || page >= p.n_pages) {
            flags |= DS_DEV_INDEX;
          } else {
            code = page * p.cache_stride[0] + slot * p.cache_stride[2];
            scale = page * p.scale_stride[0] + fast_div(slot, launch.block_div) * p.scale_stride[2];
            out = (p.out_start ? 0 : b * p.out_stride[0]) + r * p.out_stride[1];
          }
        } else if (p.out_start) {
          flags |= DS_DEV_INDEX;
        }
      }
    }
    code_s[i] = code, scale_s[i] = scale, out_s[i] = out;
  }
  __syncthreads();
  const int chunks = p.D / 8, item0 = blockIdx.y * launch.per_cta, items = min(launch.per_cta, launch.items - item0);
  const int total = n * items * chunks;
#pragma unroll 4
  for (int c = tid; c < total; c += kThreads) {
    const int q = fast_div(c, launch.chunk_div), ch = c - q * chunks, i = q / items, item = item0 + q - i * items, h = item >> 1;
    const long long code = code_s[i];
    if (code < 0) continue;
    const bool value = item & 1;
    const uint2 w = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(value ? p.v_cache : p.k_cache) + code + h * p.cache_stride[1] + 8 * ch);
    const float s = (value ? p.v_scale : p.k_scale)[scale_s[i] + h * p.scale_stride[1]];
    const float2 a0 = halves_f32(halves_lo(w.x)), a1 = halves_f32(halves_hi(w.x)), a2 = halves_f32(halves_lo(w.y)), a3 = halves_f32(halves_hi(w.y));
    T *to = reinterpret_cast<T *>(value ? p.v_out : p.k_out) + out_s[i] + h * p.out_stride[2] + 8 * ch;
    if constexpr (std::is_same<T, float>::value) {
      reinterpret_cast<float4 *>(to)[0] = make_float4(a0.x * s, a0.y * s, a1.x * s, a1.y * s);
      reinterpret_cast<float4 *>(to)[1] = make_float4(a2.x * s, a2.y * s, a3.x * s, a3.y * s);
    } else {
      const __nv_bfloat162 v[4] = {__floats2bfloat162_rn(a0.x * s, a0.y * s), __floats2bfloat162_rn(a1.x * s, a1.y * s),
                                   __floats2bfloat162_rn(a2.x * s, a2.y * s), __floats2bfloat162_rn(a3.x * s, a3.y * s)};
      *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(v);
    }
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

template <typename T, int L>
int launch_write(const ds_kv8_write_params &p, cudaStream_t stream) {
  WriteLaunch w;
  const int cap = p.max_pages * p.page_size;
  w.bound = p.max_len > 0 && p.max_len < cap ? p.max_len : cap;
  w.items = 2 * p.Hkv;
  const int at_a_time = kWarps * (32 / L);      // items of a CTA
  // One row to a CTA while the calls are few, more where the CTAs would otherwise be many waves.
  w.per_cta = w.items < at_a_time ? w.items : at_a_time;
  const long long groups = (w.items + w.per_cta - 1) / w.per_cta, enough = 8LL * sm_count();
  w.rows = 1;
  while (w.rows < 64 && (p.N + 2LL * w.rows - 1) / (2LL * w.rows) * groups >= enough) w.rows *= 2;
  w.page_div = make_fast_div(p.page_size);
  w.block_div = make_fast_div(p.scale_block);
  w.chunk_div = make_fast_div(p.D / Chunk<T>::kElems);
  const dim3 grid((unsigned)(((long long)p.N + w.rows - 1) / w.rows), (unsigned)groups);
  DS_CUDA_OK(launch_kernel(kv8_write_kernel<T, L>, grid, kThreads, 0, 0, true, stream, p, w));
  note_launch(1);
  return DS_OK;
}

template <typename T>
int launch_write_lanes(const ds_kv8_write_params &p, cudaStream_t stream) {
  // lanes of an item: a run of one row should not leave most of them idle
  const long long chunks = (long long)(p.max_q < p.scale_block ? p.max_q : p.scale_block) * (p.D / Chunk<T>::kElems);
  return chunks <= 8 ? launch_write<T, 8>(p, stream) : chunks <= 16 ? launch_write<T, 16>(p, stream) : launch_write<T, 32>(p, stream);
}

template <typename T>
int launch_read(const ds_kv8_read_params &p, cudaStream_t stream) {
  ReadLaunch w;
  w.items = 2 * p.Hkv;
  const long long units = (long long)p.D / 8 * w.items, rows = p.out_start ? p.N : (long long)p.B * p.N;
  w.rows = kReadRows;
  while (w.rows > 1 && (rows / w.rows) * ((units + 511) / 512) < 4LL * sm_count()) w.rows /= 2;
  w.per_cta = w.items;
  while (w.per_cta > 1 && (long long)w.rows * w.per_cta * (p.D / 8) > 4 * kThreads) w.per_cta = (w.per_cta + 1) / 2;
  w.per_seq = (int)(((long long)p.N + w.rows - 1) / w.rows);
  w.page_div = make_fast_div(p.page_size);
  w.block_div = make_fast_div(p.scale_block);
  w.chunk_div = make_fast_div(p.D / 8);
  w.seq_div = make_fast_div(w.per_seq);
  const long long ctas = (p.out_start ? 1LL : p.B) * w.per_seq;
  if (ctas > 0x7fffffffLL) return DS_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)ctas, (unsigned)((w.items + w.per_cta - 1) / w.per_cta));
  DS_CUDA_OK(launch_kernel(kv8_read_kernel<T>, grid, kThreads, 0, 0, true, stream, p, w));
  note_launch(1);
  return DS_OK;
}

}  // namespace

int launch_kv8_write(const ds_kv8_write_params &p, cudaStream_t stream) {
  return p.dtype == DS_BF16 ? launch_write_lanes<__nv_bfloat16>(p, stream) : launch_write_lanes<float>(p, stream);
}
int launch_kv8_read(const ds_kv8_read_params &p, cudaStream_t stream) {
  return p.dtype == DS_BF16 ? launch_read<__nv_bfloat16>(p, stream) : launch_read<float>(p, stream);
}

}  // namespace ds

// ds_kv8_write and ds_kv8_read: rows of K and V quantised into the pages of an 8-bit cache, and back.
//
// Both are bound by HBM; with few rows by launch and a chain of dependent loads (row starts, length, table, rows).
//
// Writing.  The rows of a call that fall into one block of a page are neighbours among the packed rows, a run; its first row is
// that of a sequence or of a block.  A CTA looks for the first rows of runs among its share of the packed rows.  An item is a run in one head
// of K or V and belongs to L lanes: they find the largest magnitude of the run, settle the exponent, and quantise; the run is read a
// second time (from the caches close by) where it is longer than the lanes' registers hold.  Runs of more than 4 KB get a CTA per
// item instead, whose threads stage runs in shared memory by asynchronous copies, two ahead, and quantise them from there.
// Measured: one row each of 64 requests 3.5 - 3.9 us, the floor of a launch and of the dependent loads; 32 x 32 heads x 17 .. 2048 rows in blocks
// of 64, 830 MB, 149 - 154 us = 5.4 - 5.6 TB/s of a copy's 6.55, seven tenths of the issue slots in use (184 before a thread's chunks stood at equal
// steps and full runs were told apart: addresses and conditions were most of the instructions).
// Reading.  A thread per row and 8 dimensions, four heads' loads in flight; 500 MB in 87 us = 5.7 TB/s.
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

// How many of the n values do not exceed r, by the whole warp: 128 probes at a time.  The values ascend; if they do not, some
// number between 0 and n.
__device__ __forceinline__ int count_up_to(const int32_t *values, int n, int r) {
  const int lane = threadIdx.x & 31;
  int lo = 0, hi = n;
  while (lo < hi) {
    const int step = (hi - lo + 127) / 128;
    int c = 0;      // probes that do not exceed r, up to the first that does
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = lo + (32 * k + lane + 1) * step - 1;
      const uint32_t past = ~__ballot_sync(0xffffffffu, at < hi && values[at < hi ? at : hi - 1] <= r);
      if (c == 32 * k) c += past ? __ffs(past) - 1 : 32;
    }
    const int stop = lo + (c + 1) * step - 1;
    lo = min(hi, lo + c * step);
    if (c < 128 && stop < hi) hi = stop;
  }
  return lo;
}

// Copies of 16 bytes to shared memory in the background; a thread reads back what it copied.
__device__ __forceinline__ void copy16(uint4 *to, const void *from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

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

// The scale of a run whose largest magnitude has the bits `top`, with `held` rows under the scale s0 before it in the block.
struct Scale {
  uint32_t bits;
  float by;      // 1 / scale, exactly
};
__device__ __forceinline__ Scale scale_of(uint32_t top, int held, float s0) {
  int e = (int)((min(top, kMostBits) + 0x1fffffu) >> 23) - 8;      // biased exponents
  const uint32_t b0 = __float_as_uint(s0) & 0x7fffffffu;
  if (held > 0 && b0 <= 0x7f000000u) e = max(e, (int)((b0 + 0x7fffffu) >> 23));
  e = max(e, 1);
  return {(uint32_t)e << 23, __uint_as_float(e == 254 ? 0x00400000u : (uint32_t)(254 - e) << 23)};
}
// The largest magnitude, of finite values if `finite`, else of all but NaN.
template <typename T>
__device__ __forceinline__ uint32_t peak_of(const uint4 &w, uint32_t top, bool finite) {
  if (finite) {
    float f[Chunk<T>::kElems];
    Chunk<T>::wide(w, f);
#pragma unroll
    for (int e = 0; e < Chunk<T>::kElems; ++e) {
      const uint32_t b = __float_as_uint(f[e]) & 0x7fffffffu;
      top = max(top, b < kInfBits ? b : 0u);
    }
    return top;
  }
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  if constexpr (std::is_same<T, float>::value) {
    float t = __uint_as_float(top);
#pragma unroll
    for (int k = 0; k < 4; ++k) t = fmaxf(t, fabsf(__uint_as_float(x[k])));      // NaN is not the larger
    return __float_as_uint(t);
  } else {
    // pairs: the larger of two bf16, NaN is not
    auto larger = [](uint32_t a, uint32_t b) {
      uint32_t r;
      asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
      return r;
    };
    constexpr uint32_t kAbs = 0x7fff7fffu;
    const uint32_t t = larger(larger(x[0] & kAbs, x[1] & kAbs), larger(x[2] & kAbs, x[3] & kAbs));
    return __float_as_uint(fmaxf(__uint_as_float(top), fmaxf(bf16lo_to_f32(t), bf16hi_to_f32(t))));
  }
}
// `plain`: nothing is infinite or beyond the largest value held.  NaN comes out as NaN of itself.
template <typename T>
__device__ __forceinline__ void store_codes(uint8_t *to, const uint4 &w, float by, bool plain) {
  constexpr int E = Chunk<T>::kElems;
  float f[E];
  Chunk<T>::wide(w, f);
  if (plain) {
#pragma unroll
    for (int k = 0; k < E; ++k) f[k] *= by;
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) f[k] = scaled(f[k], by);
  }
  if constexpr (E == 8) *reinterpret_cast<uint2 *>(to) = make_uint2(pack_e4m3x4(f[0], f[1], f[2], f[3]), pack_e4m3x4(f[4], f[5], f[6], f[7]));
  else *reinterpret_cast<uint32_t *>(to) = pack_e4m3x4(f[0], f[1], f[2], f[3]);
}
// Rows under the scale s0 that come under another: lane u of n.  The quotient of the scales is exact; beyond 2^60 and below 2^-60 of
// it every value but zero is the largest or zero.
__device__ __forceinline__ void rescale(uint8_t *rows, long long row_bytes, int held, int D, float s0, uint32_t now_bits, int u, int n) {
  const bool small = fabsf(s0) < 0x1p-100f;
  const uint32_t b = __float_as_uint(small ? s0 * 0x1p40f : s0), exponent = (b >> 23) & 255u;
  const int power = max(-60, min(60, (int)exponent - (small ? 40 : 0) - (int)(now_bits >> 23)));
  const float f = exponent == 255u ? __uint_as_float(0x7fffffffu) : s0 == 0.f ? s0 : __uint_as_float((b & 0x807fffffu) | (uint32_t)(127 + power) << 23);
  for (int c = u; c < held * (D / 16); c += n) {
    uint4 *at = reinterpret_cast<uint4 *>(rows + c / (D / 16) * row_bytes + c % (D / 16) * 16);
    const uint4 w = *at;
    uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 lo = halves_f32(halves_lo(x[k])), hi = halves_f32(halves_hi(x[k]));
      x[k] = pack_e4m3x4(mul_to_odd(lo.x, f), mul_to_odd(lo.y, f), mul_to_odd(hi.x, f), mul_to_odd(hi.y, f));
    }
    *at = make_uint4(x[0], x[1], x[2], x[3]);
  }
}

constexpr int kKeep = 8;      // chunks of a lane, at most

// One run in one head of K or V by L lanes (u: the lane's number), at most kKeep L chunks: `count` rows from `src` on, into rows from
// `code` on; `held` rows before them in the block, at `before`.  Every lane of the warp comes here; those without an item have count 0.
template <typename T, int L>
__device__ __forceinline__ void write_run(uint4 *buf, const T *src, long long src_row, int count, uint8_t *code, long long code_row,
                                          uint8_t *before, int held, float *scale, int D, const FastDiv &chunk_div, int u) {
  constexpr int E = Chunk<T>::kElems;
  const int chunks = (int)chunk_div.d, total = count * chunks, lane = threadIdx.x & 31;
  for (int i = 0, c = u; c < total; ++i, c += L) {
    const int row = fast_div(c, chunk_div);
    copy16(buf + 32 * i + lane, src + row * src_row + (c - row * chunks) * E);
  }
  copies_end();
  const float s0 = held > 0 ? *scale : 0.f;
  copies_wait<0>();
  auto peak = [&](bool finite) {
    uint32_t top = 0;
    for (int i = 0, c = u; c < total; ++i, c += L) top = peak_of<T>(buf[32 * i + lane], top, finite);
    __syncwarp();
#pragma unroll
    for (int off = 1; off < L; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
    return top;
  };
  uint32_t top = peak(false);
  const bool plain = top <= kMostBits;
  if (!__all_sync(0xffffffffu, plain)) top = peak(true);
  const Scale now = scale_of(top, held, s0);
  for (int i = 0, c = u; c < total; ++i, c += L) {
    const int row = fast_div(c, chunk_div);
    store_codes<T>(code + row * code_row + (c - row * chunks) * E, buf[32 * i + lane], now.by, plain);
  }
  if (count > 0) {
    const bool same = held > 0 && __float_as_uint(s0) == now.bits;
    if (held > 0 && !same) rescale(before, code_row, held, D, s0, now.bits, u, L);
    if (u == 0 && !same) *scale = __uint_as_float(now.bits);
  }
  __syncwarp();
}

// The runs that begin in a CTA's share of the packed rows, one after the other, found by every warp for itself.
struct Run {
  int row, count, held;              // packed rows; rows before them in the block, from before the call
  long long code, scale;             // offsets of its first row and of its block in head 0
};
struct RunWalk {
  int r, r_end;
  __device__ __forceinline__ RunWalk(const ds_kv8_write_params &p, const WriteLaunch &launch) {
    r = blockIdx.x * launch.rows;
    r_end = r + min(launch.rows, p.N - r);
  }
  __device__ __forceinline__ bool next(const ds_kv8_write_params &p, const WriteLaunch &launch, Run &run, uint32_t &flags) {
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
      const int pos = q.len - q.n + (r - q.lo), in_block = pos - fast_div(pos, launch.block_div) * p.scale_block, first = r;
      r = (int)min((long long)hi, (long long)r + p.scale_block - in_block);
      if (first != q.lo && in_block != 0) continue;
      const int j = fast_div(pos, launch.page_div), slot = pos - j * p.page_size;
      const int page = p.block_table[b * p.table_stride + j];
      if (page < 0 || page >= p.n_pages) {
        flags |= DS_DEV_INDEX;
        continue;
      }
      run.row = first, run.count = r - first, run.held = first == q.lo ? in_block : 0;
      run.code = page * p.cache_stride[0] + slot * p.cache_stride[2];
      run.scale = page * p.scale_stride[0] + fast_div(slot, launch.block_div) * p.scale_stride[2];
      return true;
    }
    return false;
  }
};
__device__ __forceinline__ uint32_t check_sequences(const ds_kv8_write_params &p, int bound) {
  uint32_t flags = 0;
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int b = threadIdx.x; b < p.B; b += kThreads)
      if (!new_rows(p, bound, b).ok) flags |= DS_DEV_INDEX;
  return flags;
}

template <typename T, int L>
__global__ void __launch_bounds__(kThreads, 5) kv8_write_kernel(const __grid_constant__ ds_kv8_write_params p,
                                                                const __grid_constant__ WriteLaunch launch) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, u = lane % L;
  constexpr int kGroups = 32 / L;
  __shared__ __align__(16) uint4 buf_s[kWarps][kKeep * 32];
  dependent_sync();
  uint32_t flags = check_sequences(p, launch.bound);
  const int item_end = min(launch.items, (int)(blockIdx.y + 1) * launch.per_cta);
  RunWalk walk(p, launch);
  Run run;
  while (walk.next(p, launch, run, flags)) {
    for (int first = blockIdx.y * launch.per_cta + warp * kGroups; first < item_end; first += kWarps * kGroups) {
      const int item = first + lane / L, h = item >> 1;
      const bool mine = item < item_end, value = item & 1;
      const T *src = reinterpret_cast<const T *>(value ? p.v : p.k) + run.row * p.kv_stride[0] + h * p.kv_stride[1];
      uint8_t *code = reinterpret_cast<uint8_t *>(value ? p.v_cache : p.k_cache) + run.code + h * p.cache_stride[1];
      float *scale = (value ? p.v_scale : p.k_scale) + run.scale + h * p.scale_stride[1];
      const int held = mine ? run.held : 0;
      write_run<T, L>(buf_s[warp], src, p.kv_stride[0], mine ? run.count : 0, code, p.cache_stride[2], code - held * p.cache_stride[2], held, scale, p.D,
                      launch.chunk_div, u);
    }
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

// Longer runs: the whole CTA takes an item; the next ones' first chunks are on their way while the exponent of this one is settled.
constexpr int kWideKeep = 4, kAhead = 2;      // chunks of a thread that are held; items ahead
template <typename T>
__global__ void __launch_bounds__(kThreads, 4) kv8_write_wide_kernel(const __grid_constant__ ds_kv8_write_params p,
                                                                     const __grid_constant__ WriteLaunch launch) {
  constexpr int E = Chunk<T>::kElems;
  extern __shared__ __align__(16) uint4 ring[];      // [kAhead + 1][kWideKeep][kThreads]
  __shared__ uint32_t top_s[2][kWarps];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  dependent_sync();
  uint32_t flags = check_sequences(p, launch.bound);
  const int item0 = blockIdx.y * launch.per_cta, item_end = min(launch.items, item0 + launch.per_cta);
  const int chunks = (int)launch.chunk_div.d;
  // A thread has the same chunk of every at_a_time-th row, at equal steps: with chunks dealt out one after the other the addresses were
  // most of the kernel's instructions.  (Up to chunks - 1 threads have none.)
  const int row0 = fast_div(tid, launch.chunk_div), ch = (tid - row0 * chunks) * E, at_a_time = kThreads / chunks;
  const long long src_step = at_a_time * p.kv_stride[0], code_step = at_a_time * p.cache_stride[2];
  RunWalk walk(p, launch);
  Run run;
  int turn = 0;
  while (walk.next(p, launch, run, flags)) {
    const int n_mine = row0 < at_a_time ? max(0, (run.count - row0 + at_a_time - 1) / at_a_time) : 0, n_keep = min(kWideKeep, n_mine);
    const bool full = __all_sync(0xffffffffu, n_keep == kWideKeep);      // nothing to ask for every chunk
    const long long src_at = ((long long)run.row + row0) * p.kv_stride[0] + ch;
    auto src_of = [&](int item) { return reinterpret_cast<const T *>(item & 1 ? p.v : p.k) + src_at + (item >> 1) * p.kv_stride[1]; };
    auto stage_of = [&](int item) { return ring + (item % (kAhead + 1)) * (kWideKeep * kThreads) + tid; };
    auto load = [&](int item) {
      if (item < item_end) {
        const T *src = src_of(item);
        uint4 *to = stage_of(item);
        if (full) {
#pragma unroll
          for (int i = 0; i < kWideKeep; ++i, src += src_step) copy16(to + i * kThreads, src);
        } else {
          for (int i = 0; i < n_keep; ++i, src += src_step) copy16(to + i * kThreads, src);
        }
      }
      copies_end();
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k) load(item0 + k);
#pragma unroll 1
    for (int item = item0; item < item_end; ++item) {
      const T *src = src_of(item);
      const int h = item >> 1;
      uint8_t *code = reinterpret_cast<uint8_t *>(item & 1 ? p.v_cache : p.k_cache) + run.code + h * p.cache_stride[1];
      uint8_t *mine_at = code + row0 * p.cache_stride[2] + ch;
      float *scale = (item & 1 ? p.v_scale : p.k_scale) + run.scale + h * p.scale_stride[1];
      const float s0 = run.held > 0 ? *scale : 0.f;
      load(item + kAhead);
      copies_wait<kAhead>();
      const uint4 *mine = stage_of(item);
      auto peak = [&](bool finite) {
        uint32_t top = 0;
        if (full) {
#pragma unroll
          for (int i = 0; i < kWideKeep; ++i) top = peak_of<T>(mine[i * kThreads], top, finite);
        } else {
#pragma unroll 1
          for (int i = 0; i < n_keep; ++i) top = peak_of<T>(mine[i * kThreads], top, finite);
        }
        for (int i = kWideKeep; i < n_mine; ++i) top = peak_of<T>(*reinterpret_cast<const uint4 *>(src + i * src_step), top, finite);
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) top_s[turn][warp] = top;
        turn ^= 1;
        __syncthreads();      // also: every thread has read the old scale; the buffer of two turns ago is read
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = max(top, top_s[turn ^ 1][w]);
        return top;
      };
      uint32_t top = peak(false);
      const bool plain = top <= kMostBits;
      if (!plain) top = peak(true);
      const Scale now = scale_of(top, run.held, s0);
      if (full && plain) {
#pragma unroll
        for (int i = 0; i < kWideKeep; ++i, mine_at += code_step) store_codes<T>(mine_at, mine[i * kThreads], now.by, true);
      } else {
#pragma unroll 1
        for (int i = 0; i < n_keep; ++i, mine_at += code_step) store_codes<T>(mine_at, mine[i * kThreads], now.by, plain);
      }
#pragma unroll 1
      for (int i = kWideKeep; i < n_mine; ++i, mine_at += code_step)
        store_codes<T>(mine_at, *reinterpret_cast<const uint4 *>(src + i * src_step), now.by, plain);
      const bool same = run.held > 0 && __float_as_uint(s0) == now.bits;
      if (run.held > 0 && !same) rescale(code - run.held * p.cache_stride[2], p.cache_stride[2], run.held, p.D, s0, now.bits, tid, kThreads);
      if (tid == 0 && !same) *scale = __uint_as_float(now.bits);
    }
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

// ---------------------------------------------------------------------------------------------------------------
struct ReadLaunch {
  int rows;      // of the output, per CTA; of one sequence when dense
  int per_seq;   // dense: CTAs of a sequence
  int items, per_cta;
  int groups;    // of threads, with heads of their own
  FastDiv page_div, block_div, chunk_div, seq_div, row_div;
};
constexpr int kReadRows = 32;

// Eight values times a scale of any bits, each rounded once: the products are cut off at 24 bits, to odd; small ones by way of 64 bits, as
// what is cut off has to be a number.  (Scales of ds_kv8_write do not come here.)
__device__ __noinline__ void store_any_scale(__nv_bfloat16 *to, uint32_t lo, uint32_t hi, float s) {
  __nv_bfloat162 v[4];
  if (fabsf(s) >= 0x1p-90f || s != s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 a = halves_f32(e & 1 ? halves_hi(e < 2 ? lo : hi) : halves_lo(e < 2 ? lo : hi));
      v[e] = __floats2bfloat162_rn(mul_to_odd(a.x, s), mul_to_odd(a.y, s));
    }
  } else {
    auto small = [&](float a) {
      const double x = (double)a * (double)s;
      const float r = __double2float_rz(x);
      return (double)r != x ? __uint_as_float(__float_as_uint(r) | 1u) : r;
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 a = halves_f32(e & 1 ? halves_hi(e < 2 ? lo : hi) : halves_lo(e < 2 ? lo : hi));
      v[e] = __floats2bfloat162_rn(small(a.x), small(a.y));
    }
  }
  *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(v);
}

template <typename T>
__device__ __forceinline__ void store_values(T *to, const uint2 &w, float s) {
  const float2 a0 = halves_f32(halves_lo(w.x)), a1 = halves_f32(halves_hi(w.x)), a2 = halves_f32(halves_lo(w.y)), a3 = halves_f32(halves_hi(w.y));
  if constexpr (std::is_same<T, float>::value) {
    reinterpret_cast<float4 *>(to)[0] = make_float4(a0.x * s, a0.y * s, a1.x * s, a1.y * s);
    reinterpret_cast<float4 *>(to)[1] = make_float4(a2.x * s, a2.y * s, a3.x * s, a3.y * s);
  } else {
    const uint32_t b = __float_as_uint(s) & 0x7fffffffu;
    // a power of two, as ds_kv8_write's are, and no product too small for fp32: exact; or nothing but zeros, whose scale is the smallest
    const bool exact = (b & 0x7fffffu) == 0 && (b >= (127u - 90u) << 23 || ((w.x | w.y) & 0x7f7f7f7fu) == 0);
    if (__builtin_expect(!exact, 0)) return store_any_scale(to, w.x, w.y, s);
    const __nv_bfloat162 v[4] = {__floats2bfloat162_rn(a0.x * s, a0.y * s), __floats2bfloat162_rn(a1.x * s, a1.y * s),
                                 __floats2bfloat162_rn(a2.x * s, a2.y * s), __floats2bfloat162_rn(a3.x * s, a3.y * s)};
    *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(v);
  }
}

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
  // A thread stays with a row and eight of its dimensions and goes through the heads, or some of them.
  const int chunks = (int)launch.chunk_div.d, side = fast_div(tid, launch.chunk_div), ch = tid - side * chunks;
  const int group = fast_div(side, launch.row_div), i = side - group * launch.rows;
  const int item0 = blockIdx.y * launch.per_cta, item_end = min(launch.items, item0 + launch.per_cta);
  if (group < launch.groups && i < n) {
    const long long code = code_s[i], scale = scale_s[i], out = out_s[i];
    if (code >= 0) {
      const uint8_t *from[2] = {reinterpret_cast<const uint8_t *>(p.k_cache) + code + 8 * ch, reinterpret_cast<const uint8_t *>(p.v_cache) + code + 8 * ch};
      const float *by[2] = {p.k_scale + scale, p.v_scale + scale};
      T *to[2] = {reinterpret_cast<T *>(p.k_out) + out + 8 * ch, reinterpret_cast<T *>(p.v_out) + out + 8 * ch};
      const int step = 2 * launch.groups;
      constexpr int kBatch = 4;      // heads whose loads are in flight
      for (int item = item0 + 2 * group; item < item_end; item += kBatch * step) {      // K and V of a head
        uint2 w[kBatch][2];
        float s[kBatch][2];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
#pragma unroll
          for (int x = 0; x < 2; ++x)
            if (item + k * step < item_end) {
              const int h = (item + k * step) >> 1;
              w[k][x] = *reinterpret_cast<const uint2 *>(from[x] + h * p.cache_stride[1]);
              s[k][x] = by[x][h * p.scale_stride[1]];
            }
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
#pragma unroll
          for (int x = 0; x < 2; ++x)
            if (item + k * step < item_end) store_values(to[x] + ((item + k * step) >> 1) * p.out_stride[2], w[k][x], s[k][x]);
      }
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
  // As many rows to a CTA as a run has, so that few CTAs find none, more where the CTAs would otherwise be many waves.
  w.per_cta = w.items < at_a_time ? w.items : at_a_time;
  const long long groups = (w.items + w.per_cta - 1) / w.per_cta, enough = 8LL * sm_count();
  w.rows = p.max_q < p.scale_block ? p.max_q : p.scale_block;
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
int launch_write_wide(const ds_kv8_write_params &p, cudaStream_t stream) {
  WriteLaunch w;
  const int cap = p.max_pages * p.page_size;
  w.bound = p.max_len > 0 && p.max_len < cap ? p.max_len : cap;
  w.items = 2 * p.Hkv;
  w.rows = p.scale_block < 64 ? p.scale_block : 64;
  const long long shares = ((long long)p.N + w.rows - 1) / w.rows;
  w.per_cta = w.items;      // the more the better: they overlap; but a CTA for every slot
  while (w.per_cta > 1 && shares * ((w.items + w.per_cta - 1) / w.per_cta) < 8LL * sm_count()) w.per_cta = (w.per_cta + 1) / 2;
  w.page_div = make_fast_div(p.page_size);
  w.block_div = make_fast_div(p.scale_block);
  w.chunk_div = make_fast_div(p.D / Chunk<T>::kElems);
  const dim3 grid((unsigned)shares, (unsigned)((w.items + w.per_cta - 1) / w.per_cta));
  constexpr int kBytes = (kAhead + 1) * kWideKeep * kThreads * 16;
  static std::atomic<unsigned long long> allowed{0};
  DS_CUDA_OK(allow_smem(kv8_write_wide_kernel<T>, kBytes, allowed));
  DS_CUDA_OK(launch_kernel(kv8_write_wide_kernel<T>, grid, kThreads, kBytes, 0, true, stream, p, w));
  note_launch(1);
  return DS_OK;
}

template <typename T>
int launch_write_lanes(const ds_kv8_write_params &p, cudaStream_t stream) {
  // lanes of an item: a run of one row should not leave most of them idle
  const long long chunks = (long long)(p.max_q < p.scale_block ? p.max_q : p.scale_block) * (p.D / Chunk<T>::kElems);
  if (chunks > 32 * kKeep) return launch_write_wide<T>(p, stream);
  return chunks <= 8 ? launch_write<T, 8>(p, stream) : chunks <= 16 ? launch_write<T, 16>(p, stream) : launch_write<T, 32>(p, stream);
}

template <typename T>
int launch_read(const ds_kv8_read_params &p, cudaStream_t stream) {
  ReadLaunch w;
  w.items = 2 * p.Hkv;
  // Rows of a CTA: what its threads hold at a time, fewer where there are few; then the heads are divided, too.  (Eight CTAs an SM rather than
  // three: 14.0 against 16.9 us for 50 sequences of fp32, nothing either way for 270 MB.)
  const long long rows = p.out_start ? p.N : (long long)p.B * p.N, enough = 8LL * sm_count();
  const int at_a_time = kThreads / (p.D / 8);
  w.rows = at_a_time < kReadRows ? at_a_time : kReadRows;      // kThreads / (D / 8) is at least 8
  while (w.rows > 1 && rows / w.rows < enough) w.rows = (w.rows + 1) / 2;
  w.per_cta = w.items;
  while (w.per_cta > 2 && rows / w.rows * (w.items / w.per_cta) < enough) w.per_cta = (w.per_cta / 2 + 1) / 2 * 2;
  w.groups = at_a_time / w.rows;
  w.row_div = make_fast_div(w.rows);
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

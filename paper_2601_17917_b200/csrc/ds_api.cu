// C ABI of the denoising-step library: argument validation and dispatch.
// Every step of the path runs in the CUDA kernels of the sibling files.
#include <atomic>
#include <cmath>
#include <new>

#include "ds_common.cuh"
#include "ds_paged_index.cuh"

namespace ds {

static std::atomic<long long> g_launches{0};
void note_launch(int n) { g_launches.fetch_add(n, std::memory_order_relaxed); }
thread_local int g_last_cuda_error = 0;
void note_cuda_error(int code) { g_last_cuda_error = code; }

int sm_count() {
  static int cached[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  if (cached[dev] == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
    cached[dev] = n;
  }
  return cached[dev];
}

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int validate_attn(const ds_attn_params *p) {
  if (!p) return DS_ERR_INVALID_ARG;
  if (p->dtype != DS_F32 && p->dtype != DS_BF16) return DS_ERR_INVALID_ARG;
  if (p->B < 0 || p->Hq <= 0 || p->Hkv <= 0 || p->D <= 0 || p->P < 0 || p->T <= 0) return DS_ERR_INVALID_ARG;
  if (p->Hq % p->Hkv != 0) return DS_ERR_INVALID_ARG;
  if (p->Lq < 1 || p->Lq > p->T) return DS_ERR_INVALID_ARG;
  if (!p->q_tail || !p->k_tail || !p->v_tail || !p->idx || !p->out) return DS_ERR_INVALID_ARG;
  if (p->P > 0 && (!p->k_prefix || !p->v_prefix)) return DS_ERR_INVALID_ARG;
  if (p->idx_batch_stride != 0 && p->idx_batch_stride < p->Lq) return DS_ERR_INVALID_ARG;
  if (!(p->scale == p->scale)) return DS_ERR_INVALID_ARG;
  if (p->seq_list && (p->n_seq < 0 || p->n_seq > p->B || !aligned(p->seq_list, 4) ||
                      (p->n_seq_dev && !aligned(p->n_seq_dev, 4))))
    return DS_ERR_INVALID_ARG;
  const int64_t unit = (p->dtype == DS_BF16) ? 8 : 4;  // 16 bytes
  const void *ptrs[] = {p->q_tail, p->k_tail, p->v_tail, p->out, p->P > 0 ? p->k_prefix : nullptr,
                        p->P > 0 ? p->v_prefix : nullptr};
  for (const void *q : ptrs)
    if (q && !aligned(q, 16)) return DS_ERR_INVALID_ARG;
  if (!aligned(p->idx, 4) || (p->lse && !aligned(p->lse, 4)) || (p->status && !aligned(p->status, 4)))
    return DS_ERR_INVALID_ARG;
  const int64_t *strides[] = {p->q_stride, p->kv_tail_stride, p->out_stride, p->kv_prefix_stride};
  for (int k = 0; k < 4; ++k) {
    if (k == 3 && p->P == 0) continue;
    for (int d = 0; d < 3; ++d) {
      const int64_t s = strides[k][d];
      if (s < 0 || s % unit != 0) return DS_ERR_INVALID_ARG;
    }
    if (strides[k][2] < p->D) return DS_ERR_INVALID_ARG;  // rows must not overlap
  }
  if (p->kernel != DS_ATTN_KERNEL_AUTO && p->kernel != DS_ATTN_KERNEL_ONE_TILE && p->kernel != DS_ATTN_KERNEL_TWO_TILE)
    return DS_ERR_INVALID_ARG;
  // The envelope: bf16 on the tensor cores, fp32 on the CUDA cores; nothing is rerouted.
  if (p->B > 65535 || p->Hq > 65535) return DS_ERR_UNSUPPORTED;
  if (p->dtype == DS_BF16) return attn_tc_supported(*p) ? DS_OK : DS_ERR_UNSUPPORTED;
  if (p->D != 32 && p->D != 64 && p->D != 128 && p->D != 256) return DS_ERR_UNSUPPORTED;
  if (!(p->scale > -1e30f && p->scale < 1e30f)) return DS_ERR_UNSUPPORTED;
  return DS_OK;
}

constexpr int kMaxScaleBlock = 65536;

// Strides of the paged-cache entry points: non-negative multiples of 16 bytes.
bool strides_ok(const int64_t *s, int n, int64_t unit) {
  for (int d = 0; d < n; ++d)
    if (s[d] < 0 || s[d] % unit != 0) return false;
  return true;
}

int validate_pages(const ds_page_params *p) {
  if (!p) return DS_ERR_INVALID_ARG;
  if (p->B < 0 || p->max_rows < 0 || p->page_size < 1 || p->max_pages < 1 || p->n_pages < 1) return DS_ERR_INVALID_ARG;
  if (!p->free_list || !p->free_cnt || !p->free_cnt_out || !p->row_start) return DS_ERR_INVALID_ARG;
  if (p->B > 0 && (!p->kv_len || !p->n_new || !p->block_table || !p->kv_len_out)) return DS_ERR_INVALID_ARG;
  if (p->table_stride < p->max_pages) return DS_ERR_INVALID_ARG;
  const void *words[] = {p->kv_len, p->n_new, p->block_table, p->free_list, p->free_cnt, p->kv_len_out, p->free_cnt_out,
                         p->row_start, p->positions, p->status};
  for (const void *w : words)
    if (!aligned(w, 4)) return DS_ERR_INVALID_ARG;
  if (!aligned(p->slot_map, 8)) return DS_ERR_INVALID_ARG;
  if (p->B > 8192 || (int64_t)p->max_pages * p->page_size > 0x7fffffffLL || (int64_t)p->n_pages * p->page_size > 0x7fffffffLL)
    return DS_ERR_UNSUPPORTED;
  return DS_OK;
}

int validate_qk(const ds_qk_params *p) {
  if (!p || !p->rope) return DS_ERR_INVALID_ARG;
  if (p->dtype != DS_F32 && p->dtype != DS_BF16) return DS_ERR_INVALID_ARG;
  if (p->N < 0 || p->Hq <= 0 || p->Hkv <= 0 || p->D <= 0 || !(p->eps >= 0.f)) return DS_ERR_INVALID_ARG;
  if (p->rope->rotary_dim < 2 || p->rope->rotary_dim % 2 != 0) return DS_ERR_INVALID_ARG;
  const bool cache = p->k_cache || p->v_cache;
  if (p->N > 0) {
    if (!p->q || !p->k || !p->v || !p->positions || !p->q_out) return DS_ERR_INVALID_ARG;
    if ((p->k_out == nullptr) != (p->v_out == nullptr) || (p->k_cache == nullptr) != (p->v_cache == nullptr))
      return DS_ERR_INVALID_ARG;
    if (cache && (!p->slot_map || p->page_size < 1 || p->n_pages < 1)) return DS_ERR_INVALID_ARG;
  }
  const void *ptrs[] = {p->q, p->k, p->v, p->q_weight, p->k_weight, p->q_out, p->k_out, p->v_out, p->k_cache, p->v_cache};
  for (const void *q : ptrs)
    if (!aligned(q, 16)) return DS_ERR_INVALID_ARG;
  if (!aligned(p->positions, 4) || !aligned(p->n_rows, 4) || !aligned(p->status, 4) || !aligned(p->slot_map, 8))
    return DS_ERR_INVALID_ARG;
  const int64_t unit = p->dtype == DS_BF16 ? 8 : 4;
  if (!strides_ok(p->q_stride, 2, unit) || !strides_ok(p->kv_stride, 2, unit) || !strides_ok(p->q_out_stride, 2, unit))
    return DS_ERR_INVALID_ARG;
  if (p->k_out && !strides_ok(p->kv_out_stride, 2, unit)) return DS_ERR_INVALID_ARG;
  if (cache && !strides_ok(p->cache_stride, 3, unit)) return DS_ERR_INVALID_ARG;
  if (p->D % 16 != 0 || p->D > 256 || p->rope->rotary_dim % 16 != 0 || p->rope->rotary_dim > p->D) return DS_ERR_UNSUPPORTED;
  if (cache && (int64_t)p->n_pages * p->page_size > 0x7fffffffLL) return DS_ERR_UNSUPPORTED;
  return DS_OK;
}

// `unit`: elements of the cache in 16 bytes.
int validate_paged_but_envelope(const ds_paged_params *p, int64_t unit_cache) {
  if (!p) return DS_ERR_INVALID_ARG;
  if (p->dtype != DS_F32 && p->dtype != DS_BF16) return DS_ERR_INVALID_ARG;
  if (p->B < 0 || p->Hq <= 0 || p->Hkv <= 0 || p->D <= 0 || p->N < 0 || p->max_q < 1 || p->max_len < 0) return DS_ERR_INVALID_ARG;
  if (p->page_size < 1 || p->max_pages < 1 || p->n_pages < 1 || p->window < 0 || p->sinks < 0) return DS_ERR_INVALID_ARG;
  if (p->Hq % p->Hkv != 0 || !std::isfinite(p->scale) || p->table_stride < p->max_pages) return DS_ERR_INVALID_ARG;
  if (!p->row_start && (int64_t)p->B * p->max_q > p->N) return DS_ERR_INVALID_ARG;
  if (p->B > 0 && p->N > 0 && (!p->kv_len || !p->block_table || !p->q || !p->k_cache || !p->v_cache || !p->out))
    return DS_ERR_INVALID_ARG;
  const void *ptrs[] = {p->q, p->k_cache, p->v_cache, p->out};
  for (const void *q : ptrs)
    if (!aligned(q, 16)) return DS_ERR_INVALID_ARG;
  const void *words[] = {p->row_start, p->kv_len, p->block_table, p->lse, p->status};
  for (const void *w : words)
    if (!aligned(w, 4)) return DS_ERR_INVALID_ARG;
  const int64_t unit = p->dtype == DS_BF16 ? 8 : 4;
  if (!strides_ok(p->q_stride, 2, unit) || !strides_ok(p->cache_stride, 3, unit_cache) || !strides_ok(p->out_stride, 2, unit))
    return DS_ERR_INVALID_ARG;
  return DS_OK;
}

// Sizes that the kernels count in 32 bits.
bool paged_sizes_ok(const ds_paged_params *p) {
  const int64_t rows = (int64_t)p->max_q * (p->Hq / p->Hkv), cap = (int64_t)p->max_pages * p->page_size;
  const int64_t len = p->max_len > 0 && p->max_len < cap ? p->max_len : cap;
  return p->B <= 8192 && cap <= 0x7fffffffLL && len <= kPagedMaxLen && (int64_t)p->n_pages * p->page_size <= 0x7fffffffLL && rows <= 0x3fffffffLL;
}

int validate_paged(const ds_paged_params *p) {
  const int rc = validate_paged_but_envelope(p, p && p->dtype == DS_BF16 ? 8 : 4);
  if (rc != DS_OK) return rc;
  const bool d_ok = p->dtype == DS_BF16 ? (p->D == 64 || p->D == 128) : (p->D == 32 || p->D == 64 || p->D == 128 || p->D == 256);
  // the kernels count a sequence's rows and its units of work in 32 bits
  if (!d_ok || !paged_sizes_ok(p) || !attn_paged_counts_fit(*p)) return DS_ERR_UNSUPPORTED;
  return DS_OK;
}

// The scales of an 8-bit cache.
int validate_scales(int32_t scale_block, int32_t page_size, const float *k_scale, const float *v_scale, const int64_t *stride) {
  if (scale_block < 1 || page_size % scale_block != 0) return DS_ERR_INVALID_ARG;
  if (!aligned(k_scale, 4) || !aligned(v_scale, 4) || !strides_ok(stride, 3, 1)) return DS_ERR_INVALID_ARG;
  return DS_OK;
}

int validate_paged8(const ds_paged8_params *p) {
  const int rc = validate_paged_but_envelope(p ? &p->a : nullptr, 16);
  if (rc != DS_OK) return rc;
  if (p->a.B > 0 && p->a.N > 0 && (!p->k_scale || !p->v_scale)) return DS_ERR_INVALID_ARG;
  const int rs = validate_scales(p->scale_block, p->a.page_size, p->k_scale, p->v_scale, p->scale_stride);
  if (rs != DS_OK) return rs;
  if ((p->a.D != 64 && p->a.D != 128) || p->scale_block > kMaxScaleBlock || !paged_sizes_ok(&p->a) || !attn_paged8_counts_fit(*p))
    return DS_ERR_UNSUPPORTED;
  return DS_OK;
}

// What ds_kv8_write and ds_kv8_read have in common; `rows`, `rows_stride`: the packed K and V.
template <class P>
int validate_kv8(const P *p, const void *k, const void *v, const int64_t *rows_stride, int n_strides, const int32_t *starts) {
  if (p->dtype != DS_F32 && p->dtype != DS_BF16) return DS_ERR_INVALID_ARG;
  if (p->B < 0 || p->Hkv < 1 || p->D < 1 || p->N < 0 || p->page_size < 1 || p->max_pages < 1 || p->n_pages < 1) return DS_ERR_INVALID_ARG;
  if (p->table_stride < p->max_pages) return DS_ERR_INVALID_ARG;
  const int rs = validate_scales(p->scale_block, p->page_size, p->k_scale, p->v_scale, p->scale_stride);
  if (rs != DS_OK) return rs;
  if (p->B > 0 && p->N > 0 && (!p->kv_len || !p->block_table || !k || !v || !p->k_cache || !p->v_cache || !p->k_scale || !p->v_scale))
    return DS_ERR_INVALID_ARG;
  const void *ptrs[] = {k, v, p->k_cache, p->v_cache};
  for (const void *q : ptrs)
    if (!aligned(q, 16)) return DS_ERR_INVALID_ARG;
  const void *words[] = {starts, p->kv_len, p->block_table, p->status};
  for (const void *w : words)
    if (!aligned(w, 4)) return DS_ERR_INVALID_ARG;
  if (!strides_ok(rows_stride, n_strides, p->dtype == DS_BF16 ? 8 : 4) || !strides_ok(p->cache_stride, 3, 16)) return DS_ERR_INVALID_ARG;
  if (p->D % 16 != 0 || p->D > 256 || p->B > 8192 || p->Hkv > 32767 || p->scale_block > kMaxScaleBlock ||
      (int64_t)p->max_pages * p->page_size > 0x7fffffffLL || (int64_t)p->n_pages * p->page_size > 0x7fffffffLL)
    return DS_ERR_UNSUPPORTED;
  return DS_OK;
}

int validate_kv8_write(const ds_kv8_write_params *p) {
  if (!p || p->max_q < 1 || p->max_len < 0) return DS_ERR_INVALID_ARG;
  if (!p->row_start && (int64_t)p->B * p->max_q > p->N) return DS_ERR_INVALID_ARG;
  return validate_kv8(p, p->k, p->v, p->kv_stride, 2, p->row_start);
}

int validate_kv8_read(const ds_kv8_read_params *p) {
  if (!p || !aligned(p->first, 4)) return DS_ERR_INVALID_ARG;
  const int64_t *strides = p->out_start ? p->out_stride + 1 : p->out_stride;
  const int rc = validate_kv8(p, p->k_out, p->v_out, strides, p->out_start ? 2 : 3, p->out_start);
  if (rc != DS_OK) return rc;
  return p->out_start || (int64_t)p->B * p->N <= 0x7fffffffLL ? DS_OK : DS_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace ds

extern "C" {

size_t ds_attn_pruned_workspace(const ds_attn_params *p) {
  if (ds::validate_attn(p) != DS_OK) return 0;
  // only the one-tile kernel splits the keys of an item over CTAs
  if (p->dtype == DS_BF16 && p->kernel != DS_ATTN_KERNEL_TWO_TILE) return ds::attn_tc_workspace_bytes(*p);
  return 0;
}

namespace ds {
namespace {
// Several M-tiles per KV head (wide windows, the unpruned reference, a cache-refresh step): the two-tile
// kernel fetches every KV tile once for a pair of M-tiles and keeps the softmax warps busy on one tile while
// the tensor pipe works for the other.  Measured per work item it costs about 1.88 single tiles for a full pair
// and 1.10 for a pair with one tile (which alternates between the two S buffers like the one-tile kernel), so it
// pays when the number of rounds over the SMs does not grow.
bool two_tile_kernel_pays(const ds_attn_params &p) {
  const long long rows = (long long)(p.Hq / p.Hkv) * p.Lq;
  const long long n_full = rows / 128, rem = rows % 128;
  // the one-tile kernel serves a remainder of up to 8 rows together with the last full tile
  const long long n_mt1 = (p.D == 128 && n_full >= 1 && rem >= 1 && rem <= 8) ? n_full : n_full + (rem ? 1 : 0);
  const long long n_mt = n_full + (rem ? 1 : 0), n_pr = (n_mt + 1) / 2;
  if (n_mt < 2) return false;
  const long long heads = (long long)(p.seq_list ? p.n_seq : p.B) * p.Hkv, sms = sm_count();
  const double rounds1 = (double)((heads * n_mt1 + sms - 1) / sms);
  const double rounds2 = (double)((heads * n_pr + sms - 1) / sms);
  const double pair_cost = (1.88 * (double)(n_mt / 2) + 1.10 * (double)(n_mt % 2)) / (double)n_pr;
  return rounds2 * pair_cost < 0.97 * rounds1;
}

// Validation, choice of the kernel and its parameters for one set of arguments.
int resolve_attn(const ds_attn_params *p, AttnPrepared &a) {
  const int rc = validate_attn(p);
  if (rc != DS_OK) return rc;
  a.p = *p;
  a.grid = 0;
  a.path = kAttnPathSimt;
  if (p->B == 0) return DS_OK;
  if (p->dtype == DS_BF16) {
    if (p->kernel == DS_ATTN_KERNEL_TWO_TILE) return prepare_attn_tc2(*p, a);
    if (p->kernel == DS_ATTN_KERNEL_AUTO && two_tile_kernel_pays(*p)) return prepare_attn_tc2(*p, a);
    // a missing or short workspace is not an error: the call then runs without splitting the keys
    return prepare_attn_tc(*p, a);
  }
  a.grid = 1;  // the fp32 launcher sizes its own grid from a.p
  return DS_OK;
}

int launch_resolved(const AttnPrepared &a, cudaStream_t st) {
  if (a.p.B == 0) return DS_OK;
  switch (a.path) {
    case kAttnPathTc: return launch_prepared_tc(a, st);
    case kAttnPathTc2: return launch_prepared_tc2(a, st);
    default: return launch_attn_simt(a.p, st);
  }
}
}  // namespace
}  // namespace ds

struct ds_attn_plan {
  ds::AttnPrepared a;
};

int ds_attn_pruned(const ds_attn_params *p, void *stream) {
  ds::AttnPrepared a;
  const int rc = ds::resolve_attn(p, a);
  if (rc != DS_OK) return rc;
  return ds::launch_resolved(a, reinterpret_cast<cudaStream_t>(stream));
}

int ds_attn_plan_create(const ds_attn_params *p, ds_attn_plan **plan) {
  if (!plan) return DS_ERR_INVALID_ARG;
  *plan = nullptr;
  ds_attn_plan *pl = new (std::nothrow) ds_attn_plan;
  if (!pl) return DS_ERR_CUDA;
  const int rc = ds::resolve_attn(p, pl->a);
  if (rc != DS_OK) {
    delete pl;
    return rc;
  }
  *plan = pl;
  return DS_OK;
}

int ds_attn_plan_launch(const ds_attn_plan *plan, void *stream) {
  if (!plan) return DS_ERR_INVALID_ARG;
  return ds::launch_resolved(plan->a, reinterpret_cast<cudaStream_t>(stream));
}

void ds_attn_plan_destroy(ds_attn_plan *plan) { delete plan; }

size_t ds_confidence_workspace(int64_t rows, int64_t V, int32_t dtype) {
  if (dtype != DS_F32 && dtype != DS_BF16) return 0;
  return ds::confidence_workspace_bytes(rows, V, dtype);
}

int ds_confidence(const void *logits, int32_t dtype, int64_t rows, int64_t V, int64_t ld,
                  const int32_t *row_list, int64_t n_listed, float *conf, int32_t *tok, void *workspace,
                  size_t workspace_bytes, void *stream) {
  if (dtype != DS_F32 && dtype != DS_BF16) return DS_ERR_INVALID_ARG;
  if (rows < 0 || V <= 0 || ld < V || V > 0x7fffffffLL) return DS_ERR_INVALID_ARG;
  if (rows == 0) return DS_OK;
  if (!logits || !conf || !tok) return DS_ERR_INVALID_ARG;
  const size_t esz = dtype == DS_BF16 ? 2 : 4;
  if (!ds::aligned(logits, esz) || !ds::aligned(conf, 4) || !ds::aligned(tok, 4)) return DS_ERR_INVALID_ARG;
  if (row_list && (n_listed < 0 || n_listed > rows)) return DS_ERR_INVALID_ARG;
  return ds::launch_confidence(logits, dtype, rows, V, ld, row_list, n_listed, nullptr, conf, tok, workspace,
                               workspace_bytes, reinterpret_cast<cudaStream_t>(stream));
}

int ds_confidence_listed(const void *logits, int32_t dtype, int64_t rows, int64_t V, int64_t ld,
                         const int32_t *row_list, int64_t n_listed_max, const int32_t *n_listed_dev, float *conf,
                         int32_t *tok, void *workspace, size_t workspace_bytes, void *stream) {
  if (dtype != DS_F32 && dtype != DS_BF16) return DS_ERR_INVALID_ARG;
  if (rows < 0 || V <= 0 || ld < V || V > 0x7fffffffLL) return DS_ERR_INVALID_ARG;
  if (!row_list || !n_listed_dev || n_listed_max < 0 || n_listed_max > rows) return DS_ERR_INVALID_ARG;
  if (rows == 0 || n_listed_max == 0) return DS_OK;
  if (!logits || !conf || !tok) return DS_ERR_INVALID_ARG;
  const size_t esz = dtype == DS_BF16 ? 2 : 4;
  if (!ds::aligned(logits, esz) || !ds::aligned(conf, 4) || !ds::aligned(tok, 4) || !ds::aligned(n_listed_dev, 4))
    return DS_ERR_INVALID_ARG;
  return ds::launch_confidence(logits, dtype, rows, V, ld, row_list, n_listed_max, n_listed_dev, conf, tok, workspace,
                               workspace_bytes, reinterpret_cast<cudaStream_t>(stream));
}

int ds_rope_gather(const ds_rope_params *p, void *stream) {
  if (!p) return DS_ERR_INVALID_ARG;
  if (p->B < 0 || p->Hq <= 0 || p->Hkv <= 0 || p->D <= 0 || p->T <= 0 || p->Lq < 0 || p->Lq > p->T) return DS_ERR_INVALID_ARG;
  if (p->pos_offset < 0 || !(p->rope_theta > 1.0f) || p->n_append < 0 || p->n_append > p->Lq || p->cache_row0 < 0)
    return DS_ERR_INVALID_ARG;
  if (p->D % 16 != 0) return DS_ERR_UNSUPPORTED;
  if (p->B == 0 || p->Lq == 0) return DS_OK;
  if (!p->q_raw || !p->k_raw || !p->v_raw || !p->idx || !p->q_out || !p->k_out || !p->v_out) return DS_ERR_INVALID_ARG;
  if (p->n_append > 0 && (!p->k_cache || !p->v_cache)) return DS_ERR_INVALID_ARG;
  if (p->idx_batch_stride != 0 && p->idx_batch_stride < p->Lq) return DS_ERR_INVALID_ARG;
  const void *ptrs[] = {p->q_raw, p->k_raw, p->v_raw, p->q_out, p->k_out, p->v_out, p->n_append ? p->k_cache : nullptr,
                        p->n_append ? p->v_cache : nullptr};
  for (const void *q : ptrs)
    if (q && !ds::aligned(q, 16)) return DS_ERR_INVALID_ARG;
  const int64_t *strides[] = {p->q_stride, p->kv_stride, p->q_out_stride, p->kv_out_stride, p->cache_stride};
  for (int k = 0; k < 5; ++k) {
    if (k == 4 && p->n_append == 0) continue;
    for (int d = 0; d < 3; ++d)
      if (strides[k][d] < 0 || strides[k][d] % 8 != 0) return DS_ERR_INVALID_ARG;
    if (strides[k][2] < p->D) return DS_ERR_INVALID_ARG;
  }
  return ds::launch_rope_gather(*p, reinterpret_cast<cudaStream_t>(stream));
}

size_t ds_lmhead_confidence_workspace(int64_t rows, int64_t V) { return ds::lmhead_workspace_bytes(rows, V); }

int ds_lmhead_confidence(const void *hidden, const void *weight, int64_t rows, int64_t hid, int64_t V, int64_t ld_h,
                         int64_t ld_w, float *conf, int32_t *tok, void *workspace, size_t workspace_bytes,
                         uint32_t *status, void *stream) {
  if (rows < 0 || hid <= 0 || V <= 0 || ld_h < hid || ld_w < hid) return DS_ERR_INVALID_ARG;
  if (rows > 0x7fffffffLL || V > 0x7fffffffLL || hid > 0x7fffffffLL) return DS_ERR_INVALID_ARG;
  if (rows == 0) return DS_OK;
  if (!hidden || !weight || !conf || !tok) return DS_ERR_INVALID_ARG;
  if (!ds::aligned(hidden, 16) || !ds::aligned(weight, 16) || !ds::aligned(conf, 4) || !ds::aligned(tok, 4) ||
      (status && !ds::aligned(status, 4)))
    return DS_ERR_INVALID_ARG;
  if (hid % 8 != 0 || ld_h % 8 != 0 || ld_w % 8 != 0) return DS_ERR_INVALID_ARG;
  const size_t need = ds::lmhead_workspace_bytes(rows, V);
  if (!workspace || !ds::aligned(workspace, 256) || workspace_bytes < need) return DS_ERR_WORKSPACE;
  return ds::launch_lmhead_confidence(hidden, weight, rows, hid, V, ld_h, ld_w, conf, tok, workspace, status,
                                      reinterpret_cast<cudaStream_t>(stream));
}

int ds_confidence_static(const void *logits, int32_t dtype, int64_t rows, int64_t V, int64_t ld,
                         const int32_t *row_list, int64_t n_listed, float *conf, int32_t *tok, void *stream) {
  if (dtype != DS_F32 && dtype != DS_BF16) return DS_ERR_INVALID_ARG;
  if (rows < 0 || V <= 0 || ld < V || V > 0x7fffffffLL) return DS_ERR_INVALID_ARG;
  if (rows == 0) return DS_OK;
  if (!logits || !conf || !tok) return DS_ERR_INVALID_ARG;
  const size_t esz = dtype == DS_BF16 ? 2 : 4;
  if (!ds::aligned(logits, esz) || !ds::aligned(conf, 4) || !ds::aligned(tok, 4)) return DS_ERR_INVALID_ARG;
  if (row_list && (n_listed < 0 || n_listed > rows)) return DS_ERR_INVALID_ARG;
  return ds::launch_confidence_static(logits, dtype, rows, V, ld, row_list, n_listed, conf, tok,
                                      reinterpret_cast<cudaStream_t>(stream));
}

int ds_unmask_select(const ds_select_params *p, void *stream) {
  if (!p) return DS_ERR_INVALID_ARG;
  if (p->B < 0 || p->K < 1 || p->K > 4096 || p->ratio_extra < 0) return DS_ERR_INVALID_ARG;
  if (!(p->tau0 == p->tau0) || !(p->alpha == p->alpha) || !(p->eos_tau == p->eos_tau)) return DS_ERR_INVALID_ARG;
  if (!p->active_cnt) return DS_ERR_INVALID_ARG;
  if (p->B > 0 && (!p->conf || !p->tok || !p->masked || !p->x_block || !p->sel_idx || !p->sel_cnt ||
                   !p->block_done || !p->eos_exit || !p->active_seq))
    return DS_ERR_INVALID_ARG;
  if (p->seq_list && (p->n_seq < 0 || p->n_seq > p->B)) return DS_ERR_INVALID_ARG;
  if (!p->seq_list && p->n_seq_dev) return DS_ERR_INVALID_ARG;
  if (p->masked_rows && !p->masked_cnt) return DS_ERR_INVALID_ARG;
  if ((long long)p->B * p->K > 0x7fffffffLL) return DS_ERR_UNSUPPORTED;
  return ds::launch_select(*p, reinterpret_cast<cudaStream_t>(stream));
}

int ds_block_begin(const ds_block_params *p, void *stream) {
  if (!p) return DS_ERR_INVALID_ARG;
  if (p->B < 0 || p->K < 1 || p->K > 4096) return DS_ERR_INVALID_ARG;
  if (!p->active_cnt || (p->masked_rows == nullptr) != (p->masked_cnt == nullptr)) return DS_ERR_INVALID_ARG;
  if ((long long)p->B * p->K > 0x7fffffffLL) return DS_ERR_UNSUPPORTED;
  if (p->B > 0 && (!p->eos_exit || !p->masked || !p->x_block || !p->active_seq)) return DS_ERR_INVALID_ARG;
  return ds::launch_block_begin(*p, reinterpret_cast<cudaStream_t>(stream));
}

int ds_page_update(const ds_page_params *p, void *stream) {
  const int rc = ds::validate_pages(p);
  if (rc != DS_OK) return rc;
  return ds::launch_page_update(*p, reinterpret_cast<cudaStream_t>(stream));
}

int ds_rope_table_init(ds_rope_table *t, int32_t rotary_dim, int32_t interleaved, double theta, int32_t scaling,
                       double factor, double orig_len, double beta_fast, double beta_slow) {
  if (!t || rotary_dim < 2 || rotary_dim % 2 != 0 || !(theta > 1.0) || !std::isfinite(theta)) return DS_ERR_INVALID_ARG;
  if (scaling < DS_ROPE_NONE || scaling > DS_ROPE_YARN) return DS_ERR_INVALID_ARG;
  if (scaling != DS_ROPE_NONE && (!(factor > 0.0) || !std::isfinite(factor))) return DS_ERR_INVALID_ARG;
  if (scaling == DS_ROPE_YARN && (!(orig_len >= 1.0) || !std::isfinite(orig_len) || !(beta_slow > 0.0) ||
                                  !(beta_fast > beta_slow) || !std::isfinite(beta_fast)))
    return DS_ERR_INVALID_ARG;
  if (rotary_dim > 256 || rotary_dim % 16 != 0) return DS_ERR_UNSUPPORTED;
  const long double R = rotary_dim, two_pi = 6.283185307179586476925286766559L;
  long double base = theta;
  if (scaling == DS_ROPE_NTK) base *= std::pow((long double)factor, R / (R - 2));
  long double lo = 0, hi = 0;
  if (scaling == DS_ROPE_YARN) {
    const long double per_e = R / (2 * std::log((long double)theta));
    lo = std::floor(per_e * std::log(orig_len / (beta_fast * two_pi)));
    hi = std::ceil(per_e * std::log(orig_len / (beta_slow * two_pi)));
    lo = lo > 0 ? lo : 0;
    hi = hi < R - 1 ? hi : R - 1;
  }
  t->rotary_dim = rotary_dim;
  t->interleaved = interleaved != 0;
  t->mscale = scaling == DS_ROPE_YARN && factor > 1.0 ? (float)(0.1L * std::log((long double)factor) + 1.0L) : 1.0f;
  t->reserved = 0;
  for (int d = 0; d < 128; ++d) {
    t->turn[d] = 0;
    if (d >= rotary_dim / 2) continue;
    long double f = std::pow(base, -2.0L * d / R);
    if (scaling == DS_ROPE_LINEAR) f /= factor;
    if (scaling == DS_ROPE_YARN) {
      const long double width = hi - lo > 1e-3L ? hi - lo : 1e-3L;
      long double ramp = (d - lo) / width;
      ramp = ramp < 0 ? 0 : ramp > 1 ? 1 : ramp;
      f = f * (1 - ramp) + f / factor * ramp;
    }
    long double turn = f / two_pi;
    turn -= std::floor(turn);
    // 64 fraction bits; a fraction that rounds up to a whole turn is no turn
    const long double bits = std::floor(turn * 18446744073709551616.0L + 0.5L);
    t->turn[d] = bits >= 18446744073709551616.0L ? 0 : (uint64_t)bits;
  }
  return DS_OK;
}

int ds_qk_norm_rope(const ds_qk_params *p, void *stream) {
  const int rc = ds::validate_qk(p);
  if (rc != DS_OK) return rc;
  return p->N == 0 ? (int)DS_OK : ds::launch_qk_norm_rope(*p, reinterpret_cast<cudaStream_t>(stream));
}

size_t ds_attn_paged_workspace(const ds_paged_params *p) {
  return ds::validate_paged(p) == DS_OK ? ds::attn_paged_workspace_bytes(*p) : 0;
}

int ds_attn_paged(const ds_paged_params *p, void *stream) {
  const int rc = ds::validate_paged(p);
  if (rc != DS_OK) return rc;
  if (p->B == 0 || p->N == 0) return DS_OK;
  return ds::launch_attn_paged(*p, reinterpret_cast<cudaStream_t>(stream));
}

int ds_kv8_write(const ds_kv8_write_params *p, void *stream) {
  const int rc = ds::validate_kv8_write(p);
  if (rc != DS_OK) return rc;
  if (p->B == 0 || p->N == 0) return DS_OK;
  return ds::launch_kv8_write(*p, reinterpret_cast<cudaStream_t>(stream));
}

int ds_kv8_read(const ds_kv8_read_params *p, void *stream) {
  const int rc = ds::validate_kv8_read(p);
  if (rc != DS_OK) return rc;
  if (p->B == 0 || p->N == 0) return DS_OK;
  return ds::launch_kv8_read(*p, reinterpret_cast<cudaStream_t>(stream));
}

size_t ds_attn_paged8_workspace(const ds_paged8_params *p) {
  return ds::validate_paged8(p) == DS_OK ? ds::attn_paged8_workspace_bytes(*p) : 0;
}

int ds_attn_paged8(const ds_paged8_params *p, void *stream) {
  const int rc = ds::validate_paged8(p);
  if (rc != DS_OK) return rc;
  if (p->a.B == 0 || p->a.N == 0) return DS_OK;
  return ds::launch_attn_paged8(*p, reinterpret_cast<cudaStream_t>(stream));
}

int ds_selftest_bounded_wait(uint32_t poll_limit, uint32_t *status, int32_t *report, void *stream) {
  if (poll_limit == 0 || poll_limit > (1u << 16)) return DS_ERR_INVALID_ARG;
  if ((status && !ds::aligned(status, 4)) || (report && !ds::aligned(report, 4))) return DS_ERR_INVALID_ARG;
  return ds::launch_bounded_wait_selftest(poll_limit, status, report, reinterpret_cast<cudaStream_t>(stream));
}

int ds_last_cuda_error(void) { return ds::g_last_cuda_error; }
const char *ds_last_cuda_error_name(void) {
  return cudaGetErrorName(static_cast<cudaError_t>(ds::g_last_cuda_error));
}

int ds_read_status(const uint32_t *device_status, void *stream, uint32_t *host_out) {
  if (!device_status || !host_out) return DS_ERR_INVALID_ARG;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  DS_CUDA_OK(cudaMemcpyAsync(host_out, device_status, sizeof(uint32_t), cudaMemcpyDeviceToHost, st));
  DS_CUDA_OK(cudaStreamSynchronize(st));
  return DS_OK;
}

const char *ds_strerror(int code) {
  switch (code) {
    case DS_OK: return "ok";
    case DS_ERR_INVALID_ARG: return "invalid argument";
    case DS_ERR_UNSUPPORTED: return "shape or type outside the kernels' envelope";
    case DS_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case DS_ERR_CUDA: return "CUDA call failed";
    case DS_ERR_STATIC_LIMIT:
      return "request exceeds the fixed scratch of the allocation-free entry point (too many rows)";
    default: return "unknown status";
  }
}

int ds_version(void) { return 1000; }

int64_t ds_launch_count(void) { return ds::g_launches.load(std::memory_order_relaxed); }

}  // extern "C"

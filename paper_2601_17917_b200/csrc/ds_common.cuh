// Shared host/device helpers of the sm_100a denoising-step library.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "ds.h"

namespace ds {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Count of kernels launched through the C ABI (read by ds_launch_count()).
void note_launch(int n = 1);

inline int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// Number of SMs of the current device (cached per device).
int sm_count();

#define DS_CUDA_OK(expr)                          \
  do {                                            \
    cudaError_t _e = (expr);                      \
    if (_e != cudaSuccess) {                      \
      (void)cudaGetLastError();                   \
      ::ds::note_cuda_error((int)_e);             \
      return DS_ERR_CUDA;                         \
    }                                             \
  } while (0)

// Programmatic dependent launch, for the short kernels of the paged cache: one launched with `dependent` may be set up
// while the previous kernel in the stream still runs.  dependent_sync() comes before its first access to memory: it returns
// when everything before it in the stream is done; the next kernel may then be set up in turn.
__device__ __forceinline__ void dependent_sync() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// Raises the limit of a kernel's dynamic shared memory, once per device and kernel (`done`: a static of the caller's).
template <class K>
cudaError_t allow_smem(K *kernel, int bytes, std::atomic<unsigned long long> &done) {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
  const cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (rc == cudaSuccess && dev < 64) done.fetch_or(bit, std::memory_order_release);
  return rc;
}
// Launches a kernel, on clusters of so many CTAs (0: none).
template <class... P, class... A>
cudaError_t launch_kernel(void (*kernel)(P...), dim3 grid, int threads, size_t smem, int cluster, bool dependent,
                          cudaStream_t stream, A... args) {
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (dependent) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 0) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = cluster;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

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
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float bf16lo_to_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16hi_to_f32(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Launchers implemented in the per-kernel translation units.
int launch_confidence(const void *logits, int dtype, int64_t rows, int64_t V, int64_t ld,
                      const int32_t *row_list, int64_t n_listed, const int32_t *n_listed_dev, float *conf,
                      int32_t *tok, void *workspace, size_t workspace_bytes, cudaStream_t stream);
size_t confidence_workspace_bytes(int64_t rows, int64_t V, int dtype);
int launch_confidence_static(const void *logits, int dtype, int64_t rows, int64_t V, int64_t ld,
                             const int32_t *row_list, int64_t n_listed, float *conf, int32_t *tok,
                             cudaStream_t stream);
size_t lmhead_workspace_bytes(int64_t rows, int64_t V);
int launch_lmhead_confidence(const void *hidden, const void *weight, int64_t rows, int64_t hid, int64_t V, int64_t ld_h,
                             int64_t ld_w, float *conf, int32_t *tok, void *workspace, uint32_t *status,
                             cudaStream_t stream);
int launch_block_begin(const ds_block_params &p, cudaStream_t stream);
int launch_select(const ds_select_params &p, cudaStream_t stream);
int launch_rope_gather(const ds_rope_params &p, cudaStream_t stream);
int launch_page_update(const ds_page_params &p, cudaStream_t stream);
int launch_qk_norm_rope(const ds_qk_params &p, cudaStream_t stream);
int launch_attn_paged(const ds_paged_params &p, cudaStream_t stream);
size_t attn_paged_workspace_bytes(const ds_paged_params &p);
bool attn_paged_counts_fit(const ds_paged_params &p);
bool attn_paged_tc_counts_fit(const ds_paged_params &p);
int launch_attn_paged_tc(const ds_paged_params &p, cudaStream_t stream);
size_t attn_paged_tc_workspace_bytes(const ds_paged_params &p);
int launch_kv8_write(const ds_kv8_write_params &p, cudaStream_t stream);
int launch_kv8_read(const ds_kv8_read_params &p, cudaStream_t stream);
int launch_attn_paged8(const ds_paged8_params &p, cudaStream_t stream);
size_t attn_paged8_workspace_bytes(const ds_paged8_params &p);
bool attn_paged8_counts_fit(const ds_paged8_params &p);
bool attn_paged8_tc_counts_fit(const ds_paged_params &p);
size_t attn_paged8_tc_workspace_bytes(const ds_paged_params &p);
int launch_attn_paged8_tc(const ds_paged8_params &p, cudaStream_t stream);
int launch_bounded_wait_selftest(uint32_t poll_limit, uint32_t *status, int32_t *report, cudaStream_t stream);
void note_cuda_error(int code);  // remembered per host thread for ds_last_cuda_error
int launch_attn_simt(const ds_attn_params &p, cudaStream_t stream);
int launch_attn_tc(const ds_attn_params &p, cudaStream_t stream);
int launch_attn_tc2(const ds_attn_params &p, cudaStream_t stream);

// An attention call whose kernel parameters (tensor maps included) have been worked out once: what a
// ds_attn_plan holds and what the one-shot launchers build on the stack.
enum : int { kAttnPathSimt = 0, kAttnPathTc = 1, kAttnPathTc2 = 2 };
struct AttnPrepared {
  int path;
  int grid;          // CTAs to launch; 0 = nothing to do
  ds_attn_params p;  // validated copy of the caller's arguments (the SIMT kernel takes it as it is)
  alignas(64) unsigned char kernel_params[2048];  // the tensor-core kernels' parameter struct
};
int prepare_attn_tc(const ds_attn_params &p, AttnPrepared &out);
int prepare_attn_tc2(const ds_attn_params &p, AttnPrepared &out);
int launch_prepared_tc(const AttnPrepared &a, cudaStream_t stream);
int launch_prepared_tc2(const AttnPrepared &a, cudaStream_t stream);
bool attn_tc_supported(const ds_attn_params &p);
size_t attn_tc_workspace_bytes(const ds_attn_params &p);

}  // namespace ds

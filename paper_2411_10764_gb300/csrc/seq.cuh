// Declarations shared by the sequence-model operators (sampling, embedding,
// selective scan): element types, vector access, launchers.  Not part of the
// C ABI.
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "mlt.h"
#include "mlt_internal.cuh"

namespace mlt {

// mlt_api.cu: the thread's error message, the device error word that
// mlt_sync_status reads (nullptr and *rc where it cannot be had) and the
// launch counter.
int api_fail(int code, const char* fmt, ...);
unsigned* api_error_word(int* rc);
void api_count_launches(long long n);
int api_sm_count();
unsigned long long api_take_sample_stall();  // nanoseconds, 0: not armed

inline size_t dtype_size(int dtype) { return dtype == MLT_F32 ? 4 : 2; }
inline bool dtype_ok(int dtype) { return dtype == MLT_F32 || dtype == MLT_BF16 || dtype == MLT_F16; }
inline bool aligned_to(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline size_t up256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

// Calls f with a value of the element type.
template <typename F>
auto with_dtype(int dtype, F f) {
  if (dtype == MLT_BF16) return f(__nv_bfloat16());
  if (dtype == MLT_F16) return f(__half());
  return f(float());
}

#ifdef __CUDACC__
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// V elements moved as one access (two where they are more than 16 bytes).
template <typename T, int V>
struct alignas(sizeof(T) * V > 16 ? 16 : sizeof(T) * V) Pack {
  T v[V];
};
#endif

// --- sample.cu -------------------------------------------------------------
struct SampleArgs {
  const void* scores;
  int dtype;
  unsigned stall_us;  // not 0: in teams that meet in global memory the last CTA stays away, waits last as long
  long long rows, n, row_stride;
  const float* noise;
  long long noise_stride;
  mlt_sample_rule rule;
  const mlt_sample_rule* rules;  // device, or null
  int m;
  long long* out_index;
  float* out_logprob;
  unsigned* err;
  void* ws;
};
size_t sample_workspace(int dtype, long long rows, long long n, int m, int sms);
cudaError_t launch_sample(const SampleArgs& a, int sms, long long* launches, cudaStream_t st);

// --- embed.cu --------------------------------------------------------------
struct EmbedArgs {
  const void* table;  // [vocab][dim], or the gradient of the outputs [tokens][dim]
  int in_dtype;
  long long in_stride;
  const void* ids;
  int ids_64;
  long long tokens, vocab;
  int dim;
  float scale;
  void* out;  // [tokens][dim], or the gradient of the table [vocab][dim]
  int out_dtype;
  long long out_stride;
  unsigned* err;
  void* ws;
};
cudaError_t launch_embed(const EmbedArgs& a, int sms, long long* launches, cudaStream_t st);
size_t embed_grad_workspace(long long tokens, long long vocab, int dim, int sms);
cudaError_t launch_embed_grad(const EmbedArgs& a, int sms, long long* launches, cudaStream_t st);

// --- scan.cu, scan_grad.cu -------------------------------------------------
constexpr int kScanMaxStates = 32;
constexpr int kScanMaxTaps = 4;
size_t scan_workspace(const mlt_scan_args& a, int sms);
cudaError_t launch_scan(const mlt_scan_args& a, void* ws, int sms, long long* launches, cudaStream_t st);
size_t scan_grad_workspace(const mlt_scan_args& a, int sms);
cudaError_t launch_scan_grad(const mlt_scan_args& a, const mlt_scan_grads& g, void* ws, int sms, long long* launches,
                             cudaStream_t st);

// --- norm.cu, norm_grad.cu -------------------------------------------------
cudaError_t launch_norm(const mlt_norm_args& a, int sms, long long* launches, cudaStream_t st);
size_t norm_grad_workspace(long long rows, int dim, int sms);
cudaError_t launch_norm_grad(const mlt_norm_args& a, const mlt_norm_grads& g, void* ws, int sms, long long* launches,
                             cudaStream_t st);

// --- adamw.cu --------------------------------------------------------------
cudaError_t launch_adamw(const mlt_adamw_tensor* tensors, int count, const mlt_adamw_rule& rule, void* m, void* v,
                         float* m_scale, float* v_scale, int sms, long long* launches, cudaStream_t st);

// --- beam.cu ---------------------------------------------------------------
constexpr int kBeamMostBeams = 1024;
constexpr int kBeamMostStates = 64;
size_t beam_workspace(const mlt_beam_args& a, int sms);
cudaError_t launch_beam(const mlt_beam_args& a, void* ws, int sms, long long* launches, cudaStream_t st);
cudaError_t launch_reorder(const int64_t* parent, int batch, int beams, const mlt_beam_state* tensors, int count,
                           unsigned* err, long long* launches, cudaStream_t st);

}  // namespace mlt

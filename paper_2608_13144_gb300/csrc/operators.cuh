// Internal declarations of the operators that train and serve heads.
#pragma once

#include <cuda_bf16.h>

#include <algorithm>
#include <type_traits>

#include "internal.cuh"

namespace lc {
namespace ops {

// ---------------------------------------------------------------- types
template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) {
  return __bfloat162float(v);
}
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}

inline size_t elem(int type) { return type == LIPCACHE_F32 ? 4 : 2; }
__device__ __forceinline__ int64_t ceil_div_dev(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// A launch that may begin while the kernel before it ends; `kernel` waits for
// that one's results itself (griddepcontrol.wait).
template <typename K, typename... Args>
void launch_pdl_smem(K kernel, dim3 grid, int threads, int smem, cudaStream_t s, Args... args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  LC_CUDA(cudaLaunchKernelEx(&cfg, kernel, args...));
}
template <typename K, typename... Args>
void launch_pdl(K kernel, dim3 grid, int threads, cudaStream_t s, Args... args) {
  launch_pdl_smem(kernel, grid, threads, 0, s, args...);
}
// head_mma.cu: lets `kernel` use `bytes` of dynamic shared memory on the
// current device.
void allow_smem(const void* kernel, int bytes);

// ---------------------------------------------------------------- launchers
// head_adapt.cu
size_t adapted_bytes(const lipcache_adapted& p, bool backward);
void adapted_logits(const lipcache_adapted& p, const float* bias, void* y, int64_t ldy, unsigned char* ws,
                    cudaStream_t s);
void adapted_backward(const lipcache_adapted& p, const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dA,
                      void* dB, unsigned char* ws, cudaStream_t s);
// expired bounded waits on the current device; synchronises `s`
uint64_t operator_errors(cudaStream_t s);
// head_loss.cu
void cross_entropy(int type, const void* z, int64_t ldz, int64_t tokens, int classes, const int32_t* target,
                   const float* weight, float* loss, void* dz, int64_t ldd, cudaStream_t s);
// head_ortho.cu
struct OrthoStep {  // what a step adds to an orthogonalisation; null weight: none
  const void* weight = nullptr;
  void* out_weight = nullptr;
  const float* momentum = nullptr;
  float* out_momentum = nullptr;
  int weight_type = 0;
  float beta = 0.f, keep = 1.f, rate = 0.f;  // W' = keep W - rate O
  bool nesterov = false;
};
size_t ortho_bytes(int type, int64_t batch, int rows, int cols);
void orthogonalize(int type, const void* G, int64_t ldg, int64_t batch, int rows, int cols, int steps,
                   const double* coefficients, double eps, void* out, const OrthoStep& st, unsigned char* ws,
                   cudaStream_t s);

}  // namespace ops
}  // namespace lc

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

// Two values at a time: the conversions that pack run at several times the
// rate of single ones.
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 open_f16(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
// N values as two FP16 planes, hi + lo.
template <int N>
__device__ __forceinline__ void split_f16(const float (&v)[N], uint32_t (&hi)[N / 2], uint32_t (&lo)[N / 2]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    hi[i] = pack_f16(v[2 * i], v[2 * i + 1]);
    const float2 h = open_f16(hi[i]);
    lo[i] = pack_f16(v[2 * i] - h.x, v[2 * i + 1] - h.y);
  }
}
// The same as BF16 planes.
template <int N>
__device__ __forceinline__ void split_bf16(const float (&v)[N], uint32_t (&hi)[N / 2], uint32_t (&lo)[N / 2]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    hi[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    lo[i] = pack_bf16(v[2 * i] - __uint_as_float(hi[i] << 16), v[2 * i + 1] - __uint_as_float(hi[i] & 0xffff0000u));
  }
}
// N values (a multiple of 16 bytes) rounded to T, in 32-bit words.
template <typename T, int N>
__device__ __forceinline__ void round_to(const float (&v)[N], uint32_t (&w)[N * sizeof(T) / 4]) {
#pragma unroll
  for (int i = 0; i < (int)(N * sizeof(T) / 4); ++i) {
    if constexpr (sizeof(T) == 4)
      w[i] = __float_as_uint(v[i]);
    else
      w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
  }
}

inline size_t elem(int type) { return type == LIPCACHE_F32 ? 4 : 2; }
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
  float beta = 0.f, fresh = 1.f;  // fresh: 1 - beta, rounded once
  float keep = 1.f, rate = 0.f;   // W' = keep W - rate O
  bool nesterov = false;
};
// head_ortho_small.cu: false where the matrices are not its kind (a side of at
// most 64, slices that fit)
bool ortho_small(int type, const void* G, int64_t ldg, int64_t batch, int rows, int cols, int steps,
                 const double* coefficients, double eps, void* out, const OrthoStep& st, cudaStream_t s);
size_t ortho_bytes(int type, int64_t batch, int rows, int cols);
void orthogonalize(int type, const void* G, int64_t ldg, int64_t batch, int rows, int cols, int steps,
                   const double* coefficients, double eps, void* out, const OrthoStep& st, unsigned char* ws,
                   cudaStream_t s);

}  // namespace ops
}  // namespace lc

// FP32 products on the CUDA cores for the operators of heads: D = alpha A B +
// beta E over any strides, 64 x 64 tiles, 4 x 4 sums a thread.
#pragma once

#include "operators.cuh"

namespace lc {
namespace ops {

template <typename TA, typename TB, typename TD>
struct SimpleGemm {
  const TA* a;
  const TB* b;
  const TD* e;       // nullable; same layout as d
  TD* d;
  int m, n, k;
  int64_t a_row, a_col, b_row, b_col, d_row;  // element strides: A m x k, B k x n, D m x n
  int64_t a_batch, b_batch, d_batch;
  float alpha, beta;
};

template <typename TA, typename TB, typename TD>
__global__ void __launch_bounds__(256) k_gemm_simple(const SimpleGemm<TA, TB, TD> g) {
  __shared__ float sa[16][65], sb[16][65];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int64_t m0 = (int64_t)blockIdx.x * 64, n0 = (int64_t)blockIdx.y * 64;
  const TA* a = g.a + blockIdx.z * g.a_batch;
  const TB* b = g.b + blockIdx.z * g.b_batch;
  float acc[4][4] = {};
  const bool a_k = g.a_col == 1, b_k = g.b_row == 1;  // which index neighbours in memory
  for (int k0 = 0; k0 < g.k; k0 += 16) {
    for (int i = tid; i < 1024; i += 256) {
      int r = a_k ? i >> 4 : i & 63, c = a_k ? i & 15 : i >> 6;
      sa[c][r] = m0 + r < g.m && k0 + c < g.k ? to_f32<TA>(a[(m0 + r) * g.a_row + (k0 + c) * g.a_col]) : 0.f;
      r = b_k ? i >> 4 : i & 63, c = b_k ? i & 15 : i >> 6;
      sb[c][r] = n0 + r < g.n && k0 + c < g.k ? to_f32<TB>(b[(k0 + c) * g.b_row + (n0 + r) * g.b_col]) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      float x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = sa[c][ty + 16 * i], y[i] = sb[c][tx + 16 * i];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t r = m0 + ty + 16 * i, c = n0 + tx + 16 * j;
      if (r >= g.m || c >= g.n) continue;
      const int64_t at = blockIdx.z * g.d_batch + r * g.d_row + c;
      float v = g.alpha * acc[i][j];
      if (g.e) v = fmaf(g.beta, to_f32<TD>(g.e[at]), v);
      g.d[at] = from_f32<TD>(v);
    }
}

template <typename TA, typename TB, typename TD>
void gemm_simple(const SimpleGemm<TA, TB, TD>& g, int64_t batch, cudaStream_t s) {
  const dim3 grid((unsigned)ceil_div(g.m, 64), (unsigned)ceil_div(g.n, 64), (unsigned)batch);
  k_gemm_simple<TA, TB, TD><<<grid, 256, 0, s>>>(g);
  LC_LAUNCH_CHECK("k_gemm_simple");
}

}  // namespace ops
}  // namespace lc

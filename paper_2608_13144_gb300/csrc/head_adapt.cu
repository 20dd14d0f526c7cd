// Logits under a shared head and each row's own low-rank adapter, and their
// gradients.
//   u_t = s_g A_g x_t,  y_t = W x_t + bias + B_g u_t
//   v_t = s_g B_g^T dy_t,  dx_t = W^T dy_t + A_g^T v_t
//   dA_g = sum v_t x_t^T,  dB_g = sum dy_t u_t^T
#include "head_gemm.cuh"

namespace lc {
namespace ops {

namespace {

struct AdaptLayout {
  float *u, *v, *acc;  // tokens x rank; tokens x max(d, classes)
  void take(Carve& c, const lipcache_adapted& p, bool backward) {
    const size_t r = p.adapters ? p.rank : 0;
    c.take(u, (size_t)p.tokens * r);
    c.take(v, backward ? (size_t)p.tokens * r : 0);
    c.take(acc, (size_t)p.tokens * (backward ? p.d : p.classes));
  }
};

// One warp per (row, j): out[t, j] = s_g sum_i in[t, i] F_g[j, i] (strides
// f_j, f_i), 0 for a row without an adapter.
template <typename T>
__global__ void __launch_bounds__(256)
    k_shrink(const T* in, int64_t ld, int64_t tokens, int width, const T* F, int64_t f_g, int64_t f_j, int64_t f_i,
             const int32_t* adapter, const float* scales, int G, int r, float* out) {
  const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), t = w / r;
  if (t >= tokens) return;
  const int j = (int)(w % r), lane = threadIdx.x & 31, g = adapter[t];
  if (g < 0 || g >= G) {
    if (lane == 0) out[w] = 0.f;
    return;
  }
  const T* f = F + g * f_g + j * f_j;
  float sum = 0.f;
  for (int i = lane; i < width; i += 32) sum = fmaf(to_f32<T>(in[t * ld + i]), to_f32<T>(f[i * f_i]), sum);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) out[w] = scales ? scales[g] * sum : sum;
}

// out[t, i] = acc[t, i] + bias[i] + sum_j F_g[j, i] u[t, j], rounded once.
template <typename T>
__global__ void __launch_bounds__(256)
    k_expand(const float* acc, int64_t tokens, int width, const float* bias, const float* u, int r, const T* F,
             int64_t f_g, int64_t f_j, int64_t f_i, const int32_t* adapter, int G, T* out, int64_t ld) {
  const int64_t t = blockIdx.y + (int64_t)blockIdx.z * 32768;
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= width || t >= tokens) return;
  float v = acc[t * width + i];
  if (bias) v += bias[i];
  const int g = G ? adapter[t] : -1;
  if (g >= 0 && g < G) {
    const T* f = F + g * f_g + i * f_i;
    for (int j = 0; j < r; ++j) v = fmaf(u[t * r + j], to_f32<T>(f[j * f_j]), v);
  }
  out[t * ld + i] = from_f32<T>(v);
}

// out_g[j, i] (strides f_j, f_i) = sum over g's rows of u[t, j] in[t, i].
template <typename T>
__global__ void __launch_bounds__(256)
    k_outer(const float* u, int r, const T* in, int64_t ld, int64_t tokens, int width, const int32_t* adapter, T* out,
            int64_t f_g, int64_t f_j, int64_t f_i) {
  __shared__ int ids[256];
  const int i = blockIdx.x * 256 + threadIdx.x, j = blockIdx.y, g = blockIdx.z;
  float sum = 0.f;
  for (int64_t t0 = 0; t0 < tokens; t0 += 256) {
    __syncthreads();
    ids[threadIdx.x] = t0 + threadIdx.x < tokens ? adapter[t0 + threadIdx.x] : -1;
    __syncthreads();
    for (int k = 0; k < 256; ++k)
      if (ids[k] == g && i < width) sum = fmaf(u[(t0 + k) * r + j], to_f32<T>(in[(t0 + k) * ld + i]), sum);
  }
  if (i < width) out[g * f_g + j * f_j + i * f_i] = from_f32<T>(sum);
}

template <typename T>
void shrink(const T* in, int64_t ld, const lipcache_adapted& p, int width, const T* F, int64_t f_j, int64_t f_i,
            float* out, cudaStream_t s) {
  if (!p.adapters) return;
  k_shrink<T><<<(unsigned)ceil_div(p.tokens * p.rank, 8), 256, 0, s>>>(in, ld, p.tokens, width, F, (int64_t)p.rank * width,
                                                                       f_j, f_i, p.adapter, p.scales, p.adapters,
                                                                       p.rank, out);
  LC_LAUNCH_CHECK("k_shrink");
}

template <typename T>
void expand(const float* acc, const lipcache_adapted& p, int width, const float* bias, const float* u, const T* F,
            int64_t f_j, int64_t f_i, T* out, int64_t ld, cudaStream_t s) {
  const dim3 grid((unsigned)ceil_div(width, 256), (unsigned)std::min<int64_t>(p.tokens, 32768),
                  (unsigned)ceil_div(p.tokens, 32768));
  k_expand<T><<<grid, 256, 0, s>>>(acc, p.tokens, width, bias, u, p.rank, F, (int64_t)p.rank * width, f_j, f_i,
                                   p.adapter, p.adapters, out, ld);
  LC_LAUNCH_CHECK("k_expand");
}

template <typename T>
void outer(const float* u, const T* in, int64_t ld, const lipcache_adapted& p, int width, T* out, int64_t f_j,
           int64_t f_i, cudaStream_t s) {
  const dim3 grid((unsigned)ceil_div(width, 256), (unsigned)p.rank, (unsigned)p.adapters);
  k_outer<T><<<grid, 256, 0, s>>>(u, p.rank, in, ld, p.tokens, width, p.adapter, out, (int64_t)p.rank * width, f_j, f_i);
  LC_LAUNCH_CHECK("k_outer");
}

template <typename T>
void forward(const lipcache_adapted& p, const float* bias, T* y, int64_t ldy, const AdaptLayout& l, cudaStream_t s) {
  const T *x = static_cast<const T*>(p.x), *W = static_cast<const T*>(p.W);
  shrink<T>(x, p.ldx, p, p.d, static_cast<const T*>(p.A), p.d, 1, l.u, s);
  gemm_simple<T, T, float>({x, W, nullptr, l.acc, (int)p.tokens, p.classes, p.d, p.ldx, 1, 1, p.ldw, p.classes, 0, 0, 0,
                            1.f, 0.f}, 1, s);
  expand<T>(l.acc, p, p.classes, bias, l.u, static_cast<const T*>(p.B), 1, p.rank, y, ldy, s);
}

template <typename T>
void backward(const lipcache_adapted& p, const T* dy, int64_t lddy, T* dx, int64_t lddx, T* dA, T* dB,
              const AdaptLayout& l, cudaStream_t s) {
  const T *x = static_cast<const T*>(p.x), *W = static_cast<const T*>(p.W), *A = static_cast<const T*>(p.A),
          *B = static_cast<const T*>(p.B);
  if (dB) shrink<T>(x, p.ldx, p, p.d, A, p.d, 1, l.u, s);
  if (dA || dx) shrink<T>(dy, lddy, p, p.classes, B, 1, p.rank, l.v, s);
  if (dx) {
    gemm_simple<T, T, float>({dy, W, nullptr, l.acc, (int)p.tokens, p.d, p.classes, lddy, 1, p.ldw, 1, p.d, 0, 0, 0,
                              1.f, 0.f}, 1, s);
    expand<T>(l.acc, p, p.d, nullptr, l.v, A, p.d, 1, dx, lddx, s);
  }
  if (!p.adapters) return;
  if (dA) outer<T>(l.v, x, p.ldx, p, p.d, dA, p.d, 1, s);
  if (dB) outer<T>(l.u, dy, lddy, p, p.classes, dB, 1, p.rank, s);
}

}  // namespace

size_t adapted_bytes(const lipcache_adapted& p, bool backward) {
  AdaptLayout l;
  Carve c;
  l.take(c, p, backward);
  return c.off;
}

void adapted_logits(const lipcache_adapted& p, const float* bias, void* y, int64_t ldy, unsigned char* ws,
                    cudaStream_t s) {
  AdaptLayout l;
  Carve c{ws, 0};
  l.take(c, p, false);
  if (p.type == LIPCACHE_F32)
    forward<float>(p, bias, static_cast<float*>(y), ldy, l, s);
  else
    forward<__nv_bfloat16>(p, bias, static_cast<__nv_bfloat16*>(y), ldy, l, s);
}

void adapted_backward(const lipcache_adapted& p, const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dA,
                      void* dB, unsigned char* ws, cudaStream_t s) {
  AdaptLayout l;
  Carve c{ws, 0};
  l.take(c, p, true);
  if (p.type == LIPCACHE_F32)
    backward<float>(p, static_cast<const float*>(dy), lddy, static_cast<float*>(dx), lddx, static_cast<float*>(dA),
                    static_cast<float*>(dB), l, s);
  else
    backward<__nv_bfloat16>(p, static_cast<const __nv_bfloat16*>(dy), lddy, static_cast<__nv_bfloat16*>(dx), lddx,
                            static_cast<__nv_bfloat16*>(dA), static_cast<__nv_bfloat16*>(dB), l, s);
}

}  // namespace ops
}  // namespace lc

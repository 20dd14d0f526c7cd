// Newton-Schulz orthogonalisation and the optimiser step built on it.
//   X = D / (||D||_F + eps) in its wide orientation; S = X X^T;
//   X <- a X + (b S + c S S) X
#include "head_gemm.cuh"

namespace lc {
namespace ops {
namespace {

struct OrthoLayout {
  float *x[2], *gram, *poly, *norm;
  double* part;
  static constexpr int kParts = 64;
  void take(Carve& c, int64_t batch, int rows, int cols) {
    const size_t n = (size_t)batch * rows * cols;
    const int64_t m = rows < cols ? rows : cols;
    c.take(x[0], n);
    c.take(x[1], n);
    c.take(gram, (size_t)(batch * m * m));
    c.take(poly, (size_t)(batch * m * m));
    c.take(part, (size_t)batch * kParts);
    c.take(norm, (size_t)batch);
  }
};

// The direction D into x, the momentum, and each block's sum of squares.
template <typename T>
__global__ void __launch_bounds__(256)
    k_direction(const T* g, int64_t ldg, int rows, int cols, const OrthoStep st, float* x, double* part) {
  __shared__ double red[256];
  const int64_t per = (int64_t)rows * cols, base = blockIdx.y * per;
  double sum = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < per; i += (int64_t)gridDim.x * 256) {
    float v = to_f32<T>(g[((int64_t)blockIdx.y * rows + i / cols) * ldg + i % cols]);
    if (st.weight) {
      const float m = st.beta * st.momentum[base + i] + (1.f - st.beta) * v;
      st.out_momentum[base + i] = m;
      v = st.nesterov ? st.beta * m + (1.f - st.beta) * v : m;
    }
    x[base + i] = v;
    sum += (double)v * v;
  }
  red[threadIdx.x] = sum;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if (threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) part[blockIdx.y * gridDim.x + blockIdx.x] = red[0];
}

__global__ void __launch_bounds__(256) k_normalise(float* x, int64_t per, const double* part, int parts, double eps) {
  double sum = 0.0;
  for (int i = 0; i < parts; ++i) sum += part[blockIdx.y * parts + i];
  const double norm = sqrt(sum);
  const float inv = isfinite(norm) ? (float)(1.0 / (norm + eps)) : NAN;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < per; i += (int64_t)gridDim.x * 256)
    x[blockIdx.y * per + i] *= inv;
}

template <typename T>
__global__ void __launch_bounds__(256) k_finish(const float* o, int64_t n, const OrthoStep st, T* out) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const float v = o[i];
    out[i] = from_f32<T>(st.weight ? st.keep * to_f32<T>(static_cast<const T*>(st.weight)[i]) - st.rate * v : v);
  }
}

}  // namespace

size_t ortho_bytes(int, int64_t batch, int rows, int cols) {
  OrthoLayout l;
  Carve c;
  l.take(c, batch, rows, cols);
  return c.off;
}

void orthogonalize(int type, const void* G, int64_t ldg, int64_t batch, int rows, int cols, int steps,
                   const double* coefficients, double eps, void* out, const OrthoStep& st, unsigned char* ws,
                   cudaStream_t s) {
  OrthoLayout l;
  Carve c{ws, 0};
  l.take(c, batch, rows, cols);
  const int64_t per = (int64_t)rows * cols;
  const dim3 grid(OrthoLayout::kParts, (unsigned)batch);
  if (type == LIPCACHE_F32)
    k_direction<float><<<grid, 256, 0, s>>>(static_cast<const float*>(G), ldg, rows, cols, st, l.x[0], l.part);
  else
    k_direction<__nv_bfloat16>
        <<<grid, 256, 0, s>>>(static_cast<const __nv_bfloat16*>(G), ldg, rows, cols, st, l.x[0], l.part);
  LC_LAUNCH_CHECK("k_direction");
  k_normalise<<<grid, 256, 0, s>>>(l.x[0], per, l.part, OrthoLayout::kParts, eps);
  LC_LAUNCH_CHECK("k_normalise");
  const bool tall = rows > cols;
  const int m = tall ? cols : rows, n = tall ? rows : cols;
  const int64_t xr = tall ? 1 : cols, xc = tall ? cols : 1;  // strides of the wide X
  const int64_t mm = (int64_t)m * m;
  for (int i = 0; i < steps; ++i) {
    const float a = (float)coefficients[3 * i], b = (float)coefficients[3 * i + 1], cc = (float)coefficients[3 * i + 2];
    float *x = l.x[i & 1], *y = l.x[(i & 1) ^ 1];
    gemm_simple<float, float, float>({x, x, nullptr, l.gram, m, m, n, xr, xc, xc, xr, m, per, per, mm, 1.f, 0.f}, batch, s);
    gemm_simple<float, float, float>({l.gram, l.gram, l.gram, l.poly, m, m, m, m, 1, m, 1, m, mm, mm, mm, cc, b}, batch, s);
    if (tall)
      gemm_simple<float, float, float>({x, l.poly, x, y, n, m, m, m, 1, m, 1, m, per, mm, per, 1.f, a}, batch, s);
    else
      gemm_simple<float, float, float>({l.poly, x, x, y, m, n, m, m, 1, n, 1, n, mm, per, per, 1.f, a}, batch, s);
  }
  const int out_type = st.weight ? st.weight_type : type;
  void* dst = st.weight ? st.out_weight : out;
  const unsigned blocks = (unsigned)std::min<int64_t>(ceil_div(batch * per, 1024), 1 << 20);
  if (out_type == LIPCACHE_F32)
    k_finish<float><<<blocks, 256, 0, s>>>(l.x[steps & 1], batch * per, st, static_cast<float*>(dst));
  else
    k_finish<__nv_bfloat16><<<blocks, 256, 0, s>>>(l.x[steps & 1], batch * per, st, static_cast<__nv_bfloat16*>(dst));
  LC_LAUNCH_CHECK("k_finish");
}

}  // namespace ops
}  // namespace lc

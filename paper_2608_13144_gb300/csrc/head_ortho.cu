// Newton-Schulz orthogonalisation and the optimiser step built on it.
//   X = D / (||D||_F + eps), wide (of D^T where D is tall); each step
//   S = X X^T,  P = b S + c S S,  X <- a X + P X
// Products run on the tensor cores (head_mma.cuh) from FP16 operands with FP32
// sums. An FP32 matrix is kept as two FP16 planes, hi + lo (22 bits), and a
// product is hi hi + hi lo + lo hi; a BF16 one as a single plane (11 bits): the
// iteration multiplies rounding by up to a^steps where singular values are
// small, so three bits more than the result's are kept.
//
// FP16's range: every array carries a power of two. X carries 2^13 (singular
// values up to 4 stay inside), S 2^10, P what its coefficients allow. The
// normalisation is split into a power of two that takes ||D|| below 1, applied
// exactly when the planes are written, and the rest t <= 2, which joins the
// first step's epilogues, so that the first X of a BF16 matrix is exact.
//
// S and P are symmetric: tiles on or above the diagonal are computed and
// written twice. Nothing is transposed: a tall X is contracted over its rows,
// and P X reads X along its rows, by operands stored MN-major.
#include <cuda_fp16.h>

#include "head_mma.cuh"

namespace lc {
namespace ops {
namespace {

constexpr int kParts = 128;      // partial sums of squares of a matrix, at most
constexpr float kXScale = 8192.f, kSScale = 1024.f;
constexpr int kBlock = 4;  // stages of 64 summed on the tensor cores at a time, FP32 matrices

struct OrthoLayout {
  __half *x[2], *s, *p;  // planes x batch x rows x ld
  float* t;              // batch: the rest of the normalisation
  double* part;          // batch x kParts
  int64_t ld, sld, x_plane, s_plane;
  void take(Carve& c, int planes, int64_t batch, int rows, int cols) {
    const int m = std::min(rows, cols);
    ld = round_up(cols, 8);
    sld = round_up(m, 8);
    x_plane = (int64_t)rows * ld;
    s_plane = (int64_t)m * sld;
    c.take(x[0], (size_t)(planes * batch * x_plane));
    c.take(x[1], (size_t)(planes * batch * x_plane));
    c.take(s, (size_t)(planes * batch * s_plane));
    c.take(p, (size_t)(planes * batch * s_plane));
    c.take(t, (size_t)batch);
    c.take(part, (size_t)batch * kParts);
  }
};

// ---------------------------------------------------------------- normalisation
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[VEC]) {
  if (VEC == 8 && sizeof(T) == 4) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4 % VEC] = b.x, v[5 % VEC] = b.y, v[6 % VEC] = b.z, v[7 % VEC] = b.w;
  } else if (VEC == 8) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = to_f32<T>(p[i]);
  }
}
template <int VEC>
__device__ __forceinline__ void store_vec(float* p, const float (&v)[VEC]) {
  if (VEC == 8) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1 % VEC], v[2 % VEC], v[3 % VEC]);
    *(reinterpret_cast<float4*>(p) + 1) = make_float4(v[4 % VEC], v[5 % VEC], v[6 % VEC], v[7 % VEC]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) p[i] = v[i];
  }
}

struct Direction {
  int rows, cols;
  int64_t ldg;
  int units;      // of VEC elements in a row
  OrthoStep st;
};

// Elements [VEC] of the direction D, and (FIRST) the momentum's update.
template <typename T, int VEC, bool FIRST>
__device__ __forceinline__ void direction(const Direction& a, const T* g, int64_t row, int col, float (&v)[VEC]) {
  load_vec<T, VEC>(g + row * a.ldg + col, v);
  if (!a.st.weight) return;
  const int64_t at = row * a.cols + col;
  const float b = a.st.beta, r = 1.f - b;
  float m[VEC];
  load_vec<float, VEC>((FIRST ? a.st.momentum : a.st.out_momentum) + at, m);
  if (FIRST) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) m[i] = fmaf(b, m[i], r * v[i]);
    store_vec<VEC>(a.st.out_momentum + at, m);
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = a.st.nesterov ? fmaf(b, m[i], r * v[i]) : m[i];
}

// The new momentum, and each block's sum of squares of D (runs of eight to 64
// in FP32, those in FP64, in a fixed order).
template <typename T, int VEC>
__global__ void __launch_bounds__(256) k_squares(const T* g, const Direction a, double* part) {
  __shared__ double red[8];
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const uint32_t n = (uint32_t)a.rows * (uint32_t)a.units;
  const int64_t row0 = (int64_t)blockIdx.y * a.rows;
  double sum = 0.0;
  float run = 0.f;
  int k = 0;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const uint32_t r = i / (uint32_t)a.units;
    float v[VEC];
    direction<T, VEC, true>(a, g, row0 + r, (int)(i - r * (uint32_t)a.units) * VEC, v);
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < VEC; ++j) top = fmaxf(top, fabsf(v[j]));
    if (top < 0x1p60f && (top > 0x1p-50f || top == 0.f)) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) run = fmaf(v[j], v[j], run);
    } else {  // squares that FP32 does not hold
#pragma unroll
      for (int j = 0; j < VEC; ++j) sum += (double)v[j] * v[j];
    }
    if ((++k & 7) == 0) sum += (double)run, run = 0.f;
  }
  sum += (double)run;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) sum += red[w];
    part[blockIdx.y * gridDim.x + blockIdx.x] = sum;
  }
}

// X's planes: D times 2^-e and kXScale, ||D|| < 2^e <= 2 ||D||.
template <typename T, int VEC, int PLANES>
__global__ void __launch_bounds__(256)
    k_planes(const T* g, const Direction a, const double* part, int parts, double eps, __half* x,
             int64_t ld, int64_t plane, float* t) {
  __shared__ float factor;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += 32) sum += part[blockIdx.y * parts + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x == 0) {
      const double norm = sqrt(sum);
      int e = 0;
      frexp(norm > 0.0 ? norm : 1.0, &e);  // norm < 2^e
      const bool fine = isfinite(norm) && e <= 126;
      factor = fine ? ldexpf(kXScale, min(-e, 114)) : NAN;
      if (blockIdx.x == 0) t[blockIdx.y] = fine ? (float)(ldexp(1.0, e) / (norm + eps)) : NAN;
    }
  }
  __syncthreads();
  const float f = factor;
  const uint32_t n = (uint32_t)a.rows * (uint32_t)a.units;
  const int64_t row0 = (int64_t)blockIdx.y * a.rows;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const uint32_t r = i / (uint32_t)a.units;
    const int col = (int)(i - r * (uint32_t)a.units) * VEC;
    float v[VEC];
    direction<T, VEC, false>(a, g, row0 + r, col, v);
    __half hi[VEC], lo[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      hi[j] = __float2half_rn(v[j] * f);
      lo[j] = __float2half_rn(fmaf(v[j], f, -__half2float(hi[j])));
    }
    __half* d = x + (row0 + r) * ld + col;
    if (VEC == 8) {
      *reinterpret_cast<uint4*>(d) = *reinterpret_cast<uint4*>(hi);
      if (PLANES == 2) *reinterpret_cast<uint4*>(d + plane) = *reinterpret_cast<uint4*>(lo);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        d[j] = hi[j];
        if (PLANES == 2) d[plane + j] = lo[j];
      }
    }
  }
}

// ---------------------------------------------------------------- epilogues
// 32 neighbouring values of a row as FP16 planes; columns past `cols` may be
// written up to the row's stride.
template <int PLANES>
__device__ __forceinline__ void store_planes(__half* d, int64_t plane, int left, const float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (q * 8 >= left) break;
    __half hi[8], lo[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hi[j] = __float2half_rn(v[q * 8 + j]);
      lo[j] = __float2half_rn(v[q * 8 + j] - __half2float(hi[j]));
    }
    *reinterpret_cast<uint4*>(d + q * 8) = *reinterpret_cast<uint4*>(hi);
    if (PLANES == 2) *reinterpret_cast<uint4*>(d + plane + q * 8) = *reinterpret_cast<uint4*>(lo);
  }
}
// The same 32 values down a column (row stride ld): 32 lanes write neighbours.
template <int PLANES>
__device__ __forceinline__ void store_planes_t(__half* d, int64_t ld, int64_t plane, int left, const float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    if (j >= left) break;
    const __half hi = __float2half_rn(v[j]);
    d[j * ld] = hi;
    if (PLANES == 2) d[plane + j * ld] = __float2half_rn(v[j] - __half2float(hi));
  }
}
// v += f (the values of the planes)
template <int PLANES>
__device__ __forceinline__ void add_planes(const __half* d, int64_t plane, int left, float f, float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (q * 8 >= left) break;
    uint4 w = *reinterpret_cast<const uint4*>(d + q * 8);
    const __half* h = reinterpret_cast<const __half*>(&w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[q * 8 + j] = fmaf(f, __half2float(h[j]), v[q * 8 + j]);
    if (PLANES == 2) {
      w = *reinterpret_cast<const uint4*>(d + plane + q * 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[q * 8 + j] = fmaf(f, __half2float(h[j]), v[q * 8 + j]);
    }
  }
}

// S (of = null) or P = c S S + b S, both triangles.
template <int PLANES>
struct SymEpi {
  __half* d;
  const __half* of;
  int64_t ld, mat, plane;  // row, matrix and plane strides
  int m, tile;
  float f, b;
  const float* t;  // nullable: squared into f
  __device__ __forceinline__ void store(int row0, int col0, int z, int lane, bool, const uint32_t (&acc)[32]) const {
    const int row = row0 + lane, left = m - col0;
    if (left <= 0) return;
    float g = f;
    if (t) g *= t[z] * t[z];
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = g * __uint_as_float(acc[j]);
    const int64_t at = z * mat + row * ld + col0;
    if (row < m) {
      if (of) add_planes<PLANES>(of + at, plane, left, b, v);
      store_planes<PLANES>(d + at, plane, left, v);
    }
    if (row0 / tile != col0 / tile && row < m) store_planes_t<PLANES>(d + z * mat + col0 * ld + row, ld, plane, left, v);
  }
};

// X' = a X + P X.
template <int PLANES>
struct UpdateEpi {
  __half* d;
  const __half* x;
  int64_t ld, mat, plane;
  int rows, cols;
  float f, a;
  const float* t;
  __device__ __forceinline__ void store(int row0, int col0, int z, int lane, bool, const uint32_t (&acc)[32]) const {
    const int row = row0 + lane, left = cols - col0;
    if (left <= 0 || row >= rows) return;
    const float u = t ? t[z] : 1.f, g = f * u;
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = g * __uint_as_float(acc[j]);
    const int64_t at = z * mat + row * ld + col0;
    add_planes<PLANES>(x + at, plane, left, a * u, v);
    store_planes<PLANES>(d + at, plane, left, v);
  }
};

// The last step: the result, or the weights' update, in the caller's type.
template <int PLANES, typename T>
struct LastEpi {
  T* d;
  const T* w;  // null: the result itself
  const __half* x;
  int64_t ld, mat, plane;
  int rows, cols, vec;
  float f, a, keep, rate;
  const float* t;
  __device__ __forceinline__ void store(int row0, int col0, int z, int lane, bool, const uint32_t (&acc)[32]) const {
    const int row = row0 + lane, left = cols - col0;
    if (left <= 0 || row >= rows) return;
    const float u = t ? t[z] : 1.f, g = f * u;
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = g * __uint_as_float(acc[j]);
    add_planes<PLANES>(x + z * mat + row * ld + col0, plane, left, a * u, v);
    const int64_t at = ((int64_t)z * rows + row) * cols + col0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q * 8 >= left) break;
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = v[q * 8 + j];
      if (vec) {
        if (w) {
          float old[8];
          load_vec<T, 8>(w + at + q * 8, old);
#pragma unroll
          for (int j = 0; j < 8; ++j) o[j] = fmaf(keep, old[j], -rate * o[j]);
        }
        if (sizeof(T) == 4) {
          store_vec<8>(reinterpret_cast<float*>(d + at + q * 8), o);
        } else {
          T h[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) h[j] = from_f32<T>(o[j]);
          *reinterpret_cast<uint4*>(d + at + q * 8) = *reinterpret_cast<uint4*>(h);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (q * 8 + j >= left) break;
          const int64_t i = at + q * 8 + j;
          d[i] = from_f32<T>(w ? fmaf(keep, to_f32<T>(w[i]), -rate * o[j]) : o[j]);
        }
      }
    }
  }
};

template <int PLANES, typename Epi>
void product(const mma::Tensor& A, bool a_mn, const mma::Tensor& B, bool b_mn, int M, int N, int64_t K, int batch,
             bool sym, Epi epi, cudaStream_t s) {
  mma::Args a = {};
  a.batches = batch;
  a.a_mn = a_mn;
  a.b_mn = b_mn;
  // 256 x 256 tiles of CTA pairs where they fill half the device, else 128 x 128 ones
  const int64_t big = ceil_div(M, 256) * ceil_div(N, 256) * batch / (sym ? 2 : 1);
  const bool pair = big >= mma::num_sms() / 4;
  a.bn = pair ? 256 : 128;
  const int tm = pair ? 256 : 128;
  a.m_tiles = (int)ceil_div(M, tm);
  a.n_tiles = (int)ceil_div(N, a.bn);
  a.sym = sym;
  a.block = kBlock;
  a.a_rows = 128;
  const uint32_t id = mma::idesc(tm, a.bn, false, a_mn, b_mn);
  if (PLANES == 2) {
    a.seg[a.nseg++] = mma::segment(K, 0, batch, id);
    a.seg[a.nseg++] = mma::segment(K, batch, 0, id);
  }
  a.seg[a.nseg++] = mma::segment(K, 0, 0, id);
  const CUtensorMap ma = mma::tensor_map(A, a_mn ? 64 : 128);
  const CUtensorMap mb = mma::tensor_map(B, b_mn ? 64 : pair ? 128 : a.bn);
  if (pair)
    mma::launch<2, PLANES == 2>({ma, mb, ma, mb}, a, epi, s);
  else
    mma::launch<1, PLANES == 2>({ma, mb, ma, mb}, a, epi, s);
}

template <typename T, int VEC, int PLANES>
void normalise(const T* g, Direction a, int64_t batch, double eps, const OrthoLayout& l, cudaStream_t s) {
  a.units = a.cols / VEC;
  const int64_t n = (int64_t)a.rows * a.units;
  const unsigned parts = (unsigned)std::min<int64_t>(kParts, ceil_div(n, 256));
  launch_pdl(k_squares<T, VEC>, dim3(parts, (unsigned)batch), 256, s, g, a, l.part);
  LC_LAUNCH_CHECK("k_squares");
  const unsigned blocks = (unsigned)std::min<int64_t>(ceil_div(n, 512), 1024);
  launch_pdl(k_planes<T, VEC, PLANES>, dim3(blocks, (unsigned)batch), 256, s, g, a, (const double*)l.part, (int)parts, eps,
             l.x[0], l.ld, batch * l.x_plane, l.t);
  LC_LAUNCH_CHECK("k_planes");
}

template <int PLANES, typename TO>
void iterate(int batch, int rows, int cols, int steps, const double* co, void* out, const OrthoStep& st,
             const OrthoLayout& l, cudaStream_t s) {
  const bool tall = rows > cols;
  const int m = std::min(rows, cols), n = std::max(rows, cols);
  const int64_t xp = (int64_t)batch * l.x_plane, sp = (int64_t)batch * l.s_plane;
  const mma::Tensor S{l.s, m, m, (int64_t)PLANES * batch, l.sld, l.s_plane};
  const mma::Tensor P{l.p, m, m, (int64_t)PLANES * batch, l.sld, l.s_plane};
  const int tile = ceil_div(m, 256) * ceil_div(m, 256) * batch / 2 >= mma::num_sms() / 4 ? 256 : 128;
  for (int i = 0; i < steps; ++i) {
    const float a = (float)co[3 * i], b = (float)co[3 * i + 1], c = (float)co[3 * i + 2];
    const float* t = i == 0 ? l.t : nullptr;
    __half *x = l.x[i & 1], *y = l.x[(i & 1) ^ 1];
    const mma::Tensor X{x, cols, rows, (int64_t)PLANES * batch, l.ld, l.x_plane};
    SymEpi<PLANES> gram{l.s, nullptr, l.sld, l.s_plane, sp, m, tile, kSScale / (kXScale * kXScale), 0.f, t};
    product<PLANES>(X, tall, X, tall, m, m, n, batch, true, gram, s);
    // |P| <= 16 |b| + 256 |c| for singular values up to 4
    const float bound = 16.f * fabsf(b) + 256.f * fabsf(c);
    const float ps = exp2f(floorf(fminf(12.f, log2f(32768.f / fmaxf(bound, 1.f)))));
    SymEpi<PLANES> poly{l.p, l.s, l.sld, l.s_plane, sp, m, tile, c * ps / (kSScale * kSScale), b * ps / kSScale, nullptr};
    product<PLANES>(S, false, S, false, m, m, m, batch, true, poly, s);
    auto update = [&](auto epi) {
      if (tall)
        product<PLANES>(X, false, P, false, n, m, m, batch, false, epi, s);
      else
        product<PLANES>(P, false, X, true, m, n, m, batch, false, epi, s);
    };
    if (i + 1 < steps) {
      update(UpdateEpi<PLANES>{y, x, l.ld, l.x_plane, xp, rows, cols, 1.f / ps, a, t});
    } else {
      LastEpi<PLANES, TO> e{static_cast<TO*>(st.weight ? st.out_weight : out), static_cast<const TO*>(st.weight), x,
                            l.ld, l.x_plane, xp, rows, cols, 0, 1.f / (ps * kXScale), a / kXScale, st.keep, st.rate, t};
      e.vec = cols % 8 == 0 && ((uintptr_t)e.d & 15) == 0 && ((uintptr_t)e.w & 15) == 0;
      update(e);
    }
  }
}

int planes_of(int type) { return type == LIPCACHE_F32 ? 2 : 1; }

}  // namespace

size_t ortho_bytes(int type, int64_t batch, int rows, int cols) {
  OrthoLayout l;
  Carve c;
  l.take(c, planes_of(type), batch, rows, cols);
  return c.off;
}

void orthogonalize(int type, const void* G, int64_t ldg, int64_t batch, int rows, int cols, int steps,
                   const double* coefficients, double eps, void* out, const OrthoStep& st, unsigned char* ws,
                   cudaStream_t s) {
  const int out_type = st.weight ? st.weight_type : type, planes = planes_of(out_type);
  OrthoLayout l;
  Carve c{ws, 0};
  l.take(c, planes, batch, rows, cols);
  const Direction d{rows, cols, ldg, 0, st};
  const bool vec = cols % 8 == 0 && ldg % 8 == 0 && ((uintptr_t)G & 15) == 0 && ((uintptr_t)st.momentum & 15) == 0 &&
                   ((uintptr_t)st.out_momentum & 15) == 0;
  auto go = [&](auto g) {
    using T = std::remove_const_t<std::remove_pointer_t<decltype(g)>>;
    if (planes == 2)
      vec ? normalise<T, 8, 2>(g, d, batch, eps, l, s) : normalise<T, 1, 2>(g, d, batch, eps, l, s);
    else
      vec ? normalise<T, 8, 1>(g, d, batch, eps, l, s) : normalise<T, 1, 1>(g, d, batch, eps, l, s);
  };
  if (type == LIPCACHE_F32)
    go(static_cast<const float*>(G));
  else
    go(static_cast<const __nv_bfloat16*>(G));
  if (planes == 2)
    iterate<2, float>((int)batch, rows, cols, steps, coefficients, out, st, l, s);
  else
    iterate<1, __nv_bfloat16>((int)batch, rows, cols, steps, coefficients, out, st, l, s);
}

}  // namespace ops
}  // namespace lc

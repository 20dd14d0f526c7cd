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
// A matrix far below eps stays far below 1 after that: it is kept as Y = 2^k X,
// its largest singular value near 1, and each step takes from k what it lifts X
// by (lift_steps), so that it keeps the bits of the planes all the way.
//
// S and P are symmetric: tiles on or above the diagonal are computed and
// written twice. Nothing is transposed: a tall X is contracted over its rows,
// and P X reads X along its rows, by operands stored MN-major.
#include <cuda_fp16.h>

#include "head_mma.cuh"

namespace lc {
namespace ops {
namespace {

constexpr int kBigTile = 256;  // rows and columns of a tile of a CTA pair
constexpr int kParts = 512;      // partial sums of squares of a matrix, at most
constexpr float kXScale = 8192.f, kSScale = 1024.f;
constexpr int kBlock = 4;  // stages of 64 summed on the tensor cores at a time, FP32 matrices
constexpr int kPairBlock = 2;  // the same where products with low parts share the sum

struct OrthoLayout {
  __half *x[2], *s, *p;  // planes x batch x rows x ld
  float* t;              // batch: the rest of the normalisation
  float2* lift;          // batch x LIPCACHE_MAX_NS_STEPS: factors of each step (lift_steps)
  unsigned* phases;      // CTAs past each phase of k_iterate
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
    c.take(lift, (size_t)batch * LIPCACHE_MAX_NS_STEPS);
    c.take(phases, 1);
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
  int tail;       // elements past the units (one row)
  OrthoStep st;
};

// Elements [VEC] of the direction D, and (FIRST) the momentum's update.
template <typename T, int VEC, bool FIRST>
__device__ __forceinline__ void direction(const Direction& a, const T* g, int64_t row, int col, float (&v)[VEC]) {
  load_vec<T, VEC>(g + row * a.ldg + col, v);
  if (!a.st.weight) return;
  const int64_t at = row * a.cols + col;
  const float b = a.st.beta, r = a.st.fresh;
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
// A dense matrix may be given as one row.
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
  if (blockIdx.x == 0 && threadIdx.x < a.tail) {
    float v[1];
    direction<T, 1, true>(a, g, row0, a.units * VEC + threadIdx.x, v);
    sum += (double)v[0] * v[0];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) sum += red[w];
    part[blockIdx.y * gridDim.x + blockIdx.x] = sum;
  }
}

struct Steps {
  int n;
  float coef[3 * LIPCACHE_MAX_NS_STEPS];
};

// Y = 2^k X in step i: P = b S + c q S S and Y' = w (a Y + q P Y), S = Y Y^T, with
// q = 4^-k and w = 2^(k' - k); the last step gives X itself (k' = 0). Once k = 0 it
// stays there, and both factors are 1. While it is not, singular values of Y are
// at most `top` (2 at first): p(s) / s is at most |a| + |b| q top^2 + |c| q^2 top^4,
// and k' is what keeps the next ones in [1, 2) of that bound.
__device__ __forceinline__ void lift_steps(double t, const Steps& st, float* rest, float2* lift) {
  int x;
  frexp(t, &x);
  int k = max(0, 1 - x);
  *rest = (float)ldexp(t, k);
  float top = 2.f;
  for (int i = 0; i < st.n; ++i) {
    if (k == 0) {
      lift[i] = make_float2(1.f, 1.f);
      continue;
    }
    const float q = k < 75 ? ldexpf(1.f, -2 * k) : 0.f, s = q * top * top;
    int r = k;
    if (i + 1 < st.n) {
      const float next = top * (fabsf(st.coef[3 * i]) + s * (fabsf(st.coef[3 * i + 1]) + s * fabsf(st.coef[3 * i + 2])));
      frexpf(next, &r);
      r = next > 0.f ? min(r - 1, k) : 0;
      top = ldexpf(next, -r);
    }
    lift[i] = make_float2(q, ldexpf(1.f, -r));
    k -= r;
  }
}

// X's planes: D times 2^-e and kXScale, ||D|| < 2^e <= 2 ||D||.
template <typename T, int VEC, int PLANES>
__global__ void __launch_bounds__(256)
    k_planes(const T* g, const Direction a, const double* part, int parts, double eps, const Steps steps, __half* x,
             int64_t ld, int64_t plane, float* t, float2* lift, unsigned* phases) {
  __shared__ float factor[2];  // (2^-e alone can be past FP32's range)
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *phases = 0;
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += 32) sum += part[blockIdx.y * parts + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x == 0) {
      const double norm = sqrt(sum);
      int e = 0;
      frexp(norm > 0.0 ? norm : 1.0, &e);  // norm < 2^e
      const bool fine = isfinite(norm);
      factor[0] = fine ? ldexpf(kXScale, min(-e, 100)) : NAN;
      factor[1] = ldexpf(1.f, max(-e - 100, 0));
      if (blockIdx.x == 0) {
        lift_steps(fine ? ldexp(1.0, e) / (norm + eps) : 1.0, steps, t + blockIdx.y,
                   lift + (int64_t)blockIdx.y * LIPCACHE_MAX_NS_STEPS);
        if (!fine) t[blockIdx.y] = NAN;
      }
    }
  }
  __syncthreads();
  const float f = factor[0], f1 = factor[1];
  const uint32_t n = (uint32_t)a.rows * (uint32_t)a.units;
  const int64_t row0 = (int64_t)blockIdx.y * a.rows;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const uint32_t r = i / (uint32_t)a.units;
    const int col = (int)(i - r * (uint32_t)a.units) * VEC;
    float v[VEC];
    direction<T, VEC, false>(a, g, row0 + r, col, v);
    __half* d = x + (row0 + r) * ld + col;
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[j] = v[j] * f * f1;  // powers of two
    if constexpr (VEC == 8) {
      uint32_t hi[4], lo[4];
      split_f16(v, hi, lo);
      *reinterpret_cast<uint4*>(d) = uint4{hi[0], hi[1], hi[2], hi[3]};
      if (PLANES == 2) *reinterpret_cast<uint4*>(d + plane) = uint4{lo[0], lo[1], lo[2], lo[3]};
    } else {
      const __half hi = __float2half_rn(v[0]);
      d[0] = hi;
      if (PLANES == 2) d[plane] = __float2half_rn(v[0] - __half2float(hi));
    }
  }
}

// ---------------------------------------------------------------- epilogues
// 32 columns of a row (`left` of them in the matrix; up to the row's stride may
// be written) as planes, and mirrored: down a column of stride ld, 32 lanes
// side by side.
template <int PLANES>
__device__ __forceinline__ void put_planes(__half* d, int64_t plane, __half* mirror, int64_t ld, int left,
                                           const float (&v)[32]) {
  uint32_t hi[16], lo[16];
  split_f16(v, hi, lo);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (q * 8 >= left) break;
    *reinterpret_cast<uint4*>(d + q * 8) = uint4{hi[4 * q], hi[4 * q + 1], hi[4 * q + 2], hi[4 * q + 3]};
    if (PLANES == 2)
      *reinterpret_cast<uint4*>(d + plane + q * 8) = uint4{lo[4 * q], lo[4 * q + 1], lo[4 * q + 2], lo[4 * q + 3]};
  }
  if (mirror) {
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      if (j >= left) break;
      mirror[j * ld] = __ushort_as_half((uint16_t)(hi[j / 2] >> (j & 1) * 16));
      if (PLANES == 2) mirror[plane + j * ld] = __ushort_as_half((uint16_t)(lo[j / 2] >> (j & 1) * 16));
    }
  }
}
// v += f (eight FP16 values)
__device__ __forceinline__ void add_f16(const uint4& w, float f, float* v) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 h = open_f16(x[i]);
    v[2 * i] = fmaf(f, h.x, v[2 * i]);
    v[2 * i + 1] = fmaf(f, h.y, v[2 * i + 1]);
  }
}
// v += f (the values of the planes)
template <int PLANES>
__device__ __forceinline__ void add_planes(const __half* d, int64_t plane, int left, float f, float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (q * 8 >= left) break;
    const uint4 w = __ldcg(reinterpret_cast<const uint4*>(d + q * 8));
    add_f16(w, f, &v[q * 8]);
    if (PLANES == 2) add_f16(__ldcg(reinterpret_cast<const uint4*>(d + plane + q * 8)), f, &v[q * 8]);
  }
}

struct Nothing {};

// S (of = null) or P = c q S S + b S, both triangles.
template <int PLANES>
struct SymEpi {
  static constexpr bool kTurns = false, kEarly = false;
  using Head = Nothing;
  __device__ __forceinline__ void load(int, int, int, int, Nothing&) const {}
  __half* d;
  const __half* of;
  int64_t ld, mat, plane;  // row, matrix and plane strides
  int m;
  float f, b;
  const float* t;      // nullable: squared into f
  const float2* lift;  // of this step (P)
  __device__ __forceinline__ void store(int row0, int col0, int z, int lane, bool, uint32_t, const uint32_t (&acc)[32], const Nothing&, int) const {
    const int row = row0 + lane, left = m - col0;
    if (left <= 0) return;
    float g = f;
    if (t) g *= __ldcg(t + z) * __ldcg(t + z);
    if (of) g *= __ldg(lift + (int64_t)z * LIPCACHE_MAX_NS_STEPS).x;
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = g * __uint_as_float(acc[j]);
    const int64_t at = z * mat + row * ld + col0;
    if (row >= m) return;
    if (of) add_planes<PLANES>(of + at, plane, left, b, v);
    const bool off_diagonal = row0 / kBigTile != col0 / kBigTile;
    put_planes<PLANES>(d + at, plane, off_diagonal ? d + z * mat + col0 * ld + row : nullptr, ld, left, v);
  }
};

// X' = w (a X + q P X).
template <int PLANES>
struct UpdateEpi {
  static constexpr bool kTurns = false, kEarly = false;
  using Head = Nothing;
  __device__ __forceinline__ void load(int, int, int, int, Nothing&) const {}
  __half* d;
  const __half* x;
  int64_t ld, mat, plane;
  int rows, cols;
  float f, a;
  const float* t;
  const float2* lift;
  __device__ __forceinline__ void store(int row0, int col0, int z, int lane, bool, uint32_t, const uint32_t (&acc)[32], const Nothing&, int) const {
    const int row = row0 + lane, left = cols - col0;
    if (left <= 0 || row >= rows) return;
    const float2 qw = __ldg(lift + (int64_t)z * LIPCACHE_MAX_NS_STEPS);
    const float u = (t ? __ldcg(t + z) : 1.f) * qw.y, g = f * u * qw.x;
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = g * __uint_as_float(acc[j]);
    const int64_t at = z * mat + row * ld + col0;
    add_planes<PLANES>(x + at, plane, left, a * u, v);
    put_planes<PLANES>(d + at, plane, nullptr, 0, left, v);
  }
};

// The last step: the result, or the weights' update, in the caller's type.
template <int PLANES, typename T>
struct LastEpi {
  static constexpr bool kTurns = false, kEarly = false;
  using Head = Nothing;
  __device__ __forceinline__ void load(int, int, int, int, Nothing&) const {}
  T* d;
  const T* w;  // null: the result itself
  const __half* x;
  int64_t ld, mat, plane;
  int rows, cols, vec;
  float f, a, keep, rate;
  const float* t;
  const float2* lift;
  __device__ __forceinline__ void store(int row0, int col0, int z, int lane, bool, uint32_t, const uint32_t (&acc)[32], const Nothing&, int) const {
    const int row = row0 + lane, left = cols - col0;
    if (left <= 0 || row >= rows) return;
    const float2 qw = __ldg(lift + (int64_t)z * LIPCACHE_MAX_NS_STEPS);
    const float u = (t ? __ldcg(t + z) : 1.f) * qw.y, g = f * u * qw.x;
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
          *reinterpret_cast<uint4*>(d + at + q * 8) =
              uint4{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]), pack_bf16(o[4], o[5]), pack_bf16(o[6], o[7])};
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

// The power of two P carries: |P| <= 16 |b| + 256 |c| for singular values up
// to 4 stays below 2^15.
float poly_scale(float b, float c) {
  const float bound = 16.f * fabsf(b) + 256.f * fabsf(c);
  return exp2f(floorf(fminf(12.f, log2f(32768.f / fmaxf(bound, 1.f)))));
}

// ---------------------------------------------------------------- one launch
// Matrices whose tiles do not fill the device several times over: all steps in
// one cooperative launch, their products (phases) parted by a barrier over the
// grid. Tiles of 128 x 128, or x 64 where those leave CTAs idle, one CTA each; a
// stage holds 64 of the contracted index of every plane of both operands, so that
// the three products of FP32 planes read each once. Where a phase has few tiles, a
// cluster of `split` CTAs shares one: each sums a part of the contracted index,
// and the parts meet in the shared memory of the CTA that writes that slice of the
// tile's columns. Products with a low part have a sum of their own, 2^-11 of the
// other, so that this is cut off a third as often (an addition in tensor memory is
// not rounded). The blocks of a sum meet in tensor memory, eight columns a turn of
// a loop: straight-line code for a whole tile is fetched anew in every phase (10 to
// 30 us a phase). What a tile gives leaves through TMA, as does its mirror
// image.
// Bound by the phases' latency (a barrier, the first loads, the join, the writes:
// 4 to 6 us) until the products take longer. Five steps: 200 x 256 FP32 120 us (141
// with tiles of 128 columns only), 2,001 x 1,003 FP32 255 us (a launch a product
// 598), 137 TFLOP/s.
constexpr int kCluster = 4;
constexpr int kTile = 128, kTileBytes = 128 * 128;
// What a warp of the epilogue has to itself: others' parts of its 32 rows (three
// of 32 columns, or one of 64; four columns of the rows side by side), then what
// it sends to memory.
constexpr int kPartBytes = 12 * 1024;

struct IterateArgs {
  CUtensorMap xk[2], xm[2], s, p, s64, p64;  // X's two buffers, S and P with boxes of 128 rows, and of 64
  CUtensorMap to[4];               // X's buffers, S and P to write to (boxes of 32 x 32)
  int tall, batch, m, n, steps;
  int split[3], bn[3];             // of S, P and X' phases; bn: columns of a tile, 128 or (unsplit) 64
  float coef[3 * LIPCACHE_MAX_NS_STEPS], ps[LIPCACHE_MAX_NS_STEPS];
  const float* t;
  const float2* lift;
  void* out;
  const void* weight;
  int rows, cols, vec;
  float keep, rate;
  unsigned* phases;
  unsigned long long* errors;
};

// Tiles on or above the diagonal of rt x ct ones that are `wide` to a square.
__host__ __device__ inline int upper_tiles(int rt, int ct, int wide) { return rt * ct - wide * (rt * (rt - 1) / 2); }

__device__ __forceinline__ unsigned load_acquire(const unsigned* p) {
  unsigned v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void add_release(unsigned* p) {
  asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p) : "memory");
}
// Waits until `want` CTAs have passed; false when it gives up.
__device__ __forceinline__ bool wait_phase(const unsigned* p, unsigned want, volatile int* abort) {
  const long long t0 = clock64();
  while (load_acquire(p) < want) {
    if (*abort) return false;
    if (clock64() - t0 > mma::kWaitLimit) {
      *abort = 1;
      return false;
    }
  }
  return true;
}

// The same as the result, or the weights' update, in the caller's type.
template <typename TO>
__device__ __forceinline__ void put_result(const IterateArgs& a, int64_t at, int left, const float (&v)[32]) {
  TO* o = static_cast<TO*>(a.out) + at;
  const TO* w = a.weight ? static_cast<const TO*>(a.weight) + at : nullptr;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (q * 8 >= left) break;
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = v[q * 8 + j];
    if (a.vec) {
      if (w) {
        float old[8];
        load_vec<TO, 8>(w + q * 8, old);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = fmaf(a.keep, old[j], -a.rate * r[j]);
      }
      if constexpr (sizeof(TO) == 4) {
        store_vec<8>(reinterpret_cast<float*>(o + q * 8), r);
      } else {
        *reinterpret_cast<uint4*>(o + q * 8) =
            uint4{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3]), pack_bf16(r[4], r[5]), pack_bf16(r[6], r[7])};
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (q * 8 + j < left) o[q * 8 + j] = from_f32<TO>(w ? fmaf(a.keep, to_f32<TO>(w[q * 8 + j]), -a.rate * r[j]) : r[j]);
    }
  }
}

// Counts the epilogue's warps as they pass; true for the eighth (nobody waits,
// so that a warp that has given up holds up no other).
__device__ __forceinline__ bool last_of_eight(uint32_t* count) {
  __threadfence_block();
  if (atomicAdd(count, 1u) + 1 < mma::kEpiWarps) return false;
  *reinterpret_cast<volatile uint32_t*>(count) = 0;
  __threadfence_block();
  return true;
}

template <int PLANES, typename TO>
__global__ void __launch_bounds__(mma::kThreads, 1) k_iterate(const __grid_constant__ IterateArgs a) {
  constexpr int kStageBytes = 2 * PLANES * kTileBytes, kStages = PLANES == 2 ? 2 : 5;
  constexpr int kSendBytes = 6144 * PLANES;  // two blocks of 32 x 32 and a mirror image, in planes
  constexpr int kRegionBytes = 4 * kPartBytes > 8 * kSendBytes ? 4 * kPartBytes : 8 * kSendBytes;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t region = base + kStages * kStageBytes;
  const uint32_t full = region + kRegionBytes, empty = full + 8 * kStages, acc_full = empty + 8 * kStages,
                 acc_empty = acc_full + 16, ready = acc_empty + 16, got = ready + 8, drain = got + 8,
                 go = drain + 8, low_empty = go + 8, misc = low_empty + 8;
  unsigned char* misc_p = smem_raw + (misc - ptx::smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc_p);
  volatile int* abort_s = reinterpret_cast<volatile int*>(misc_p + 4);
  // warps done with what is added to even tiles and to odd ones, with the phase
  uint32_t* counts = reinterpret_cast<uint32_t*>(misc_p + 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)ptx::cluster_ctarank();
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(full + 8 * s, 1);
      ptx::mbar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(acc_full + 8 * b, 1);
      ptx::mbar_init(acc_empty + 8 * b, mma::kEpiWarps);
    }
    // the join: every CTA is done with the parts of the join before; the others' parts are here
    ptx::mbar_init(ready, kCluster * mma::kEpiWarps);
    ptx::mbar_init(got, (kCluster - 1) * mma::kEpiWarps);
    ptx::mbar_init(drain, 1);
    ptx::mbar_init(go, 1);  // the producer has seen the barrier over the grid
    ptx::mbar_init(low_empty, mma::kEpiWarps);
    *abort_s = 0;
    counts[0] = counts[1] = counts[2] = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 1) {
    ptx::tmem_alloc(misc, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  ptx::cluster_sync();
  ptx::wait_prerequisites();
  const uint32_t tmem = *tmem_slot;
  const int rows_x = a.tall ? a.n : a.m, cols_x = a.tall ? a.m : a.n;  // of X as it is stored

  // The work of a phase, the same for every role.
  struct Work {
    int kind, split, bn, rt, ct, per, tiles, chunks, workers, me;
  };
  auto phase_of = [&](int i, int k) {
    Work w;
    w.kind = k == 2 ? (i == a.steps - 1 ? 3 : 2) : k;
    w.split = a.split[k];
    w.bn = a.bn[k];
    w.rt = ((k == 2 ? rows_x : a.m) + kTile - 1) / kTile;
    w.ct = ((k == 2 ? cols_x : a.m) + w.bn - 1) / w.bn;
    w.per = k == 2 ? w.rt * w.ct : upper_tiles(w.rt, w.ct, kTile / w.bn);
    w.tiles = w.per * a.batch;
    w.chunks = ((k == 0 ? a.n : a.m) + 63) / 64;
    w.workers = w.split > 1 ? (int)gridDim.x / kCluster : (int)gridDim.x;
    w.me = w.split > 1 ? (int)blockIdx.x / kCluster : (int)blockIdx.x;
    return w;
  };
  // (a split of two uses half the cluster)
  auto tile = [&](const Work& w, int t, int& r, int& c, int& z) {
    z = t / w.per;
    t -= z * w.per;
    if (w.kind < 2) {
      // on or above the diagonal, row by row
      const int wide = kTile / w.bn;
      r = 0;
      while (t >= w.ct - r * wide) t -= w.ct - r * wide, ++r;
      c = r * wide + t;
    } else {
      r = t / w.ct;
      c = t - r * w.ct;
    }
  };
  auto range = [&](const Work& w, int& c0, int& c1) {
    const int part = w.split > 1 ? rank : 0;
    c0 = part >= w.split ? 0 : w.chunks * part / w.split;
    c1 = part >= w.split ? 0 : w.chunks * (part + 1) / w.split;
  };

  // whether this CTA's tiles have something added to the product
  auto adds = [&](const Work& w) { return w.kind > 0 && (w.split == 1 || rank < w.split); };

  if (warp == 0) {
    // ------------------------------------------------------------ producer
    if (lane == 0) {
      int st = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int i = 0; i < a.steps && ok; ++i)
        for (int k = 0; k < 3 && ok; ++k) {
          const Work w = phase_of(i, k);
          const bool kx = i & 1;
          ok = wait_phase(a.phases, (unsigned)(3 * i + k) * gridDim.x, abort_s);
          if (!ok) break;
          ptx::mbar_arrive(go);
          asm volatile("fence.proxy.async.global;" ::: "memory");
          const bool amn = k == 0 && a.tall, bmn = amn || (k == 2 && !a.tall);
          const CUtensorMap* ma = k == 0 ? (a.tall ? &a.xm[kx] : &a.xk[kx]) : k == 1 ? &a.s : a.tall ? &a.xk[kx] : &a.p;
          const bool half = w.bn == 64;  // B K-major: a box of 64 rows
          const CUtensorMap* mb = bmn ? &a.xm[kx] : k == 0 ? (half ? &a.xm[kx] : &a.xk[kx]) : k == 1 ? (half ? &a.s64 : &a.s) : half ? &a.p64 : &a.p;
          int c0, c1;
          range(w, c0, c1);
          for (int t = w.me; t < w.tiles && ok; t += w.workers) {
            int r, c, z;
            tile(w, t, r, c, z);
            for (int q = c0; q < c1 && ok; ++q) {
              ok = ptx::mbar_wait(empty + 8 * st, ph ^ 1u, abort_s, mma::kWaitLimit);
              if (!ok) break;
              const uint32_t dst = base + st * kStageBytes, bar = full + 8 * st;
              ptx::mbar_expect_tx(bar, (uint32_t)(PLANES * (kTileBytes + w.bn * 128)));
              for (int pl = 0; pl < PLANES; ++pl) {
                const int zz = pl * a.batch + z;
                const uint32_t da = dst + pl * kTileBytes, db = dst + (PLANES + pl) * kTileBytes;
                if (amn) {
                  mma::load_3d(da, ma, r * kTile, q * 64, zz, bar);
                  mma::load_3d(da + 8192, ma, r * kTile + 64, q * 64, zz, bar);
                } else {
                  mma::load_3d(da, ma, q * 64, r * kTile, zz, bar);
                }
                if (bmn) {
                  mma::load_3d(db, mb, c * w.bn, q * 64, zz, bar);
                  if (!half) mma::load_3d(db + 8192, mb, c * w.bn + 64, q * 64, zz, bar);
                } else {
                  mma::load_3d(db, mb, q * 64, c * w.bn, zz, bar);
                }
              }
              if (++st == kStages) st = 0, ph ^= 1u;
            }
            if (ok && adds(w)) {
              // what the epilogue adds to the product, a stage of its own: the halves of the tile this CTA writes
              ok = ptx::mbar_wait(empty + 8 * st, ph ^ 1u, abort_s, mma::kWaitLimit);
              if (!ok) break;
              const uint32_t dst = base + st * kStageBytes, bar = full + 8 * st;
              const CUtensorMap* mi = k == 1 ? &a.s : &a.xk[kx];
              const int h0 = w.split == 1 ? 0 : w.split == 2 ? rank : rank >> 1, h1 = w.split == 1 ? w.bn / 64 : h0 + 1;
              ptx::mbar_expect_tx(bar, (uint32_t)((h1 - h0) * PLANES * kTileBytes));
              for (int h = h0; h < h1; ++h)
                for (int pl = 0; pl < PLANES; ++pl)
                  mma::load_3d(dst + (h * PLANES + pl) * kTileBytes, mi, c * w.bn + 64 * h, r * kTile, pl * a.batch + z, bar);
              if (++st == kStages) st = 0, ph ^= 1u;
            }
          }
        }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    const bool lead = ptx::elect_one();
    int st = 0, n = 0, lows = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int i = 0; i < a.steps && ok; ++i)
      for (int k = 0; k < 3 && ok; ++k) {
        const Work w = phase_of(i, k);
        const bool amn = k == 0 && a.tall, bmn = amn || (k == 2 && !a.tall);
        const uint32_t id = mma::idesc(128, w.bn, false, amn, bmn);
        int c0, c1;
        range(w, c0, c1);
        const int last_steps = ((k == 0 ? a.n : a.m) - (w.chunks - 1) * 64 + 15) / 16;
        for (int t = w.me; t < w.tiles && ok; t += w.workers) {
          uint32_t acc_low = 0;
          if (PLANES == 2 && c1 > c0) {
            // the tile's sum of products with low parts, read by the epilogue of the tile before
            ok = ptx::mbar_wait_warp(low_empty, (uint32_t)(lows & 1) ^ 1u, abort_s, mma::kWaitLimit);
            ptx::tc_fence_after();
            ++lows;
          }
          for (int b0 = c0; b0 < c1 && ok; b0 += kBlock, ++n) {
            ok = ptx::mbar_wait_warp(acc_empty + 8 * (n & 1), (uint32_t)((n >> 1) & 1) ^ 1u, abort_s, mma::kWaitLimit);
            if (!ok) break;
            ptx::tc_fence_after();
            const uint32_t d = tmem + (uint32_t)(n & 1) * 128u;
            const int b1 = PLANES == 2 ? min(b0 + kBlock, c1) : c1;
            for (int q = b0; q < b1 && ok; ++q) {
              ok = ptx::mbar_wait_warp(full + 8 * st, ph, abort_s, mma::kWaitLimit);
              if (!ok) break;
              ptx::tc_fence_after();
              if (lead) {
                const uint32_t sa = base + st * kStageBytes, sb = sa + PLANES * kTileBytes;
                const int steps = q == w.chunks - 1 ? last_steps : 4;
                uint32_t acc = q > b0;
                // lo hi, hi lo, hi hi
                for (int pr = PLANES == 2 ? 0 : 2; pr < 3; ++pr) {
                  uint64_t da = mma::desc(sa + (pr == 0 ? kTileBytes : 0), amn), db = mma::desc(sb + (pr == 1 ? kTileBytes : 0), bmn);
                  for (int e = 0; e < steps; ++e, da += amn ? 2048 >> 4 : 32 >> 4, db += bmn ? 2048 >> 4 : 32 >> 4) {
                    if (pr < 2) {
                      ptx::mma_f16(tmem + 384u, da, db, id, acc_low);
                      acc_low = 1;
                    } else {
                      ptx::mma_f16(d, da, db, id, acc);
                      acc = 1;
                    }
                  }
                }
                ptx::mma_commit(empty + 8 * st);
              }
              if (++st == kStages) st = 0, ph ^= 1u;
            }
            if (ok && lead) ptx::mma_commit(acc_full + 8 * (n & 1));
            if (PLANES == 1) b0 = c1;
          }
          if (adds(w) && ++st == kStages) st = 0, ph ^= 1u;
        }
      }
    if (lead) {
      volatile int never = 0;
      ptx::mma_commit(drain);
      ptx::mbar_wait(drain, 0, &never, mma::kWaitLimit);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ epilogue
    // A warp: 32 rows, half the columns as blocks of 32 x 32. Blocks go to memory
    // by way of shared memory and TMA, mirror images too: a store a row from
    // registers takes a cycle for every 16 bytes (128 x 128 FP32 tiles: 9,000
    // clocks of a phase).
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    int n = 0, joins = 0, st = 0, added = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int i = 0; i < a.steps && ok; ++i)
      for (int k = 0; k < 3 && ok; ++k) {
        const Work w = phase_of(i, k);
        ok = ptx::mbar_wait_warp(go, (uint32_t)(3 * i + k) & 1u, abort_s, mma::kWaitLimit);
        const float ps = a.ps[i];
        const bool split = w.split > 1;
        const int slice = w.bn / w.split, hw = w.bn / 2;  // hw: this warp's columns
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + half * hw, sums = lanes + 256, lows = lanes + 384;
        const int rows = k < 2 ? a.m : a.rows, cols = k < 2 ? a.m : a.cols;
        const bool mine = !split || half * hw / slice == rank || (half * hw + 32) / slice == rank;
        const uint32_t own = region + (split ? quarter * kPartBytes : (half * 4 + quarter) * kSendBytes);
        const CUtensorMap* to = k == 0 ? &a.to[2] : k == 1 ? &a.to[3] : &a.to[(i & 1) ^ 1];
        int c0, c1;
        range(w, c0, c1);
        for (int t = w.me; t < w.tiles && ok; t += w.workers) {
          int r, c, z;
          tile(w, t, r, c, z);
          const float tn = i == 0 ? __ldcg(a.t + z) : 1.f;
          const float2 qw = __ldg(a.lift + (int64_t)z * LIPCACHE_MAX_NS_STEPS + i);
          float f, g = 0.f;
          if (k == 0) {
            f = tn * tn * (kSScale / (kXScale * kXScale));
          } else if (k == 1) {
            f = a.coef[3 * i + 2] * ps / (kSScale * kSScale) * qw.x;
            g = a.coef[3 * i + 1] * ps / kSScale;
          } else {
            const float last = w.kind == 3 ? qw.y / kXScale : qw.y;
            f = tn * last / ps * qw.x;
            g = tn * last * a.coef[3 * i];
          }
          const int row = r * kTile + quarter * 32 + lane, col = c * w.bn + half * hw;
          // blocks of the sum meet in tensor memory
          uint32_t src = sums;
          const int blocks = c1 <= c0 ? 0 : PLANES == 2 ? (c1 - c0 + kBlock - 1) / kBlock : 1;
          for (int b = 0; b < blocks; ++b, ++n) {
            ok = ptx::mbar_wait_warp(acc_full + 8 * (n & 1), (uint32_t)((n >> 1) & 1), abort_s, mma::kWaitLimit);
            if (!ok) break;
            ptx::tc_fence_after();
            src = lanes + (uint32_t)(n & 1) * 128u;
            if (blocks == 1) break;
#pragma unroll 1
            for (int q = 0; q < hw; q += 8) {
              float v[8];
              mma::tmem_ld8(src + q, v);
              if (b > 0) {
                float s[8];
                mma::tmem_ld8(sums + q, s);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += s[j];
              }
              mma::tmem_st8(sums + q, v);
            }
            mma::tmem_wait_st();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(acc_empty + 8 * (n & 1));
            src = sums;
          }
          if (!ok) break;
          st += c1 - c0;
          while (st >= kStages) st -= kStages, ph ^= 1u;
          if (split) {
            // every CTA has read the parts of the join before
            if (joins) ok = ptx::mbar_wait_warp<true>(ready, (uint32_t)(joins - 1) & 1u, abort_s, mma::kWaitLimit);
            if (!ok) break;
            // columns [slice o, + slice) go to CTA o, into the sender's slot there
            if (blocks) {
#pragma unroll 1
              for (int p = 0; p < 2; ++p) {
                const int first = half * hw + p * 32, owner = first / slice;
                if (owner == rank) continue;
                uint32_t v[32];
                ptx::tmem_ld32(src + p * 32, v);
                if (PLANES == 2) {
                  uint32_t low[32];
                  ptx::tmem_ld32(lows + p * 32, low);
                  ptx::tmem_wait_ld();
#pragma unroll
                  for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + __uint_as_float(low[j]));
                }
                ptx::tmem_wait_ld();
                const int slot = rank < owner ? rank : rank - 1;
                const uint32_t dst = ptx::mapa(region + quarter * kPartBytes, owner) +
                                     (uint32_t)(slot * slice * 128 + (first - owner * slice) * 128 + lane * 16);
#pragma unroll
                for (int j = 0; j < 32; j += 4)
                  asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + j * 128), "r"(v[j]),
                               "r"(v[j + 1]), "r"(v[j + 2]), "r"(v[j + 3])
                               : "memory");
              }
            }
            __syncwarp();
            if (lane < kCluster && lane != rank) ptx::mbar_arrive_cluster(ptx::mapa(got, lane));
            ok = ptx::mbar_wait_warp<true>(got, (uint32_t)joins & 1u, abort_s, mma::kWaitLimit);
            if (!ok) break;
          }
          const uint32_t in = base + st * kStageBytes + (quarter * 32 + lane) * 128;
          if (adds(w)) {
            ok = ptx::mbar_wait_warp(full + 8 * st, ph, abort_s, mma::kWaitLimit);
            if (!ok) break;
          }
          float v[2][32];
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const int first = half * hw + p * 32, owner = first / slice;
            if (p * 32 >= hw || (split && owner != rank)) continue;
            uint32_t bits[32];
            ptx::tmem_ld32(src + p * 32, bits);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) v[p][j] = blocks ? __uint_as_float(bits[j]) : 0.f;
            if (PLANES == 2 && blocks) {
              ptx::tmem_ld32(lows + p * 32, bits);
              ptx::tmem_wait_ld();
#pragma unroll
              for (int j = 0; j < 32; ++j) v[p][j] += __uint_as_float(bits[j]);
            }
            if (split) {
              // the parts in their order: those of lower CTAs, this one's, those of higher ones
              float s[32];
#pragma unroll
              for (int j = 0; j < 32; ++j) s[j] = 0.f;
#pragma unroll 1
              for (int part = 0; part < w.split; ++part) {
                if (part == rank) {
#pragma unroll
                  for (int j = 0; j < 32; ++j) s[j] += v[p][j];
                  continue;
                }
                const uint32_t o = own + (uint32_t)((part < rank ? part : part - 1) * slice * 128 +
                                                    (first - owner * slice) * 128 + lane * 16);
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                  float e[4];
                  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                               : "=f"(e[0]), "=f"(e[1]), "=f"(e[2]), "=f"(e[3])
                               : "r"(o + j * 128)
                               : "memory");
#pragma unroll
                  for (int q = 0; q < 4; ++q) s[j + q] += e[q];
                }
              }
#pragma unroll
              for (int j = 0; j < 32; ++j) v[p][j] = s[j];
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) v[p][j] *= f;
            if (k > 0) {
#pragma unroll
              for (int l = 0; l < PLANES; ++l)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                  uint4 e;
                  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                               : "=r"(e.x), "=r"(e.y), "=r"(e.z), "=r"(e.w)
                               : "r"(in + ((first >> 6) * PLANES + l) * kTileBytes + ((((first & 63) / 8 + q) ^ (lane & 7)) << 4))
                               : "memory");
                  add_f16(e, g, &v[p][q * 8]);
                }
            }
          }
          if (adds(w)) {
            // The last of the eight warps gives the stage back. Tiles count apart by turns: with one
            // sum a tile (one plane) a warp may be a tile ahead of another, but not two, since the
            // accumulator of the tile after next waits for all eight, who count before they free it.
            __syncwarp();
            if (lane == 0 && last_of_eight(counts + (added & 1))) ptx::mbar_arrive(empty + 8 * st);
            ++added;
            if (++st == kStages) st = 0, ph ^= 1u;
          }
          ptx::tc_fence_before();
          __syncwarp();
          if (PLANES == 2 && blocks && lane == 0) ptx::mbar_arrive(low_empty);
          if (blocks == 1) {
            if (lane == 0) ptx::mbar_arrive(acc_empty + 8 * (n & 1));
            ++n;
          }
          __syncwarp();  // the warp has read its parts
          if (mine && w.kind < 3) {
            const bool mirror = k < 2 && r != c * w.bn / kTile;
            bool busy = false;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              const int first = half * hw + p * 32;
              if (p * 32 >= hw || (split && first / slice != rank)) continue;
              uint32_t hl[2][16];
              split_f16(v[p], hl[0], hl[1]);
              // what stood there has left: the tile before, or the mirror image before
              if (!busy || (mirror && p == 1)) {
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                __syncwarp();
                busy = true;
              }
#pragma unroll
              for (int l = 0; l < PLANES; ++l) {
                const uint32_t at = own + (p * PLANES + l) * 2048 + lane * 64;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + ((q ^ ((lane >> 1) & 3)) << 4)),
                               "r"(hl[l][4 * q]), "r"(hl[l][4 * q + 1]), "r"(hl[l][4 * q + 2]), "r"(hl[l][4 * q + 3])
                               : "memory");
                if (mirror) {
                  // lanes in pairs: the even one writes its and its neighbour's column 2 q, the odd one 2 q + 1
                  const uint32_t to_m = own + (2 * PLANES + l) * 2048 + ((lane & 7) >> 1) * 4;
#pragma unroll
                  for (int q = 0; q < 16; ++q) {
                    const uint32_t other = __shfl_xor_sync(0xffffffffu, hl[l][q], 1);
                    const int j = 2 * q + (lane & 1);
                    const uint32_t word = lane & 1 ? __byte_perm(other, hl[l][q], 0x7632) : __byte_perm(hl[l][q], other, 0x5410);
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(to_m + j * 64 + (((lane >> 3) ^ ((j >> 1) & 3)) << 4)), "r"(word)
                                 : "memory");
                  }
                }
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) {
                const int x = col + p * 32, y = r * kTile + quarter * 32;
                for (int l = 0; l < PLANES; ++l) {
                  if (x < cols && y < rows) mma::store_3d(to, x, y, l * a.batch + z, own + (p * PLANES + l) * 2048);
                  if (mirror && x < cols && y < rows) mma::store_3d(to, y, x, l * a.batch + z, own + (2 * PLANES + l) * 2048);
                }
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
              }
            }
          } else if (mine) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              const int first = half * hw + p * 32, left = cols - col - p * 32;
              if (p * 32 >= hw || (split && first / slice != rank) || left <= 0 || row >= rows) continue;
              put_result<TO>(a, ((int64_t)z * a.rows + row) * a.cols + col + p * 32, left, v[p]);
            }
          }
          if (split) {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
            if (lane < kCluster) ptx::mbar_arrive_cluster(ptx::mapa(ready, lane));
            ++joins;
          }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        // written, and readable by copies of other CTAs; the last warp says so
        asm volatile("fence.proxy.async.global;" ::: "memory");
        __syncwarp();
        if (lane == 0 && last_of_eight(counts + 2)) add_release(a.phases);
      }
  }
  __syncthreads();
  if (*abort_s) {
    const long long t0 = clock64();
    while (clock64() - t0 < (1LL << 23)) {
    }
    if (threadIdx.x == 0) atomicAdd(a.errors, 1ull);
    __syncthreads();
  }
  ptx::tc_fence_after();
  ptx::cluster_sync();
  if (warp == 1) ptx::tmem_dealloc(tmem, 512);
}

template <int PLANES, typename TO>
int iterate_ctas() {
  static int known[64] = {};
  int dev = 0;
  LC_CUDA(cudaGetDevice(&dev));
  if (dev < 64 && known[dev]) return known[dev];
  allow_smem(reinterpret_cast<const void*>(k_iterate<PLANES, TO>), mma::kSmem);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kCluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(mma::num_sms() / kCluster * kCluster));
  cfg.blockDim = dim3(mma::kThreads);
  cfg.dynamicSmemBytes = mma::kSmem;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int clusters = 0;
  LC_CUDA(cudaOccupancyMaxActiveClusters(&clusters, k_iterate<PLANES, TO>, &cfg));
  LC_REQUIRE(clusters >= 1, LIPCACHE_E_CUDA, "no cluster of the iteration kernel fits on this device");
  const int ctas = std::min(clusters, mma::num_sms() / kCluster) * kCluster;
  if (dev < 64) known[dev] = ctas;
  return ctas;
}

template <int PLANES, typename TO>
void iterate_at_once(int batch, int rows, int cols, int steps, const double* co, void* out, const OrthoStep& st,
                     const OrthoLayout& l, cudaStream_t s) {
  const bool tall = rows > cols;
  const int m = std::min(rows, cols), n = std::max(rows, cols);
  IterateArgs a = {};
  for (int i = 0; i < 2; ++i) {
    const mma::Tensor X{l.x[i], cols, rows, (int64_t)PLANES * batch, l.ld, l.x_plane};
    a.xk[i] = mma::tensor_map(X, 128);
    a.xm[i] = mma::tensor_map(X, 64);
    a.to[i] = mma::tensor_map(X, 32, 32);
  }
  const mma::Tensor S{l.s, m, m, (int64_t)PLANES * batch, l.sld, l.s_plane},
      P{l.p, m, m, (int64_t)PLANES * batch, l.sld, l.s_plane};
  a.s = mma::tensor_map(S, 128);
  a.p = mma::tensor_map(P, 128);
  a.s64 = mma::tensor_map(S, 64);
  a.p64 = mma::tensor_map(P, 64);
  a.to[2] = mma::tensor_map(S, 32, 32);
  a.to[3] = mma::tensor_map(P, 32, 32);
  a.tall = tall;
  a.batch = batch;
  a.m = m;
  a.n = n;
  a.steps = steps;
  for (int i = 0; i < 3 * steps; ++i) a.coef[i] = (float)co[i];
  for (int i = 0; i < steps; ++i) a.ps[i] = poly_scale(a.coef[3 * i + 1], a.coef[3 * i + 2]);
  a.phases = l.phases;
  a.errors = mma::error_counter();
  const int ctas = iterate_ctas<PLANES, TO>();
  // The tile and split that end first, in clocks: a stage's loads from L2 (64
  // bytes a clock and SM; two stages of planes in flight take no less for 64
  // columns), the tile's epilogue, the join (measured, 2001 x 1003
  // FP32: 8,000 to 9,600 with the epilogue of a slice).
  int64_t grid = 0;  // no more CTAs than have work: each takes part in every barrier
  for (int k = 0; k < 3; ++k) {
    const int64_t chunks = ceil_div(k == 0 ? n : m, 64);
    int64_t best = -1, most = 0;
    for (int c = 0; c < 4; ++c) {
      const int bn = c == 0 ? 64 : 128, sp = c == 3 ? 4 : c == 2 ? 2 : 1;
      if (sp > chunks) continue;
      const int rt = (int)ceil_div(k == 2 ? rows : m, kTile), ct = (int)ceil_div(k == 2 ? cols : m, bn);
      const int64_t tiles = (k == 2 ? (int64_t)rt * ct : upper_tiles(rt, ct, kTile / bn)) * (int64_t)batch;
      const int64_t workers = sp > 1 ? ctas / kCluster : ctas;
      const int stage = PLANES == 2 ? 1024 : 2 * (kTile + bn);
      const int64_t cost = ceil_div(tiles, workers) * (ceil_div(chunks, sp) * stage +
                                                       (sp > 1 ? 12000 : 2000 + 12 * PLANES * bn));
      if (best < 0 || cost < best) {
        best = cost;
        a.split[k] = sp;
        a.bn[k] = bn;
        most = tiles * (sp > 1 ? kCluster : 1);
      }
    }
    grid = std::max(grid, most);
  }
  grid = std::min<int64_t>(round_up(grid, kCluster), ctas);
  a.t = l.t;
  a.lift = l.lift;
  a.out = st.weight ? st.out_weight : out;
  a.weight = st.weight;
  a.rows = rows;
  a.cols = cols;
  a.vec = cols % 8 == 0 && ((uintptr_t)a.out & 15) == 0 && ((uintptr_t)a.weight & 15) == 0;
  a.keep = st.keep;
  a.rate = st.rate;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kCluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeCooperative;
  attr[1].val.cooperative = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(mma::kThreads);
  cfg.dynamicSmemBytes = mma::kSmem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  LC_CUDA(cudaLaunchKernelEx(&cfg, k_iterate<PLANES, TO>, a));
  LC_LAUNCH_CHECK("k_iterate");
}

// Large matrices: tiles of 256 x 256 of CTA pairs, a launch a product. Bound by the
// tensor cores, under the power limit in a long run: 2 x (4,096 x 4,096) BF16, five
// steps, 2.13 ms, 1.29 PFLOP/s of the operations that symmetry leaves (S, P, X' of a
// step: 89, 93 and 177 us alone).
template <int PLANES, typename Epi>
void product(const mma::Tensor& A, bool a_mn, const mma::Tensor& B, bool b_mn, int M, int N, int64_t K, int batch,
             bool sym, Epi epi, cudaStream_t s) {
  mma::Args a = {};
  a.batches = batch;
  a.a_mn = a_mn;
  a.b_mn = b_mn;
  a.bn = kBigTile;
  a.m_tiles = (int)ceil_div(M, kBigTile);
  a.n_tiles = (int)ceil_div(N, kBigTile);
  a.sym = sym;
  a.block = kPairBlock;
  a.a_rows = 128;
  a.seg = mma::segment(K, mma::idesc(kBigTile, kBigTile, false, a_mn, b_mn));
  a.a_planes = a.b_planes = batch;
  const CUtensorMap ma = mma::tensor_map(A, a_mn ? 64 : 128);
  const CUtensorMap mb = mma::tensor_map(B, b_mn ? 64 : 128);
  mma::launch<2, PLANES>({ma, mb, ma, mb}, a, epi, s);
}

template <typename T, int VEC, int PLANES>
void normalise(const T* g, Direction a, int64_t batch, double eps, const Steps& steps, const OrthoLayout& l,
               cudaStream_t s) {
  a.units = a.cols / VEC;
  const int64_t n = (int64_t)a.rows * a.units, per = (int64_t)a.rows * a.cols;
  // dense matrices on 16-byte boundaries: eight elements at a time whatever the rows
  const bool flat = VEC == 1 && a.ldg == a.cols && (batch == 1 || per % 8 == 0) && per < (1LL << 31) &&
                    (((uintptr_t)g | (uintptr_t)a.st.momentum | (uintptr_t)a.st.out_momentum) & 15) == 0;
  unsigned parts = (unsigned)std::min<int64_t>(kParts, ceil_div(flat ? per / 8 + 1 : n, 512));
  if (flat) {
    Direction f = a;
    f.rows = 1;
    f.cols = (int)per;
    f.ldg = per;
    f.units = (int)(per / 8);
    f.tail = (int)(per % 8);
    launch_pdl(k_squares<T, 8>, dim3(parts, (unsigned)batch), 256, s, g, f, l.part);
  } else {
    launch_pdl(k_squares<T, VEC>, dim3(parts, (unsigned)batch), 256, s, g, a, l.part);
  }
  LC_LAUNCH_CHECK("k_squares");
  const unsigned blocks = (unsigned)std::min<int64_t>(ceil_div(n, 512), 1024);
  launch_pdl(k_planes<T, VEC, PLANES>, dim3(blocks, (unsigned)batch), 256, s, g, a, (const double*)l.part, (int)parts, eps,
             steps, l.x[0], l.ld, batch * l.x_plane, l.t, l.lift, l.phases);
  LC_LAUNCH_CHECK("k_planes");
}

template <int PLANES, typename TO>
void iterate(int batch, int rows, int cols, int steps, const double* co, void* out, const OrthoStep& st,
             const OrthoLayout& l, cudaStream_t s) {
  const bool tall = rows > cols;
  const int m = std::min(rows, cols), n = std::max(rows, cols);
  const int64_t xp = (int64_t)batch * l.x_plane, sp = (int64_t)batch * l.s_plane;
  if (ceil_div(m, kBigTile) * ceil_div(m, kBigTile) * batch / 2 < mma::num_sms() / 4) {
    iterate_at_once<PLANES, TO>(batch, rows, cols, steps, co, out, st, l, s);
    return;
  }
  const mma::Tensor S{l.s, m, m, (int64_t)PLANES * batch, l.sld, l.s_plane};
  const mma::Tensor P{l.p, m, m, (int64_t)PLANES * batch, l.sld, l.s_plane};
  for (int i = 0; i < steps; ++i) {
    const float a = (float)co[3 * i], b = (float)co[3 * i + 1], c = (float)co[3 * i + 2];
    const float* t = i == 0 ? l.t : nullptr;
    __half *x = l.x[i & 1], *y = l.x[(i & 1) ^ 1];
    const mma::Tensor X{x, cols, rows, (int64_t)PLANES * batch, l.ld, l.x_plane};
    const float2* lift = l.lift + i;
    SymEpi<PLANES> gram{l.s, nullptr, l.sld, l.s_plane, sp, m, kSScale / (kXScale * kXScale), 0.f, t, lift};
    product<PLANES>(X, tall, X, tall, m, m, n, batch, true, gram, s);
    const float ps = poly_scale(b, c);
    SymEpi<PLANES> poly{l.p, l.s, l.sld, l.s_plane, sp, m, c * ps / (kSScale * kSScale), b * ps / kSScale, nullptr, lift};
    product<PLANES>(S, false, S, false, m, m, m, batch, true, poly, s);
    auto update = [&](auto epi) {
      if (tall)
        product<PLANES>(X, false, P, false, n, m, m, batch, false, epi, s);
      else
        product<PLANES>(P, false, X, true, m, n, m, batch, false, epi, s);
    };
    if (i + 1 < steps) {
      update(UpdateEpi<PLANES>{y, x, l.ld, l.x_plane, xp, rows, cols, 1.f / ps, a, t, lift});
    } else {
      LastEpi<PLANES, TO> e{static_cast<TO*>(st.weight ? st.out_weight : out), static_cast<const TO*>(st.weight), x,
                            l.ld, l.x_plane, xp, rows, cols, 0, 1.f / (ps * kXScale), a / kXScale, st.keep, st.rate, t, lift};
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
  if (ortho_small(type, G, ldg, batch, rows, cols, steps, coefficients, eps, out, st, s)) return;
  const int out_type = st.weight ? st.weight_type : type, planes = planes_of(out_type);
  OrthoLayout l;
  Carve c{ws, 0};
  l.take(c, planes, batch, rows, cols);
  const Direction d{rows, cols, ldg, 0, 0, st};
  const bool vec = cols % 8 == 0 && ldg % 8 == 0 && ((uintptr_t)G & 15) == 0 && ((uintptr_t)st.momentum & 15) == 0 &&
                   ((uintptr_t)st.out_momentum & 15) == 0;
  Steps poly = {steps, {}};
  for (int i = 0; i < 3 * steps; ++i) poly.coef[i] = (float)coefficients[i];
  auto go = [&](auto g) {
    using T = std::remove_const_t<std::remove_pointer_t<decltype(g)>>;
    if (planes == 2)
      vec ? normalise<T, 8, 2>(g, d, batch, eps, poly, l, s) : normalise<T, 1, 2>(g, d, batch, eps, poly, l, s);
    else
      vec ? normalise<T, 8, 1>(g, d, batch, eps, poly, l, s) : normalise<T, 1, 1>(g, d, batch, eps, poly, l, s);
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

// Logits under a shared head and each row's own low-rank adapter, and their
// gradients.
//   u_t = s_g A_g x_t,  y_t = W x_t + bias + B_g u_t
//   v_t = s_g B_g^T dy_t,  dx_t = W^T dy_t + A_g^T v_t
//   dA_g = sum v_t x_t^T,  dB_g = sum dy_t u_t^T
//
// The shared product and the low-rank one of a tile are one sum in tensor
// memory: after the stages of W come, for each run of rows in the tile with
// the same adapter (head_plan.cuh), the few stages of that adapter's factor,
// limited to the run's rows by the MMA's lane mask. u and v are kept to 16 bits
// of mantissa or more (BF16 operands: two BF16 planes, hi + lo; FP32: three),
// so the split costs less than the operands' own rounding.
//
// FP32 rows become two FP16 planes under a power of two of each row's own (rows
// of W likewise), undone in the epilogue; u is divided by its row's before it
// is split, and the factors of W's rows are folded into dy where W is
// contracted over them, so each output keeps its precision relative to its own
// terms. A few FP32 rows go through the CUDA cores instead.
#include <cuda_fp16.h>

#include "head_plan.cuh"

namespace lc {
namespace ops {
namespace {

using mma::Tensor;
typedef __nv_bfloat16 bf16;

constexpr int kBlock = 4;  // stages of 64 the tensor cores sum before the sum is drained, FP32

// ---------------------------------------------------------------- staging
// The place's row of the input: `perm` where the plan sorted.
__device__ __forceinline__ int64_t row_at(const int* flags, const int* perm, int64_t p) {
  return flags && __ldg(flags + 1) ? (int64_t)__ldg(perm + p) : p;
}

struct Stage {
  int64_t rows, ld;     // of the input
  int cols;
  const int* flags;     // nullable: rows in their own order
  const int* perm;
  int only_sorted;      // nothing to do where rows keep their order
  const float* fold;    // FP32, nullable: a factor of each column
  int64_t ldo, plane;
  float* undo;          // FP32: what undoes each row's power of two
  int most;             // the largest power used
};

// A warp a row. BF16 rows are copied, FP32 rows scaled and split.
template <typename T>
__global__ void __launch_bounds__(256) k_stage(const T* in, const Stage a, uint16_t* out) {
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  if (a.only_sorted && !__ldg(a.flags + 1)) return;
  const int lane = threadIdx.x & 31;
  for (int64_t p = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); p < a.rows; p += (int64_t)gridDim.x * 8) {
    const T* r = in + row_at(a.flags, a.perm, p) * a.ld;
    uint16_t* o = out + p * a.ldo;
    if constexpr (sizeof(T) == 2) {
      const uint16_t* w = reinterpret_cast<const uint16_t*>(r);
      if ((((uintptr_t)w | (uintptr_t)(a.cols * 2)) & 15) == 0) {
        for (int i = lane; i < a.cols / 8; i += 32) reinterpret_cast<uint4*>(o)[i] = reinterpret_cast<const uint4*>(w)[i];
      } else {
        for (int i = lane; i < a.cols; i += 32) o[i] = w[i];
      }
    } else {
      auto value = [&](int i) { return a.fold ? to_f32<T>(r[i]) * __ldg(a.fold + i) : to_f32<T>(r[i]); };
      float top = 0.f;
      for (int i = lane; i < a.cols; i += 32) top = fmaxf(top, fabsf(value(i)));
#pragma unroll
      for (int s = 16; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
      // the largest element lands in [2^14, 2^15)
      int k = top > 0.f && top < INFINITY ? 14 - ilogbf(top) : 0;
      k = max(-a.most, min(a.most, k));
      const float f = ldexpf(1.f, k);
      for (int i = lane; i < a.cols; i += 32) {
        const float v = value(i) * f;
        const __half hi = __float2half_rn(v), lo = __float2half_rn(v - __half2float(hi));
        o[i] = __half_as_ushort(hi);
        o[a.plane + i] = __half_as_ushort(lo);
      }
      if (lane == 0) a.undo[p] = ldexpf(1.f, -k);
    }
  }
}

// An adapter factor in rows of ldo: BF16 copied, FP32 (over its row's power of
// two, nullable, one for `div_rows` rows in turn) as three BF16 planes.
template <typename T>
__global__ void __launch_bounds__(256)
    k_factor(const T* in, int64_t rows, int cols, int64_t ldo, int64_t plane, const float* undo, int div_rows,
             uint16_t* out) {
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int64_t n = rows * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / cols;
    uint16_t* o = out + r * ldo + (i - r * cols);
    if constexpr (sizeof(T) == 2) {
      *o = reinterpret_cast<const uint16_t*>(in)[i];
    } else {
      float v = in[i];
      if (undo) v /= __ldg(undo + r % div_rows);  // a power of two
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const bf16 h = __float2bfloat16_rn(v);
        o[q * plane] = __bfloat16_as_ushort(h);
        v -= __bfloat162float(h);
      }
    }
  }
}

// ---------------------------------------------------------------- shrink
struct Shrink {
  int64_t tokens, ld;
  int width, r, G;
  const int* flags;     // nullable, with perm: the plan's order
  const int* perm;
  const int32_t* adapter;
  const float* scales;
  int64_t f_g, f_j, f_i;  // strides of the factor
  float* out;             // nullable: tokens x r
  uint16_t* planes;       // nullable: BF16 planes of tokens x ldo
  int64_t ldo, plane;
  int n_planes;
  const float* undo;      // nullable: over each row's power of two in the planes
};

// Four values' worth of rows a warp, eight columns at a time: the sums of 32
// (row, j) pairs end on 32 lanes.
template <typename T>
__global__ void __launch_bounds__(128) k_shrink(const T* in, const T* F, const Shrink a) {
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t p0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 5)) * 4;
  if (p0 >= a.tokens) return;
  const int j0 = blockIdx.y * 8, nj = min(8, a.r - j0);
  const T* x[4];
  int g[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int64_t p = p0 + k;
    const int64_t t = p < a.tokens ? row_at(a.flags, a.perm, p) : 0;
    const int id = p < a.tokens ? __ldg(a.adapter + t) : -1;
    g[k] = id >= 0 && id < a.G ? id : -1;
    x[k] = in + t * a.ld;
  }
  float acc[32];
#pragma unroll
  for (int k = 0; k < 32; ++k) acc[k] = 0.f;
  bool done[4] = {g[0] < 0, g[1] < 0, g[2] < 0, g[3] < 0};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (done[k]) continue;
    bool in_g[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      in_g[q] = !done[q] && g[q] == g[k];
      done[q] |= in_g[q];
    }
    const T* f = F + g[k] * a.f_g + j0 * a.f_j;
#pragma unroll 2
    for (int i = lane; i < a.width; i += 32) {
      float xv[4], fv[8];
#pragma unroll
      for (int q = 0; q < 4; ++q) xv[q] = in_g[q] ? to_f32<T>(x[q][i]) : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) fv[j] = j < nj ? to_f32<T>(f[j * a.f_j + i * a.f_i]) : 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (in_g[q]) {
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[q * 8 + j] = fmaf(xv[q], fv[j], acc[q * 8 + j]);
        }
    }
  }
  // halve the values and double the lanes that share one, five times
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    const bool up = lane & s;
#pragma unroll
    for (int k = 0; k < s; ++k) {
      const float keep = up ? acc[k + s] : acc[k], give = up ? acc[k] : acc[k + s];
      acc[k] = keep + __shfl_xor_sync(0xffffffffu, give, s);
    }
  }
  const int q = lane >> 3, j = j0 + (lane & 7);
  const int64_t p = p0 + q;
  if (p >= a.tokens) return;
  const int id = q == 0 ? g[0] : q == 1 ? g[1] : q == 2 ? g[2] : g[3];
  float v = acc[0];
  if (id < 0) v = 0.f;
  else if (a.scales) v *= __ldg(a.scales + id);
  if (a.out && j < a.r) a.out[p * a.r + j] = v;
  if (a.planes && j < a.ldo) {
    if (j >= a.r) v = 0.f;
    if (a.undo) v /= __ldg(a.undo + p);
    uint16_t* o = a.planes + p * a.ldo + j;
    for (int k = 0; k < a.n_planes; ++k) {
      const bf16 h = __float2bfloat16_rn(v);
      o[k * a.plane] = __bfloat16_as_ushort(h);
      v -= __bfloat162float(h);
    }
  }
}

// The same product on the tensor cores (BF16): two planes.
struct ShrinkEpi {
  uint16_t* planes;
  const int* row_g;
  const float* scales;
  int64_t ldo, plane, tokens;
  int G;
  __device__ __forceinline__ void store(int row0, int col0, int, int lane, const uint32_t (&acc)[32]) const {
    const int64_t row = row0 + lane;
    if (row >= tokens || col0 >= ldo) return;
    const int g = __ldg(row_g + row);
    const float s = g >= G ? 0.f : scales ? __ldg(scales + g) : 1.f;
    uint16_t* o = planes + row * ldo + col0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (col0 + q * 8 >= ldo) break;
      uint16_t hi[8], lo[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = g >= G ? 0.f : s * __uint_as_float(acc[q * 8 + j]);
        const bf16 h = __float2bfloat16_rn(v);
        hi[j] = __bfloat16_as_ushort(h);
        lo[j] = __bfloat16_as_ushort(__float2bfloat16_rn(v - __bfloat162float(h)));
      }
      *reinterpret_cast<uint4*>(o + q * 8) = *reinterpret_cast<uint4*>(hi);
      *reinterpret_cast<uint4*>(o + plane + q * 8) = *reinterpret_cast<uint4*>(lo);
    }
  }
};

// ---------------------------------------------------------------- shared product
template <typename T>
struct AdaptEpi {
  T* y;
  int64_t ldy, rows;
  int cols, vec;
  const float *bias, *undo_row, *undo_col;  // nullable
  const int *flags, *perm;                  // nullable
  // few rows: the low-rank product here, from FP32 u (B: G x cols x r)
  const float* u;
  const T* B;
  const int32_t* adapter;
  int G, r;
  __device__ __forceinline__ void store(int row0, int col0, int, int lane, const uint32_t (&acc)[32]) const {
    const int left = cols - col0;
    const int64_t p = row0 + lane;
    if (left <= 0 || p >= rows) return;
    float v[32];
    const float f = undo_row ? __ldg(undo_row + p) : 1.f;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      v[j] = __uint_as_float(acc[j]) * f;
      if (undo_col && j < left) v[j] *= __ldg(undo_col + col0 + j);
      if (bias && j < left) v[j] += __ldg(bias + col0 + j);
    }
    if (u) {
      const int g = __ldg(adapter + p);
      if (g >= 0 && g < G) {
        const T* b = B + ((int64_t)g * cols + col0) * r;
        for (int k = 0; k < r; ++k) {
          const float uk = __ldg(u + p * r + k);
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (j < left) v[j] = fmaf(uk, to_f32<T>(b[j * r + k]), v[j]);
        }
      }
    }
    T* o = y + row_at(flags, perm, p) * ldy + col0;
    constexpr int kVec = 16 / sizeof(T);
#pragma unroll
    for (int q = 0; q < 32 / kVec; ++q) {
      if (q * kVec >= left) break;
      __align__(16) T h[kVec];
#pragma unroll
      for (int j = 0; j < kVec; ++j) h[j] = from_f32<T>(v[q * kVec + j]);
      if (vec && left >= (q + 1) * kVec) {
        *reinterpret_cast<uint4*>(o + q * kVec) = *reinterpret_cast<const uint4*>(h);
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
          if (q * kVec + j < left) o[q * kVec + j] = h[j];
      }
    }
  }
};

// A few rows on the CUDA cores (FP32, or BF16 that TMA cannot read): a warp
// takes four rows of W against eight of x.
template <typename T>
__global__ void __launch_bounds__(128)
    k_rows(const T* x, int64_t ldx, int64_t tokens, const T* W, int64_t ldw, int classes, int d, const float* bias,
           const float* u, const T* B, const int32_t* adapter, int G, int r, T* y, int64_t ldy) {
  ptx::launch_dependents();
  const int lane = threadIdx.x & 31;
  const int c0 = (blockIdx.x * 4 + (threadIdx.x >> 5)) * 4;
  const int64_t t0 = (int64_t)blockIdx.y * 8;
  if (c0 >= classes) return;
  const T *w[4], *xr[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = W + (int64_t)min(c0 + k, classes - 1) * ldw;
  ptx::wait_prerequisites();
#pragma unroll
  for (int k = 0; k < 8; ++k) xr[k] = x + min(t0 + k, tokens - 1) * ldx;
  float acc[32];
#pragma unroll
  for (int k = 0; k < 32; ++k) acc[k] = 0.f;
#pragma unroll 2
  for (int i = lane; i < d; i += 32) {
    float wv[4], xv[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) wv[k] = to_f32<T>(w[k][i]);
#pragma unroll
    for (int k = 0; k < 8; ++k) xv[k] = to_f32<T>(xr[k][i]);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[q * 8 + k] = fmaf(wv[q], xv[k], acc[q * 8 + k]);
  }
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    const bool up = lane & s;
#pragma unroll
    for (int k = 0; k < s; ++k) {
      const float keep = up ? acc[k + s] : acc[k], give = up ? acc[k] : acc[k + s];
      acc[k] = keep + __shfl_xor_sync(0xffffffffu, give, s);
    }
  }
  const int c = c0 + (lane >> 3);
  const int64_t t = t0 + (lane & 7);
  if (c >= classes || t >= tokens) return;
  float v = acc[0];
  if (bias) v += __ldg(bias + c);
  const int g = G ? __ldg(adapter + t) : -1;
  if (g >= 0 && g < G) {
    const T* b = B + ((int64_t)g * classes + c) * r;
    for (int k = 0; k < r; ++k) v = fmaf(__ldg(u + t * r + k), to_f32<T>(b[k]), v);
  }
  y[t * ldy + c] = from_f32<T>(v);
}

// ---------------------------------------------------------------- outer products
// F_g[j, i] = sum over g's places p of c[p, j] in[row(p), i], on the tensor
// cores: D^T, 128 of i x r of j (both planes of c side by side), one CTA each,
// contracted over each run's whole groups of 16 rows; what is left of a run is
// added in the epilogue, so that no row of another adapter is touched.
struct Outer {
  int r, width, rb;       // rb: columns of a plane in the tile, 64 or 128
  const int* flags;
  const int *off, *next, *first;
  const bf16 *in, *in2;   // elements of the rows: in place, or staged where sorted
  int64_t ld, ld2;
  const uint16_t* c;      // planes of tokens x ldc
  int64_t ldc, plane;
  bf16* out;
  int64_t f_g, f_j, f_i;
  unsigned long long* errors;
};
constexpr int kOuterThreads = 192;

__global__ void __launch_bounds__(kOuterThreads)
    k_outer(const __grid_constant__ CUtensorMap tm, const __grid_constant__ CUtensorMap tm2,
            const __grid_constant__ CUtensorMap tmC, const Outer a) {
  constexpr int kStages = 4;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const int stage_bytes = 16384 + a.rb * 256;
  const uint32_t full = base + kStages * stage_bytes, empty = full + 8 * kStages, done = empty + 8 * kStages,
                 misc = done + 8;
  unsigned char* misc_p = smem_raw + (misc - ptx::smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc_p);
  volatile int* abort_s = reinterpret_cast<volatile int*>(misc_p + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = blockIdx.y, i0 = blockIdx.x * 128;
  const uint32_t cols = (uint32_t)a.rb * 2;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      ptx::mbar_init(full + 8 * s, 1);
      ptx::mbar_init(empty + 8 * s, 1);
    }
    ptx::mbar_init(done, 1);
    *abort_s = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 1) {
    ptx::tmem_alloc(misc, cols);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const uint32_t tmem = *tmem_slot;
  const bool sorted = __ldg(a.flags + 1) != 0;
  const int head = __ldg(a.first + g);
  if (warp == 0) {
    if (lane == 0) {
      const CUtensorMap* m = sorted ? &tm2 : &tm;
      int st = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int i = head; i >= 0 && ok; i = __ldg(a.next + i)) {
        const int r0 = __ldg(a.off + i), whole = (__ldg(a.off + i + 1) - r0) & ~15;
        for (int k = 0; k < whole && ok; k += 64) {
          ok = ptx::mbar_wait(empty + 8 * st, ph ^ 1u, abort_s, mma::kWaitLimit);
          if (!ok) break;
          ptx::mbar_expect_tx(full + 8 * st, (uint32_t)stage_bytes);
          const uint32_t sa = base + st * stage_bytes, sb = sa + 16384;
          mma::load_3d(sa, m, i0, r0 + k, 0, full + 8 * st);
          mma::load_3d(sa + 8192, m, i0 + 64, r0 + k, 0, full + 8 * st);
          for (int q = 0; q < 2; ++q)
            for (int j = 0; j < a.rb; j += 64)
              mma::load_3d(sb + (q * a.rb + j) * 128, &tmC, j, r0 + k, q, full + 8 * st);
          if (++st == kStages) st = 0, ph ^= 1u;
        }
      }
    }
  } else if (warp == 1) {
    const bool lead = ptx::elect_one();
    const uint32_t id = mma::idesc(128, a.rb * 2, true, true, true);
    int st = 0;
    uint32_t ph = 0, acc = 0;
    bool ok = true;
    for (int i = head; i >= 0 && ok; i = __ldg(a.next + i)) {
      const int whole = (__ldg(a.off + i + 1) - __ldg(a.off + i)) & ~15;
      for (int k = 0; k < whole && ok; k += 64) {
        ok = ptx::mbar_wait_warp(full + 8 * st, ph, abort_s, mma::kWaitLimit);
        if (!ok) break;
        ptx::tc_fence_after();
        if (lead) {
          uint64_t da = mma::desc(base + st * stage_bytes, true), db = mma::desc(base + st * stage_bytes + 16384, true);
          const int steps = min(4, (whole - k) / 16);
          for (int q = 0; q < steps; ++q, da += 2048 >> 4, db += 2048 >> 4) {
            ptx::mma_f16(tmem, da, db, id, acc);
            acc = 1;
          }
          ptx::mma_commit(empty + 8 * st);
        }
        if (++st == kStages) st = 0, ph ^= 1u;
      }
    }
    if (lead) {
      volatile int never = 0;
      ptx::mma_commit(done);
      ptx::mbar_wait(done, 0, &never, mma::kWaitLimit);
    }
    __syncwarp();
  } else {
    const int i = i0 + (warp & 3) * 32 + lane;
    bool ok = ptx::mbar_wait(done, 0, abort_s, mma::kWaitLimit);
    ok = __all_sync(0xffffffffu, ok);
    ptx::tc_fence_after();
    bool any = false;  // rows on the tensor cores
    for (int q = head; q >= 0; q = __ldg(a.next + q)) any |= __ldg(a.off + q + 1) - __ldg(a.off + q) >= 16;
    const bf16* in = sorted ? a.in2 : a.in;
    const int64_t ld = sorted ? a.ld2 : a.ld;
    bf16* out = a.out + g * a.f_g + (int64_t)i * a.f_i;
    for (int j0 = 0; ok && j0 < a.r; j0 += 32) {
      uint32_t hi[32], lo[32];
      float v[32];
      const uint32_t src = tmem + ((uint32_t)((warp & 3) * 32) << 16) + j0;
      ptx::tmem_ld32(src, hi);
      ptx::tmem_ld32(src + a.rb, lo);
      ptx::tmem_wait_ld();
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = any ? __uint_as_float(hi[j]) + __uint_as_float(lo[j]) : 0.f;
      for (int q = head; q >= 0; q = __ldg(a.next + q)) {
        const int r0 = __ldg(a.off + q), r1 = __ldg(a.off + q + 1);
        for (int p = r0 + ((r1 - r0) & ~15); p < r1; ++p) {
          const float xv = i < a.width ? to_f32<bf16>(in[p * ld + i]) : 0.f;
          const uint16_t* c = a.c + p * a.ldc + j0;
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (j0 + j < a.r)
              v[j] = fmaf(xv, __uint_as_float((uint32_t)__ldg(c + j) << 16) +
                                  __uint_as_float((uint32_t)__ldg(c + a.plane + j) << 16), v[j]);
        }
      }
      if (i < a.width) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (j0 + j < a.r) out[(j0 + j) * a.f_j] = from_f32<bf16>(v[j]);
      }
    }
    ptx::tc_fence_before();
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
  if (warp == 1) ptx::tmem_dealloc(tmem, cols);
}

// The same in FP32 on the CUDA cores: 128 of i, eight of j, the places dealt
// over eight groups of threads.
__global__ void __launch_bounds__(1024)
    k_outer_f32(const float* in, int64_t ld, int width, const float* c, int r, const Plan p, float* out, int64_t f_g,
                int64_t f_j, int64_t f_i) {
  __shared__ float red[8][8][128];
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int g = blockIdx.z, j0 = blockIdx.y * 8, ti = threadIdx.x & 127, q = threadIdx.x >> 7;
  const int i = blockIdx.x * 128 + ti;
  const int nj = min(8, r - j0);
  const bool sorted = __ldg(p.flags + 1) != 0;
  float acc[8] = {};
  for (int run = __ldg(p.first + g); run >= 0; run = __ldg(p.next + run)) {
    const int r1 = __ldg(p.off + run + 1);
#pragma unroll 4
    for (int at = __ldg(p.off + run) + q; at < r1; at += 8) {
      const int64_t t = sorted ? __ldg(p.perm + at) : at;
      const float x = i < width ? in[t * ld + i] : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < nj) acc[j] = fmaf(x, __ldg(c + (int64_t)at * r + j0 + j), acc[j]);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) red[q][j][ti] = acc[j];
  __syncthreads();
  for (int e = threadIdx.x; e < nj * 128; e += 1024) {
    const int j = e >> 7, k = e & 127, at = blockIdx.x * 128 + k;
    float s = red[0][j][k];
#pragma unroll
    for (int w = 1; w < 8; ++w) s += red[w][j][k];
    if (at < width) out[g * f_g + (j0 + j) * f_j + (int64_t)at * f_i] = s;
  }
}

// ---------------------------------------------------------------- host side
constexpr int64_t kFewF32 = 64, kFewBf16 = 128;  // rows that need no plan

// What one product with the shared head needs: its rows' input (x or dy), its
// contracted width and the factor its low-rank part shrinks by.
struct Side {
  const void* in;
  int64_t ld;
  int width;       // contracted
  int out;         // columns of the result
  int64_t f_j, f_i;  // strides of the shrinking factor
};

struct Layout {
  Plan plan;
  uint16_t* in[2];                       // staged rows: of x, of dy
  uint16_t* w;                           // staged W
  uint16_t *a, *b;                       // staged factors
  float *undo_in, *undo_w, *u[2];        // u, v in FP32
  uint16_t* up[2];                       // their planes
  int64_t ld_in[2], ld_w, ld_a, ld_b, ld_u;
  void take(Carve& c, const lipcache_adapted& p, bool backward) {
    const bool f32 = p.type == LIPCACHE_F32;
    const int64_t T = p.tokens, G = p.adapters, r = G ? p.rank : 1;
    const int planes = f32 ? 2 : 1;
    ld_in[0] = round_up(p.d, 8);
    ld_in[1] = round_up(p.classes, 8);
    ld_w = round_up(p.d, 8);
    ld_a = round_up(p.d, 8);
    ld_b = ld_u = round_up(r, 8);
    plan.take(c, G ? T : 0, p.adapters);
    const bool stage_x = !(f32 && backward);
    c.take(in[0], stage_x ? (size_t)(planes * T * ld_in[0]) : 0);
    c.take(in[1], backward ? (size_t)(planes * T * ld_in[1]) : 0);
    c.take(w, (size_t)(planes * p.classes * ld_w));
    const int fp = f32 ? 3 : 1;
    c.take(a, (size_t)(fp * G * r * ld_a));
    c.take(b, (size_t)(fp * G * p.classes * ld_b));
    c.take(undo_in, (size_t)T);
    c.take(undo_w, (size_t)p.classes);
    for (int i = 0; i < 2; ++i) {
      c.take(u[i], G ? (size_t)(T * r) : 0);
      c.take(up[i], G ? (size_t)(3 * T * ld_u) : 0);
    }
  }
};

template <typename T>
struct Op {
  static constexpr bool f32 = sizeof(T) == 4;
  const lipcache_adapted& p;
  const Layout& l;
  cudaStream_t s;
  const T *x = static_cast<const T*>(p.x), *W = static_cast<const T*>(p.W), *A = static_cast<const T*>(p.A),
          *B = static_cast<const T*>(p.B);
  const int* flags = p.adapters ? l.plan.flags : nullptr;

  void stage(const T* in, int64_t ld, int64_t rows, int cols, bool sort, bool only_sorted, const float* fold,
             uint16_t* out, int64_t ldo, float* undo) {
    // (W's powers are folded into dy: less room)
    Stage a{rows, ld, cols, sort ? flags : nullptr, l.plan.perm, only_sorted, fold, ldo, rows * ldo, undo, sort ? 100 : 60};
    launch_pdl(k_stage<T>, dim3((unsigned)std::min<int64_t>(ceil_div(rows, 8), 1 << 16)), 256, s, in, a, out);
    LC_LAUNCH_CHECK("k_stage");
  }
  void factor(const T* in, int64_t rows, int cols, int64_t ldo, const float* undo, int div, uint16_t* out) {
    launch_pdl(k_factor<T>, dim3((unsigned)std::min<int64_t>(ceil_div(rows * cols, 1024), 1 << 16)), 256, s, in, rows,
               cols, ldo, rows * ldo, undo, div, out);
    LC_LAUNCH_CHECK("k_factor");
  }
  // u (i = 0) or v (1) of every row, in FP32 and/or planes.
  void shrink(const Side& d, const T* F, int i, bool planned, bool want_f32, bool want_planes, const float* undo) {
    Shrink a{p.tokens, d.ld, d.width, p.rank, p.adapters, planned ? flags : nullptr, l.plan.perm, p.adapter, p.scales,
             (int64_t)p.rank * d.width, d.f_j, d.f_i, want_f32 ? l.u[i] : nullptr, want_planes ? l.up[i] : nullptr,
             l.ld_u, p.tokens * l.ld_u, f32 ? 3 : 2, undo};
    const dim3 grid((unsigned)ceil_div(p.tokens, 16), (unsigned)ceil_div(p.rank, 8));
    launch_pdl(k_shrink<T>, grid, 128, s, static_cast<const T*>(d.in), F, a);
    LC_LAUNCH_CHECK("k_shrink");
  }
  // The same on the tensor cores; rows: the maps of the input in place and staged.
  void shrink_mma(const Side& d, const CUtensorMap& rows, const CUtensorMap& staged, const Tensor& F, bool f_mn, int i) {
    mma::Args a = {};
    a.m_tiles = (int)ceil_div(p.tokens, 128);
    a.n_tiles = a.batches = 1;
    a.bn = p.rank <= 64 ? 64 : 128;
    a.a_rows = 128;
    a.lb_mn = f_mn;
    a.alt = flags + 1;
    a.low.runs = l.plan.runs();
    a.low.from_a = 1;
    a.low.G = p.adapters;
    a.low.pairs = 1;
    const mma::Seg g = mma::segment(d.width, 0, 0, mma::idesc(128, a.bn, true, false, f_mn));
    a.low.chunks = g.chunks;
    a.low.last = g.last;
    a.low.idesc = g.idesc;
    const CUtensorMap f = mma::tensor_map(F, f_mn ? 64 : a.bn);
    const ShrinkEpi e{l.up[i], l.plan.row_g, p.scales, l.ld_u, p.tokens * l.ld_u, p.tokens, p.adapters};
    mma::launch<1, false>({rows, staged, f, rows, f}, a, e, s);
  }

  // out = rows . W (both as tensors) + low-rank: M tokens, N d.out, K d.width.
  void product(const Side& d, const CUtensorMap& rows, const CUtensorMap& staged, const Tensor& w, bool w_mn, int a_rows,
               int i, const Tensor* F, bool f_mn, AdaptEpi<T> e) {
    mma::Args a = {};
    const int64_t tiles = ceil_div(p.tokens, 256) * ceil_div(d.out, 256);
    // CTA pairs where their tiles fill half the device; else single CTAs, the tile narrowed until they do
    const bool pair = tiles >= mma::num_sms() / 4;
    const int step = w_mn ? (pair ? 128 : 64) : 32;
    a.bn = (int)std::min<int64_t>(pair ? 256 : 128, round_up(d.out, step));
    if (!pair)
      while (a.bn > step && ceil_div(p.tokens, 128) * ceil_div(d.out, a.bn) < mma::num_sms() / 2)
        a.bn = (int)round_up(a.bn / 2, step);
    const int tm = pair ? 256 : 128;
    a.m_tiles = (int)ceil_div(p.tokens, tm);
    a.n_tiles = (int)ceil_div(d.out, a.bn);
    a.batches = 1;
    a.b_mn = w_mn;
    a.a_rows = a_rows;
    a.alt = flags ? flags + 1 : nullptr;
    a.block = kBlock;
    const uint32_t id = mma::idesc(tm, a.bn, !f32, false, w_mn);
    if (f32) {
      a.seg[a.nseg++] = mma::segment(d.width, 0, 1, id);
      a.seg[a.nseg++] = mma::segment(d.width, 1, 0, id);
    }
    a.seg[a.nseg++] = mma::segment(d.width, 0, 0, id);
    const CUtensorMap mw = mma::tensor_map(w, w_mn ? 64 : a.bn / (pair ? 2 : 1));
    CUtensorMap la = rows, lb = mw;
    if (F) {
      a.lb_mn = f_mn;
      a.low.runs = l.plan.runs();
      a.low.G = p.adapters;
      const mma::Seg g = mma::segment(p.rank, 0, 0, mma::idesc(tm, a.bn, true, false, f_mn));
      a.low.chunks = g.chunks;
      a.low.last = g.last;
      a.low.idesc = g.idesc;
      static const int pu[6] = {2, 0, 1, 1, 0, 0}, pf[6] = {0, 2, 1, 0, 1, 0};
      a.low.pairs = f32 ? 6 : 2;
      for (int k = 0; k < a.low.pairs; ++k) {
        a.low.a_z[k] = f32 ? pu[k] : 1 - k;
        a.low.b_z[k] = f32 ? pf[k] : 0;
      }
      la = mma::tensor_map(Tensor{l.up[i], l.ld_u, p.tokens, f32 ? 3 : 2, l.ld_u, p.tokens * l.ld_u}, 128);
      lb = mma::tensor_map(*F, f_mn ? 64 : a.bn / (pair ? 2 : 1));
    }
    const mma::Maps maps{rows, staged, mw, la, lb};
    if (pair)
      mma::launch<2, f32>(maps, a, e, s);
    else
      mma::launch<1, f32>(maps, a, e, s);
  }

  AdaptEpi<T> epilogue(T* y, int64_t ldy, int cols) {
    AdaptEpi<T> e = {};
    e.y = y;
    e.ldy = ldy;
    e.rows = p.tokens;
    e.cols = cols;
    e.vec = ((uintptr_t)y & 15) == 0 && ldy * sizeof(T) % 16 == 0;
    e.flags = flags;
    e.perm = l.plan.perm;
    return e;
  }

  // W's planes or its own rows; `undo_w` is set for FP32.
  Tensor shared() {
    if (f32 || !mma::mappable(W, p.ldw)) {
      stage(W, p.ldw, p.classes, p.d, false, false, nullptr, l.w, l.ld_w, l.undo_w);
      return Tensor{l.w, p.d, p.classes, f32 ? 2 : 1, l.ld_w, p.classes * l.ld_w};
    }
    return Tensor{W, p.d, p.classes, 1, p.ldw, 0};
  }
  Tensor factor_a() {  // G x r x d
    const int64_t rows = (int64_t)p.adapters * p.rank;
    if (f32 || !mma::mappable(A, p.d)) {
      factor(A, rows, p.d, l.ld_a, nullptr, 1, l.a);
      return Tensor{l.a, p.d, p.rank, (f32 ? 3 : 1) * (int64_t)p.adapters, l.ld_a, p.rank * l.ld_a};
    }
    return Tensor{A, p.d, p.rank, p.adapters, p.d, (int64_t)p.rank * p.d};
  }
  Tensor factor_b(const float* undo) {  // G x classes x r
    const int64_t rows = (int64_t)p.adapters * p.classes;
    if (f32 || !mma::mappable(B, p.rank)) {
      factor(B, rows, p.rank, l.ld_b, undo, p.classes, l.b);
      return Tensor{l.b, p.rank, p.classes, (f32 ? 3 : 1) * (int64_t)p.adapters, l.ld_b, p.classes * l.ld_b};
    }
    return Tensor{B, p.rank, p.classes, p.adapters, p.rank, (int64_t)p.classes * p.rank};
  }
  // The maps of the rows of x (i = 0) or dy (1): in place, and staged in the plan's order.
  void rows(const Side& d, int i, const float* fold, CUtensorMap& in, CUtensorMap& staged) {
    const bool direct = !f32 && mma::mappable(d.in, d.ld);
    staged = mma::tensor_map(Tensor{l.in[i], d.width, p.tokens, f32 ? 2 : 1, l.ld_in[i], p.tokens * l.ld_in[i]}, 128);
    in = direct ? mma::tensor_map(Tensor{d.in, d.width, p.tokens, 1, d.ld, 0}, 128) : staged;
    if (!direct || flags)
      stage(static_cast<const T*>(d.in), d.ld, p.tokens, d.width, true, direct, fold, l.in[i], l.ld_in[i], l.undo_in);
  }
  // Whether an adapter has rows enough for its factor to be worth the tensor
  // cores' stages (a factor's stages are loaded again for every run).
  bool dense() const { return !f32 && p.tokens >= 16 * (int64_t)p.adapters; }

  void forward(const float* bias, T* y, int64_t ldy) {
    const Side d{x, p.ldx, p.d, p.classes, p.d, 1};
    const bool tma = !f32 && mma::mappable(x, p.ldx) && mma::mappable(W, p.ldw);
    if (p.tokens <= (tma ? kFewBf16 : kFewF32)) {
      if (p.adapters) shrink(d, A, 0, false, true, false, nullptr);
      if (tma) {
        AdaptEpi<T> e = epilogue(y, ldy, p.classes);
        e.bias = bias;
        e.flags = nullptr;
        if (p.adapters) e.u = l.u[0], e.B = B, e.adapter = p.adapter, e.G = p.adapters, e.r = p.rank;
        const int a_rows = (int)round_up(p.tokens, 8);
        const CUtensorMap in = mma::tensor_map(Tensor{x, p.d, p.tokens, 1, p.ldx, 0}, a_rows);
        const int* keep = flags;
        flags = nullptr;
        product(d, in, in, Tensor{W, p.d, p.classes, 1, p.ldw, 0}, false, a_rows, 0, nullptr, false, e);
        flags = keep;
      } else {
        launch_pdl(k_rows<T>, dim3((unsigned)ceil_div(p.classes, 16), (unsigned)ceil_div(p.tokens, 8)), 128, s, x,
                   p.ldx, p.tokens, W, p.ldw, (int)p.classes, (int)p.d, bias, (const float*)l.u[0], B, p.adapter,
                   (int)p.adapters, (int)p.rank, y, ldy);
        LC_LAUNCH_CHECK("k_rows");
      }
      return;
    }
    if (p.adapters) make_plan(p.adapter, p.tokens, p.adapters, l.plan, s);
    CUtensorMap in, staged;
    const Tensor w = shared();
    rows(d, 0, nullptr, in, staged);
    Tensor fb = {};
    if (p.adapters) {
      if (dense())
        shrink_mma(d, in, staged, factor_a(), false, 0);
      else
        shrink(d, A, 0, true, false, true, f32 ? l.undo_in : nullptr);
      fb = factor_b(f32 ? l.undo_w : nullptr);
    }
    AdaptEpi<T> e = epilogue(y, ldy, p.classes);
    e.bias = bias;
    if (f32) e.undo_row = l.undo_in, e.undo_col = l.undo_w;
    product(d, in, staged, w, false, 128, 0, p.adapters ? &fb : nullptr, false, e);
  }

  void outer(const Side& d, int in_i, int c_i, T* out, const CUtensorMap& in, const CUtensorMap& staged) {
    // d: the side whose rows are contracted; the factor's gradient has its strides
    if constexpr (f32) {
      k_outer_f32_launch(d, c_i, out);
    } else {
      Outer a = {};
      a.r = p.rank;
      a.width = d.width;
      a.rb = p.rank <= 64 ? 64 : 128;
      a.flags = flags;
      a.off = l.plan.off;
      a.next = l.plan.next;
      a.first = l.plan.first;
      const bool direct = mma::mappable(d.in, d.ld);
      a.in2 = reinterpret_cast<const bf16*>(l.in[in_i]);
      a.ld2 = l.ld_in[in_i];
      a.in = direct ? static_cast<const bf16*>(d.in) : a.in2;
      a.ld = direct ? d.ld : a.ld2;
      a.c = l.up[c_i];
      a.ldc = l.ld_u;
      a.plane = p.tokens * l.ld_u;
      a.out = out;
      a.f_g = (int64_t)p.rank * d.width;
      a.f_j = d.f_j;
      a.f_i = d.f_i;
      a.errors = mma::error_counter();
      // boxes of 64 x 64: the rows are contracted
      const Tensor ti{a.in, d.width, p.tokens, 1, a.ld, 0}, ts{a.in2, d.width, p.tokens, 1, a.ld2, 0},
          tc{a.c, l.ld_u, p.tokens, 2, l.ld_u, a.plane};
      const CUtensorMap m1 = mma::tensor_map(ti, 64), m2 = mma::tensor_map(ts, 64), mc = mma::tensor_map(tc, 64);
      const int smem = 1024 + 4 * (16384 + a.rb * 256) + 128;
      allow_smem(reinterpret_cast<const void*>(k_outer), 1024 + 4 * (16384 + 128 * 256) + 128);
      cudaLaunchAttribute attr;
      attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
      attr.val.programmaticStreamSerializationAllowed = 1;
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3((unsigned)ceil_div(d.width, 128), (unsigned)p.adapters);
      cfg.blockDim = dim3(kOuterThreads);
      cfg.dynamicSmemBytes = (size_t)smem;
      cfg.stream = s;
      cfg.attrs = &attr;
      cfg.numAttrs = 1;
      LC_CUDA(cudaLaunchKernelEx(&cfg, k_outer, m1, m2, mc, a));
      LC_LAUNCH_CHECK("k_outer");
    }
  }
  void k_outer_f32_launch(const Side& d, int c_i, T* out) {
    const dim3 grid((unsigned)ceil_div(d.width, 128), (unsigned)ceil_div(p.rank, 8), (unsigned)p.adapters);
    launch_pdl(k_outer_f32, grid, 1024, s, reinterpret_cast<const float*>(d.in), d.ld, d.width, (const float*)l.u[c_i],
               (int)p.rank, l.plan, reinterpret_cast<float*>(out), (int64_t)p.rank * d.width, d.f_j, d.f_i);
    LC_LAUNCH_CHECK("k_outer_f32");
  }

  void backward(const T* dy, int64_t lddy, T* dx, int64_t lddx, T* dA, T* dB) {
    const Side sx{x, p.ldx, p.d, p.classes, p.d, 1}, sy{dy, lddy, p.classes, p.d, 1, p.rank};
    const bool low = p.adapters > 0;
    if (!low && !dx) return;
    if (low) make_plan(p.adapter, p.tokens, p.adapters, l.plan, s);
    CUtensorMap in_x, staged_x, in_y, staged_y;
    Tensor w = {}, fa = {};
    if (dx) w = shared();
    // BF16 rows of x are read through the tensor cores for dA and u, those of dy for all else
    if (!f32 && low && (dA || dB)) rows(sx, 0, nullptr, in_x, staged_x);
    if (!f32 || dx) rows(sy, 1, f32 ? l.undo_w : nullptr, in_y, staged_y);
    if (low && (dx || dA)) {
      if (dense())
        shrink_mma(sy, in_y, staged_y, factor_b(nullptr), true, 1);
      else
        shrink(sy, B, 1, true, f32, !f32 || dx != nullptr, f32 && dx ? l.undo_in : nullptr);
    }
    if (low && (dx || (dB && dense()))) fa = factor_a();
    if (low && dB) {
      if (dense())
        shrink_mma(sx, in_x, staged_x, fa, false, 0);
      else
        shrink(sx, A, 0, true, f32, !f32, nullptr);
    }
    if (dx) {
      AdaptEpi<T> e = epilogue(dx, lddx, p.d);
      if (f32) e.undo_row = l.undo_in;
      product(sy, in_y, staged_y, w, true, 128, 1, low ? &fa : nullptr, true, e);
    }
    if (low && dA) outer(sx, 0, 1, dA, in_x, staged_x);
    if (low && dB) outer(sy, 1, 0, dB, in_y, staged_y);
  }
};

}  // namespace

size_t adapted_bytes(const lipcache_adapted& p, bool backward) {
  Layout l;
  Carve c;
  l.take(c, p, backward);
  return c.off;
}

void adapted_logits(const lipcache_adapted& p, const float* bias, void* y, int64_t ldy, unsigned char* ws,
                    cudaStream_t s) {
  Layout l;
  Carve c{ws, 0};
  l.take(c, p, false);
  if (p.type == LIPCACHE_F32)
    Op<float>{p, l, s}.forward(bias, static_cast<float*>(y), ldy);
  else
    Op<bf16>{p, l, s}.forward(bias, static_cast<bf16*>(y), ldy);
}

void adapted_backward(const lipcache_adapted& p, const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dA,
                      void* dB, unsigned char* ws, cudaStream_t s) {
  Layout l;
  Carve c{ws, 0};
  l.take(c, p, true);
  if (p.type == LIPCACHE_F32)
    Op<float>{p, l, s}.backward(static_cast<const float*>(dy), lddy, static_cast<float*>(dx), lddx,
                                static_cast<float*>(dA), static_cast<float*>(dB));
  else
    Op<bf16>{p, l, s}.backward(static_cast<const bf16*>(dy), lddy, static_cast<bf16*>(dx), lddx,
                               static_cast<bf16*>(dA), static_cast<bf16*>(dB));
}

}  // namespace ops
}  // namespace lc

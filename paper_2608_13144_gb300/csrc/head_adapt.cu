// Logits under a shared head and each row's own low-rank adapter, and their
// gradients.
//   u_t = s_g A_g x_t,  y_t = W x_t + bias + B_g u_t
//   v_t = s_g B_g^T dy_t,  dx_t = W^T dy_t + A_g^T v_t
//   dA_g = sum v_t x_t^T,  dB_g = sum dy_t u_t^T
//
// Rows stay where they stand, in any order of adapters.
// - The shared product runs on the tensor cores (head_mma.cuh). BF16: a tile
//   with few adapters among its rows takes the low-rank product into the same
//   sum, each adapter's few stages limited to its rows by the MMA's lane mask;
//   a tile with many adds it in the epilogue from u in FP32. FP32: one more
//   product, of u and of B with every adapter's side by side (zeros but in a
//   row's own) as three BF16 planes each, up to 256 columns; in the epilogue
//   beyond.
// - u and v (shrink): BF16 on the tensor cores, a tile's adapters side by side,
//   the rows loaded once for all of them; FP32 a warp for four rows of an adapter.
// - dA and dB: the rows of an adapter, listed by the CTA that sums them, are
//   gathered row by row, so that no other adapter's row is touched.
// On the tensor cores u and v are two BF16 planes, hi + lo (16 bits): their
// rounding stays below that of the operands.
//
// FP32 rows become two FP16 planes under a power of two of each row's own (rows
// of W likewise), undone in the epilogue; where W is contracted over its rows,
// their powers are folded into dy: each output keeps its precision relative to
// its own terms. A few rows go through the CUDA cores instead.
#include <cuda_fp16.h>

#include "head_mma.cuh"

namespace lc {
namespace ops {
namespace {

using mma::Tensor;
typedef __nv_bfloat16 bf16;

constexpr int kBlock = 4;  // stages of 64 the tensor cores sum before the sum is drained, FP32
// Powers of two of FP32 rows, at most. Rows of x, dy and (logits) W: what FP32 can undo;
// the smallest numbers still have the planes' bits. Where W is contracted over its rows,
// rows of dy are taken times the inverse, which has to leave them in range: rows of W
// below 2^-62 lose bits there.
constexpr int kRowPower = 126, kFoldPower = 60;
// B set side by side stands over the power of its class's row of W: under 2^kSidePower
// then, that sums of its products stay in range. Values of B and A that are not below
// kAside, which a power would take out of range for the rows of other adapters too, are
// set aside and added in the epilogue.
constexpr int kSidePower = 92;
constexpr float kAside = 0x1p32f;

// ---------------------------------------------------------------- copies
// A BF16 matrix whose rows TMA cannot read, in rows of ldo: 2048 columns of a
// row a block. Bound by memory.
__global__ void __launch_bounds__(256)
    k_copy_rows(const uint16_t* in, int64_t ld, int cols, int parts, uint16_t* out, int64_t ldo) {
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int64_t row = blockIdx.x / parts;
  const int c0 = (int)(blockIdx.x - row * parts) * 2048 + threadIdx.x;
  uint16_t v[8];
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (c0 + k * 256 < cols) v[k] = in[row * ld + c0 + k * 256];
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (c0 + k * 256 < cols) out[row * ldo + c0 + k * 256] = v[k];
}

// ---------------------------------------------------------------- FP32 rows
// A warp a row, in registers between its maximum and its planes. Kinds of rows
// in a launch: planes of a row (of W, with the B of all adapters for that class
// side by side); rows of A set side by side. Bound by memory: 65,536 x 256 rows,
// 134 MB, 26 us (5.2 TB/s).
struct RowJob {
  int set_aside = 0;            // a row of A
  const float* in = nullptr;
  int64_t ld = 0, rows = 0;
  int width = 0, vec = 0;       // vec: elements of a row that can be read together, 4, 2 or 1
  const float* fold = nullptr;  // a factor of each column
  int most = 0;                 // the largest power of two used
  __half* planes = nullptr;     // two FP16 planes under a power of two
  int64_t ldo = 0, plane = 0;
  float* undo = nullptr;        // what undoes each row's power of two
  bf16* wide = nullptr;         // three BF16 planes of what is set side by side
  const float* side = nullptr;  // nullable: B, of which row c of every adapter is set side by side in `wide`
  int64_t ldw = 0, wplane = 0;
  int* odd = nullptr;           // whether a value set into `wide` was not below kAside (0 there instead)
};
constexpr int kRowJobs = 3;
struct RowJobs {
  RowJob job[kRowJobs];
  int G, r;
  int blocks[kRowJobs];
};

// Sums of eight values over a warp: lane l ends with the sum of value l & 7.
__device__ __forceinline__ float sum8(float (&v)[8], int lane) {
#pragma unroll
  for (int s = 4; s > 0; s >>= 1) {
    const bool up = lane & s;
#pragma unroll
    for (int k = 0; k < s; ++k) {
      const float keep = up ? v[k + s] : v[k], give = up ? v[k] : v[k + s];
      v[k] = keep + __shfl_xor_sync(0xffffffffu, give, s);
    }
  }
  float r = v[0];
  r += __shfl_xor_sync(0xffffffffu, r, 8);
  return r + __shfl_xor_sync(0xffffffffu, r, 16);
}

// v as three BF16 planes (24 bits).
__device__ __forceinline__ void put3(bf16* o, int64_t plane, float v) {
#pragma unroll
  for (int q = 0; q < 3; ++q) {
    const bf16 h = __float2bfloat16_rn(v);
    o[q * plane] = h;
    v -= __bfloat162float(h);
  }
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, s));
  return v;
}
// The exponent that takes the largest element of a row into [2^14, 2^15), at
// most `most` (below, no finite row asks for less than -113).
__device__ __forceinline__ int row_power(float top, int most) {
  top = warp_max(top);
  const int e = top > 0.f ? 14 - ilogbf(top) : 0;
  return min(most, e);
}

// The planes of a row; returns its factor.
template <int VEC>
__device__ __forceinline__ float row_planes(const RowJob& a, const float* r, int64_t row, int lane, int most) {
  constexpr int kHeld = 2;  // vectors that a lane keeps between the two passes
  auto get = [&](int i, float (&v)[VEC]) {
    if constexpr (VEC == 4) {
      const float4 q = __ldg(reinterpret_cast<const float4*>(r + i));
      v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else if constexpr (VEC == 2) {
      const float2 q = __ldg(reinterpret_cast<const float2*>(r + i));
      v[0] = q.x, v[1] = q.y;
    } else {
      v[0] = __ldg(r + i);
    }
    if (a.fold) {
      if constexpr (VEC == 4) {
        const float4 q = __ldg(reinterpret_cast<const float4*>(a.fold + i));
        v[0] *= q.x, v[1] *= q.y, v[2] *= q.z, v[3] *= q.w;
      } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) v[k] *= __ldg(a.fold + i + k);
      }
    }
  };
  // (infinities leave the others of their row their bits)
  auto size = [](float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.f; };
  float held[kHeld][VEC];
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int i = (k * 32 + lane) * VEC;
#pragma unroll
    for (int q = 0; q < VEC; ++q) held[k][q] = 0.f;
    if (i < a.width) get(i, held[k]);
  }
#pragma unroll
  for (int k = 0; k < kHeld; ++k)
#pragma unroll
    for (int q = 0; q < VEC; ++q) top = fmaxf(top, size(held[k][q]));
#pragma unroll 4
  for (int i = (kHeld * 32 + lane) * VEC; i < a.width; i += 32 * VEC) {
    float v[VEC];
    get(i, v);
#pragma unroll
    for (int q = 0; q < VEC; ++q) top = fmaxf(top, size(v[q]));
  }
  const float f = ldexpf(1.f, row_power(top, most));
  __half* o = a.planes + row * a.ldo;
  auto put = [&](int i, float (&v)[VEC]) {
#pragma unroll
    for (int q = 0; q < VEC; ++q) v[q] *= f;
    if constexpr (VEC == 4) {
      uint32_t hi[2], lo[2];
      split_f16(v, hi, lo);
      *reinterpret_cast<uint2*>(o + i) = uint2{hi[0], hi[1]};
      *reinterpret_cast<uint2*>(o + a.plane + i) = uint2{lo[0], lo[1]};
    } else if constexpr (VEC == 2) {
      uint32_t hi[1], lo[1];
      split_f16(v, hi, lo);
      *reinterpret_cast<uint32_t*>(o + i) = hi[0];
      *reinterpret_cast<uint32_t*>(o + a.plane + i) = lo[0];
    } else {
      const __half hi = __float2half_rn(v[0]);
      o[i] = hi;
      o[a.plane + i] = __float2half_rn(v[0] - __half2float(hi));
    }
  };
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int i = (k * 32 + lane) * VEC;
    if (i < a.width) put(i, held[k]);
  }
#pragma unroll 4
  for (int i = (kHeld * 32 + lane) * VEC; i < a.width; i += 32 * VEC) {
    float v[VEC];
    get(i, v);
    put(i, v);
  }
  if (lane == 0) a.undo[row] = 1.f / f;  // a power of two
  return f;
}

__global__ void __launch_bounds__(128, 6) k_rows_f32(const __grid_constant__ RowJobs jobs) {
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int lane = threadIdx.x & 31, R = jobs.r;
  // a block has one kind of rows
  const int b0 = jobs.blocks[0], b1 = b0 + jobs.blocks[1], b = blockIdx.x;
  const int which = b < b0 ? 0 : b < b1 ? 1 : 2, first = b < b0 ? b : b < b1 ? b - b0 : b - b1;
  const RowJob& a = jobs.job[which];
  const int64_t step = (int64_t)jobs.blocks[which] * 4;
  for (int64_t row = (int64_t)first * 4 + (threadIdx.x >> 5); row < a.rows; row += step) {
    const float* r = a.in + row * a.ld;
    float f = 1.f;
    int most = a.most;
    if (a.side) {
      float top = 0.f;
      for (int i = lane; i < jobs.G * R; i += 32) {
        const int h = i / R;
        const float v = fabsf(__ldg(a.side + ((int64_t)h * a.rows + row) * R + i - h * R));
        if (v < kAside) top = fmaxf(top, v);
      }
      top = warp_max(top);
      if (top > 0.f) most = min(most, kSidePower - ilogbf(top));
    }
    if (a.planes)
      f = a.vec == 4   ? row_planes<4>(a, r, row, lane, most)
          : a.vec == 2 ? row_planes<2>(a, r, row, lane, most)
                       : row_planes<1>(a, r, row, lane, most);
    if (a.side || a.set_aside) {
      // B of this class, over the class's power of two; or a row of A
      bool odd = false;
      for (int i = lane; i < (a.side ? jobs.G * R : a.width); i += 32) {
        const int h = i / R;
        float v = __ldg(a.side ? a.side + ((int64_t)h * a.rows + row) * R + i - h * R : r + i);
        if (!(fabsf(v) < kAside)) v = 0.f, odd = true;
        put3(a.wide + row * a.ldw + i, a.wplane, v * f);
      }
      odd = __any_sync(0xffffffffu, odd);
      if (lane == 0) a.odd[row] = odd;
    }
  }
}

// u (or v) of FP32 rows. A block sorts its rows by adapter, so that a warp has
// four rows of one adapter against eight columns of its factor: three loads for
// eight multiplications of a lane, where a row alone takes nine. The products of
// a row can be set side by side too (three BF16 planes, 0 but at its adapter's
// place), over the row's power of two. 65,536 x 256 rows, ten adapters of rank 8:
// 41 us (67 MB read, 31 written; half of it outside the sums and the rows set
// side by side), bound by the latency of a warp's groups, one after another, at 16
// warps an SM: 128 registers hold four rows against eight columns.
struct LowJob {
  const float* in;
  int64_t ld;
  int width, vec;
  const float* F;
  int64_t f_g, f_j, f_i;
  float* u;
  bf16* wide;         // nullable
  const float* undo;
};
struct LowJobs {
  LowJob job[2];
  const int32_t* adapter;
  const float* scales;
  int64_t tokens, ldw;
  int G, r, tile, share;  // share: warps on a group, each a part of the width
};
constexpr int kLowTile = 128;  // rows of a block, at most

template <int VEC, bool J_INNER>
__device__ __forceinline__ void low_dots(const LowJob& a, const float* const (&x)[4], const float* F, int nj, int at,
                                         int step, float (&acc)[32]) {
#pragma unroll(VEC == 4 ? 1 : VEC == 2 ? 2 : 4)
  for (int i = at * VEC; i < a.width; i += step * VEC) {
    float v[4][VEC], f[8][VEC];
    if constexpr (J_INNER) {  // eight neighbours of the factor (VEC = 1)
      const float* fp = F + (int64_t)i * a.f_i;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j][0] = j < nj ? __ldg(fp + j) : 0.f;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (VEC == 4) {
          const float4 q = j < nj ? __ldg(reinterpret_cast<const float4*>(F + j * a.f_j + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
          f[j][0] = q.x, f[j][1] = q.y, f[j][2] = q.z, f[j][3] = q.w;
        } else if constexpr (VEC == 2) {
          const float2 q = j < nj ? __ldg(reinterpret_cast<const float2*>(F + j * a.f_j + i)) : make_float2(0.f, 0.f);
          f[j][0] = q.x, f[j][1] = q.y;
        } else {
          f[j][0] = j < nj ? __ldg(F + j * a.f_j + i) : 0.f;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (VEC == 4) {
        const float4 q = __ldg(reinterpret_cast<const float4*>(x[k] + i));
        v[k][0] = q.x, v[k][1] = q.y, v[k][2] = q.z, v[k][3] = q.w;
      } else if constexpr (VEC == 2) {
        const float2 q = __ldg(reinterpret_cast<const float2*>(x[k] + i));
        v[k][0] = q.x, v[k][1] = q.y;
      } else {
        v[k][0] = __ldg(x[k] + i);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int q = 0; q < VEC; ++q) acc[k * 8 + j] = fmaf(v[k][q], f[j][q], acc[k * 8 + j]);
  }
}

// A group of rows of one adapter: its place in the order, rows, adapter.
__device__ __forceinline__ uint32_t group_of(int first, int count, int g) { return (uint32_t)(first | count << 8 | g << 16); }

__global__ void __launch_bounds__(256, 2) k_low_f32(const __grid_constant__ LowJobs a) {
  __shared__ int bins[LIPCACHE_MAX_ADAPTERS + 1];
  __shared__ int id[kLowTile], order[kLowTile], total;
  __shared__ uint32_t group[kLowTile];
  __shared__ float parts[8][32];
  __shared__ __align__(16) bf16 own[3][kLowTile][8];
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const LowJob& job = a.job[blockIdx.z];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, R = a.r;
  const int64_t t0 = (int64_t)blockIdx.x * a.tile;
  const int n = (int)min((int64_t)a.tile, a.tokens - t0);
  const int j0 = blockIdx.y * 8, nj = min(8, R - j0);
  // Rows by adapter, those without one last: counted, the counts summed up, each
  // row put in its place. (Which rows of an adapter share a group is left to
  // chance; no row's sums depend on it.)
  int mine = a.G, place = 0;
  if (tid < n) {
    const int g = __ldg(a.adapter + t0 + tid);
    mine = g >= 0 && g < a.G ? g : a.G;
  }
  for (int i = tid; i <= a.G; i += 256) bins[i] = 0;
  __syncthreads();
  if (tid < n) place = atomicAdd(&bins[mine], 1);
  __syncthreads();
  if (warp == 0) {
    int rows = 0, groups = 0;
    for (int i0 = 0; i0 <= a.G; i0 += 32) {
      const int c = i0 + lane <= a.G ? bins[i0 + lane] : 0;
      int sum = c | (c + 3) / 4 << 16;
      const int one = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
      }
      const int before = sum - one;  // rows and groups before this adapter's
      if (i0 + lane <= a.G) bins[i0 + lane] = rows + (before & 0xffff) | (groups + (before >> 16)) << 8 | c << 16;
      const int all = __shfl_sync(0xffffffffu, sum, 31);
      rows += all & 0xffff;
      groups += all >> 16;
    }
    if (lane == 0) total = groups;
  }
  __syncthreads();
  if (tid < n) {
    const int b = bins[mine], at = (b & 255) + place;
    id[tid] = mine;
    order[at] = tid;
    if ((place & 3) == 0) group[(b >> 8 & 255) + place / 4] = group_of(at, min(4, (b >> 16) - place), mine);
  }
  __syncthreads();
  const int groups = total, share = a.share, part = warp % share;
  for (int q0 = 0; q0 < groups; q0 += 8 / share) {
    const int q = q0 + warp / share;
    const bool live = q < groups;
    const uint32_t it = live ? group[q] : 0u;
    const int first = it & 255, count = it >> 8 & 255, g = it >> 16;
    const bool any = live && g < a.G;
    const int64_t t = t0 + order[first + min(lane >> 3, max(count - 1, 0))];  // this lane's row of the results
    const float scale = any && a.scales ? __ldg(a.scales + g) : 1.f;
    const float over = any && job.wide ? __ldg(job.undo + t) : 1.f;
    float acc[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) acc[k] = 0.f;
    if (any) {
      const int at = part * 32 + lane, step = share * 32;
      const float* x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = job.in + __shfl_sync(0xffffffffu, t, k * 8) * job.ld;
      const float* F = job.F + g * job.f_g + j0 * job.f_j;
      if (job.f_j == 1)
        low_dots<1, true>(job, x, F, nj, at, step, acc);
      else if (job.vec == 4)
        low_dots<4, false>(job, x, F, nj, at, step, acc);
      else if (job.vec == 2)
        low_dots<2, false>(job, x, F, nj, at, step, acc);
      else
        low_dots<1, false>(job, x, F, nj, at, step, acc);
    }
    // 32 sums on 32 lanes: halve the values, double the lanes that share one
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
      const bool up = lane & s;
#pragma unroll
      for (int k = 0; k < s; ++k) {
        const float keep = up ? acc[k + s] : acc[k], give = up ? acc[k] : acc[k + s];
        acc[k] = keep + __shfl_xor_sync(0xffffffffu, give, s);
      }
    }
    if (share > 1) {  // the parts of the width, in order
      __syncthreads();
      parts[warp][lane] = acc[0];
      __syncthreads();
      if (part > 0) continue;
      for (int o = 1; o < share; ++o) acc[0] += parts[warp + o][lane];
    }
    if (!live) continue;
    const int k = lane >> 3, j = lane & 7;
    const float v = any ? scale * acc[0] : 0.f;
    if (k < count && j < nj) job.u[t * R + j0 + j] = v;
    // over a power of two
    if (job.wide && any && k < count) put3(own[0][t - t0] + j, kLowTile * 8, j < nj ? v / over : 0.f);
  }
  if (!job.wide) return;
  __syncthreads();
  // the rows set side by side: 16 bytes of a plane a lane
  const int words = (int)(a.ldw / 8);
  for (int row = warp; row < n; row += 8) {
    const int g = id[row], low = g < a.G ? g * R : -R;  // the adapter's columns
    bf16* o = job.wide + (t0 + row) * a.ldw;
    for (int e = lane; e < 3 * words; e += 32) {
      const int p = (e >= words) + (e >= 2 * words), w = e - p * words;
      const bf16* from = own[p][row];
      bf16* to = o + p * a.tokens * a.ldw + w * 8;
      const int at = low + j0 - w * 8;  // of this block's columns in the word
      if (w * 8 + 8 <= low || w * 8 >= low + R) {
        if (blockIdx.y == 0) *reinterpret_cast<uint4*>(to) = uint4{0, 0, 0, 0};
      } else if (R <= 8 || (at == 0 && nj == 8)) {
        // the row's own columns (zeros past them), moved to their place in the word
        ulonglong2 v = *reinterpret_cast<const ulonglong2*>(from);
        const int up = at * 16;
        if (up > 0) {
          v.y = up < 64 ? v.y << up | v.x >> (64 - up) : v.x << (up - 64);
          v.x = up < 64 ? v.x << up : 0;
        } else if (up < 0) {
          v.x = up > -64 ? v.x >> -up | v.y << (64 + up) : v.y >> (-up - 64);
          v.y = up > -64 ? v.y >> -up : 0;
        }
        *reinterpret_cast<ulonglong2*>(to) = v;
      } else {
        // the first of the blocks along j clears what is no block's
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          if (c >= at && c < at + nj)
            to[c] = from[c - at];
          else if (blockIdx.y == 0 && (w * 8 + c < low || w * 8 + c >= low + R))
            to[c] = __float2bfloat16_rn(0.f);
        }
      }
    }
  }
}

// ---------------------------------------------------------------- shrink, few rows
// u of one row (blockIdx.x), eight columns (blockIdx.y) in FP32. Bound by
// latency: 48 BF16 rows of 4,096, r = 16: 7.5 us.
template <typename T>
__global__ void __launch_bounds__(128)
    k_shrink_few(const T* x, int64_t ldx, int width, const T* A, int vec, int G, int r, const int32_t* adapter,
                 const float* scales, float* u) {
  __shared__ float red[4][8];
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int64_t t = blockIdx.x;
  const int j0 = blockIdx.y * 8, nj = min(8, r - j0), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = __ldg(adapter + t);
  const bool any = g >= 0 && g < G;
  float acc[8] = {};
  if (any) {
    const T* row = x + t * ldx;
    const T* F = A + ((int64_t)g * r + j0) * width;
    constexpr int N = 16 / sizeof(T);
    auto dot = [](const uint4& p, const uint4& q, float s) {
      const uint32_t a[4] = {p.x, p.y, p.z, p.w}, b[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (sizeof(T) == 4) {
          s = fmaf(__uint_as_float(a[k]), __uint_as_float(b[k]), s);
        } else {
          s = fmaf(__uint_as_float(a[k] << 16), __uint_as_float(b[k] << 16), s);
          s = fmaf(__uint_as_float(a[k] & 0xffff0000u), __uint_as_float(b[k] & 0xffff0000u), s);
        }
      }
      return s;
    };
    if (vec) {
      for (int i = threadIdx.x * N; i < width; i += 128 * N) {
        const uint4 xv = *reinterpret_cast<const uint4*>(row + i);
        uint4 f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < nj) f[j] = __ldg(reinterpret_cast<const uint4*>(F + (int64_t)j * width + i));
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < nj) acc[j] = dot(xv, f[j], acc[j]);
      }
    } else {
#pragma unroll 2
      for (int i = threadIdx.x; i < width; i += 128) {
        const float xv = to_f32<T>(row[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < nj) acc[j] = fmaf(xv, to_f32<T>(F[(int64_t)j * width + i]), acc[j]);
      }
    }
  }
  const float v = sum8(acc, lane);
  if (lane < 8) red[warp][lane] = v;
  __syncthreads();
  if (threadIdx.x < nj) {
    const int k = threadIdx.x;
    const float s = ((red[0][k] + red[1][k]) + red[2][k]) + red[3][k];
    u[t * r + j0 + k] = any ? (scales ? __ldg(scales + g) * s : s) : 0.f;
  }
}

// ---------------------------------------------------------------- shrink, tensor cores
// u of 128 rows. The factors of a tile's adapters stand side by side along N, so
// that the rows are read, and the MMAs issued, once for all of them (up to 256
// columns a pass); the epilogue takes each row's own columns. A cluster splits
// the contracted width; its first CTA joins the parts in order. Bound by
// reading the rows once (8,192 x 4,096 BF16 rows, r = 16: 25 us, 5.5 TB/s after
// 11 us that any size takes), and by latency where they are few. Twelve smaller
// stages in place of three took no less.
constexpr int kShrinkThreads = 192, kShrinkStages = 3, kShrinkStage = 48 * 1024;
struct ShrinkJob {
  CUtensorMap rows, factor;
  int chunks, last;
  int f_mn;       // the factor's contracted index is not its innermost
  int f_bytes;    // of a factor's part of a stage
  int per;        // factors in a stage
  int cols;       // columns of D a factor
  float* u;       // tokens x r
  uint16_t* planes;
};
struct ShrinkJobs {
  ShrinkJob job[2];
  const int32_t* adapter;
  const float* scales;
  int64_t tokens, ldo, plane;
  int G, r, rn;   // rn: r up to a multiple of 16, the columns of D
  unsigned long long* errors;
};

__device__ __forceinline__ void store_cluster(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

__global__ void __launch_bounds__(kShrinkThreads, 1) k_shrink(const __grid_constant__ ShrinkJobs a) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  float* part = reinterpret_cast<float*>(smem_raw + (base - ptx::smem_u32(smem_raw)));  // others', in the stages
  const uint32_t own_s = base + kShrinkStages * kShrinkStage;  // this CTA's u: [column][row]
  float* own = part + kShrinkStages * kShrinkStage / 4;
  const uint32_t full = own_s + 128 * 128 * 4, empty = full + 8 * kShrinkStages, acc_full = empty + 8 * kShrinkStages,
                 acc_empty = acc_full + 16, misc = acc_empty + 16;
  unsigned char* misc_p = smem_raw + (misc - ptx::smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc_p);
  volatile int* abort_s = reinterpret_cast<volatile int*>(misc_p + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const ShrinkJob& job = a.job[blockIdx.z];
  uint32_t splits;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(splits));
  const uint32_t rank = ptx::cluster_ctarank();
  const int64_t m0 = (int64_t)(blockIdx.x / splits) * 128;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kShrinkStages; ++s) {
      ptx::mbar_init(full + 8 * s, 1);
      ptx::mbar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(acc_full + 8 * b, 1);
      ptx::mbar_init(acc_empty + 8 * b, 4);
    }
    *abort_s = 0;
    ptx::fence_mbar_init();
    ptx::tma_prefetch_desc(&job.rows);
    ptx::tma_prefetch_desc(&job.factor);
  }
  if (warp == 1) {
    ptx::tmem_alloc(misc, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const uint32_t tmem = *tmem_slot;
  const int c0 = (int)((int64_t)job.chunks * rank / splits), c1 = (int)((int64_t)job.chunks * (rank + 1) / splits);
  const int cols = job.cols, row = (warp & 3) * 32 + lane;
  bool ok = true;
  {
    // every role walks the same passes: up to `per` adapters of the tile each
    mma::Groups<128> gr;
    gr.begin(a.adapter, a.tokens, a.G, m0, lane);
    const bool lead = ptx::elect_one();
    const int my = gr.id[warp & 3];  // (epilogue) this thread's row's adapter
    int st = 0, passes = 0;
    uint32_t ph = 0;
    for (bool more = gr.next(); more && ok; ++passes) {
      int g[8], n = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (k >= job.per || !more) continue;
        g[k] = gr.g;
        n = k + 1;
        more = gr.next();
      }
      const int buf = passes & 1;
      const uint32_t use = (uint32_t)(passes >> 1) & 1u;
      if (warp == 0) {
        for (int c = c0; c < c1 && ok; ++c) {
          ok = ptx::mbar_wait_warp(empty + 8 * st, ph ^ 1u, abort_s, mma::kWaitLimit);
          if (!ok) break;
          if (lane == 0) {
            const uint32_t sa = base + st * kShrinkStage, bar = full + 8 * st;
            ptx::mbar_expect_tx(bar, (uint32_t)(16384 + n * job.f_bytes));
            mma::load_3d(sa, &job.rows, c * 64, (int)m0, 0, bar);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              if (k >= n) break;
              const uint32_t sb = sa + 16384 + k * job.f_bytes;
              if (job.f_mn)
                for (int j = 0; j * 8192 < job.f_bytes; ++j) mma::load_3d(sb + j * 8192, &job.factor, j * 64, c * 64, g[k], bar);
              else
                mma::load_3d(sb, &job.factor, c * 64, 0, g[k], bar);
            }
          }
          if (++st == kShrinkStages) st = 0, ph ^= 1u;
        }
      } else if (warp == 1) {
        ok = ptx::mbar_wait_warp(acc_empty + 8 * buf, use ^ 1u, abort_s, mma::kWaitLimit);
        ptx::tc_fence_after();
        const uint32_t id = mma::idesc(128, n * cols, true, false, job.f_mn), d = tmem + (uint32_t)buf * 256u;
        for (int c = c0; c < c1 && ok; ++c) {
          ok = ptx::mbar_wait_warp(full + 8 * st, ph, abort_s, mma::kWaitLimit);
          if (!ok) break;
          ptx::tc_fence_after();
          if (lead) {
            const uint32_t sa = base + st * kShrinkStage;
            const int steps = c == job.chunks - 1 ? job.last : 4;
            uint64_t da = mma::desc(sa, false), db = mma::desc(sa + 16384, job.f_mn);
            for (int q = 0; q < steps; ++q, da += 32 >> 4, db += job.f_mn ? 2048 >> 4 : 32 >> 4)
              ptx::mma_f16(d, da, db, id, c > c0 || q > 0);
            ptx::mma_commit(empty + 8 * st);
          }
          if (++st == kShrinkStages) st = 0, ph ^= 1u;
        }
        if (ok && lead) ptx::mma_commit(acc_full + 8 * buf);
      } else {
        ok = ptx::mbar_wait_warp(acc_full + 8 * buf, use, abort_s, mma::kWaitLimit);
        if (!ok) break;
        ptx::tc_fence_after();
        // each row's own columns, eight at a time
        for (int k = 0; k < n; ++k) {
          int gk = g[0];
#pragma unroll
          for (int q = 1; q < 8; ++q)
            if (q == k) gk = g[q];
          if (!__any_sync(0xffffffffu, my == gk)) continue;
#pragma unroll 1
          for (int j = 0; j < a.r; j += 8) {
            float v[8];
            mma::tmem_ld8(tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(buf * 256 + k * cols + j), v);
            if (my == gk) {
#pragma unroll
              for (int q = 0; q < 8; ++q) own[(j + q) * 128 + row] = v[q];
            }
            __syncwarp();
          }
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(acc_empty + 8 * buf);
      }
    }
  }
  __syncwarp();
  const int64_t t = m0 + row;
  const int id = t < a.tokens ? __ldg(a.adapter + t) : -1;
  const bool any = id >= 0 && id < a.G;
  if (splits > 1) {
    // the first CTA's stages are free once all of them have their sums
    ptx::cluster_sync();
    if (warp >= 2 && rank > 0) {
      const uint32_t dst = ptx::mapa(base, 0) + (uint32_t)((rank - 1) * 128 * a.rn + row) * 4;
#pragma unroll 8
      for (int j = 0; j < a.r; ++j) store_cluster(dst + (uint32_t)(j * 128) * 4, own[j * 128 + row]);
    }
    ptx::cluster_sync();
  }
  if (warp >= 2 && rank == 0 && ok && t < a.tokens) {
    const float s = any && a.scales ? __ldg(a.scales + id) : 1.f;
#pragma unroll 1
    for (int j0 = 0; j0 < a.ldo; j0 += 8) {
      float f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int j = j0 + k;
        f[k] = 0.f;
        if (any && j < a.r) {
          f[k] = own[j * 128 + row];
          for (uint32_t p = 1; p < splits; ++p) f[k] += part[((p - 1) * a.rn + j) * 128 + row];
          f[k] *= s;
        }
        if (j < a.r) job.u[t * a.r + j] = f[k];
      }
      uint32_t hi[4], lo[4];
      split_bf16(f, hi, lo);
      uint16_t* o = job.planes + t * a.ldo + j0;
      *reinterpret_cast<uint4*>(o) = uint4{hi[0], hi[1], hi[2], hi[3]};
      *reinterpret_cast<uint4*>(o + a.plane) = uint4{lo[0], lo[1], lo[2], lo[3]};
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (*abort_s) {
    const long long t1 = clock64();
    while (clock64() - t1 < (1LL << 23)) {
    }
    if (threadIdx.x == 0) atomicAdd(a.errors, 1ull);
    __syncthreads();
  }
  ptx::tc_fence_after();
  if (warp == 1) ptx::tmem_dealloc(tmem, 512);
}

// ---------------------------------------------------------------- shared product
// EARLY: the few-rows form, whose epilogue takes the low-rank product of its
// tile while the shared one is summed.
template <typename T, bool EARLY = false>
struct AdaptEpi {
  static constexpr bool kTurns = true, kEarly = EARLY;
  static constexpr float kFar = 0x1p64f;
  T* y;
  int64_t ldy, rows;
  int cols, vec;
  const float *bias, *undo_row, *undo_col;  // nullable
  // the low-rank product: u (tokens x r) times the factor of cols x r
  // (f_col = r, f_j = 1) or r x cols (1, cols)
  const float* u;
  const T* F;
  const int32_t* adapter;
  int G, r, f_vec;
  int64_t f_col, f_j;
  // set-aside values of a dense low-rank product (not below kAside, or NaN), a
  // flag for each column (n_odd = 0) or for each of n_odd rows of A
  const int* odd;
  int n_odd;

  // Of a row, and of a lane's columns in each of up to four blocks of 32, 64 apart.
  struct Head {
    float f, uc[4], bc[4];
    bool odd;
  };
  __device__ __forceinline__ void load(int row0, int col0, int wide, int lane, Head& h) const {
    const int64_t p = (int64_t)row0 + lane;
    h.f = undo_row && p < rows ? __ldg(undo_row + p) : 1.f;
    h.odd = false;
    if (odd && n_odd)
      for (int i = lane; i < n_odd; i += 32) h.odd |= __ldg(odd + i) != 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = col0 + 64 * i + lane;
      const bool in = 64 * i < wide && c < cols;
      h.uc[i] = undo_col && in ? __ldg(undo_col + c) : 1.f;
      h.bc[i] = bias && in ? __ldg(bias + c) : 0.f;
      if (odd && !n_odd && in) h.odd |= __ldg(odd + c) != 0;
    }
    h.odd = __any_sync(0xffffffffu, h.odd);
  }
  // Rare rows, in shared memory, a row a lane: the columns' factors, what is left of the row's
  // (a sum times the whole of a large one may be past FP32's range before the column's), and what
  // was set aside of the row's adapter.
  __device__ __forceinline__ void strange(int64_t p, int col0, int left, int lane, uint32_t turn, float uc, float rest,
                                          bool aside) const {
    const int g = aside && p < rows ? __ldg(adapter + p) : -1;
    const bool any = g >= 0 && g < G;
    const T* f = any ? F + (int64_t)g * cols * r + col0 * f_col : nullptr;
#pragma unroll 1
    for (int j = 0; j < 32; ++j) {
      const uint32_t at = turn + (uint32_t)(lane * 128 + ((j >> 2 ^ (lane & 7)) << 4) + (j & 3) * 4);
      float x;
      asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
      x = x * __shfl_sync(0xffffffffu, uc, j) * rest;
      if (any && j < left) {
#pragma unroll 1
        for (int k = 0; k < r; ++k) {
          const float q = to_f32<T>(f[j * f_col + k * f_j]);
          if (!(fabsf(q) < kAside)) x = fmaf(__ldg(u + p * r + k), q, x);
        }
      }
      asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory");
    }
  }

  // element i of a 16-byte vector
  static __device__ __forceinline__ float part(const uint4& q, int i) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    return __uint_as_float(sizeof(T) == 4 ? w[i % 4] : i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  // v += the row's low-rank product in 32 columns, `left` of them in the matrix
  // (few rows: a factor of cols x r; loads in groups, all of a group in flight;
  // past the matrix the last column is read again).
  __device__ __forceinline__ void low(int64_t p, int col0, int left, float (&v)[32]) const {
    constexpr int N = 16 / sizeof(T);
    const int g = __ldg(adapter + p);
    if (g < 0 || g >= G) return;
    const T* f = F + (int64_t)g * cols * r + col0 * f_col;
    const float* up = u + p * r;
    const int last = min(left, 32) - 1;
    if (f_vec) {
      for (int k = 0; k < r; k += N) {
        float uk[N];
#pragma unroll
        for (int i = 0; i < N; ++i) uk[i] = __ldg(up + k + i);
#pragma unroll
        for (int j0 = 0; j0 < 32; j0 += 8) {
          uint4 q[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) q[j] = __ldg(reinterpret_cast<const uint4*>(f + min(j0 + j, last) * r + k));
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < N; ++i) v[j0 + j] = fmaf(uk[i], part(q[j], i), v[j0 + j]);
        }
      }
    } else {
      for (int k = 0; k < r; ++k) {
        const float uk = __ldg(up + k);
#pragma unroll
        for (int j0 = 0; j0 < 32; j0 += 16) {
          float q[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) q[j] = to_f32<T>(f[min(j0 + j, last) * r + k]);
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j0 + j] = fmaf(uk, q[j], v[j0 + j]);
        }
      }
    }
  }

  // x += the low-rank product of row p in the N columns from col on, `left` of
  // them in the matrix.
  template <int N>
  __device__ __forceinline__ void low_part(int64_t p, int col, int left, float (&x)[N]) const {
    const int g = __ldg(adapter + p);
    if (g < 0 || g >= G) return;
    const T* f = F + (int64_t)g * cols * r + col * f_col;
    const float* up = u + p * r;
    if (f_vec && f_j == 1 && N > 1) {
#pragma unroll 1
      for (int k = 0; k < r; k += N) {
        float uk[N];
#pragma unroll
        for (int i = 0; i < N; ++i) uk[i] = __ldg(up + k + i);
        uint4 q[N];
#pragma unroll
        for (int i = 0; i < N; ++i) q[i] = __ldg(reinterpret_cast<const uint4*>(f + min(i, left - 1) * r + k));
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
          for (int j = 0; j < N; ++j) x[i] = fmaf(uk[j], part(q[i], j), x[i]);
      }
    } else if (f_vec && N > 1) {
#pragma unroll 4
      for (int k = 0; k < r; ++k) {
        const float uk = __ldg(up + k);
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(f + k * f_j));  // (rows are whole vectors)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(uk, part(q, i), x[i]);
      }
    } else {
#pragma unroll 4
      for (int k = 0; k < r; ++k) {
        const float uk = __ldg(up + k);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(uk, to_f32<T>(f[min(i, left - 1) * f_col + k * f_j]), x[i]);
      }
    }
  }

  // The low-rank product of 32 columns before the shared one is there (unscaled
  // sums, every tile's: the few-rows form).
  __device__ __forceinline__ bool ahead(int row0, int col0, int lane, float (&v)[32]) const {
    if (!u) return false;
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = 0.f;
    if (row0 + lane < rows && col0 < cols) low(row0 + lane, col0, cols - col0, v);
    return true;
  }
  __device__ __forceinline__ void store(int row0, int col0, int, int lane, bool many, uint32_t turn,
                                        const uint32_t (&acc)[32], const Head& h, int block) const {
    const int left = cols - col0;
    const int64_t p = (int64_t)row0 + lane;
    if (left <= 0) return;
    const float f = h.f;
    float uc = h.uc[0], bc = h.bc[0];
#pragma unroll
    for (int i = 1; i < 4; ++i)
      if (block == i) uc = h.uc[i], bc = h.bc[i];
    const bool after = many && u && !odd;
    float v[32];
    const float near = sizeof(T) == 4 ? fminf(f, kFar) : f;
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(acc[j]) * near;
    // Turned in shared memory, 16 bytes at a time, places mixed by the row: a row
    // from a thread would take a cycle for every 16 bytes, or for every element
    // where rows are not whole vectors. Scales (powers of two) and biases of the
    // columns come after, a few shuffles instead of 64, and so does the low-rank
    // product of mixed rows, whose factors the lanes of a row then read side by side.
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q)
      asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(turn + (uint32_t)(lane * 128 + ((q ^ (lane & 7)) << 4))),
                   "f"(v[4 * q]), "f"(v[4 * q + 1]), "f"(v[4 * q + 2]), "f"(v[4 * q + 3])
                   : "memory");
    if (sizeof(T) == 4 && (h.odd || __any_sync(0xffffffffu, f > kFar))) {
      strange(p, col0, left, lane, turn, uc, f > kFar ? f / kFar : 1.f, h.odd);
      uc = 1.f;
    }
    __syncwarp();
    const int have = (int)min((int64_t)32, rows - row0);
    constexpr int N = 16 / sizeof(T), kLanes = 32 / N;  // columns of a lane, lanes of a row
    if (vec && (left >= 32 || left % N == 0)) {
      const int first = lane / kLanes, q = lane % kLanes;
      float cu[N], cb[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        cu[i] = __shfl_sync(0xffffffffu, uc, q * N + i);
        cb[i] = __shfl_sync(0xffffffffu, bc, q * N + i);
      }
      T* o = y + ((int64_t)row0 + first) * ldy + col0 + q * N;
      const bool inside = q * N < left;
#pragma unroll
      for (int r0 = 0; r0 < 32; r0 += N) {
        const int r = r0 + first;
        float x[N];
#pragma unroll
        for (int i = 0; i < N; i += 4)
          asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                       : "=f"(x[i]), "=f"(x[i + 1]), "=f"(x[i + 2]), "=f"(x[i + 3])
                       : "r"(turn + (uint32_t)(r * 128 + (((q * N + i) / 4 ^ (r & 7)) << 4)))
                       : "memory");
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(x[i], cu[i], cb[i]);
        if (after && inside && r < have) low_part<N>((int64_t)row0 + r, col0 + q * N, left - q * N, x);
        round_to<T>(x, w);
        if (inside && r < have) *reinterpret_cast<uint4*>(o + r0 * ldy) = uint4{w[0], w[1], w[2], w[3]};
      }
    } else if (lane < left) {
      T* o = y + (int64_t)row0 * ldy + col0 + lane;
#pragma unroll 8
      for (int r = 0; r < have; ++r) {
        float x;
        asm volatile("ld.shared.f32 %0, [%1];"
                     : "=f"(x)
                     : "r"(turn + (uint32_t)(r * 128 + ((lane >> 2 ^ (r & 7)) << 4) + (lane & 3) * 4))
                     : "memory");
        float z[1] = {fmaf(x, uc, bc)};
        if (after) low_part<1>((int64_t)row0 + r, col0 + lane, 1, z);
        o[r * ldy] = from_f32<T>(z[0]);
      }
    }
  }
};

// A few rows on the CUDA cores (FP32, or BF16 that TMA cannot read): a warp
// takes four rows of W against eight of x; VEC: four FP32 columns a load. Bound by
// the latency of the loads in flight (4,096 x 4,096 FP32, W from memory: eight rows
// 32 us, 2.1 TB/s; 16 rows 51, one column a load 57; 48 rows 103, 157 by ones).
// Up to 64 rows stay here: at 64 the tensor cores take 106 us for 128 at the shape
// above, but 25 for 13 at 1,024 x 1,000.
// u: the rows' low-rank products, or null where a block works them out itself,
// kRowsDots of them at most (as many rows of A as the block has of W) of kRowsOwn
// features: a launch of its own costs the host 3 us and the GPU under one, four
// dots a warp of 4,096 features 14.
constexpr int kRowsDots = 16, kRowsOwn = 512;
template <typename T, bool VEC>
__global__ void __launch_bounds__(128)
    k_rows(const T* x, int64_t ldx, int64_t tokens, const T* W, int64_t ldw, int classes, int d, const float* bias,
           const float* u, const T* A, const float* scales, const T* B, const int32_t* adapter, int G, int r, T* y,
           int64_t ldy) {
  __shared__ float own[kRowsDots];
  ptx::launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = (blockIdx.x * 4 + warp) * 4;
  const int64_t t0 = (int64_t)blockIdx.y * 8;
  const T *w[4], *xr[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = W + (int64_t)min(c0 + k, classes - 1) * ldw;
  ptx::wait_prerequisites();
#pragma unroll
  for (int k = 0; k < 8; ++k) xr[k] = x + min(t0 + k, tokens - 1) * ldx;
  float acc[32];
#pragma unroll
  for (int k = 0; k < 32; ++k) acc[k] = 0.f;
  if constexpr (VEC) {
#pragma unroll 2
    for (int i = lane * 4; i < d; i += 128) {
      float4 wv[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) wv[k] = __ldg(reinterpret_cast<const float4*>(w[k] + i));
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float4 xv = __ldg(reinterpret_cast<const float4*>(xr[k] + i));
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc[q * 8 + k] =
              fmaf(wv[q].x, xv.x, fmaf(wv[q].y, xv.y, fmaf(wv[q].z, xv.z, fmaf(wv[q].w, xv.w, acc[q * 8 + k]))));
      }
    }
  } else {
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
  if (G && !u) {
    // four of the rows' low-rank products a warp
    const T *xd[4], *ad[4];
    const int dots = (int)min((int64_t)8, tokens - t0) * r;
    float dot[4], scale[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = min(warp * 4 + k, dots - 1), row = e / r;
      const int g = __ldg(adapter + t0 + row);
      const bool any = g >= 0 && g < G;
      xd[k] = x + (t0 + row) * ldx;
      ad[k] = A + ((int64_t)(any ? g : 0) * r + e - row * r) * d;
      scale[k] = any && scales ? __ldg(scales + g) : 1.f;
      dot[k] = 0.f;
    }
#pragma unroll 2
    for (int i = lane; i < d; i += 32)
#pragma unroll
      for (int k = 0; k < 4; ++k) dot[k] = fmaf(to_f32<T>(xd[k][i]), to_f32<T>(ad[k][i]), dot[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) dot[k] += __shfl_xor_sync(0xffffffffu, dot[k], o);
      if (lane == 0 && warp * 4 + k < dots) own[warp * 4 + k] = scale[k] * dot[k];
    }
    __syncthreads();
  }
  const int c = c0 + lane / 8, row = lane % 8;
  const int64_t t = t0 + row;
  if (c >= classes || t >= tokens) return;
  float v = acc[0];
  if (bias) v += __ldg(bias + c);
  const int g = G ? __ldg(adapter + t) : -1;
  if (g >= 0 && g < G) {
    const T* b = B + ((int64_t)g * classes + c) * r;
    const float* ut = u ? u + t * r : own + row * r;
    for (int k = 0; k < r; ++k) v = fmaf(ut[k], to_f32<T>(b[k]), v);
  }
  y[t * ldy + c] = from_f32<T>(v);
}

// ---------------------------------------------------------------- outer products
// F_g[j, i] = sum over g's rows t of c[t, j] in[t, i]. A CTA lists the rows of
// its adapter, a window of rows at a time, in order.
constexpr int kWindow = 4096;  // (lists of 8 KB: two CTAs an SM)

// The rows of `g` among [t0, t1), as offsets from t0, by THREADS threads;
// returns their number. `count`: THREADS / 32 ints.
template <int THREADS>
__device__ __forceinline__ int list_rows(const int32_t* adapter, int64_t t0, int64_t t1, int g, uint16_t* list,
                                         int* count, int tid) {
  constexpr int kPer = kWindow / THREADS;  // neighbouring rows a thread
  static_assert(kPer <= 32 && kPer % 4 == 0, "a bit for each");
  const int n = (int)(t1 - t0), first = tid * kPer;
  uint32_t hits = 0;
  if ((((uintptr_t)(adapter + t0)) & 15) == 0 && first + kPer <= n) {
    int4 v[kPer / 4];
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i) v[i] = __ldg(reinterpret_cast<const int4*>(adapter + t0 + first) + i);
#pragma unroll
    for (int i = 0; i < kPer / 4; ++i)
      hits |= ((v[i].x == g ? 1u : 0u) | (v[i].y == g ? 2u : 0u) | (v[i].z == g ? 4u : 0u) | (v[i].w == g ? 8u : 0u)) << (4 * i);
  } else {
#pragma unroll 8
    for (int i = 0; i < kPer; ++i)
      if (first + i < n && __ldg(adapter + t0 + first + i) == g) hits |= 1u << i;
  }
  const int mine = __popc(hits);
  int at = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, at, o);
    if ((tid & 31) >= o) at += v;
  }
  if ((tid & 31) == 31) count[tid >> 5] = at;
  asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
  int all = 0;
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < tid >> 5) at += count[w];
    all += count[w];
  }
  at -= mine;
  while (hits) {
    list[at++] = (uint16_t)(first + __ffs(hits) - 1);
    hits &= hits - 1;
  }
  asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
  return all;
}

// BF16, on the tensor cores: D^T, 128 of i x r of j (both planes of c side by
// side). Four warps gather 64 rows a stage with 16-byte copies (past the list
// and the width: zeros), one issues the MMAs. A cluster shares the rows of one
// tile; its first CTA joins the parts in order. Bound by latency (the list, the
// first rows) and by the adapter with the most rows: 4,096 rows of eight adapters,
// r = 32, widths 2,048 and 4,096: 30 us.
struct OuterJob {
  const bf16* in;
  int64_t ld;
  int width;
  const uint16_t* c;  // planes of tokens x ldc
  bf16* out;
  int64_t f_g, f_j, f_i;
};
struct OuterJobs {
  OuterJob job[2];
  const int32_t* adapter;
  int64_t tokens, ldc, plane;
  int r, rb;          // rb: columns of a plane in the tile, 64 or 128
  unsigned long long* errors;
};
constexpr int kOuterThreads = 160, kOuterStages = 3;

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

__global__ void __launch_bounds__(kOuterThreads) k_outer(const OuterJobs a) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ int count[4];
  const OuterJob& job = a.job[blockIdx.z];
  uint32_t splits;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(splits));
  const uint32_t rank = ptx::cluster_ctarank();
  const int i0 = (int)(blockIdx.x / splits) * 128, g = blockIdx.y;
  if (i0 >= job.width) return;  // (the whole cluster)
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const int stage_bytes = 16384 + a.rb * 256;
  const uint32_t lists = base + kOuterStages * stage_bytes, full = lists + 2 * kWindow, empty = full + 8 * kOuterStages,
                 done = empty + 8 * kOuterStages, misc = done + 8;
  uint16_t* list = reinterpret_cast<uint16_t*>(smem_raw + (lists - ptx::smem_u32(smem_raw)));
  unsigned char* misc_p = smem_raw + (misc - ptx::smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc_p);
  volatile int* abort_s = reinterpret_cast<volatile int*>(misc_p + 4);
  volatile int* total_s = reinterpret_cast<volatile int*>(misc_p + 8);  // chunks of the window, or -1
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t cols = (uint32_t)a.rb * 2;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kOuterStages; ++s) {
      ptx::mbar_init(full + 8 * s, 128);
      ptx::mbar_init(empty + 8 * s, 1);
    }
    ptx::mbar_init(done, 1);
    *abort_s = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 4) {
    ptx::tmem_alloc(misc, cols);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const uint32_t tmem = *tmem_slot;
  const uint32_t id = mma::idesc(128, a.rb * 2, true, true, true);
  int st = 0, issued = 0;  // stage and chunks so far, on every thread alike
  uint32_t ph = 0, acc = 0;
  bool ok = true;
  const bool lead = warp == 4 && ptx::elect_one();
  for (int64_t t0 = 0; t0 < a.tokens; t0 += kWindow) {
    const int64_t t1 = min(t0 + kWindow, a.tokens);
    if (warp < 4) {
      const int n = list_rows<128>(a.adapter, t0, t1, g, list, count, threadIdx.x);
      if (threadIdx.x == 0) *total_s = n;
    }
    __syncthreads();
    const int n = *total_s, all = (n + 63) / 64;
    const int first = all * (int)rank / (int)splits, chunks = all * (int)(rank + 1) / (int)splits - first;
    issued += chunks;
    if (warp < 4) {
      auto arrive = [&](int s) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        ptx::mbar_arrive(full + 8 * s);
      };
      auto before = [&](int k) { return st >= k ? st - k : st - k + kOuterStages; };
      for (int k = 0; k < chunks && ok; ++k) {
        ok = ptx::mbar_wait(empty + 8 * st, ph ^ 1u, abort_s, mma::kWaitLimit);
        const uint32_t sa = base + st * stage_bytes;
        // 16-byte pieces of a row: 16 of `in`, rb / 8 of each plane of c; a lane
        // has the same piece of all its warp's rows
        for (int q = lane; q < 16 + a.rb / 4; q += 32) {
          const char* src;
          int64_t stride;
          uint32_t dst;
          int bytes, swz;
          if (q < 16) {
            const int i = i0 + q * 8;
            bytes = max(0, min(16, (job.width - i) * 2));
            src = reinterpret_cast<const char*>(job.in + (bytes ? i : 0));
            stride = job.ld * 2;
            dst = sa + (q >> 3) * 8192;
            swz = q & 7;
          } else {
            const int p = (q - 16) / (a.rb / 8), j = (q - 16) - p * (a.rb / 8);
            bytes = j * 8 < a.ldc ? 16 : 0;
            src = reinterpret_cast<const char*>(job.c + a.plane * p + (bytes ? j * 8 : 0));
            stride = a.ldc * 2;
            dst = sa + 16384 + (p * a.rb + (j >> 3) * 64) * 128;
            swz = j & 7;
          }
          src += t0 * stride;
          const uint16_t* rows = list + (first + k) * 64;
          const int left = n - (first + k) * 64;
#pragma unroll 4
          for (int r = warp; r < 64; r += 4)
            copy16(dst + r * 128 + ((swz ^ (r & 7)) << 4), src + (r < left ? rows[r] * stride : 0), r < left ? bytes : 0);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        // the stage two before this one has arrived; at the end, all have
        if (k >= 2) {
          asm volatile("cp.async.wait_group 2;" ::: "memory");
          arrive(before(2));
        }
        if (k == chunks - 1) {
          asm volatile("cp.async.wait_group 0;" ::: "memory");
          if (k >= 1) arrive(before(1));
          arrive(st);
        }
        if (++st == kOuterStages) st = 0, ph ^= 1u;
      }
    } else {
      for (int k = 0; k < chunks && ok; ++k) {
        ok = ptx::mbar_wait_warp(full + 8 * st, ph, abort_s, mma::kWaitLimit);
        if (!ok) break;
        ptx::tc_fence_after();
        if (lead) {
          uint64_t da = mma::desc(base + st * stage_bytes, true), db = mma::desc(base + st * stage_bytes + 16384, true);
          const int steps = min(4, (n - (first + k) * 64 + 15) / 16);
          for (int q = 0; q < steps; ++q, da += 2048 >> 4, db += 2048 >> 4) {
            ptx::mma_f16(tmem, da, db, id, acc);
            acc = 1;
          }
          ptx::mma_commit(empty + 8 * st);
        }
        if (++st == kOuterStages) st = 0, ph ^= 1u;
      }
    }
    __syncthreads();  // the list is free
  }
  if (warp == 4) {
    if (lead) {
      volatile int never = 0;
      ptx::mma_commit(done);
      ptx::mbar_wait(done, 0, &never, mma::kWaitLimit);
    }
    __syncwarp();
  } else {
    ok = ptx::mbar_wait(done, 0, abort_s, mma::kWaitLimit);
    ok = __all_sync(0xffffffffu, ok);
    ptx::tc_fence_after();
  }
  // hi + lo of 32 columns
  auto sums = [&](int j0, float (&v)[32]) {
    uint32_t hi[32], lo[32];
    const uint32_t src = tmem + ((uint32_t)(warp * 32) << 16) + j0;
    ptx::tmem_ld32(src, hi);
    ptx::tmem_ld32(src + a.rb, lo);
    ptx::tmem_wait_ld();
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = issued ? __uint_as_float(hi[j]) + __uint_as_float(lo[j]) : 0.f;
  };
  const int row = warp * 32 + lane;
  if (splits > 1) {
    ptx::cluster_sync();  // the first CTA's stages are free: its products are done
    if (warp < 4 && rank > 0) {
      const uint32_t dst = ptx::mapa(base, 0) + (rank - 1) * (uint32_t)(128 * a.rb * 4);
      for (int j0 = 0; j0 < a.r; j0 += 32) {
        float v[32];
        sums(j0, v);
#pragma unroll
        for (int j = 0; j < 32; ++j) store_cluster(dst + (uint32_t)((j0 + j) * 128 + row) * 4, v[j]);
      }
    }
    ptx::cluster_sync();
  }
  if (warp < 4 && rank == 0) {
    const float* part = reinterpret_cast<const float*>(smem_raw + (base - ptx::smem_u32(smem_raw)));
    const int i = i0 + row;
    bf16* out = job.out + g * job.f_g + (int64_t)i * job.f_i;
    const bool vec = job.f_j == 1 && a.r % 8 == 0 && ((uintptr_t)job.out & 15) == 0;
    for (int j0 = 0; ok && j0 < a.r; j0 += 32) {
      float v[32];
      sums(j0, v);
      for (uint32_t p = 1; p < splits; ++p) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] += part[(p - 1) * 128 * a.rb + (j0 + j) * 128 + row];
      }
      if (i >= job.width) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (j0 + q * 8 >= a.r) break;
        if (vec) {
          *reinterpret_cast<uint4*>(out + j0 + q * 8) =
              uint4{pack_bf16(v[q * 8], v[q * 8 + 1]), pack_bf16(v[q * 8 + 2], v[q * 8 + 3]),
                    pack_bf16(v[q * 8 + 4], v[q * 8 + 5]), pack_bf16(v[q * 8 + 6], v[q * 8 + 7])};
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j0 + q * 8 + j < a.r) out[(j0 + q * 8 + j) * job.f_j] = __float2bfloat16_rn(v[q * 8 + j]);
        }
      }
    }
    ptx::tc_fence_before();
  }
  __syncthreads();
  if (threadIdx.x == 0 && *abort_s) atomicAdd(a.errors, 1ull);
  ptx::tc_fence_after();
  if (warp == 4) ptx::tmem_dealloc(tmem, cols);
}

// FP32, on the CUDA cores: 64 COLS of i, eight of j at a time, the listed rows
// dealt over GROUPS groups of threads. Where adapters have 256 rows or more, 16
// groups and blocks of 64 columns, so that there are blocks enough (4,095 rows
// of five, r = 6, widths 500 and 1,000: 24 us). With fewer, most blocks find few
// rows or none, and eight groups of two columns a thread cost less (402 rows,
// nearly all of one adapter of 36, r = 16, widths 384 and 3,520: 42 us; with
// four groups of one column 80). Bound by the latency of a group's rows.
struct OuterJobF32 {
  const float* in;
  int64_t ld;
  int width;
  const float* c;  // tokens x r
  float* out;
  int64_t f_g, f_j, f_i;
};
struct OuterJobsF32 {
  OuterJobF32 job[2];
  const int32_t* adapter;
  int64_t tokens;
  int r;
};

template <int GROUPS, int COLS>
__global__ void __launch_bounds__(64 * GROUPS) k_outer_f32(const __grid_constant__ OuterJobsF32 a) {
  constexpr int kWide = 64 * COLS;
  __shared__ float red[GROUPS][8][kWide];
  __shared__ uint16_t list[kWindow];
  __shared__ int count[2 * GROUPS];
  const OuterJobF32& job = a.job[blockIdx.z];
  const int g = blockIdx.y;
  const int ti = threadIdx.x & 63, q = threadIdx.x >> 6, i = blockIdx.x * kWide + ti;
  if (blockIdx.x * kWide >= job.width) return;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  int n = 0;
  int64_t t0 = 0;
  const bool once = a.tokens <= kWindow;  // one list serves all j
  if (once) n = list_rows<64 * GROUPS>(a.adapter, 0, a.tokens, g, list, count, threadIdx.x);
  for (int j0 = 0; j0 < a.r; j0 += 8) {
    const int nj = min(8, a.r - j0);
    float acc[COLS][8] = {};
    for (t0 = 0; t0 < a.tokens; t0 += kWindow) {
      if (!once) n = list_rows<64 * GROUPS>(a.adapter, t0, min(t0 + kWindow, a.tokens), g, list, count, threadIdx.x);
#pragma unroll 4
      for (int k = q; k < n; k += GROUPS) {
        const int64_t t = t0 + list[k];
        const float* in = job.in + t * job.ld + i;
        const float* c = job.c + t * a.r + j0;
        float x[COLS], v[8];
#pragma unroll
        for (int m = 0; m < COLS; ++m) x[m] = i + 64 * m < job.width ? __ldg(in + 64 * m) : 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < nj ? __ldg(c + j) : 0.f;
#pragma unroll
        for (int m = 0; m < COLS; ++m)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < nj) acc[m][j] = fmaf(x[m], v[j], acc[m][j]);
      }
      if (!once) __syncthreads();
    }
#pragma unroll
    for (int m = 0; m < COLS; ++m)
#pragma unroll
      for (int j = 0; j < 8; ++j) red[q][j][ti + 64 * m] = acc[m][j];
    __syncthreads();
    // neighbouring threads along memory: along j or i
    float* out = job.out + g * job.f_g + j0 * job.f_j;
    for (int e = threadIdx.x; e < nj * kWide; e += 64 * GROUPS) {
      int j = e / kWide, k = e % kWide;
      if (job.f_j == 1) j = nj == 8 ? e & 7 : e % nj, k = nj == 8 ? e >> 3 : e / nj;
      const int at = blockIdx.x * kWide + k;
      float s = red[0][j][k];
#pragma unroll
      for (int w = 1; w < GROUPS; ++w) s += red[w][j][k];
      if (at < job.width) out[j * job.f_j + (int64_t)at * job.f_i] = s;
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- host side
constexpr int64_t kFewF32 = 64, kFewBf16 = 128;  // rows of the single-token form

// One product with the shared head: its rows' input (x or dy), its contracted
// width, its columns and the strides of the factor that shrinks it.
struct Side {
  const void* in;
  int64_t ld;
  int width, out;
  int64_t f_j, f_i;
};

struct Layout {
  uint16_t* in[2];        // rows of x, of dy: planes (FP32), copies (BF16 that TMA cannot read)
  uint16_t *w, *a, *b;    // the same of W and of the factors (BF16)
  float *undo_in, *undo_w;
  float* u[2];            // u, v: tokens x r
  uint16_t* up[2];        // their planes (BF16)
  // FP32 with few adapters: u (or v) and the factor, every adapter's side by side, in three BF16 planes
  bool dense;
  bf16 *wide_u, *wide_f;
  int* odd;
  int64_t ld_x, ld_y, ld_r, ld_g;
  void take(Carve& c, const lipcache_adapted& p, bool backward) {
    const bool f32 = p.type == LIPCACHE_F32;
    const int64_t T = p.tokens, G = p.adapters, r = G ? p.rank : 1;
    const int planes = f32 ? 2 : 1;
    ld_x = round_up(p.d, 8);
    ld_y = round_up(p.classes, 8);
    ld_r = round_up(r, 8);
    c.take(in[0], f32 && backward ? 0 : (size_t)(planes * T * ld_x));
    c.take(in[1], backward ? (size_t)(planes * T * ld_y) : 0);
    c.take(w, (size_t)(planes * p.classes * ld_x));
    c.take(a, f32 ? 0 : (size_t)(G * r * ld_x));
    c.take(b, f32 ? 0 : (size_t)(G * p.classes * ld_r));
    c.take(undo_in, (size_t)T);
    c.take(undo_w, (size_t)p.classes);
    // up to 256 columns: eight stages of two planes each (in the epilogue,
    // 65,536 x 200 with ten adapters of rank 8, the low-rank product took 100 of
    // 138 us)
    dense = f32 && G > 0 && G * r <= 256;
    ld_g = round_up(G * r, 8);
    c.take(wide_u, dense ? (size_t)(3 * T * ld_g) : 0);
    c.take(wide_f, dense ? (size_t)(3 * (backward ? G * r * ld_x : p.classes * ld_g)) : 0);
    c.take(odd, dense ? (size_t)(backward ? G * r : p.classes) : 0);
    for (int i = 0; i < 2; ++i) {
      c.take(u[i], G ? (size_t)(T * r) : 0);
      c.take(up[i], G && !f32 ? (size_t)(2 * T * ld_r) : 0);
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

  // A BF16 tensor as TMA can read it: itself, or a copy.
  Tensor readable(const void* in, int64_t ld, int64_t rows, int cols, int64_t planes, uint16_t* copy, int64_t ldo) {
    if (mma::mappable(in, ld)) return Tensor{in, cols, rows, planes, ld, rows * ld};
    const int64_t all = rows * planes;
    const int parts = (int)ceil_div(cols, 2048);
    launch_pdl(k_copy_rows, dim3((unsigned)(all * parts)), 256, s, reinterpret_cast<const uint16_t*>(in), ld, cols, parts,
               copy, ldo);
    LC_LAUNCH_CHECK("k_copy_rows");
    return Tensor{copy, cols, rows, planes, ldo, rows * ldo};
  }
  Tensor rows_of(const Side& d, int i) {
    return readable(d.in, d.ld, p.tokens, d.width, 1, l.in[i], i ? l.ld_y : l.ld_x);
  }
  Tensor head() { return readable(W, p.ldw, p.classes, p.d, 1, l.w, l.ld_x); }
  Tensor factor_a() { return readable(A, p.d, p.rank, p.d, p.adapters, l.a, l.ld_x); }
  Tensor factor_b() { return readable(B, p.rank, p.classes, p.rank, p.adapters, l.b, l.ld_r); }

  RowJob row_job(const void* in, int64_t ld, int64_t rows, int width) {
    RowJob j;
    j.in = static_cast<const float*>(in);
    j.ld = ld;
    j.rows = rows;
    j.width = width;
    j.vec = width % 4 == 0 && ld % 4 == 0 && ((uintptr_t)in & 15) == 0 ? 4
            : width % 2 == 0 && ld % 2 == 0 && ((uintptr_t)in & 7) == 0 ? 2
                                                                        : 1;
    return j;
  }
  RowJob planes_job(const void* in, int64_t ld, int64_t rows, int width, uint16_t* out, int64_t ldo, float* undo, int most) {
    RowJob j = row_job(in, ld, rows, width);
    j.planes = reinterpret_cast<__half*>(out);
    j.ldo = ldo;
    j.plane = rows * ldo;
    j.undo = undo;
    j.most = most;
    return j;
  }
  // u (i = 0) or v (1); `wide`: set side by side too, over the rows' powers of two
  LowJob low_job(const Side& d, const T* F, int i, bool wide) {
    LowJob j = {};
    j.in = static_cast<const float*>(d.in);
    j.ld = d.ld;
    j.width = d.width;
    const uintptr_t both = (uintptr_t)d.in | (uintptr_t)F;
    j.vec = d.width % 4 == 0 && d.ld % 4 == 0 && both % 16 == 0 ? 4 : d.width % 2 == 0 && d.ld % 2 == 0 && both % 8 == 0 ? 2 : 1;
    j.F = reinterpret_cast<const float*>(F);
    j.f_g = (int64_t)p.rank * d.width;
    j.f_j = d.f_j;
    j.f_i = d.f_i;
    j.u = l.u[i];
    j.wide = wide && l.dense ? l.wide_u : nullptr;
    j.undo = l.undo_in;
    return j;
  }
  void run_low(const LowJob* jobs, int n) {
    if (!n) return;
    LowJobs a = {};
    for (int k = 0; k < n; ++k) a.job[k] = jobs[k];
    a.adapter = p.adapter;
    a.scales = p.scales;
    a.tokens = p.tokens;
    a.ldw = l.ld_g;
    a.G = p.adapters;
    a.r = p.rank;
    // more rows a block leave fewer groups short; fewer fill the device, and then warps share them (4,095 rows of
    // five adapters: 8 rows, four warps a group 41 us; 16, two 32; 32, two 40; 9,095 rows of one: 32, one 52; 16, two 58)
    const int64_t sms = mma::num_sms();
    a.tile = p.tokens >= 128 * sms ? 128 : p.tokens >= 32 * sms ? 32 : p.tokens >= 16 * sms ? 16 : 8;
    a.share = a.tile == 8 ? 4 : a.tile == 16 ? 2 : 1;
    launch_pdl(k_low_f32, dim3((unsigned)ceil_div(p.tokens, a.tile), (unsigned)ceil_div(p.rank, 8), (unsigned)n), 256, s, a);
    LC_LAUNCH_CHECK("k_low_f32");
  }
  void run_rows(const RowJob& a, const RowJob& b, const RowJob& c) {
    RowJobs j{{a, b, c}, p.adapters, p.rank, {}};
    unsigned all = 0;
    for (int k = 0; k < kRowJobs; ++k) {
      j.blocks[k] = (int)std::min<int64_t>(ceil_div(j.job[k].rows, 4), 32 * mma::num_sms());
      all += (unsigned)j.blocks[k];
    }
    if (!all) return;
    launch_pdl(k_rows_f32, dim3(all), 128, s, j);
    LC_LAUNCH_CHECK("k_rows_f32");
  }

  // u and/or v on the tensor cores.
  struct Shrinking {
    Tensor rows, factor;
    bool f_mn;
    int i;
  };
  void shrink(const Shrinking* jobs, int n) {
    ShrinkJobs a = {};
    int chunks = 1 << 30;
    const int rn = (int)round_up(p.rank, 16), rb = p.rank <= 64 ? 64 : 128;
    for (int k = 0; k < n; ++k) {
      ShrinkJob& j = a.job[k];
      const Shrinking& d = jobs[k];
      j.rows = mma::tensor_map(d.rows, 128);
      j.f_mn = d.f_mn;
      j.cols = d.f_mn ? rb : rn;
      j.factor = mma::tensor_map(d.factor, d.f_mn ? 64 : rn);
      j.f_bytes = j.cols * 128;
      j.per = std::min(8, 256 / j.cols);
      const mma::Seg g = mma::segment(d.rows.cols, 0);
      j.chunks = g.chunks;
      j.last = g.last;
      j.u = l.u[d.i];
      j.planes = l.up[d.i];
      chunks = std::min(chunks, j.chunks);
    }
    a.adapter = p.adapter;
    a.scales = p.scales;
    a.tokens = p.tokens;
    a.ldo = l.ld_r;
    a.plane = p.tokens * l.ld_r;
    a.G = p.adapters;
    a.r = p.rank;
    a.rn = rn;
    a.errors = mma::error_counter();
    const int64_t tiles = ceil_div(p.tokens, 128);
    // the width split until the device is filled, two stages or more a CTA
    int splits = 1;
    while (splits < (rn <= 64 ? 4 : 2) && tiles * n * splits * 2 <= mma::num_sms() && chunks >= 4 * splits) splits *= 2;
    const int smem = 1024 + kShrinkStages * kShrinkStage + 128 * 128 * 4 + 128;
    allow_smem(reinterpret_cast<const void*>(k_shrink), smem);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)splits;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(splits * tiles), 1, (unsigned)n);
    cfg.blockDim = dim3(kShrinkThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    LC_CUDA(cudaLaunchKernelEx(&cfg, k_shrink, a));
    LC_LAUNCH_CHECK("k_shrink");
  }

  // out = rows . W + low-rank: M tokens, N d.out, K d.width. F: the low-rank
  // factor as the tensor cores read it, or null
  // (FP32: as FP32 planes with every adapter's side by side).
  template <bool EARLY>
  void product(const Side& d, const Tensor& rows, const Tensor& w, bool w_mn, int i, const Tensor* F, bool f_mn,
               AdaptEpi<T, EARLY> e) {
    mma::Args a = {};
    const int64_t tiles = ceil_div(p.tokens, 256) * ceil_div(d.out, 256);
    // CTA pairs where their tiles fill half the device; else single CTAs, the tile narrowed until they do
    const bool pair = !EARLY && tiles >= mma::num_sms() / 4;
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
    a.a_rows = (int)std::min<int64_t>(128, round_up(p.tokens, 8));
    a.block = kBlock;
    const uint32_t id = mma::idesc(tm, a.bn, !f32, false, w_mn);
    a.seg = mma::segment(d.width, id);
    a.a_planes = a.b_planes = 1;
    a.low_after = e.u && !F;
    mma::Maps maps;
    maps.a = mma::tensor_map(rows, a.a_rows);
    maps.b = mma::tensor_map(w, w_mn ? 64 : a.bn / (pair ? 2 : 1));
    maps.la = maps.a;
    maps.lb = maps.b;
    if (F) {
      a.lb_mn = f_mn;
      a.low.adapter = p.adapter;
      a.low.tokens = p.tokens;
      a.low.G = p.adapters;
      a.low.dense = f32;
      const int64_t k = f32 ? (int64_t)p.adapters * p.rank : p.rank;
      const mma::Seg g = mma::segment(k, mma::idesc(tm, a.bn, true, false, f_mn));
      a.low.chunks = g.chunks;
      a.low.last = g.last;
      a.low.idesc = g.idesc;
      maps.la = f32 ? mma::tensor_map(Tensor{l.wide_u, k, p.tokens, 3, l.ld_g, p.tokens * l.ld_g}, a.a_rows)
                    : mma::tensor_map(Tensor{l.up[i], l.ld_r, p.tokens, 2, l.ld_r, p.tokens * l.ld_r}, a.a_rows);
      maps.lb = mma::tensor_map(*F, f_mn ? 64 : a.bn / (pair ? 2 : 1));
    }
    if constexpr (EARLY) {
      mma::launch<1, 1>(maps, a, e, s);
    } else {
      if (pair)
        mma::launch<2, f32 ? 2 : 1>(maps, a, e, s);
      else
        mma::launch<1, f32 ? 2 : 1>(maps, a, e, s);
    }
  }

  template <bool EARLY = false>
  AdaptEpi<T, EARLY> epilogue(T* y, int64_t ldy, int cols) {
    AdaptEpi<T, EARLY> e = {};
    e.y = y;
    e.ldy = ldy;
    e.rows = p.tokens;
    e.cols = cols;
    e.vec = ((uintptr_t)y & 15) == 0 && ldy * sizeof(T) % 16 == 0;
    return e;
  }
  // the low-rank product in the epilogue: F of cols x r (by_col) or r x cols
  template <bool EARLY>
  void epilogue_low(AdaptEpi<T, EARLY>& e, int i, const T* F, bool by_col) {
    if (!p.adapters) return;
    constexpr int N = 16 / sizeof(T);
    e.u = l.u[i];
    e.F = F;
    e.adapter = p.adapter;
    e.G = p.adapters;
    e.r = p.rank;
    e.f_col = by_col ? p.rank : 1;
    e.f_j = by_col ? 1 : e.cols;
    e.f_vec = (by_col ? p.rank : e.cols) % N == 0 && ((uintptr_t)F & 15) == 0;
  }

  void forward(const float* bias, T* y, int64_t ldy) {
    const Side d{x, p.ldx, p.d, p.classes, p.d, 1};
    const bool low = p.adapters > 0, tma = !f32 && mma::mappable(x, p.ldx) && mma::mappable(W, p.ldw);
    if (p.tokens <= (tma ? kFewBf16 : kFewF32)) {
      const bool own = !tma && p.tokens * p.rank <= kRowsDots && p.d <= kRowsOwn;
      if (low && !own) {
        const int vec = ((uintptr_t)x & 15) == 0 && ((uintptr_t)A & 15) == 0 && p.ldx * sizeof(T) % 16 == 0 &&
                        p.d * sizeof(T) % 16 == 0;
        launch_pdl(k_shrink_few<T>, dim3((unsigned)p.tokens, (unsigned)ceil_div(p.rank, 8)), 128, s, x, p.ldx,
                   (int)p.d, A, vec, (int)p.adapters, (int)p.rank, p.adapter, p.scales, l.u[0]);
        LC_LAUNCH_CHECK("k_shrink_few");
      }
      if constexpr (!f32) {
        if (tma) {
          AdaptEpi<T, true> e = epilogue<true>(y, ldy, p.classes);
          e.bias = bias;
          epilogue_low(e, 0, B, true);
          product(d, rows_of(d, 0), head(), false, 0, nullptr, false, e);
          return;
        }
      }
      const bool wide = f32 && p.d % 4 == 0 && p.ldx % 4 == 0 && p.ldw % 4 == 0 && (((uintptr_t)x | (uintptr_t)W) & 15) == 0;
      launch_pdl(wide ? k_rows<T, f32> : k_rows<T, false>,
                 dim3((unsigned)ceil_div(p.classes, 16), (unsigned)ceil_div(p.tokens, 8)), 128, s, x, p.ldx, p.tokens, W,
                 p.ldw, (int)p.classes, (int)p.d, bias, own ? (const float*)nullptr : (const float*)l.u[0], A, p.scales,
                 B, p.adapter, (int)p.adapters, (int)p.rank, y, ldy);
      LC_LAUNCH_CHECK("k_rows");
      return;
    }
    AdaptEpi<T> e = epilogue(y, ldy, p.classes);
    e.bias = bias;
    epilogue_low(e, 0, B, true);
    if constexpr (f32) {
      RowJob jw = planes_job(W, p.ldw, p.classes, p.d, l.w, l.ld_x, l.undo_w, kRowPower);
      if (l.dense) {
        jw.side = B;
        jw.wide = l.wide_f;
        jw.ldw = l.ld_g;
        jw.wplane = p.classes * l.ld_g;
        jw.odd = l.odd;
        e.odd = l.odd;
      }
      run_rows(jw, planes_job(x, p.ldx, p.tokens, p.d, l.in[0], l.ld_x, l.undo_in, kRowPower), RowJob{});
      const LowJob ju = low_job(d, A, 0, true);
      run_low(&ju, low ? 1 : 0);
      e.undo_row = l.undo_in;
      e.undo_col = l.undo_w;
      const Tensor fb{l.wide_f, (int64_t)p.adapters * p.rank, p.classes, 3, l.ld_g, p.classes * l.ld_g};
      product(d, Tensor{l.in[0], p.d, p.tokens, 2, l.ld_x, p.tokens * l.ld_x},
              Tensor{l.w, p.d, p.classes, 2, l.ld_x, p.classes * l.ld_x}, false, 0, l.dense ? &fb : nullptr, false, e);
    } else {
      const Tensor rows = rows_of(d, 0), w = head();
      Tensor fb = {};
      if (low) {
        const Shrinking j{rows, factor_a(), false, 0};
        shrink(&j, 1);
        fb = factor_b();
      }
      product(d, rows, w, false, 0, low ? &fb : nullptr, false, e);
    }
  }

  void backward(const T* dy, int64_t lddy, T* dx, int64_t lddx, T* dA, T* dB) {
    const Side sx{x, p.ldx, p.d, p.classes, p.d, 1}, sy{dy, lddy, p.classes, p.d, 1, p.rank};
    const bool low = p.adapters > 0, want_v = low && (dx || dA), want_u = low && dB;
    if (!dx && !(low && (dA || dB))) return;
    AdaptEpi<T> e = epilogue(dx, lddx, p.d);
    if (dx) epilogue_low(e, 1, A, false);
    if constexpr (f32) {
      RowJob jw, ja, jy;
      if (dx) {
        jw = planes_job(W, p.ldw, p.classes, p.d, l.w, l.ld_x, l.undo_w, kFoldPower);
        if (l.dense) {
          ja = row_job(A, p.d, (int64_t)p.adapters * p.rank, p.d);
          ja.set_aside = 1;
          ja.wide = l.wide_f;
          ja.ldw = l.ld_x;
          ja.wplane = ja.rows * l.ld_x;
          ja.odd = l.odd;
          e.odd = l.odd;
          e.n_odd = (int)ja.rows;
        }
        run_rows(jw, ja, RowJob{});
        jy = planes_job(dy, lddy, p.tokens, p.classes, l.in[1], l.ld_y, l.undo_in, kRowPower);
        jy.fold = l.undo_w;  // W's planes are W over these
        run_rows(jy, RowJob{}, RowJob{});
      }
      LowJob jl[2];
      int nl = 0;
      if (want_v) jl[nl++] = low_job(sy, B, 1, dx != nullptr);
      if (want_u) jl[nl++] = low_job(sx, A, 0, false);
      run_low(jl, nl);
      if (dx) {
        e.undo_row = l.undo_in;
        const Tensor fa{l.wide_f, p.d, (int64_t)p.adapters * p.rank, 3, l.ld_x, p.adapters * p.rank * l.ld_x};
        product(sy, Tensor{l.in[1], p.classes, p.tokens, 2, l.ld_y, p.tokens * l.ld_y},
                Tensor{l.w, p.d, p.classes, 2, l.ld_x, p.classes * l.ld_x}, true, 1, l.dense ? &fa : nullptr, true, e);
      }
      if (low && (dA || dB)) {
        OuterJobsF32 o = {};
        int n = 0, wide = 0;
        if (dA) o.job[n++] = OuterJobF32{x, p.ldx, p.d, l.u[1], dA, (int64_t)p.rank * p.d, p.d, 1}, wide = p.d;
        if (dB)
          o.job[n++] = OuterJobF32{dy, lddy, p.classes, l.u[0], dB, (int64_t)p.rank * p.classes, 1, p.rank},
          wide = std::max(wide, p.classes);
        o.adapter = p.adapter;
        o.tokens = p.tokens;
        o.r = p.rank;
        const bool many = p.tokens >= 256 * (int64_t)p.adapters;
        const dim3 grid((unsigned)ceil_div(wide, many ? 64 : 128), (unsigned)p.adapters, (unsigned)n);
        if (many)
          launch_pdl(k_outer_f32<16, 1>, grid, 1024, s, o);
        else
          launch_pdl(k_outer_f32<8, 2>, grid, 512, s, o);
        LC_LAUNCH_CHECK("k_outer_f32");
      }
    } else {
      Tensor rx = {}, ry = {}, w = {}, fa = {}, fb = {};
      if (dx || want_v || want_u) ry = rows_of(sy, 1);
      if (low && (dA || dB)) rx = rows_of(sx, 0);
      if (dx) w = head();
      if (low && (dx || want_u)) fa = factor_a();
      if (want_v) fb = factor_b();
      if (want_u || want_v) {
        Shrinking j[2];
        int n = 0;
        if (want_v) j[n++] = Shrinking{ry, fb, true, 1};
        if (want_u) j[n++] = Shrinking{rx, fa, false, 0};
        shrink(j, n);
      }
      if (dx) product(sy, ry, w, true, 1, low ? &fa : nullptr, true, e);
      if (low && (dA || dB)) {
        OuterJobs o = {};
        int n = 0, wide = 0;
        if (dA)
          o.job[n++] = OuterJob{static_cast<const bf16*>(rx.base), rx.ld, (int)p.d, l.up[1], dA, (int64_t)p.rank * p.d, p.d, 1},
          wide = p.d;
        if (dB)
          o.job[n++] = OuterJob{static_cast<const bf16*>(ry.base), ry.ld, (int)p.classes, l.up[0], dB,
                                (int64_t)p.rank * p.classes, 1, p.rank},
          wide = std::max(wide, p.classes);
        o.adapter = p.adapter;
        o.tokens = p.tokens;
        o.ldc = l.ld_r;
        o.plane = p.tokens * l.ld_r;
        o.r = p.rank;
        o.rb = p.rank <= 64 ? 64 : 128;
        o.errors = mma::error_counter();
        const int smem = 1024 + kOuterStages * (16384 + o.rb * 256) + 2 * kWindow + 128;
        allow_smem(reinterpret_cast<const void*>(k_outer), 1024 + kOuterStages * (16384 + 128 * 256) + 2 * kWindow + 128);
        // CTAs a tile: as long as an adapter has some eight stages of rows for each (four: 37 us for 30 at 4,096 rows of 8), and a slot for its parts
        unsigned splits = 1;
        while (splits < (o.rb == 64 ? 4u : 2u) && p.tokens >= (int64_t)p.adapters * splits * 1024) splits *= 2;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = splits;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)ceil_div(wide, 128) * splits, (unsigned)p.adapters, (unsigned)n);
        cfg.blockDim = dim3(kOuterThreads);
        cfg.dynamicSmemBytes = (size_t)smem;
        cfg.stream = s;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        LC_CUDA(cudaLaunchKernelEx(&cfg, k_outer, o));
        LC_LAUNCH_CHECK("k_outer");
      }
    }
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

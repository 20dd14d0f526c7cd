// Newton-Schulz orthogonalisation of matrices with a side of at most 64, all
// steps in one launch and in FP32 on the CUDA cores.
//
// A cluster of CTAs keeps one matrix in shared memory for all steps: each CTA a
// slice of the columns of the wide X (m x n, m <= 64). A step sums S over the
// slice (4 x 4 sums a thread, rows interleaved so that neighbouring threads
// read neighbouring banks), joins the slices' S through the cluster's shared
// memory in a fixed order, squares it, and updates the slice in place (8 rows x
// 4 columns a thread). Memory is touched once: the gradient (momentum, weight)
// is read and the result written. Bound by the steps' latency (a join through
// the cluster, six block barriers): 64 matrices of 16 x 1024 with momentum and
// weights, FP32: 36 us a step.
#include <cooperative_groups.h>

#include "head_mma.cuh"

namespace lc {
namespace ops {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kMaxSide = 64;

struct SmallArgs {
  int rows, cols, tall, m, mp, n, nc, stride, steps;  // mp: m up to a multiple of 8; stride of a row of the slice
  int64_t ldg;
  float coef[3 * LIPCACHE_MAX_NS_STEPS];
  double eps;
  OrthoStep st;
};

// S[i][j] (+)= sum over k of X[i][k] X[j][k] for the 4 x 4 rows of a tile pair,
// k4 of every `step` groups of four columns from `k4`.
__device__ __forceinline__ void dot16(const float* x, int stride, int ti, int tj, int nb, int k4, int step, int groups,
                                      float (&acc)[16]) {
  const float *pi = x + ti * stride, *pj = x + tj * stride;
  for (; k4 < groups; k4 += step) {
    float4 a[4], b[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      a[q] = *reinterpret_cast<const float4*>(pi + q * nb * stride + 4 * k4);
      b[q] = *reinterpret_cast<const float4*>(pj + q * nb * stride + 4 * k4);
    }
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        acc[p * 4 + q] = fmaf(a[p].x, b[q].x, fmaf(a[p].y, b[q].y, fmaf(a[p].z, b[q].z, fmaf(a[p].w, b[q].w, acc[p * 4 + q]))));
  }
}

// X <- a X + P X in the slice: columns in passes, ROWS rows x four columns a
// thread.
template <int ROWS>
__device__ __forceinline__ void update(float* x, const float* p, int mp, int ss, int stride, int groups, float ca) {
  const int rg = mp / ROWS, per = kThreads / rg;  // groups of rows; groups of columns a pass
  const int r = threadIdx.x % rg, q0 = threadIdx.x / rg;
  for (int c0 = 0; c0 < groups; c0 += per) {
    const int c = c0 + q0;
    const bool live = q0 < per && c < groups;
    float4 acc[ROWS];
    if (live) {
      const float* xc = x + 4 * c;
      const float* pr = p + ROWS * r;
#pragma unroll
      for (int q = 0; q < ROWS; ++q) {
        const float4 v = *reinterpret_cast<const float4*>(xc + (ROWS * r + q) * stride);
        acc[q] = make_float4(ca * v.x, ca * v.y, ca * v.z, ca * v.w);
      }
#pragma unroll 4
      for (int k = 0; k < mp; ++k) {
        const float4 v = *reinterpret_cast<const float4*>(xc + k * stride);
        float pk[ROWS];
#pragma unroll
        for (int q = 0; q < ROWS; q += 4) {
          const float4 f = *reinterpret_cast<const float4*>(pr + k * ss + q);
          pk[q] = f.x, pk[q + 1] = f.y, pk[q + 2] = f.z, pk[q + 3] = f.w;
        }
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
          acc[q].x = fmaf(pk[q], v.x, acc[q].x);
          acc[q].y = fmaf(pk[q], v.y, acc[q].y);
          acc[q].z = fmaf(pk[q], v.z, acc[q].z);
          acc[q].w = fmaf(pk[q], v.w, acc[q].w);
        }
      }
    }
    __syncthreads();  // the pass's columns have been read
    if (live) {
#pragma unroll
      for (int q = 0; q < ROWS; ++q) *reinterpret_cast<float4*>(x + (ROWS * r + q) * stride + 4 * c) = acc[q];
    }
  }
}

template <typename T, typename TO>
__global__ void __launch_bounds__(kThreads) k_small(const T* g, TO* out, const SmallArgs a) {
  extern __shared__ float4 smem4[];
  __shared__ double norm_s;
  __shared__ double red[kThreads / 32];
  __shared__ float factor_s[3];
  float* smem = reinterpret_cast<float*>(smem4);
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
  const int64_t z = blockIdx.x / ctas;
  const int tid = threadIdx.x, mp = a.mp, ss = mp + 4;  // ss: row stride of S and P
  float* x = smem;                                      // mp x stride
  float* part = x + mp * a.stride;                      // two of mp x ss: this slice's S, by turns
  float* s = part + 2 * mp * ss;
  float* p = s + mp * ss;
  const int j0 = rank * a.nc, j1 = min(j0 + a.nc, a.n), nj = max(j1 - j0, 0);
  ptx::wait_prerequisites();
  ptx::launch_dependents();

  // the slice of D, and its sum of squares
  const int64_t grow = z * a.rows;  // first row of the matrix in g
  auto at = [&](int i, int j) { return a.tall ? (grow + j) * a.cols + i : (grow + i) * a.cols + j; };
  double sum = 0.0;
  float run = 0.f;
  for (int e = tid; e < mp * a.stride; e += kThreads) x[e] = 0.f;
  __syncthreads();
  // neighbouring threads along memory: along j (wide) or i (tall)
  const int len = a.tall ? a.m : nj, lines = a.tall ? nj : a.m;
  constexpr int kBatch = 8;  // elements of a thread whose loads are in flight together
  for (int e0 = tid; e0 < len * lines; e0 += kThreads * kBatch) {
    float v[kBatch], m[kBatch];
    int at_x[kBatch];
    int64_t o[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int e = e0 + q * kThreads;
      v[q] = m[q] = 0.f;
      at_x[q] = -1;
      if (e >= len * lines) continue;
      const int l = e / len, c = e - l * len, i = a.tall ? c : l, j = a.tall ? l : c;
      v[q] = to_f32<T>(g[a.tall ? (grow + j0 + j) * a.ldg + i : (grow + i) * a.ldg + j0 + j]);
      o[q] = at(i, j0 + j);
      if (a.st.weight) m[q] = a.st.momentum[o[q]];
      at_x[q] = i * a.stride + j;
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      if (at_x[q] < 0) continue;
      if (a.st.weight) {
        const float b = a.st.beta, r = a.st.fresh * v[q], n = fmaf(b, m[q], r);
        a.st.out_momentum[o[q]] = n;
        v[q] = a.st.nesterov ? fmaf(b, n, r) : n;
      }
      x[at_x[q]] = v[q];
      const float w = fabsf(v[q]);
      if (w < 0x1p60f && (w > 0x1p-50f || w == 0.f))
        run = fmaf(v[q], v[q], run);
      else  // squares that FP32 does not hold
        sum += (double)v[q] * v[q];
    }
  }
  sum += (double)run;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((tid & 31) == 0) red[tid >> 5] = sum;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kThreads / 32; ++w) sum += red[w];
    norm_s = sum;
  }
  cluster.sync();
  if (tid == 0) {  // (one thread: FP64 is slow)
    sum = 0.0;
    for (int r = 0; r < ctas; ++r) sum += *cluster.map_shared_rank(&norm_s, r);
    const double norm = sqrt(sum);
    int e2 = 0;
    frexp(norm > 0.0 ? norm : 1.0, &e2);
    // 2^-e2 (past FP32's range for the smallest matrices, so in two), then the rest
    const bool fine = isfinite(norm);
    factor_s[0] = fine ? ldexpf(1.f, min(-e2, 100)) : NAN;
    factor_s[1] = ldexpf(1.f, max(-e2 - 100, 0));
    factor_s[2] = fine ? (float)(ldexp(1.0, e2) / (norm + a.eps)) : NAN;
  }
  __syncthreads();
  const float f0 = factor_s[0], f1 = factor_s[1], f2 = factor_s[2];
  for (int e = tid; e < a.m * a.stride; e += kThreads) x[e] = x[e] * f0 * f1 * f2;
  __syncthreads();

  const int nb = mp / 4, tiles = nb * (nb + 1) / 2;
  int ks = 1;  // threads that share a tile
  while (ks < 32 && tiles * ks * 2 <= kThreads) ks *= 2;
  const int groups = (nj + 3) / 4;
  for (int it = 0; it < a.steps; ++it) {
    const float ca = a.coef[3 * it], cb = a.coef[3 * it + 1], cc = a.coef[3 * it + 2];
    float* mine = part + (it & 1) * mp * ss;
    // S of the slice
    for (int w = tid; w < (tiles * ks + 31) / 32 * 32; w += kThreads) {
      const int t = w / ks;
      float acc[16] = {};
      int tj = 0;
      while ((tj + 1) * (tj + 2) / 2 <= t) ++tj;
      const int ti = t - tj * (tj + 1) / 2;
      if (t < tiles) dot16(x, a.stride, ti, tj, nb, w & (ks - 1), ks, groups, acc);
      if (ks >= 16) {
        // 16 sums on 16 lanes: halve the values, double the lanes that share one
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
          const bool up = w & o;
#pragma unroll
          for (int q = 0; q < o; ++q) {
            const float keep = up ? acc[q + o] : acc[q], give = up ? acc[q] : acc[q + o];
            acc[q] = keep + __shfl_xor_sync(0xffffffffu, give, o);
          }
        }
        if (ks == 32) acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], 16);
        if (t < tiles && (w & (ks - 1)) < 16) {
          const int q = w & 15, i = ti + nb * (q >> 2), j = tj + nb * (q & 3);
          mine[i * ss + j] = acc[0];
          mine[j * ss + i] = acc[0];
        }
        continue;
      }
      for (int o = ks / 2; o > 0; o >>= 1) {
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[q] += __shfl_xor_sync(0xffffffffu, acc[q], o);
      }
      if (t < tiles && (w & (ks - 1)) == 0) {
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          const int i = ti + nb * (q >> 2), j = tj + nb * (q & 3);
          mine[i * ss + j] = acc[q];
          mine[j * ss + i] = acc[q];
        }
      }
    }
    if (ctas > 1) {
      cluster.sync();
      for (int e = tid; e < mp * ss; e += kThreads) {
        float v = 0.f;
        for (int r = 0; r < ctas; ++r) v += cluster.map_shared_rank(mine, r)[e];
        s[e] = v;
      }
      __syncthreads();
    } else {
      __syncthreads();
    }
    const float* sm = ctas > 1 ? s : mine;
    // P = b S + c S S (S is symmetric: rows against rows)
    if (mp <= 32) {  // an element a thread: too few tiles for them
      for (int e = tid; e < mp * mp; e += kThreads) {
        const int i = e / mp, j = e - i * mp;
        float acc = 0.f;
#pragma unroll 4
        for (int k = 0; k < mp; k += 4) {
          const float4 u = *reinterpret_cast<const float4*>(sm + i * ss + k), v = *reinterpret_cast<const float4*>(sm + j * ss + k);
          acc = fmaf(u.x, v.x, fmaf(u.y, v.y, fmaf(u.z, v.z, fmaf(u.w, v.w, acc))));
        }
        p[i * ss + j] = fmaf(cc, acc, cb * sm[i * ss + j]);
      }
    } else
    for (int w = tid; w < tiles; w += kThreads) {
      float acc[16] = {};
      int tj = 0;
      while ((tj + 1) * (tj + 2) / 2 <= w) ++tj;
      const int ti = w - tj * (tj + 1) / 2;
      dot16(sm, ss, ti, tj, nb, 0, 1, mp / 4, acc);
#pragma unroll
      for (int q = 0; q < 16; ++q) {
        const int i = ti + nb * (q >> 2), j = tj + nb * (q & 3);
        const float v = fmaf(cc, acc[q], cb * sm[i * ss + j]);
        p[i * ss + j] = v;
        p[j * ss + i] = v;
      }
    }
    __syncthreads();
    // X <- a X + P X: four rows a thread where eight leave threads idle
    if (mp / 8 * groups < kThreads)
      update<4>(x, p, mp, ss, a.stride, groups, ca);
    else
      update<8>(x, p, mp, ss, a.stride, groups, ca);
    __syncthreads();
  }
  for (int e0 = tid; e0 < len * lines; e0 += kThreads * kBatch) {
    float v[kBatch], w[kBatch];
    int64_t o[kBatch];
#pragma unroll
    for (int q = 0; q < kBatch; ++q) {
      const int e = e0 + q * kThreads;
      o[q] = -1;
      if (e >= len * lines) continue;
      const int l = e / len, c = e - l * len, i = a.tall ? c : l, j = a.tall ? l : c;
      o[q] = at(i, j0 + j);
      v[q] = x[i * a.stride + j];
      if (a.st.weight) w[q] = to_f32<TO>(static_cast<const TO*>(a.st.weight)[o[q]]);
    }
#pragma unroll
    for (int q = 0; q < kBatch; ++q)
      if (o[q] >= 0) out[o[q]] = from_f32<TO>(a.st.weight ? fmaf(a.st.keep, w[q], -a.st.rate * v[q]) : v[q]);
  }
  if (ctas > 1) cluster.sync();  // no CTA leaves while another reads its part
}

int smem_bytes(int mp, int stride) { return (mp * stride + 4 * mp * (mp + 4)) * 4; }
int slice_stride(int nc) { return (int)round_up(nc, 32) + 4; }

}  // namespace

bool ortho_small(int type, const void* G, int64_t ldg, int64_t batch, int rows, int cols, int steps,
                 const double* coefficients, double eps, void* out, const OrthoStep& st, cudaStream_t s) {
  SmallArgs a = {};
  a.rows = rows;
  a.cols = cols;
  a.tall = rows > cols;
  a.m = std::min(rows, cols);
  a.n = std::max(rows, cols);
  if (a.m > kMaxSide) return false;
  a.mp = (int)round_up(a.m, 8);
  // CTAs a matrix: until the slices have 256 columns or the device is full, and at least what shared memory asks for
  int ctas = 1;
  while (ctas < 8 && ((ceil_div(a.n, ctas) > 256 && batch * ctas * 2 <= 2 * mma::num_sms()) ||
                      smem_bytes(a.mp, slice_stride((int)round_up(ceil_div(a.n, ctas), 4))) > 200 * 1024))
    ctas *= 2;
  a.nc = (int)round_up(ceil_div(a.n, ctas), 4);
  a.stride = slice_stride(a.nc);
  const int smem = smem_bytes(a.mp, a.stride);
  if (smem > 200 * 1024) return false;
  a.steps = steps;
  a.ldg = ldg;
  for (int i = 0; i < 3 * steps; ++i) a.coef[i] = (float)coefficients[i];
  a.eps = eps;
  a.st = st;
  const int out_type = st.weight ? st.weight_type : type;
  void* dst = st.weight ? st.out_weight : out;
  auto go = [&](auto g, auto o) {
    using T = std::remove_const_t<std::remove_pointer_t<decltype(g)>>;
    using TO = std::remove_pointer_t<decltype(o)>;
    allow_smem(reinterpret_cast<const void*>(k_small<T, TO>), 200 * 1024);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(batch * ctas));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    LC_CUDA(cudaLaunchKernelEx(&cfg, k_small<T, TO>, g, o, a));
    LC_LAUNCH_CHECK("k_small");
  };
  typedef __nv_bfloat16 bf16;
  if (type == LIPCACHE_F32 && out_type == LIPCACHE_F32)
    go(static_cast<const float*>(G), static_cast<float*>(dst));
  else if (type == LIPCACHE_F32)
    go(static_cast<const float*>(G), static_cast<bf16*>(dst));
  else if (out_type == LIPCACHE_F32)
    go(static_cast<const bf16*>(G), static_cast<float*>(dst));
  else
    go(static_cast<const bf16*>(G), static_cast<bf16*>(dst));
  return true;
}

}  // namespace ops
}  // namespace lc

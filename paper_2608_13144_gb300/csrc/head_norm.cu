// Layer norm of feature rows and its gradients.
//   mean, rstd = 1 / sqrt(var + eps);  xh = (x - mean) rstd;  y = xh w + b
//   g = dy w;  dx = rstd (g - sum g / d - xh sum(g xh) / d)
//   dw = sum over rows of dy xh;  db = sum over rows of dy
// G threads a row, each with P of its columns in registers; a group takes rows in
// turn, so that weight, bias and the columns' sums stay with their thread. Columns'
// sums are written once a block and joined by a second kernel, in a fixed order.
//
// Sums are taken about a first mean, and what that mean is off by is taken out
// again: a row far from 0 loses nothing. The gradient does the same about the
// rounded mean that it is given.
#include "head_mma.cuh"
#include "head_rows.cuh"

namespace lc {
namespace ops {
namespace {

struct NormArgs {
  int64_t ldx, ldy, lddy, lddx, tokens;
  int d;
  float eps;
  const float *weight, *bias;
  float* stats;
  float* parts;  // gradient: blocks x 2 x d
};

constexpr uint32_t kAll = 0xffffffffu;

// A unit of B bytes.
template <int B>
struct Unit;
template <>
struct Unit<16> {
  using type = uint4;
};
template <>
struct Unit<8> {
  using type = uint2;
};
template <>
struct Unit<4> {
  using type = uint32_t;
};
template <>
struct Unit<2> {
  using type = uint16_t;
};

// The columns of a thread: units of B bytes, unit u at G u + rank, so that
// neighbours read next to each other.
template <typename T, int B, int G, int P>
struct Columns {
  static constexpr int E = B / (int)sizeof(T), U = P / E;  // values of a unit, units
  using Word = typename Unit<B>::type;
  struct Raw {
    Word w[U];
  };
  __device__ static __forceinline__ int column(int u, int rank) { return (u * G + rank) * E; }
  __device__ static __forceinline__ Raw load(const T* p, int d, int rank) {
    Raw r{};
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (column(u, rank) < d) r.w[u] = *reinterpret_cast<const Word*>(p + column(u, rank));
    return r;
  }
  __device__ static __forceinline__ void open(const Raw& r, float (&v)[P]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) v[u * E + e] = to_f32<T>(reinterpret_cast<const T*>(&r.w[u])[e]);
  }
  __device__ static __forceinline__ void store(T* p, int d, int rank, const float (&v)[P]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Word w;
#pragma unroll
      for (int e = 0; e < E; ++e) reinterpret_cast<T*>(&w)[e] = from_f32<T>(v[u * E + e]);
      if (column(u, rank) < d) *reinterpret_cast<Word*>(p + column(u, rank)) = w;
    }
  }
  // an FP32 array's values at the thread's columns, `other` past d
  __device__ static __forceinline__ void floats(const float* p, int d, int rank, float other, float (&v)[P]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) v[u * E + e] = p && column(u, rank) < d ? __ldg(p + column(u, rank) + e) : other;
  }
};

// Sums over a group of a cluster's blocks, on every thread. `turn`: this thread's
// count of sums, whose two buffers take turns: with one barrier between, a slow
// thread's reading is safe from the sum after next.
template <int G, int K, int CL>
struct GroupSum {
  float warps[2][K][G == 32 ? 1 : G / 32];
  float blocks[2][K];
  __device__ __forceinline__ void operator()(float (&v)[K], int& turn) {
#pragma unroll
    for (int i = 0; i < K; ++i) v[i] = warp_sum(v[i]);
    if constexpr (G > 32) {
      const int lane = threadIdx.x & 31;
      if (lane == 0) {
#pragma unroll
        for (int i = 0; i < K; ++i) warps[turn][i][threadIdx.x >> 5] = v[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < K; ++i) v[i] = warp_sum(lane < G / 32 ? warps[turn][i][lane] : 0.f);
      if constexpr (CL > 1) {
        if (threadIdx.x == 0) {
#pragma unroll
          for (int i = 0; i < K; ++i) blocks[turn][i] = v[i];
        }
        ptx::cluster_sync();
#pragma unroll
        for (int i = 0; i < K; ++i) {
          float s = 0.f;
#pragma unroll
          for (int b = 0; b < CL; ++b) {
            float o;
            asm volatile("ld.shared::cluster.f32 %0, [%1];"
                         : "=f"(o)
                         : "r"(ptx::mapa(ptx::smem_u32(&blocks[turn][i]), b))
                         : "memory");
            s += o;
          }
          v[i] = s;
        }
      }
      turn ^= 1;
    }
  }
};

template <int G>
constexpr int kBlock = G == 32 ? 256 : G;

// Whose rows a group takes: `first`, then every `step`-th; and where its columns
// begin. A cluster of CL blocks shares a row.
template <int G, int P, int CL>
struct Share {
  int64_t first, step;
  int base, d, rank;
  __device__ __forceinline__ explicit Share(int all) {
    constexpr int kGroups = kBlock<G> / G;
    const int block = (int)(blockIdx.x / CL);
    first = (int64_t)block * kGroups + (G == 32 ? threadIdx.x >> 5 : 0);
    step = (int64_t)(gridDim.x / CL) * kGroups;
    base = CL > 1 ? (int)ptx::cluster_ctarank() * G * P : 0;
    d = min(max(all - base, 0), CL > 1 ? G * P : all);
    rank = group_rank<G>();
  }
};

template <typename T, int B, int G, int P, int CL>
__global__ void __launch_bounds__(kBlock<G>) k_norm(const T* x, T* y, const NormArgs a) {
  using Cols = Columns<T, B, G, P>;
  __shared__ GroupSum<G, 1, CL> sum1;
  __shared__ GroupSum<G, 2, CL> sum2;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const Share<G, P, CL> at(a.d);
  float w[P], b[P];
  Cols::floats(a.weight ? a.weight + at.base : nullptr, at.d, at.rank, 1.f, w);
  Cols::floats(a.bias ? a.bias + at.base : nullptr, at.d, at.rank, 0.f, b);
  const float over = 1.f / (float)a.d;
  int turn1 = 0, turn2 = 0;
  typename Cols::Raw next = {};
  if (at.first < a.tokens) next = Cols::load(x + at.first * a.ldx + at.base, at.d, at.rank);
  for (int64_t t = at.first; t < a.tokens; t += at.step) {
    float v[P];
    Cols::open(next, v);
    if (t + at.step < a.tokens) next = Cols::load(x + (t + at.step) * a.ldx + at.base, at.d, at.rank);
    float s1[1] = {0.f};
#pragma unroll
    for (int i = 0; i < P; ++i) s1[0] += v[i];
    sum1(s1, turn1);
    float mean = s1[0] * over, off = mean, var = 0.f;
    // once, but for rows whose spread is lost in the first mean's rounding
    for (int round = 0; round < 8; ++round) {
      float s2[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < P; ++i) {
        v[i] = Cols::column(i / Cols::E, at.rank) < at.d ? v[i] - off : 0.f;
        s2[0] += v[i];
        s2[1] += v[i] * v[i];
      }
      sum2(s2, turn2);
      off = s2[0] * over;
      var = s2[1] * over - off * off;
      if (!(off * off > var * 0.00390625f)) break;
      mean += off;
    }
    const float rstd = 1.f / sqrtf((var < 0.f ? 0.f : var) + a.eps);
    if (a.stats && at.rank == 0 && at.base == 0) {
      a.stats[2 * t] = mean + off;
      a.stats[2 * t + 1] = rstd;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = (v[i] - off) * rstd * w[i] + b[i];
    Cols::store(y + t * a.ldy + at.base, at.d, at.rank, v);
  }
  if (CL > 1) ptx::cluster_sync();  // (others may still read this block's sums)
}

template <typename T, int B, int G, int P, int CL>
__global__ void __launch_bounds__(kBlock<G>) k_norm_grad(const T* dy, const T* x, T* dx, const NormArgs a) {
  using Cols = Columns<T, B, G, P>;
  constexpr int kGroups = kBlock<G> / G;
  __shared__ GroupSum<G, 3, CL> sum;
  extern __shared__ float cols_s[];  // G == 32: the warps' columns, 2 x d each
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const Share<G, P, CL> at(a.d);
  float w[P], dw[P], db[P];
  Cols::floats(a.weight ? a.weight + at.base : nullptr, at.d, at.rank, 1.f, w);
#pragma unroll
  for (int i = 0; i < P; ++i) dw[i] = db[i] = 0.f;
  const float over = 1.f / (float)a.d;
  int turn = 0;
  typename Cols::Raw next_x = {}, next_dy = {};
  float next_mean = 0.f, next_rstd = 0.f;
  auto load = [&](int64_t t) {
    if (t >= a.tokens) return;
    next_x = Cols::load(x + t * a.ldx + at.base, at.d, at.rank);
    next_dy = Cols::load(dy + t * a.lddy + at.base, at.d, at.rank);
    next_mean = __ldg(a.stats + 2 * t);
    next_rstd = __ldg(a.stats + 2 * t + 1);
  };
  load(at.first);
  for (int64_t t = at.first; t < a.tokens; t += at.step) {
    float v[P], g[P];
    Cols::open(next_x, v);
    Cols::open(next_dy, g);
    const float mean = next_mean, rstd = next_rstd;
    load(t + at.step);
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < P; ++i) {
      v[i] = Cols::column(i / Cols::E, at.rank) < at.d ? (v[i] - mean) * rstd : 0.f;
      s[0] += v[i];
      s[1] += g[i] * w[i];
      s[2] += g[i] * w[i] * v[i];
    }
    sum(s, turn);
    // xh is v less `off`, what the rounded mean leaves
    const float off = s[0] * over, mean_g = s[1] * over, mean_gx = s[2] * over - off * mean_g;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float xh = v[i] - off;
      dw[i] += g[i] * xh;
      db[i] += g[i];
      g[i] = rstd * (g[i] * w[i] - mean_g - xh * mean_gx);
    }
    if (dx) Cols::store(dx + t * a.lddx + at.base, at.d, at.rank, g);
  }
  if (CL > 1) ptx::cluster_sync();
  if (!a.parts) return;
  float* out = a.parts + (int64_t)(blockIdx.x / CL) * 2 * a.d + at.base;
  if constexpr (G == 32) {
    float* own = cols_s + (threadIdx.x >> 5) * 2 * a.d;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = Cols::column(i / Cols::E, at.rank) + i % Cols::E;
      if (c < at.d) {
        own[c] = dw[i];
        own[a.d + c] = db[i];
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.d; c += kBlock<G>) {
      float t = 0.f;
#pragma unroll
      for (int r = 0; r < kGroups; ++r) t += cols_s[r * 2 * a.d + c];
      out[c] = t;
    }
  } else {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = Cols::column(i / Cols::E, at.rank) + i % Cols::E;
      if (c < at.d) {
        out[c] = dw[i];
        out[a.d + c] = db[i];
      }
    }
  }
}

// The columns' sums of `blocks` blocks: a block takes 32 columns, a warp every 16th
// block's part.
__global__ void __launch_bounds__(512) k_norm_columns(const float* parts, int blocks, int d, float* dweight, float* dbias) {
  __shared__ float s[16][33];
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float t = 0.f;
  if (c < 2 * d) {
#pragma unroll 4
    for (int b = warp; b < blocks; b += 16) t += parts[(int64_t)b * 2 * d + c];
  }
  s[warp][lane] = t;
  __syncthreads();
  if (warp == 0 && c < 2 * d) {
    t = s[0][lane];
#pragma unroll
    for (int i = 1; i < 16; ++i) t += s[i][lane];
    if (c < d) {
      if (dweight) dweight[c] = t;
    } else if (dbias) {
      dbias[c - d] = t;
    }
  }
}

// Blocks (clusters) that take rows in turn: as many as a GB300's 152 SMs hold.
int norm_blocks(int64_t tokens, int d) {
  const int groups = d <= 512 ? 8 : 1;
  const int most = d <= 2048 ? 608 : d <= 8192 ? 304 : d <= 16384 ? 76 : d <= 32768 ? 38 : 19;
  return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(tokens, groups), most));
}

template <int CL, typename K, typename... Args>
void launch_cluster(K kernel, int blocks, int threads, int smem, cudaStream_t s, Args... args) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CL;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(blocks * CL));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 2 : 1;
  LC_CUDA(cudaLaunchKernelEx(&cfg, kernel, args...));
}

// f(G, P, CL) for rows of d columns.
template <typename F>
void by_width(int d, F&& f) {
  using std::integral_constant;
  auto with = [&](auto g, auto p, auto cl) { f(g, p, cl); };
  integral_constant<int, 1> one;
  if (d <= 256)
    with(integral_constant<int, 32>{}, integral_constant<int, 8>{}, one);
  else if (d <= 512)
    with(integral_constant<int, 32>{}, integral_constant<int, 16>{}, one);
  else if (d <= 2048)
    with(integral_constant<int, 128>{}, integral_constant<int, 16>{}, one);
  else if (d <= 4096)
    with(integral_constant<int, 256>{}, integral_constant<int, 16>{}, one);
  else if (d <= 8192)
    with(integral_constant<int, 512>{}, integral_constant<int, 16>{}, one);
  else if (d <= 16384)
    with(integral_constant<int, 512>{}, integral_constant<int, 16>{}, integral_constant<int, 2>{});
  else if (d <= 32768)
    with(integral_constant<int, 512>{}, integral_constant<int, 16>{}, integral_constant<int, 4>{});
  else
    with(integral_constant<int, 512>{}, integral_constant<int, 16>{}, integral_constant<int, 8>{});
}
// f(B) with the largest unit that divides every address and row.
template <typename T, typename F>
void by_alignment(uintptr_t bits, F&& f) {
  if (bits % 16 == 0)
    f(std::integral_constant<int, 16>{});
  else if (sizeof(T) == 2 && bits % 4 == 0)
    f(std::integral_constant<int, 4>{});
  else
    f(std::integral_constant<int, (int)sizeof(T)>{});
}

template <typename T>
void launch_norm(const T* x, T* y, const NormArgs& a, cudaStream_t s) {
  const uintptr_t bits = (uintptr_t)x | (uintptr_t)y | (uintptr_t)(a.ldx * sizeof(T)) | (uintptr_t)(a.ldy * sizeof(T)) |
                         (uintptr_t)(a.d * sizeof(T));
  by_width(a.d, [&](auto g, auto p, auto cl) {
    by_alignment<T>(bits, [&](auto b) {
      constexpr int G = decltype(g)::value, CL = decltype(cl)::value;
      launch_cluster<CL>(k_norm<T, decltype(b)::value, G, decltype(p)::value, CL>, norm_blocks(a.tokens, a.d), kBlock<G>, 0,
                         s, x, y, a);
    });
  });
  LC_LAUNCH_CHECK("k_norm");
}

template <typename T>
void launch_norm_grad(const T* dy, const T* x, T* dx, const NormArgs& a, float* dweight, float* dbias, cudaStream_t s) {
  const uintptr_t bits = (uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx | (uintptr_t)(a.ldx * sizeof(T)) |
                         (uintptr_t)(a.lddy * sizeof(T)) | (uintptr_t)(dx ? a.lddx * sizeof(T) : 0) |
                         (uintptr_t)(a.d * sizeof(T));
  const int blocks = norm_blocks(a.tokens, a.d);
  by_width(a.d, [&](auto g, auto p, auto cl) {
    by_alignment<T>(bits, [&](auto b) {
      constexpr int G = decltype(g)::value, CL = decltype(cl)::value;
      launch_cluster<CL>(k_norm_grad<T, decltype(b)::value, G, decltype(p)::value, CL>, blocks, kBlock<G>,
                         G == 32 ? 8 * 2 * a.d * 4 : 0, s, dy, x, dx, a);
    });
  });
  LC_LAUNCH_CHECK("k_norm_grad");
  if (!a.parts) return;
  launch_pdl(k_norm_columns, dim3((unsigned)ceil_div(2 * (int64_t)a.d, 32)), 512, s, (const float*)a.parts, blocks, a.d,
             dweight, dbias);
  LC_LAUNCH_CHECK("k_norm_columns");
}

}  // namespace

size_t layer_norm_bytes(int64_t tokens, int d) {
  return tokens == 0 ? 0 : (size_t)norm_blocks(tokens, d) * 2 * d * 4;
}

void layer_norm(int type, const void* x, int64_t ldx, int64_t tokens, int d, const float* weight, const float* bias,
                double eps, void* y, int64_t ldy, float* stats, cudaStream_t s) {
  NormArgs a{};
  a.ldx = ldx, a.ldy = ldy, a.tokens = tokens, a.d = d, a.eps = (float)eps;
  a.weight = weight, a.bias = bias, a.stats = stats;
  if (type == LIPCACHE_F32)
    launch_norm(static_cast<const float*>(x), static_cast<float*>(y), a, s);
  else
    launch_norm(static_cast<const __nv_bfloat16*>(x), static_cast<__nv_bfloat16*>(y), a, s);
}

void layer_norm_backward(int type, const void* dy, int64_t lddy, const void* x, int64_t ldx, int64_t tokens, int d,
                         const float* stats, const float* weight, void* dx, int64_t lddx, float* dweight, float* dbias,
                         unsigned char* ws, cudaStream_t s) {
  NormArgs a{};
  a.ldx = ldx, a.lddy = lddy, a.lddx = lddx, a.tokens = tokens, a.d = d;
  a.weight = weight, a.stats = const_cast<float*>(stats);
  a.parts = dweight || dbias ? reinterpret_cast<float*>(ws) : nullptr;
  if (type == LIPCACHE_F32)
    launch_norm_grad(static_cast<const float*>(dy), static_cast<const float*>(x), static_cast<float*>(dx), a, dweight,
                     dbias, s);
  else
    launch_norm_grad(static_cast<const __nv_bfloat16*>(dy), static_cast<const __nv_bfloat16*>(x),
                     static_cast<__nv_bfloat16*>(dx), a, dweight, dbias, s);
}

}  // namespace ops
}  // namespace lc

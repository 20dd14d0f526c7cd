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
  int d, rank;
  __device__ __forceinline__ int column(int u) const { return (u * G + rank) * E; }
  __device__ __forceinline__ bool inside(int u) const { return column(u) < d; }
  // f(index of a value, its column) for the thread's values
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (inside(u)) {
#pragma unroll
        for (int e = 0; e < E; ++e) f(u * E + e, column(u) + e);
      }
  }
  __device__ __forceinline__ void store(T* p, const float (&v)[P]) const {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (inside(u)) {
        float part[E];
#pragma unroll
        for (int e = 0; e < E; ++e) part[e] = v[u * E + e];
        Word w;
        if constexpr (sizeof(T) == 2 && E >= 2)
          round_to<T, E>(part, reinterpret_cast<uint32_t(&)[E / 2]>(w));
        else
#pragma unroll
          for (int e = 0; e < E; ++e) reinterpret_cast<T*>(&w)[e] = from_f32<T>(part[e]);
        *reinterpret_cast<Word*>(p + column(u)) = w;
      }
  }
  // an FP32 array's values, `other` without one
  __device__ __forceinline__ void floats(const float* p, float other, float (&v)[P]) const {
#pragma unroll
    for (int i = 0; i < P; ++i) v[i] = other;
    if (p) each([&](int i, int c) { v[i] = __ldg(p + c); });
  }
};

// Rows on their way to a thread: asynchronous copies of its columns into its own
// places of a ring in shared memory, D rows ahead, or one row ahead in registers
// (units of two bytes, which cannot be copied so).
template <typename T, int B, int G, int P, int D>
struct Feed {
  using Cols = Columns<T, B, G, P>;
  using Word = typename Cols::Word;
  static constexpr int U = Cols::U, E = Cols::E;
  static constexpr bool kRing = B >= 4;
  static constexpr int kDepth = kRing ? D : 1;
  static constexpr int kBytes = kRing ? D * P * G * (int)sizeof(T) : 0;  // of a group
  Word* ring;
  Word next[kRing ? 1 : U];
  __device__ __forceinline__ void issue(const Cols& at, int slot, const T* p) {
    if constexpr (kRing) {
      if (p) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (at.inside(u)) {
            const uint32_t to = ptx::smem_u32(ring + (slot * U + u) * G + at.rank);
            if constexpr (B == 16)
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p + at.column(u)) : "memory");
            else
              asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(p + at.column(u)), "n"(B) : "memory");
          }
      }
    } else if (p) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at.inside(u)) next[u] = *reinterpret_cast<const Word*>(p + at.column(u));
    }
  }
  __device__ __forceinline__ void take(const Cols& at, int slot, float (&v)[P]) const {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at.inside(u)) {
        const Word w = kRing ? ring[(slot * U + u) * G + at.rank] : next[kRing ? 0 : u];
#pragma unroll
        for (int e = 0; e < E; ++e) v[u * E + e] = to_f32<T>(reinterpret_cast<const T*>(&w)[e]);
      }
  }
};
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

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
      if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < K; ++i) warps[turn][i][threadIdx.x >> 5] = v[i];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < K; ++i) {
        v[i] = warps[turn][i][0];
#pragma unroll
        for (int j = 1; j < G / 32; ++j) v[i] += warps[turn][i][j];
      }
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

// Whose rows a group takes: `first`, then every `step`-th; and its columns, from
// `base` on. A cluster of CL blocks shares a row.
template <typename T, int B, int G, int P, int CL>
struct Share {
  int64_t first, step;
  int base, slot;
  Columns<T, B, G, P> cols;
  __device__ __forceinline__ explicit Share(int d) {
    constexpr int kGroups = kBlock<G> / G;
    slot = G == 32 ? threadIdx.x >> 5 : 0;
    first = (int64_t)(blockIdx.x / CL) * kGroups + slot;
    step = (int64_t)(gridDim.x / CL) * kGroups;
    base = CL > 1 ? (int)ptx::cluster_ctarank() * G * P : 0;
    cols.d = CL > 1 ? min(max(d - base, 0), G * P) : d;
    cols.rank = group_rank<G>();
  }
};

constexpr int kNormDepth = 4, kGradDepth = 3;

template <typename T, int B, int G, int P, int CL>
__global__ void __launch_bounds__(kBlock<G>) k_norm(const T* x, T* y, const NormArgs a) {
  extern __shared__ uint4 ring_s[];
  __shared__ GroupSum<G, 1, CL> sum1;
  __shared__ GroupSum<G, 2, CL> sum2;
  using Rows = Feed<T, B, G, P, kNormDepth>;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const Share<T, B, G, P, CL> at(a.d);
  Rows feed;
  feed.ring = reinterpret_cast<typename Rows::Word*>(reinterpret_cast<char*>(ring_s) + at.slot * Rows::kBytes);
  auto row = [&](int64_t t) { return t < a.tokens ? x + t * a.ldx + at.base : nullptr; };
#pragma unroll
  for (int i = 0; i < Rows::kDepth; ++i) {
    feed.issue(at.cols, i, row(at.first + i * at.step));
    commit_copies();
  }
  float w[P], b[P];
  at.cols.floats(a.weight ? a.weight + at.base : nullptr, 1.f, w);
  at.cols.floats(a.bias ? a.bias + at.base : nullptr, 0.f, b);
  const float over = 1.f / (float)a.d;
  int turn1 = 0, turn2 = 0, slot = 0;
  for (int64_t t = at.first; t < a.tokens; t += at.step) {
    float v[P];
    wait_copies<Rows::kDepth - 1>();
    feed.take(at.cols, slot, v);
    feed.issue(at.cols, slot, row(t + Rows::kDepth * at.step));
    commit_copies();
    slot = slot + 1 == Rows::kDepth ? 0 : slot + 1;
    float s1[1] = {0.f};
    at.cols.each([&](int i, int) { s1[0] += v[i]; });
    sum1(s1, turn1);
    float mean = s1[0] * over, off = mean, var = 0.f;
    // once, but for rows whose spread is lost in the first mean's rounding
    for (int again = 0; again < 8; ++again) {
      float s2[2] = {0.f, 0.f};
      at.cols.each([&](int i, int) {
        v[i] -= off;
        s2[0] += v[i];
        s2[1] += v[i] * v[i];
      });
      sum2(s2, turn2);
      off = s2[0] * over;
      var = s2[1] * over - off * off;
      if (!(off * off > var * 0.00390625f)) break;
      mean += off;
    }
    const float rstd = 1.f / sqrtf((var < 0.f ? 0.f : var) + a.eps);
    if (a.stats && at.cols.rank == 0 && at.base == 0) {
      a.stats[2 * t] = mean + off;
      a.stats[2 * t + 1] = rstd;
    }
    at.cols.each([&](int i, int) { v[i] = (v[i] - off) * rstd * w[i] + b[i]; });
    at.cols.store(y + t * a.ldy + at.base, v);
  }
  if (CL > 1) ptx::cluster_sync();  // (others may still read this block's sums)
}

template <typename T, int B, int G, int P, int CL>
__global__ void __launch_bounds__(kBlock<G>) k_norm_grad(const T* dy, const T* x, T* dx, const NormArgs a) {
  constexpr int kGroups = kBlock<G> / G;
  extern __shared__ uint4 ring_s[];  // the rows' rings; after them G == 32's warps' columns, 2 x d each
  __shared__ GroupSum<G, 3, CL> sum;
  using Rows = Feed<T, B, G, P, kGradDepth>;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const Share<T, B, G, P, CL> at(a.d);
  Rows feed_x, feed_dy;
  feed_x.ring = reinterpret_cast<typename Rows::Word*>(reinterpret_cast<char*>(ring_s) + at.slot * 2 * Rows::kBytes);
  feed_dy.ring = feed_x.ring + Rows::kBytes / B;
  float2 ahead[2] = {};  // the statistics of the next two rows
  auto issue = [&](int64_t t, int slot) {
    const bool is = t < a.tokens;
    feed_x.issue(at.cols, slot, is ? x + t * a.ldx + at.base : nullptr);
    feed_dy.issue(at.cols, slot, is ? dy + t * a.lddy + at.base : nullptr);
    commit_copies();
  };
  auto stats_of = [&](int64_t t) { return t < a.tokens ? float2{__ldg(a.stats + 2 * t), __ldg(a.stats + 2 * t + 1)} : float2{}; };
#pragma unroll
  for (int i = 0; i < Rows::kDepth; ++i) issue(at.first + i * at.step, i);
  ahead[0] = stats_of(at.first);
  ahead[1] = stats_of(at.first + at.step);
  float w[P], dw[P], db[P];
  at.cols.floats(a.weight ? a.weight + at.base : nullptr, 1.f, w);
#pragma unroll
  for (int i = 0; i < P; ++i) dw[i] = db[i] = 0.f;
  const float over = 1.f / (float)a.d;
  int turn = 0, slot = 0;
  for (int64_t t = at.first; t < a.tokens; t += at.step) {
    float v[P], g[P];
    wait_copies<Rows::kDepth - 1>();
    feed_x.take(at.cols, slot, v);
    feed_dy.take(at.cols, slot, g);
    issue(t + Rows::kDepth * at.step, slot);
    slot = slot + 1 == Rows::kDepth ? 0 : slot + 1;
    const float mean = ahead[0].x, rstd = ahead[0].y;
    ahead[0] = ahead[1];
    ahead[1] = stats_of(t + 2 * at.step);
    float s[3] = {0.f, 0.f, 0.f};
    at.cols.each([&](int i, int) {
      v[i] = (v[i] - mean) * rstd;
      const float gw = g[i] * w[i];
      s[0] += v[i];
      s[1] += gw;
      s[2] += gw * v[i];
    });
    sum(s, turn);
    // xh is v less `off`, what the rounded mean leaves
    const float off = s[0] * over, mean_g = s[1] * over, mean_gx = s[2] * over - off * mean_g;
    at.cols.each([&](int i, int) {
      const float xh = v[i] - off;
      dw[i] += g[i] * xh;
      db[i] += g[i];
      g[i] = rstd * (g[i] * w[i] - mean_g - xh * mean_gx);
    });
    if (dx) at.cols.store(dx + t * a.lddx + at.base, g);
  }
  if (CL > 1) ptx::cluster_sync();
  if (!a.parts) return;
  float* out = a.parts + (int64_t)(blockIdx.x / CL) * 2 * a.d + at.base;
  if constexpr (G == 32) {
    float* all = reinterpret_cast<float*>(reinterpret_cast<char*>(ring_s) + kGroups * 2 * Rows::kBytes);
    float* own = all + at.slot * 2 * a.d;
    at.cols.each([&](int i, int c) {
      own[c] = dw[i];
      own[a.d + c] = db[i];
    });
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.d; c += kBlock<G>) {
      float t = 0.f;
#pragma unroll
      for (int r = 0; r < kGroups; ++r) t += all[r * 2 * a.d + c];
      out[c] = t;
    }
  } else {
    at.cols.each([&](int i, int c) {
      out[c] = dw[i];
      out[a.d + c] = db[i];
    });
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

// Blocks (clusters of CL) that take rows in turn: what a GB300's 152 SMs hold at once
// of the kernel, whose rows are then dealt evenly.
constexpr int kSms = 152, kMostOnSm = 4;
template <typename K>
int resident_blocks(K kernel, int threads, int smem) {
  int n = 0;
  LC_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, (size_t)smem));
  return std::max(1, std::min(n, kMostOnSm)) * kSms;
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
      constexpr int G = decltype(g)::value, P = decltype(p)::value, CL = decltype(cl)::value, B = decltype(b)::value;
      constexpr int kSmem = kBlock<G> / G * Feed<T, B, G, P, kNormDepth>::kBytes;
      if (kSmem > 40 * 1024) allow_smem(reinterpret_cast<const void*>(k_norm<T, B, G, P, CL>), kSmem);
      static const int kResident = resident_blocks(k_norm<T, B, G, P, CL>, kBlock<G>, kSmem);
      const int blocks = (int)std::min<int64_t>(ceil_div(a.tokens, kBlock<G> / G), kResident / CL);
      launch_cluster<CL>(k_norm<T, B, G, P, CL>, blocks, kBlock<G>, kSmem, s, x, y, a);
    });
  });
  LC_LAUNCH_CHECK("k_norm");
}

template <typename T>
void launch_norm_grad(const T* dy, const T* x, T* dx, const NormArgs& a, float* dweight, float* dbias, cudaStream_t s) {
  const uintptr_t bits = (uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx | (uintptr_t)(a.ldx * sizeof(T)) |
                         (uintptr_t)(a.lddy * sizeof(T)) | (uintptr_t)(dx ? a.lddx * sizeof(T) : 0) |
                         (uintptr_t)(a.d * sizeof(T));
  int blocks = 0;
  by_width(a.d, [&](auto g, auto p, auto cl) {
    by_alignment<T>(bits, [&](auto b) {
      constexpr int G = decltype(g)::value, P = decltype(p)::value, CL = decltype(cl)::value, B = decltype(b)::value;
      constexpr int kSmem = kBlock<G> / G * (2 * Feed<T, B, G, P, kGradDepth>::kBytes + (G == 32 ? 2 * G * P * 4 : 0));
      if (kSmem > 40 * 1024) allow_smem(reinterpret_cast<const void*>(k_norm_grad<T, B, G, P, CL>), kSmem);
      static const int kResident = resident_blocks(k_norm_grad<T, B, G, P, CL>, kBlock<G>, kSmem);
      blocks = (int)std::min<int64_t>(ceil_div(a.tokens, kBlock<G> / G), kResident / CL);
      launch_cluster<CL>(k_norm_grad<T, B, G, P, CL>, blocks, kBlock<G>, kSmem, s, dy, x, dx, a);
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
  return (size_t)std::min<int64_t>(tokens, kSms * kMostOnSm) * 2 * d * 4;
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

// Layer norm of feature rows and its gradients.
//   mean, rstd = 1 / sqrt(var + eps);  xh = (x - mean) rstd;  y = xh w + b
//   g = dy w;  dx = rstd (g - sum g / d - xh sum(g xh) / d)
//   dw = sum over rows of dy xh;  db = sum over rows of dy
// G threads a row, each with P of its columns in registers; a group takes rows in
// turn, so that weight, bias and the columns' sums stay with their thread. Columns'
// sums are written once a block and joined by a second kernel, in a fixed order.
//
// A row's moments are taken by warps about the warp's own mean, rounded, and joined by
// their distances, which are small: a row far from 0 loses nothing, and one barrier a row
// is enough. (No value lies between a mean and the FP32 numbers beside it: the square of
// what the rounding takes from the mean is at most the variance.) The gradient takes out
// what the rounded mean that it is given is off by.
//
// Bound by memory, then by the latency of the sums' shuffles: 16,384 x 4,096 BF16 47
// us, 5.7 TB/s, the gradients 71 us, 5.7 TB/s, of which the columns' second kernel is 6;
// 65,536 x 256 FP32 gradients 36 us, 5.6 TB/s. 32 columns a thread where registers hold
// them (the gradient of BF16 rows: with weights in shared memory and values kept packed),
// since what a row costs a warp beside its values weighs less (16 columns: 54 us). Rows
// that are not aligned take two to three times as long (16,384 x 4,001 BF16 105 us, the
// gradients 165), bound by instructions: loads and stores of 4 bytes, shifts between them.
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
  float* parts;  // gradient: blocks x 2 x d, or null where one block writes the sums itself
  float *dweight, *dbias;
};

constexpr uint32_t kAll = 0xffffffffu;

// The columns of a thread: units of 16 bytes, or, where rows start anywhere or their
// width is not one of whole units (SHIFTED), of 4. A warp's units follow one another,
// each of a thread's 32 after the one before, so that neighbours read next to each
// other. Values are held in pairs, for instructions that take two. ALL: every place of
// the warp is a column of the row (of all warps of a row but its last ones).
template <typename T, int G, int P, bool SHIFTED>
struct Columns {
  static constexpr int B = SHIFTED ? 4 : 16, E = B / (int)sizeof(T), U = P / E;  // bytes, values of a unit; units
  using Word = typename std::conditional<SHIFTED, uint32_t, uint4>::type;
  int d, rank;
  __device__ __forceinline__ int column(int u) const { return ((rank & ~31) * U + u * 32 + (rank & 31)) * E; }
  template <bool ALL>
  __device__ __forceinline__ bool inside(int u) const {
    return ALL || column(u) < d;
  }
  __device__ __forceinline__ bool all() const { return ((rank & ~31) + 32) * P <= d; }
  // f(pair) for each pair with a column
  template <bool ALL, typename F>
  __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
    for (int k = 0; k < P / 2; ++k)
      if (inside<ALL>(2 * k / E)) f(k);
  }
  // the column of a pair's second value
  __device__ __forceinline__ int second(int k) const {
    return E == 1 ? column(2 * k + 1) : column(2 * k / E) + 2 * k % E + 1;
  }
  // a pair with a column; its second value 0 if that has none
  template <bool ALL>
  __device__ __forceinline__ uint64_t masked(uint64_t v, int k) const {
    return ALL || !SHIFTED || second(k) < d ? v : v & 0xffffffffull;
  }
  // how many columns the thread has
  __device__ __forceinline__ int count() const {
    int n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) n += min(max(d - column(u), 0), E);
    return n;
  }
  // The compiler takes units for new ones from here on.
  __device__ static __forceinline__ void forget(Word (&w)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (SHIFTED)
        asm volatile("" : "+r"(w[u]));
      else
        asm volatile("" : "+r"(w[u].x), "+r"(w[u].y), "+r"(w[u].z), "+r"(w[u].w));
    }
  }
  // a pair of the thread's units
  __device__ static __forceinline__ uint64_t pair(const Word (&w)[U], int k) {
    if constexpr (E == 1) {
      return ptx::pack_f32x2(w[2 * k], w[2 * k + 1]);
    } else if constexpr (SHIFTED) {
      return ptx::pack_f32x2(w[k] << 16, w[k] & 0xffff0000u);
    } else {
      const uint4& x = w[2 * k / E];
      const uint32_t v[4] = {x.x, x.y, x.z, x.w};
      if constexpr (sizeof(T) == 4)
        return ptx::pack_f32x2(v[(2 * k) & 3], v[(2 * k + 1) & 3]);
      else
        return ptx::pack_f32x2(v[k & 3] << 16, v[k & 3] & 0xffff0000u);
    }
  }
  // To a row: f(pair)'s values, a unit (or two of one value) at a time. BF16 rows that
  // start between two words: a thread writes the word that its unit's first value ends,
  // with the unit before it; at the ends of the warp's units and of the row single values.
  template <bool ALL, typename F>
  __device__ __forceinline__ void put(T* p, F&& f) const {
    if constexpr (!SHIFTED) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (inside<ALL>(u)) {
          uint32_t x[4];
#pragma unroll
          for (int k = 0; k < E / 2; ++k) {
            const uint64_t v = f(u * E / 2 + k);
            if constexpr (sizeof(T) == 4) {
              x[2 * k] = (uint32_t)v;
              x[2 * k + 1] = (uint32_t)(v >> 32);
            } else {
              x[k] = pack_bf16(lo_f32(v), hi_f32(v));
            }
          }
          *reinterpret_cast<uint4*>(p + column(u)) = uint4{x[0], x[1], x[2], x[3]};
        }
    } else if constexpr (E == 1) {
#pragma unroll
      for (int k = 0; k < P / 2; ++k)
        if (inside<ALL>(2 * k)) {
          const uint64_t v = f(k);
          p[column(2 * k)] = lo_f32(v);
          if (inside<ALL>(2 * k + 1)) p[column(2 * k + 1)] = hi_f32(v);
        }
    } else {
      const bool between = (uintptr_t)p & 2;
      const int lane = threadIdx.x & 31;
      auto one = [&](int c, uint32_t bits) { p[c] = __ushort_as_bfloat16((unsigned short)bits); };
      uint32_t x = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t last = x;
        const int c = column(u);
        if (inside<ALL>(u)) {
          const uint64_t v = f(u);
          x = pack_bf16(lo_f32(v), hi_f32(v));
        }
        if (!between) {
          if (ALL || c + 1 < d)
            *reinterpret_cast<uint32_t*>(p + c) = x;
          else if (c < d)
            one(c, x);
        } else {
          // (the first lane's unit follows the last lane's unit before)
          const uint32_t before = __shfl_sync(kAll, lane == 31 ? last : x, (lane + 31) & 31);
          if (ALL || c < d) {
            if (u > 0 || lane > 0)
              *reinterpret_cast<uint32_t*>(p + c - 1) = __funnelshift_r(before, x, 16);
            else
              one(c, x);
            if (u == U - 1 && lane == 31 ? ALL || c + 1 < d : !ALL && c + 2 == d) one(c + 1, x >> 16);
          }
        }
      }
    }
  }
  // f(value of the pair array, column) for each value
  template <typename F>
  __device__ __forceinline__ void each_value(const uint64_t (&v)[P / 2], F&& f) const {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int c = column(i / E) + i % E;
      if (c < d) f(i & 1 ? hi_f32(v[i / 2]) : lo_f32(v[i / 2]), c);
    }
  }
  // an FP32 array's values, `other` without one
  __device__ __forceinline__ void floats(const float* p, float other, uint64_t (&v)[P / 2]) const {
#pragma unroll
    for (int k = 0; k < P / 2; ++k) {
      float x[2] = {other, other};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = column((2 * k + h) / E) + (2 * k + h) % E;
        if (p && c < d) x[h] = __ldg(p + c);
      }
      v[k] = ptx::pack_f32x2(__float_as_uint(x[0]), __float_as_uint(x[1]));
    }
  }
};

// Rows on their way to a group of threads: asynchronous copies of 16 bytes, D rows
// ahead, to a ring in shared memory. A thread reads what it copied itself; of shifted
// rows also others' granules: barriers stand before the reading and before the next
// copy to the same place.
template <typename T, int G, int P, bool SHIFTED, int D>
struct Feed {
  using Cols = Columns<T, G, P, SHIFTED>;
  using Word = typename Cols::Word;
  static constexpr int N = 16 / (int)sizeof(T), C = P / N;  // values of a granule, granules of a thread
  static constexpr int kGranules = C * G + (SHIFTED ? 1 : 0);
  static constexpr int kBytes = D * kGranules * 16;  // of a group
  uint4* ring;
  template <bool ALL>
  __device__ __forceinline__ void issue(const Cols& at, int slot, const T* p) {
    if (!p || at.d == 0) return;  // (a cluster's block past the row has nothing)
    const int lead = SHIFTED ? (int)((uintptr_t)p & 15) / (int)sizeof(T) : 0;
    const uint4* from = reinterpret_cast<const uint4*>(p - lead);
    auto copy = [&](int j) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(ring + slot * kGranules + j)), "l"(from + j)
                   : "memory");
    };
#pragma unroll
    for (int v = 0; v < C; ++v) {
      const int j = (at.rank & ~31) * C + v * 32 + (at.rank & 31);
      if (ALL || j * N < at.d + lead) copy(j);
    }
    if (SHIFTED && at.rank == 0 && C * G * N < at.d + lead) copy(C * G);
  }
  // the thread's units of the row at p
  template <bool ALL>
  __device__ __forceinline__ void take(const Cols& at, int slot, const T* p, Word (&w)[Cols::U]) const {
    const Word* in = reinterpret_cast<const Word*>(ring + slot * kGranules);
    if constexpr (!SHIFTED) {
#pragma unroll
      for (int u = 0; u < Cols::U; ++u)
        if (at.template inside<ALL>(u)) w[u] = in[at.column(u) / Cols::E];
    } else {
      in += ((uintptr_t)p & 15) / 4;
      const bool between = sizeof(T) == 2 && ((uintptr_t)p & 2);
#pragma unroll
      for (int u = 0; u < Cols::U; ++u) {
        w[u] = 0;
        if (at.template inside<ALL>(u)) {
          const int i = at.column(u) / Cols::E;
          w[u] = in[i];
          if (between) w[u] = __funnelshift_r(w[u], in[i + 1], 16);
          if (!ALL && sizeof(T) == 2 && at.column(u) + 1 >= at.d) w[u] &= 0xffffu;
        }
      }
    }
  }
};
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ float sum_of(uint64_t v) { return lo_f32(v) + hi_f32(v); }
__device__ __forceinline__ float xor_sum(float v, int lanes) { return v + __shfl_xor_sync(kAll, v, lanes); }
// Two sums at once over a warp: a's on lanes below 16, b's on the others.
__device__ __forceinline__ float warp_sum2(float a, float b) {
  const bool high = threadIdx.x & 16;
  float v = (high ? b : a) + __shfl_xor_sync(kAll, high ? a : b, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = xor_sum(v, o);
  return v;
}
// Three: a's on lane 0, b's on lane 16, c's on lanes 8 and 24 (and those after them).
__device__ __forceinline__ float warp_sum3(float a, float b, float c) {
  const bool high = threadIdx.x & 16, odd = threadIdx.x & 8;
  const float ab = (high ? b : a) + __shfl_xor_sync(kAll, high ? a : b, 16);
  c = xor_sum(c, 16);
  float v = (odd ? c : ab) + __shfl_xor_sync(kAll, odd ? ab : c, 8);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) v = xor_sum(v, o);
  return v;
}

// What joins the warps of a row, and the blocks of a cluster. Two buffers take
// turns: with one barrier between, a slow thread's reading is safe from the join
// after next.
template <int G, int CL>
struct NormShared {
  float4 warp[2][G == 32 ? 1 : G / 32];
  float4 block[2];
};
// Every block's `mine` of the cluster, in order, to f(rank, value).
template <int CL, typename F>
__device__ __forceinline__ void over_cluster(float4& place, const float4& mine, F&& f) {
  if (threadIdx.x == 0) place = mine;
  ptx::cluster_sync();
#pragma unroll
  for (int b = 0; b < CL; ++b) {
    float4 o;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(o.x), "=f"(o.y), "=f"(o.z), "=f"(o.w)
                 : "r"(ptx::mapa(ptx::smem_u32(&place), b))
                 : "memory");
    f(b, o);
  }
}

template <int G>
constexpr int kBlock = G == 32 ? 256 : G;
// The barrier of a group of G threads among the block's GROUPS.
template <int G, int GROUPS>
__device__ __forceinline__ void group_barrier(int group) {
  if constexpr (G == 32)
    __syncwarp();
  else if constexpr (GROUPS == 1)
    __syncthreads();
  else
    asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "n"(G) : "memory");
}

// f(ALL) for a warp's columns: known before where rows are aligned (FULL: as wide as
// their threads' places), warp by warp where they are shifted and checks cost more.
template <bool FULL, bool SHIFTED, typename F>
__device__ __forceinline__ void by_warp(bool all, F& f) {
  if constexpr (FULL) {
    f(std::true_type{});
  } else {
    if constexpr (SHIFTED) {
      if (all) {
        f(std::true_type{});
        return;
      }
    }
    f(std::false_type{});
  }
}

// Blocks of an SM whose threads have so many registers.
template <int THREADS, int REGISTERS>
constexpr int kFitting = 65536 / (THREADS * REGISTERS) > 1 ? 65536 / (THREADS * REGISTERS) : 1;

// Whose rows a group takes: `first`, then every `step`-th; and its columns, from
// `base` on. A cluster of CL blocks shares a row.
template <typename T, int G, int P, bool SHIFTED, int CL, int GROUPS>
struct Share {
  int64_t first, step;
  int base, slot;
  Columns<T, G, P, SHIFTED> cols;
  __device__ __forceinline__ explicit Share(int d) {
    slot = GROUPS == 1 ? 0 : threadIdx.x / G;
    first = (int64_t)(blockIdx.x / CL) * GROUPS + slot;
    step = (int64_t)(gridDim.x / CL) * GROUPS;
    base = CL > 1 ? (int)ptx::cluster_ctarank() * G * P : 0;
    cols.d = CL > 1 ? min(max(d - base, 0), G * P) : d;
    cols.rank = threadIdx.x % G;
  }
};

// Rows ahead of a group (what shared memory holds of the widest).
template <typename T, int G, int P>
constexpr int kNormDepth = G * P * (int)sizeof(T) > 48 * 1024 ? 3 : 4;
constexpr int kGradDepth = 3;

template <typename T, int G, int P, bool FULL, bool SHIFTED, int CL>
__global__ void __launch_bounds__(kBlock<G>, SHIFTED ? kFitting<kBlock<G>, P == 8 ? 48 : P == 16 ? 80 : 128> : 1)
    k_norm(const T* x, T* y, const NormArgs a) {
  extern __shared__ uint4 ring_s[];
  __shared__ NormShared<G, CL> shared;
  using Rows = Feed<T, G, P, SHIFTED, kNormDepth<T, G, P>>;
  using Cols = typename Rows::Cols;
  constexpr int D = kNormDepth<T, G, P>;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const Share<T, G, P, SHIFTED, CL, kBlock<G> / G> at(a.d);
  Rows feed;
  feed.ring = ring_s + at.slot * (Rows::kBytes / 16);
  auto row = [&](int64_t t) { return t < a.tokens ? x + t * a.ldx + at.base : nullptr; };
#pragma unroll
  for (int i = 0; i < D; ++i) {
    feed.template issue<false>(at.cols, i, row(at.first + i * at.step));
    commit_copies();
  }
  uint64_t w[P / 2], b[P / 2];
  at.cols.floats(a.weight ? a.weight + at.base : nullptr, 1.f, w);
  at.cols.floats(a.bias ? a.bias + at.base : nullptr, 0.f, b);
  constexpr int W = G / 32;
  const int warp = G == 32 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int mine = __reduce_add_sync(kAll, at.cols.count());  // the warp's columns
  const float n = (float)mine, over_n = mine ? 1.f / n : 0.f, over = 1.f / (float)a.d;
  int turn = 0, slot = 0;
  T* out = y + at.first * a.ldy + at.base;
  auto rows = [&](auto whole) {
    constexpr bool ALL = decltype(whole)::value;
    for (int64_t t = at.first; t < a.tokens; t += at.step, out += at.step * a.ldy) {
      uint64_t v[P / 2];
      wait_copies<D - 1>();
      if (SHIFTED) group_barrier<G, kBlock<G> / G>(at.slot);
      {
        typename Rows::Word raw[Cols::U];
        feed.template take<ALL>(at.cols, slot, x + t * a.ldx + at.base, raw);
        at.cols.template each<ALL>([&](int k) { v[k] = Cols::pair(raw, k); });
      }
      auto refill = [&] {
        feed.template issue<ALL>(at.cols, slot, row(t + D * at.step));
        commit_copies();
        slot = slot + 1 == D ? 0 : slot + 1;
      };
      if (SHIFTED && G == 32) __syncwarp();
      if (!SHIFTED || G == 32) refill();
      // the warp's mean c, and its sums s and m2 of x - c and their squares
      uint64_t p = 0;
      at.cols.template each<ALL>([&](int k) { p = ptx::add_f32x2(p, v[k]); });
      float c = warp_sum(sum_of(p)) * over_n, off = c, s, m2;
      // once, but for rows whose spread is lost in the mean's rounding
      for (int again = 0;; ++again) {
        uint64_t s2 = 0, q2 = 0;
        at.cols.template each<ALL>([&](int k) {
          v[k] = at.cols.template masked<ALL>(ptx::add_f32x2(v[k], both(-off)), k);
          s2 = ptx::add_f32x2(s2, v[k]);
          q2 = ptx::fma_f32x2(v[k], v[k], q2);
        });
        const float sq = warp_sum2(sum_of(s2), sum_of(q2)), other = __shfl_xor_sync(kAll, sq, 16);
        s = lane < 16 ? sq : other;
        m2 = lane < 16 ? other : sq;
        off = (c + s * over_n) - c;  // by as much as c moves, so that v stays the distance from c
        if (!(s * s > m2 * n * 0.00390625f) || off == 0.f || again == 7) break;
        c += off;
      }
      // e: the warp's c less the row's mean
      float mean, e, var;
      if constexpr (W == 1) {
        e = -s * over_n;
        mean = c - e;
        var = (m2 + e * (2.f * s + n * e)) * over;
      } else {
        if (lane == 0) shared.warp[turn][warp] = float4{c, s, m2, n};
        __syncthreads();
        if (SHIFTED) refill();
        const float4 o = shared.warp[turn][lane % W];
        const float first = __shfl_sync(kAll, o.x, 0), away = o.x - first;
        float sum = away * o.w + o.y, count = o.w;
#pragma unroll
        for (int l = 1; l < W; l <<= 1) {
          sum = xor_sum(sum, l);
          if (CL > 1) count = xor_sum(count, l);
        }
        const float middle = sum * (CL > 1 ? (count > 0.f ? 1.f / count : 0.f) : over);
        const float apart = o.w > 0.f ? away - middle : 0.f;
        float q = o.z + apart * (2.f * o.y + o.w * apart);
#pragma unroll
        for (int l = 1; l < W; l <<= 1) q = xor_sum(q, l);
        e = __shfl_sync(kAll, apart, warp);
        mean = first + middle;
        if constexpr (CL > 1) {
          float4 part[CL];
          over_cluster<CL>(shared.block[turn], float4{first, middle, q, count}, [&](int r, const float4& o) { part[r] = o; });
          float all = 0.f;
#pragma unroll
          for (int r = 0; r < CL; ++r) all += ((part[r].x - part[0].x) + part[r].y) * part[r].w;
          const float centre = all * over;
          q = 0.f;
#pragma unroll
          for (int r = 0; r < CL; ++r) {
            const float apart = (part[r].x - part[0].x) + part[r].y - centre;
            q += part[r].w > 0.f ? part[r].z + part[r].w * apart * apart : 0.f;
          }
          e += (first - part[0].x) + middle - centre;
          mean = part[0].x + centre;
        }
        var = q * over;
        turn ^= 1;
      }
      const float rstd = 1.f / sqrtf((var < 0.f ? 0.f : var) + a.eps);
      if (a.stats && at.cols.rank == 0 && at.base == 0) {
        a.stats[2 * t] = mean;
        a.stats[2 * t + 1] = rstd;
      }
      at.cols.template put<ALL>(out, [&](int k) {
        return ptx::fma_f32x2(ptx::mul_f32x2(ptx::add_f32x2(v[k], both(e)), both(rstd)), w[k], b[k]);
      });
    }
  };
  by_warp<FULL, SHIFTED>(at.cols.all(), rows);
  if (CL > 1) ptx::cluster_sync();  // (others may still read this block's sums)
}

// Values wait as they were loaded, not as FP32, between the row's sums and its
// gradient; GROUPS groups of G threads a block, whose columns' sums join there.
template <typename T, int G, int P, bool FULL, bool SHIFTED, int CL, int GROUPS>
__global__ void __launch_bounds__(G* GROUPS, kFitting<G * GROUPS, P == 8 ? 80 : P == 16 ? 128 : 168>)
    k_norm_grad(const T* dy, const T* x, T* dx, const NormArgs a) {
  extern __shared__ uint4 ring_s[];  // the rows' rings; in the end the groups' columns, 2 x d each
  __shared__ NormShared<G, CL> shared_s[GROUPS];
  constexpr int D = kGradDepth;
  using Rows = Feed<T, G, P, SHIFTED, D>;
  using Cols = typename Rows::Cols;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const Share<T, G, P, SHIFTED, CL, GROUPS> at(a.d);
  NormShared<G, CL>& shared = shared_s[at.slot];
  Rows feed_x, feed_dy;
  feed_x.ring = ring_s + at.slot * 2 * (Rows::kBytes / 16);
  feed_dy.ring = feed_x.ring + Rows::kBytes / 16;
  float2 ahead = {};  // the next row's statistics
  auto issue = [&](auto whole, int64_t t, int slot) {
    constexpr bool ALL = decltype(whole)::value;
    const bool is = t < a.tokens;
    feed_x.template issue<ALL>(at.cols, slot, is ? x + t * a.ldx + at.base : nullptr);
    feed_dy.template issue<ALL>(at.cols, slot, is ? dy + t * a.lddy + at.base : nullptr);
    commit_copies();
  };
  auto stats_of = [&](int64_t t) {
    return t < a.tokens ? float2{__ldg(a.stats + 2 * t), __ldg(a.stats + 2 * t + 1)} : float2{};
  };
#pragma unroll
  for (int i = 0; i < D; ++i) issue(std::false_type{}, at.first + i * at.step, i);
  ahead = stats_of(at.first);
  // Weights in registers; where a thread holds 32 columns, in shared memory, a
  // thread's pairs G apart (each thread reads what a thread of its place wrote).
  constexpr bool kSharedWeight = P >= 32;
  __shared__ uint64_t weight_s[kSharedWeight ? P / 2 * G : 1];
  uint64_t w[P / 2], dw[P / 2], db[P / 2];
  if (!kSharedWeight || at.slot == 0) at.cols.floats(a.weight ? a.weight + at.base : nullptr, 1.f, w);
  if (kSharedWeight) {
    if (at.slot == 0) {
#pragma unroll
      for (int k = 0; k < P / 2; ++k) weight_s[k * G + at.cols.rank] = w[k];
    }
    __syncthreads();
  }
  auto weight = [&](int k) { return kSharedWeight ? weight_s[k * G + at.cols.rank] : w[k]; };
#pragma unroll
  for (int k = 0; k < P / 2; ++k) dw[k] = db[k] = 0;
  constexpr int W = G / 32;
  const int warp = (threadIdx.x % G) >> 5, lane = threadIdx.x & 31;
  const float over = 1.f / (float)a.d;
  int turn = 0, slot = 0;
  auto rows = [&](auto whole) {
    constexpr bool ALL = decltype(whole)::value;
    for (int64_t t = at.first; t < a.tokens; t += at.step) {
      typename Rows::Word raw_x[Cols::U], raw_dy[Cols::U];
      wait_copies<D - 1>();
      if (SHIFTED) group_barrier<G, GROUPS>(at.slot);
      feed_x.template take<ALL>(at.cols, slot, x + t * a.ldx + at.base, raw_x);
      feed_dy.template take<ALL>(at.cols, slot, dy + t * a.lddy + at.base, raw_dy);
      auto refill = [&] {
        issue(whole, t + D * at.step, slot);
        slot = slot + 1 == D ? 0 : slot + 1;
      };
      if (SHIFTED && G == 32) __syncwarp();
      if (!SHIFTED || G == 32) refill();
      const float mean = ahead.x, rstd = ahead.y;
      ahead = stats_of(t + at.step);
      const uint64_t minus_mean = both(-mean), r = both(rstd);
      uint64_t s0 = 0, s1 = 0, s2 = 0;
      at.cols.template each<ALL>([&](int k) {
        const uint64_t xh = at.cols.template masked<ALL>(ptx::mul_f32x2(ptx::add_f32x2(Cols::pair(raw_x, k), minus_mean), r), k);
        const uint64_t gw = ptx::mul_f32x2(Cols::pair(raw_dy, k), weight(k));
        s0 = ptx::add_f32x2(s0, xh);
        s1 = ptx::add_f32x2(s1, gw);
        s2 = ptx::fma_f32x2(gw, xh, s2);
      });
      float sum[3];
      const float part = warp_sum3(sum_of(s0), sum_of(s1), sum_of(s2));
      if constexpr (W == 1) {
        sum[0] = __shfl_sync(kAll, part, 0);
        sum[1] = __shfl_sync(kAll, part, 16);
        sum[2] = __shfl_sync(kAll, part, 8);
      } else {
        if ((lane & 7) == 0 && lane != 24) reinterpret_cast<float*>(&shared.warp[turn][warp])[lane == 8 ? 2 : lane >> 4] = part;
        group_barrier<G, GROUPS>(at.slot);
        if (SHIFTED) refill();
        const float4 o = shared.warp[turn][lane % W];
        sum[0] = o.x, sum[1] = o.y, sum[2] = o.z;
#pragma unroll
        for (int l = 1; l < W; l <<= 1)
#pragma unroll
          for (int i = 0; i < 3; ++i) sum[i] = xor_sum(sum[i], l);
        if constexpr (CL > 1) {
          float all[3] = {0.f, 0.f, 0.f};
          over_cluster<CL>(shared.block[turn], float4{sum[0], sum[1], sum[2], 0.f}, [&](int, const float4& o) {
            all[0] += o.x, all[1] += o.y, all[2] += o.z;
          });
          sum[0] = all[0], sum[1] = all[1], sum[2] = all[2];
        }
        turn ^= 1;
      }
      // (opened anew below: kept as FP32 since above, the values would take twice the registers)
      Cols::forget(raw_x);
      Cols::forget(raw_dy);
      // xh less `off`, what the rounded mean leaves
      const float off = sum[0] * over, mean_g = sum[1] * over, mean_gx = sum[2] * over - off * mean_g;
      const uint64_t less = both(-off), down = both(-mean_g * rstd), along = both(-mean_gx * rstd);
      auto step = [&](int k) {
        const uint64_t g = Cols::pair(raw_dy, k);
        const uint64_t xh = ptx::add_f32x2(ptx::mul_f32x2(ptx::add_f32x2(Cols::pair(raw_x, k), minus_mean), r), less);
        dw[k] = ptx::fma_f32x2(g, xh, dw[k]);
        db[k] = ptx::add_f32x2(db[k], g);
        return ptx::fma_f32x2(xh, along, ptx::fma_f32x2(ptx::mul_f32x2(g, weight(k)), r, down));
      };
      if (dx)
        at.cols.template put<ALL>(dx + t * a.lddx + at.base, step);
      else
        at.cols.template each<ALL>(step);
    }
  };
  by_warp<FULL, SHIFTED>(at.cols.all(), rows);
  if (CL > 1) ptx::cluster_sync();
  if (!a.dweight && !a.dbias) return;
  // one after the other in the block's part, or to the gradients themselves
  float* part = a.parts ? a.parts + (int64_t)(blockIdx.x / CL) * 2 * a.d : nullptr;
  if constexpr (GROUPS > 1) {
    // (all copies have arrived: the last rows' were waited for, the others are empty)
    __syncthreads();
    float* all = reinterpret_cast<float*>(ring_s);
    float* own = all + at.slot * 2 * a.d;
    at.cols.each_value(dw, [&](float v, int c) { own[c] = v; });
    at.cols.each_value(db, [&](float v, int c) { own[a.d + c] = v; });
    __syncthreads();
    auto join = [&](float* to, int from, int n) {
      for (int c = threadIdx.x; c < n; c += G * GROUPS) {
        float t = 0.f;
#pragma unroll
        for (int r = 0; r < GROUPS; ++r) t += all[r * 2 * a.d + from + c];
        to[c] = t;
      }
    };
    if (part) {
      join(part, 0, 2 * a.d);
    } else {
      if (a.dweight) join(a.dweight, 0, a.d);
      if (a.dbias) join(a.dbias, a.d, a.d);
    }
  } else {
    float *to_dw = part ? part : a.dweight, *to_db = part ? part + a.d : a.dbias;
    if (to_dw) at.cols.each_value(dw, [&](float v, int c) { to_dw[at.base + c] = v; });
    if (to_db) at.cols.each_value(db, [&](float v, int c) { to_db[at.base + c] = v; });
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
constexpr int kSms = 152;
template <typename K>
int resident_blocks(K kernel, int threads, int smem) {
  int n = 0;
  LC_CUDA(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, (size_t)smem));
  return std::max(1, n) * kSms;
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

template <int V>
using Int = std::integral_constant<int, V>;
// f(G, P, CL) for rows of d columns: as many columns a thread as registers hold
// (sums over threads cost more than values), more threads beyond, then blocks.
template <typename F>
void by_width(int d, F&& f) {
  if (d <= 256)
    f(Int<32>{}, Int<8>{}, Int<1>{});
  else if (d <= 512)
    f(Int<32>{}, Int<16>{}, Int<1>{});
  else if (d <= 1024)
    f(Int<32>{}, Int<32>{}, Int<1>{});
  else if (d <= 2048)
    f(Int<64>{}, Int<32>{}, Int<1>{});
  else if (d <= 4096)
    f(Int<128>{}, Int<32>{}, Int<1>{});
  else if (d <= 8192)
    f(Int<256>{}, Int<32>{}, Int<1>{});
  else if (d <= 16384)
    f(Int<512>{}, Int<32>{}, Int<1>{});
  else if (d <= 32768)
    f(Int<512>{}, Int<32>{}, Int<2>{});
  else
    f(Int<512>{}, Int<32>{}, Int<4>{});
}
// f(G, P, CL, GROUPS) of the gradient, which holds a thread's columns four times over
// (FP32 values; BF16 ones of aligned rows take half the registers).
template <typename T, bool SHIFTED, typename F>
void by_width_grad(int d, F&& f) {
  constexpr bool kPacked = sizeof(T) == 2 && !SHIFTED;
  if (d <= 256) {
    f(Int<32>{}, Int<8>{}, Int<1>{}, Int<8>{});
  } else if (d <= 512) {
    f(Int<32>{}, Int<16>{}, Int<1>{}, Int<8>{});
  } else if (d <= 1024) {
    if constexpr (kPacked)
      f(Int<32>{}, Int<32>{}, Int<1>{}, Int<12>{});
    else
      f(Int<64>{}, Int<16>{}, Int<1>{}, Int<8>{});
  } else if (d <= 2048) {
    if constexpr (kPacked)
      f(Int<64>{}, Int<32>{}, Int<1>{}, Int<6>{});
    else
      f(Int<128>{}, Int<16>{}, Int<1>{}, Int<4>{});
  } else if (d <= 4096) {
    if constexpr (kPacked)
      f(Int<128>{}, Int<32>{}, Int<1>{}, Int<3>{});
    else
      f(Int<256>{}, Int<16>{}, Int<1>{}, Int<2>{});
  } else if (d <= 8192) {
    f(Int<512>{}, Int<16>{}, Int<1>{}, Int<1>{});
  } else if (d <= 16384) {
    f(Int<512>{}, Int<16>{}, Int<2>{}, Int<1>{});
  } else if (d <= 32768) {
    f(Int<512>{}, Int<16>{}, Int<4>{}, Int<1>{});
  } else {
    f(Int<512>{}, Int<16>{}, Int<8>{}, Int<1>{});
  }
}
// The gradients' blocks (clusters) at most, each with its columns' sums in the workspace:
// as many as the registers of by_width_grad's kernels let the SMs hold.
int most_parts(int d) {
  return kSms * (d <= 256 ? 3 : d <= 512 ? 2 : 1) / (d <= 8192 ? 1 : d <= 16384 ? 2 : d <= 32768 ? 4 : 8);
}
// f(FULL)
template <bool SHIFTED, typename F>
void by_fullness(bool full, F&& f) {
  if constexpr (!SHIFTED) {
    if (full) return f(std::true_type{});
  }
  f(std::false_type{});
}

template <typename T>
void launch_norm(const T* x, T* y, const NormArgs& a, cudaStream_t s) {
  const uintptr_t bits = (uintptr_t)x | (uintptr_t)y | (uintptr_t)(a.ldx * sizeof(T)) | (uintptr_t)(a.ldy * sizeof(T)) |
                         (uintptr_t)(a.d * sizeof(T));
  auto launch = [&](auto shifted) {
    constexpr bool SHIFTED = decltype(shifted)::value;
    by_width(a.d, [&](auto g, auto p, auto cl) {
      by_fullness<SHIFTED>(a.d == g * p * cl, [&](auto full) {
        constexpr int G = decltype(g)::value, P = decltype(p)::value, CL = decltype(cl)::value;
        constexpr int kSmem = kBlock<G> / G * Feed<T, G, P, SHIFTED, kNormDepth<T, G, P>>::kBytes;
        const auto kernel = k_norm<T, G, P, decltype(full)::value, SHIFTED, CL>;
        if (kSmem > 40 * 1024) allow_smem(reinterpret_cast<const void*>(kernel), kSmem);
        static const int kResident = resident_blocks(kernel, kBlock<G>, kSmem);
        const int blocks = (int)std::min<int64_t>(ceil_div(a.tokens, kBlock<G> / G), kResident / CL);
        launch_cluster<CL>(kernel, blocks, kBlock<G>, kSmem, s, x, y, a);
      });
    });
  };
  if (bits % 16)
    launch(std::true_type{});
  else
    launch(std::false_type{});
  LC_LAUNCH_CHECK("k_norm");
}

template <typename T>
void launch_norm_grad(const T* dy, const T* x, T* dx, const NormArgs& a, cudaStream_t s) {
  const uintptr_t bits = (uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx | (uintptr_t)(a.ldx * sizeof(T)) |
                         (uintptr_t)(a.lddy * sizeof(T)) | (uintptr_t)(dx ? a.lddx * sizeof(T) : 0) |
                         (uintptr_t)(a.d * sizeof(T));
  int blocks = 0;
  auto launch = [&](auto shifted) {
    constexpr bool SHIFTED = decltype(shifted)::value;
    by_width_grad<T, SHIFTED>(a.d, [&](auto g, auto p, auto cl, auto groups) {
      // (a warp of 32 columns a thread: rows of 1,024 as any others, for want of registers)
      constexpr bool kChecked = SHIFTED || (decltype(g)::value == 32 && decltype(p)::value == 32);
      by_fullness<kChecked>(a.d == g * p * cl, [&](auto full) {
        constexpr int G = decltype(g)::value, P = decltype(p)::value, CL = decltype(cl)::value;
        constexpr int GROUPS = decltype(groups)::value;
        constexpr int kRing = GROUPS * 2 * Feed<T, G, P, SHIFTED, kGradDepth>::kBytes;
        constexpr int kSums = GROUPS > 1 ? GROUPS * 2 * G * P * 4 : 0, kSmem = kRing > kSums ? kRing : kSums;
        const auto kernel = k_norm_grad<T, G, P, decltype(full)::value, SHIFTED, CL, GROUPS>;
        if (kSmem > 40 * 1024) allow_smem(reinterpret_cast<const void*>(kernel), kSmem);
        static const int kResident = resident_blocks(kernel, G * GROUPS, kSmem);
        const bool sums = a.dweight || a.dbias;
        const int most = std::min(kResident / CL, most_parts(a.d));
        blocks = sums && !a.parts ? 1 : (int)std::min<int64_t>(ceil_div(a.tokens, GROUPS), most);
        launch_cluster<CL>(kernel, blocks, G * GROUPS, kSmem, s, dy, x, dx, a);
      });
    });
  };
  if (bits % 16)
    launch(std::true_type{});
  else
    launch(std::false_type{});
  LC_LAUNCH_CHECK("k_norm_grad");
  if (!a.parts) return;
  launch_pdl(k_norm_columns, dim3((unsigned)ceil_div(2 * (int64_t)a.d, 32)), 512, s, (const float*)a.parts, blocks, a.d,
             a.dweight, a.dbias);
  LC_LAUNCH_CHECK("k_norm_columns");
}

// Few rows, which one block (or cluster) takes and writes the columns' sums of itself:
// a second kernel and its workspace cost a call more than the rows one after another.
// Calls from Python take 15 us, 19 to 20 with both, until the rows' time shows; of the
// GPU's time at the limits (with both): 64 x 256 FP32 8 us (7), 64 x 500 12 (8; BF16 22,
// a call 20, and 9), 8 x 4,096 13 (10), 2 x 20,000 14 (14); 128 x 256 10 (6).
bool one_block(int64_t tokens, int d) { return tokens <= (d <= 512 ? 64 : d <= 4096 ? 8 : 2); }

}  // namespace

size_t layer_norm_bytes(int64_t tokens, int d) {
  return one_block(tokens, d) ? 0 : (size_t)std::min<int64_t>(tokens, most_parts(d)) * 2 * d * 4;
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
  a.dweight = dweight, a.dbias = dbias;
  a.parts = (dweight || dbias) && !one_block(tokens, d) ? reinterpret_cast<float*>(ws) : nullptr;
  if (type == LIPCACHE_F32)
    launch_norm_grad(static_cast<const float*>(dy), static_cast<const float*>(x), static_cast<float*>(dx), a, s);
  else
    launch_norm_grad(static_cast<const __nv_bfloat16*>(dy), static_cast<const __nv_bfloat16*>(x),
                     static_cast<__nv_bfloat16*>(dx), a, s);
}

}  // namespace ops
}  // namespace lc

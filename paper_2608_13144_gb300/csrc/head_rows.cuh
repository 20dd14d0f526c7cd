// Rows of logits and features: what the kernels that read them share. A row is
// covered by granules of 16 bytes (the first and last one may hold values of
// nothing's, which are masked); a group of G threads works on it, granule i being
// thread i % G's.
#pragma once

#include "operators.cuh"
#include "tc_ptx.cuh"

namespace lc {
namespace ops {

// exp(x) for x <= 0 on the special function unit: 2^(x log2 e).
__device__ __forceinline__ float exp2_of(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f;

// A granule of 16 bytes: its values as pairs of FP32 (two values an
// instruction), their maximum (NaN ignored), and FP32 pairs put back.
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  __device__ static __forceinline__ void open(const uint4& w, uint64_t (&v)[N / 2]) {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < N / 2; ++i)
      v[i] = sizeof(T) == 4 ? ptx::pack_f32x2(x[(2 * i) & 3], x[(2 * i + 1) & 3])
                            : ptx::pack_f32x2(x[i & 3] << 16, x[i & 3] & 0xffff0000u);
  }
  __device__ static __forceinline__ float top(const uint4& w) {
    if constexpr (sizeof(T) == 4) {
      return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    } else {
      const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w);
      const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
      return fmaxf(__low2float(m), __high2float(m));
    }
  }
  __device__ static __forceinline__ uint4 close(const uint64_t (&v)[N / 2]) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[2 * i] = (uint32_t)v[i];
        x[2 * i + 1] = (uint32_t)(v[i] >> 32);
      } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float((uint32_t)v[i]), __uint_as_float((uint32_t)(v[i] >> 32)));
        x[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    return uint4{x[0], x[1], x[2], x[3]};
  }
  // element j of a granule
  __device__ static __forceinline__ float at(const uint4& w, int j) {
    return to_f32<T>(reinterpret_cast<const T*>(&w)[j]);
  }
};
__device__ __forceinline__ uint64_t both(float f) {
  return ptx::pack_f32x2(__float_as_uint(f), __float_as_uint(f));
}
// exp(v - m) of a pair
__device__ __forceinline__ uint64_t exp_pair(uint64_t v, uint64_t minus_m) {
  const uint64_t x = ptx::mul_f32x2(ptx::add_f32x2(v, minus_m), both(kLog2e));
  return ptx::pack_f32x2(__float_as_uint(exp2_of(__uint_as_float((uint32_t)x))),
                         __float_as_uint(exp2_of(__uint_as_float((uint32_t)(x >> 32)))));
}

template <int W>
__device__ __forceinline__ uint4 window_at(const uint4& a, const uint4& b, bool half) {
  const uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint4 r{x[W], x[W + 1], x[W + 2], x[W + 3]};
  if (half) {
    r.x = __funnelshift_r(x[W], x[W + 1], 16);
    r.y = __funnelshift_r(x[W + 1], x[W + 2], 16);
    r.z = __funnelshift_r(x[W + 2], x[W + 3], 16);
    r.w = __funnelshift_r(x[W + 3], x[W + 4], 16);
  }
  return r;
}
// The 16 bytes at byte `m` (< 16, the same for the whole row) of granules a, b.
__device__ __forceinline__ uint4 window(const uint4& a, const uint4& b, int m) {
  const bool half = m & 2;
  switch (m >> 2) {
    case 0: return window_at<0>(a, b, half);
    case 1: return window_at<1>(a, b, half);
    case 2: return window_at<2>(a, b, half);
    default: return window_at<3>(a, b, half);
  }
}

__device__ __forceinline__ float lo_f32(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float hi_f32(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
// The larger one; NaN if either is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// The largest value of a granule, NaN if one is.
template <typename T>
__device__ __forceinline__ float top_nan(const uint4& w) {
  if constexpr (sizeof(T) == 4) {
    return max_nan(max_nan(__uint_as_float(w.x), __uint_as_float(w.y)),
                   max_nan(__uint_as_float(w.z), __uint_as_float(w.w)));
  } else {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w);
    const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
    return max_nan(__low2float(m), __high2float(m));
  }
}

// Values as integers of the same order (-0 as 0); kUnmasked: the lowest finite
// value's, which -inf stands below.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
constexpr uint32_t kUnmasked = 0x00800000u;
constexpr uint32_t kNanKey = 0xff800000u;  // +inf's: it and NaN (made positive by max_nan) are from here

// A row's granules.
template <typename T>
struct RowSpan {
  static constexpr int N = Vec<T>::N;
  const uint4* granules;
  int lead, count;
  __device__ __forceinline__ RowSpan(const T* p, int n) {
    const int off = (int)((uintptr_t)p & 15);
    granules = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) - off);
    lead = off / (int)sizeof(T);
    count = (lead + n + N - 1) / N;
  }
  __device__ __forceinline__ int first(int granule) const { return granule * N - lead; }
  // whether a granule holds values outside the row
  __device__ __forceinline__ bool edge(int granule, int n) const {
    return (granule == 0 && lead) || (granule == count - 1 && first(granule) + N > n);
  }
};
// What lies outside [0, n) becomes -inf.
template <typename T>
__device__ __forceinline__ uint4 masked_outside(uint4 w, int first, int n) {
  constexpr int N = Vec<T>::N;
  __align__(16) T v[N];
  *reinterpret_cast<uint4*>(v) = w;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (first + j < 0 || first + j >= n) v[j] = from_f32<T>(-INFINITY);
  return *reinterpret_cast<const uint4*>(v);
}

// A granule of outputs to the row at dr; `same`: dr is aligned as the row whose
// granules are counted.
template <typename T>
__device__ __forceinline__ void put_granule(T* dr, bool same, const uint4& o, int first, int n) {
  constexpr int N = Vec<T>::N;
  if (same && first >= 0 && first + N <= n) {
    *reinterpret_cast<uint4*>(dr + first) = o;
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (first + j >= 0 && first + j < n) dr[first + j] = reinterpret_cast<const T*>(&o)[j];
  }
}

// The threads of a row: all of a block, or a warp.
template <int G>
__device__ __forceinline__ int group_rank() {
  return G == 32 ? (int)(threadIdx.x & 31) : (int)threadIdx.x;
}
template <int G>
__device__ __forceinline__ void group_sync() {
  if constexpr (G == 32)
    __syncwarp();
  else
    __syncthreads();
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ---------------------------------------------------------------- softmax sums
// Of a set of logits with t = (z - m) / T, in units of log 2: m its maximum,
// 1 + others the sum of exp2(t), q the sum of exp2(t) t (<= 0). One of the values
// that are m stands outside `others`, so that a sure row's logarithm is
// log1p(others) to its last bits. none: no value above -inf.
struct RowSums {
  float m, others, q;
  bool none;
};

// BF16 values, for which bounding t costs less before they are opened: a value twice,
// so far below m that its t is at most -500 (reach = 500 / c) but finite, for
// |m| < 2^100.
__device__ __forceinline__ uint32_t floor_below(float m, float reach) {
  const uint32_t bits = __float_as_uint(m - reach - fabsf(m) * 0.015625f);
  // (rounded down: two steps of BF16 below m at least)
  const uint32_t low = (bits >> 31 ? bits + 0xffffu : bits) >> 16;
  return low | low << 16;
}
__device__ __forceinline__ bool has_floor(float m) { return fabsf(m) < 1.2676506e30f; }
__device__ __forceinline__ uint4 raised(uint4 w, uint32_t floor) {
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&w);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __hmax2(h[i], *reinterpret_cast<const __nv_bfloat162*>(&floor));
  return w;
}
// v - m of a granule's values: differences first, so that logits may stand at any
// offset (BF16 ones are opened by the subtraction itself).
template <typename T>
__device__ __forceinline__ void differences(const uint4& w, float m, uint64_t (&v)[Vec<T>::N / 2]) {
  if constexpr (sizeof(T) == 4) {
    Vec<T>::open(w, v);
#pragma unroll
    for (int i = 0; i < Vec<T>::N / 2; ++i) v[i] = ptx::add_f32x2(v[i], both(-m));
  } else {
    const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      asm("{\n\t.reg .b16 l, h;\n\t"
          "mov.b32 {l, h}, %2;\n\t"
          "sub.rn.f32.bf16 %0, l, %3;\n\t"
          "sub.rn.f32.bf16 %1, h, %3;\n\t}"
          : "=f"(lo), "=f"(hi)
          : "r"(x[i]), "f"(m));
      v[i] = ptx::pack_f32x2(__float_as_uint(lo), __float_as_uint(hi));
    }
  }
}
__device__ __forceinline__ uint64_t exp2_pair(uint64_t t) {
  return ptx::pack_f32x2(__float_as_uint(exp2_of(lo_f32(t))), __float_as_uint(exp2_of(hi_f32(t))));
}
// exp2 of anything from here down is 0; of -inf, too, but 0 * -inf is NaN.
constexpr float kLeast = -1000.f;
__device__ __forceinline__ uint64_t bounded(uint64_t t) {
  return ptx::pack_f32x2(__float_as_uint(fmaxf(lo_f32(t), kLeast)), __float_as_uint(fmaxf(hi_f32(t), kLeast)));
}

// What t and its bounds go by: c = log2(e) / T.
struct Scale {
  float c, reach;  // reach = 500 / c
};

// A thread's part of a row: the largest value, and the sums relative to m, which is
// at least that (the warp's largest at the start, so that few of a thread's later
// values move it); with MEAN, q too. NaN or +inf: top is.
template <typename T, bool MEAN>
struct RowPart {
  static constexpr int N = Vec<T>::N;
  static constexpr bool kFloor = MEAN && sizeof(T) == 2;
  float top = -INFINITY, m = -3.402823466e38f;
  uint64_t s = 0, q = 0;
  uint32_t floor = 0;
  template <int U>
  __device__ __forceinline__ static float top_of(const uint4 (&w)[U]) {
    if constexpr (sizeof(T) == 4) {
      float top = top_nan<T>(w[0]);
#pragma unroll
      for (int u = 1; u < U; ++u) top = max_nan(top, top_nan<T>(w[u]));
      return top;
    } else {
      __nv_bfloat162 m = *reinterpret_cast<const __nv_bfloat162*>(&w[0].x);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w[u]);
        m = __hmax2_nan(m, __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
      }
      return max_nan(__low2float(m), __high2float(m));
    }
  }
  // m before anything is added, by the whole warp; `first`: the thread's first value,
  // or -inf
  __device__ __forceinline__ void start(float first, const Scale& k) {
    m = fmaxf(value_of(__reduce_max_sync(0xffffffffu, key_of(first))), -3.402823466e38f);
    if (kFloor) floor = floor_below(m, k.reach);
  }
  template <int U>
  __device__ __forceinline__ void add(const uint4 (&w)[U], const Scale& k) {
    const float here = top_of(w);
    top = max_nan(top, here);
    if (!(here <= m)) {
      const float delta = fmaxf((m - here) * k.c, kLeast), f = exp2_of(delta);
      if (MEAN) q = ptx::mul_f32x2(both(f), ptx::fma_f32x2(both(delta), s, q));
      s = ptx::mul_f32x2(both(f), s);
      m = here;
      if (kFloor) floor = floor_below(m, k.reach);
    }
    if (!kFloor || has_floor(m))
      accumulate<kFloor>(w, k.c);
    else
      accumulate<false>(w, k.c);
  }
  template <bool FLOOR, int U>
  __device__ __forceinline__ void accumulate(const uint4 (&w)[U], float c) {
    const uint64_t cc = both(c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint64_t v[N / 2];
      differences<T>(FLOOR ? raised(w[u], floor) : w[u], m, v);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        uint64_t t = ptx::mul_f32x2(v[i], cc);
        if (MEAN && !FLOOR) t = bounded(t);
        const uint64_t e = exp2_pair(t);
        s = ptx::add_f32x2(s, e);
        if (MEAN) q = ptx::fma_f32x2(e, t, q);
      }
    }
  }
  // 0: nothing above -inf
  __device__ __forceinline__ uint32_t key() const { return top == -INFINITY ? 0u : key_of(top); }
};

// Which granules of [begin, end) of a row are a thread's: those inside the row go
// round robin, the first and last one, if they reach outside, are thread 0's and 1's.
struct Slice {
  int first, last;  // granules inside the row, from first up to last
  int head, tail;   // the others, -1: none
  template <typename T>
  __device__ __forceinline__ Slice(const RowSpan<T>& row, int begin, int end, int n) : first(begin), last(end), head(-1), tail(-1) {
    if (begin < end && row.edge(begin, n)) head = first++;
    if (first < last && row.edge(last - 1, n)) tail = --last;
  }
};

// The part of thread `rank` of G: U granules at a time.
template <typename T, int G, bool MEAN, int U, typename Get>
__device__ __forceinline__ RowPart<T, MEAN> sum_part(const RowSpan<T>& row, const Slice& at, int n, int rank,
                                                     const Scale& k, Get get) {
  RowPart<T, MEAN> part;
  int i = at.first + rank;
  const bool whole = i + (U - 1) * G < at.last;
  uint4 w[U];
  float first = -INFINITY;
  if (whole) {
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = get(i + u * G);
    first = RowPart<T, MEAN>::top_of(w);
  }
  part.start(first, k);
  if (whole) {
    part.add(w, k);
    for (i += U * G; i + (U - 1) * G < at.last; i += U * G) {
#pragma unroll
      for (int u = 0; u < U; ++u) w[u] = get(i + u * G);
      part.add(w, k);
    }
  }
  for (; i < at.last; i += G) {
    const uint4 one[1] = {get(i)};
    part.add(one, k);
  }
  const int edge = rank == 0 ? at.head : rank == 1 ? at.tail : -1;
  if (edge >= 0) {
    const uint4 one[1] = {masked_outside<T>(get(edge), row.first(edge), n)};
    part.add(one, k);
  }
  return part;
}

// What a group's warps leave for each other between barriers.
template <int G>
struct JoinShared {
  static constexpr int W = G / 32;
  uint32_t top[W];
  float s[W], q[W], own, again;
};

// The block's sums from its G threads', of which STRIDE have granules. Where the row is nearly sure, the sum of the
// thread that holds the maximum has lost the others' last bits beside it: its warp
// takes that thread's granules again. meanwhile(): what warps do besides, between the
// two barriers.
template <typename T, int G, int STRIDE, bool MEAN, typename Get, typename F>
__device__ __forceinline__ RowSums join_block(const RowPart<T, MEAN>& part, const RowSpan<T>& row, const Slice& at, int n,
                                              float c, Get get, JoinShared<G>& sh, F&& meanwhile) {
  constexpr int W = G / 32;
  constexpr uint32_t kAll = 0xffffffffu;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t key = part.key(), warp_key = __reduce_max_sync(kAll, key);
  if (lane == 0) sh.top[warp] = warp_key;
  __syncthreads();
  const uint32_t other = sh.top[lane % W], top = __reduce_max_sync(kAll, other);
  const int winner_warp = __ffs(__ballot_sync(kAll, other == top)) - 1;
  RowSums r;
  r.none = top == 0;
  r.m = r.none ? -INFINITY : top >= kNanKey ? NAN : value_of(top);
  const float delta = fmaxf((part.m - r.m) * c, kLeast), f = exp2_of(delta);
  float s = lo_f32(part.s) + hi_f32(part.s), q = 0.f;
  if (MEAN) q = s == 0.f ? 0.f : f * (lo_f32(part.q) + hi_f32(part.q) + delta * s);
  s = s == 0.f ? 0.f : f * s;
  int winner = -1;
  if (warp == winner_warp) {
    winner = __ffs(__ballot_sync(kAll, key == top)) - 1;
    if (lane == winner) {
      sh.own = s - 1.f;
      s = 0.f;
    }
  }
  s = warp_sum(s);
  if (MEAN) q = warp_sum(q);
  if (lane == 0) {
    sh.s[warp] = s;
    sh.q[warp] = q;
  }
  meanwhile();
  __syncthreads();
  s = sh.s[0];
  q = sh.q[0];
#pragma unroll
  for (int i = 1; i < W; ++i) {
    s += sh.s[i];
    if (MEAN) q += sh.q[i];
  }
  float own = sh.own;
  if (s + own < 0.0625f && !r.none) {  // (the same for the whole block)
    if (warp == winner_warp) {
      const int thread = warp * 32 + winner;
      float again = 0.f;
      auto take = [&](int i, bool edge) {
        uint4 w = get(i);
        if (edge) w = masked_outside<T>(w, row.first(i), n);
#pragma unroll
        for (int j = 0; j < Vec<T>::N; ++j) {
          const float z = Vec<T>::at(w, j);
          if (z < r.m) again += exp2_of((z - r.m) * c);
        }
      };
      for (int i = at.first + thread + lane * STRIDE; i < at.last; i += 32 * STRIDE) take(i, false);
      const int edge = thread == 0 ? at.head : thread == 1 ? at.tail : -1;
      if (lane == 0 && edge >= 0) take(edge, true);
      again = warp_sum(again);
      if (lane == 0) sh.again = again;
    }
    __syncthreads();
    own = sh.again;
  }
  r.others = s + own;
  r.q = q;
  return r;
}

// ---------------------------------------------------------------- rows on a few lanes
// A row on L lanes of a warp, all of it in their registers: U granules a lane, granule
// u L + lane. What lies outside the row is -inf.
template <typename T, int L, int U>
struct LaneRow {
  static constexpr int N = Vec<T>::N;
  uint4 w[U];
  __device__ __forceinline__ void load(const RowSpan<T>& row, int n, int lane, bool live) {
    const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
#pragma unroll
    for (int u = 0; u < U; ++u)
      w[u] = live && u * L + lane < row.count ? row.granules[u * L + lane] : uint4{none, none, none, none};
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * L + lane < row.count && row.edge(u * L + lane, n)) w[u] = masked_outside<T>(w[u], row.first(u * L + lane), n);
  }
  __device__ __forceinline__ float at(int u, int j) const { return Vec<T>::at(w[u], j); }
};
// Sum, and maximum of keys, over the L lanes.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
  if constexpr (L == 32) {
    return __reduce_max_sync(0xffffffffu, v);
  } else {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
  }
}
// Its sums, on all of its lanes; `mine`: the lane's own maximum's key.
template <typename T, int L, int U, bool MEAN>
__device__ __forceinline__ RowSums sum_lanes(const LaneRow<T, L, U>& row, int lane, float c, uint32_t& mine) {
  constexpr int N = Vec<T>::N;
  RowPart<T, MEAN> part;
  const float own = RowPart<T, MEAN>::top_of(row.w);
  mine = own == -INFINITY ? 0u : key_of(own);
  const uint32_t top = lanes_max<L>(mine);
  RowSums r;
  r.none = top == 0;
  r.m = r.none ? 0.f : top >= kNanKey ? NAN : value_of(top);
  part.m = r.m;
  part.template accumulate<false>(row.w, c);
  float s = lo_f32(part.s) + hi_f32(part.s), q = MEAN ? lo_f32(part.q) + hi_f32(part.q) : 0.f;
  const uint32_t holders = __ballot_sync(0xffffffffu, mine == top) >> (threadIdx.x & 31 & ~(L - 1));
  const bool holds = mine == top && !(holders & ((1u << lane) - 1));
  if (holds) s -= 1.f;
  r.others = lanes_sum<L>(s);
  if (__any_sync(0xffffffffu, r.others < 0.0625f && !r.none)) {
    // a nearly sure row: beside its maximum the lane's sum has lost the others' last bits
    float again = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float z = row.at(u, j);
        if (z < r.m) again += exp2_of((z - r.m) * c);
      }
    const float anew = lanes_sum<L>(holds ? again : s);
    if (r.others < 0.0625f) r.others = anew;
  }
  r.q = MEAN ? lanes_sum<L>(q) : 0.f;
  if (r.none) r.m = -INFINITY;
  return r;
}

}  // namespace ops
}  // namespace lc

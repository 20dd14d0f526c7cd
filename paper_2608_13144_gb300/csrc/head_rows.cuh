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
// What a group leaves for its threads between two barriers.
template <int G>
struct JoinShared {
  static constexpr int W = G / 32;
  uint32_t top[W];
  float s[W], q[W], own[W];
};

// Of a set of logits with t = (z - m) / T, in units of log 2: m its maximum,
// 1 + others the sum of exp2(t), q the sum of exp2(t) t (<= 0). One of the values
// that are m stands outside `others`, so that a sure row's logarithm is
// log1p(others) to its last bits. none: no value above -inf.
struct RowSums {
  float m, others, q;
  bool none;
};

// t of a pair: differences first, so that logits may stand at any offset.
__device__ __forceinline__ uint64_t shifted(uint64_t v, uint64_t minus_m, uint64_t c) {
  return ptx::mul_f32x2(ptx::add_f32x2(v, minus_m), c);
}
__device__ __forceinline__ uint64_t exp2_pair(uint64_t t) {
  return ptx::pack_f32x2(__float_as_uint(exp2_of(lo_f32(t))), __float_as_uint(exp2_of(hi_f32(t))));
}
// exp2 of anything from here down is 0; of -inf, too, but 0 * -inf is NaN.
constexpr float kLeast = -1000.f;
__device__ __forceinline__ uint64_t bounded(uint64_t t) {
  return ptx::pack_f32x2(__float_as_uint(fmaxf(lo_f32(t), kLeast)), __float_as_uint(fmaxf(hi_f32(t), kLeast)));
}

// A thread's part of a row: the running maximum (from the lowest finite value up),
// and the sums relative to it; with MEAN, q too. NaN or +inf: m is.
template <typename T, bool MEAN>
struct RowPart {
  static constexpr int N = Vec<T>::N;
  float m = -3.402823466e38f;
  uint64_t s = 0, q = 0;
  template <int U>
  __device__ __forceinline__ void add(const uint4 (&w)[U], float c) {
    float top = top_nan<T>(w[0]);
#pragma unroll
    for (int u = 1; u < U; ++u) top = max_nan(top, top_nan<T>(w[u]));
    top = max_nan(top, m);
    if (top != m) {
      const float delta = fmaxf((m - top) * c, kLeast);
      const uint64_t f = both(exp2_of(delta));
      if (MEAN) q = ptx::mul_f32x2(f, ptx::fma_f32x2(both(delta), s, q));
      s = ptx::mul_f32x2(f, s);
      m = top;
    }
    const uint64_t minus_m = both(-m), cc = both(c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint64_t v[N / 2];
      Vec<T>::open(w[u], v);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        uint64_t t = shifted(v[i], minus_m, cc);
        if (MEAN) t = bounded(t);
        const uint64_t e = exp2_pair(t);
        s = ptx::add_f32x2(s, e);
        if (MEAN) q = ptx::fma_f32x2(e, t, q);
      }
    }
  }
};

// The part of thread `rank` of G in granules [begin, end) of a row: U at a time.
template <typename T, int G, bool MEAN, int U, typename Get>
__device__ __forceinline__ RowPart<T, MEAN> sum_part(const RowSpan<T>& row, int begin, int end, int n, int rank, float c,
                                                     Get get) {
  RowPart<T, MEAN> part;
  const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  for (int i = begin + rank; i < end; i += U * G) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = i + u * G < end ? get(i + u * G) : uint4{none, none, none, none};
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * G < end && row.edge(i + u * G, n)) w[u] = masked_outside<T>(w[u], row.first(i + u * G), n);
    part.add(w, c);
  }
  return part;
}

// The group's sums from its threads'. Where the row is nearly sure, the sum of the
// thread that holds the maximum has lost the others' last bits beside it: its warp
// takes that thread's granules again.
template <typename T, int G, bool MEAN, typename Get>
__device__ __forceinline__ RowSums join_group(const RowPart<T, MEAN>& part, const RowSpan<T>& row, int begin, int end,
                                              int n, float c, Get get, JoinShared<G>& sh) {
  constexpr int W = G / 32;
  constexpr uint32_t kAll = 0xffffffffu;
  const int lane = threadIdx.x & 31, warp = G == 32 ? 0 : threadIdx.x >> 5;
  float s = lo_f32(part.s) + hi_f32(part.s), q = MEAN ? lo_f32(part.q) + hi_f32(part.q) : 0.f;
  // (a thread that saw nothing above -inf has s = 0; one that saw NaN may have)
  const uint32_t key = s == 0.f && part.m <= 3.402823466e38f ? 0u : key_of(part.m);
  const uint32_t warp_key = __reduce_max_sync(kAll, key);
  uint32_t top = warp_key;
  int winner_warp = 0;
  if (W > 1) {
    if (lane == 0) sh.top[warp] = warp_key;
    __syncthreads();
    const uint32_t other = sh.top[lane % W];
    top = __reduce_max_sync(kAll, other);
    winner_warp = __ffs(__ballot_sync(kAll, other == top)) - 1;
  }
  RowSums r;
  r.none = top == 0;
  r.m = r.none ? -INFINITY : value_of(top);
  if (top >= kNanKey) r.m = NAN;
  const float delta = fmaxf((part.m - r.m) * c, kLeast), f = exp2_of(delta);
  if (MEAN) q = s == 0.f ? 0.f : f * (q + delta * s);
  s = s == 0.f ? 0.f : f * s;
  const int winner = warp == winner_warp ? __ffs(__ballot_sync(kAll, key == top)) - 1 : -1;
  float own = 0.f;
  if (lane == winner) {
    own = s - 1.f;
    s = 0.f;
  }
  s = warp_sum(s);
  if (MEAN) q = warp_sum(q);
  if (winner >= 0) own = __shfl_sync(kAll, own, winner);
  if (W > 1) {
    if (lane == 0) {
      sh.s[warp] = s;
      sh.q[warp] = q;
      if (warp == winner_warp) sh.own[0] = own;
    }
    __syncthreads();
    s = warp_sum(lane < W ? sh.s[lane % W] : 0.f);
    if (MEAN) q = warp_sum(lane < W ? sh.q[lane % W] : 0.f);
    own = sh.own[0];
  }
  if (s + own < 0.0625f && !r.none) {  // (the same for the whole group)
    if (warp == winner_warp) {
      const int thread = warp * 32 + winner;
      float again = 0.f;
      for (int i = begin + thread + lane * G; i < end; i += 32 * G) {
        uint4 w = get(i);
        if (row.edge(i, n)) w = masked_outside<T>(w, row.first(i), n);
#pragma unroll
        for (int j = 0; j < Vec<T>::N; ++j) {
          const float z = Vec<T>::at(w, j);
          if (z < r.m) again += exp2_of((z - r.m) * c);
        }
      }
      own = warp_sum(again);
      if (W > 1 && lane == 0) sh.own[1] = own;
    }
    if (W > 1) {
      __syncthreads();
      own = sh.own[1];
    }
  }
  r.others = s + own;
  r.q = q;
  return r;
}

}  // namespace ops
}  // namespace lc

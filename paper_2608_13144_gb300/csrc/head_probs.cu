// What a head answers: of each row of logits the log-probability of a given class,
// the entropy, and the most probable classes, the logits read once; and the
// gradient of the log-probabilities and entropies.
//   t = (z - m) / T, m = max z;  log_sum = log sum exp t;  mean = -sum p t
//   logprob = t_y - log_sum;  entropy = log_sum + mean;  norm = (m, log_sum, mean)
//   dz_c = (g ([c = y] - p_c) - h p_c (t_c + mean)) / T
// All terms of the entropy are positive: nothing cancels.
//
// The k largest: of the G threads' own maxima (which the sums need anyway) one that
// at least k of them reach is found by halving; only threads that reach it hold
// values that count, so only their granules are read again (from L2), and the few
// values at or above it are ranked against each other by (value, lowest index).
#include "head_mma.cuh"
#include "head_rows.cuh"

namespace lc {
namespace ops {
namespace {

struct ProbArgs {
  int64_t ldz, tokens;
  int classes, k;
  float temperature, c;  // c = log2(e) / temperature
  const int32_t* target;
  float *logprob, *entropy, *norm, *top;
  int32_t* index;
};

constexpr float kLn2 = 0.6931471805599453f;

// ---------------------------------------------------------------- the k largest
template <int G>
struct SelectShared {
  static constexpr int kCap = G == 32 ? 128 : G == 128 ? 512 : 1024;
  uint32_t key[G];
  uint16_t live[G];
  uint32_t tau;
  int n_live, n;
  int total[G / 32];
  unsigned long long found[kCap];
};

// Sum over the group, on every thread.
template <int G>
__device__ __forceinline__ int group_count(int v, int (&total)[G / 32]) {
  v = __reduce_add_sync(0xffffffffu, v);
  if constexpr (G > 32) {
    __syncthreads();
    if ((threadIdx.x & 31) == 0) total[threadIdx.x >> 5] = v;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    v = __reduce_add_sync(0xffffffffu, lane < G / 32 ? total[lane] : 0);
  }
  return v;
}

// How many of a granule's values inside the row have a key of at least `tau`.
template <typename T>
__device__ __forceinline__ int count_from(const uint4& w, int first, int n, uint32_t tau) {
  int c = 0;
#pragma unroll
  for (int j = 0; j < Vec<T>::N; ++j) c += first + j >= 0 && first + j < n && key_of(Vec<T>::at(w, j)) >= tau;
  return c;
}

// The group's k largest unmasked values in granules [begin, end) of a row without
// NaN or +inf, to emit(rank, key, index), each rank from one thread; returns how
// many there are (at most k). `mine`: the key of this thread's own maximum, 0 if it
// holds none.
template <typename T, int G, typename Get, typename Emit>
__device__ __forceinline__ int select_largest(const RowSpan<T>& row, int begin, int end, int n, int k, uint32_t mine,
                                              Get get, SelectShared<G>& sh, Emit emit) {
  constexpr uint32_t kAll = 0xffffffffu;
  constexpr int N = Vec<T>::N, R = G / 32, kCap = SelectShared<G>::kCap;
  const int rank = group_rank<G>(), lane = threadIdx.x & 31;
  sh.key[rank] = mine;
  group_sync<G>();
  if (G == 32 || threadIdx.x < 32) {
    uint32_t v[R];
    uint32_t high = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      v[i] = sh.key[i * 32 + lane];
      high = max(high, v[i]);
    }
    // [lo, hi): k threads or more reach lo (or it is the lowest there is), fewer hi
    uint32_t lo = kUnmasked, hi = __reduce_max_sync(kAll, high) + 1;
    while (hi > lo + 1) {
      const uint32_t mid = lo + (hi - lo) / 2;
      int c = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) c += v[i] >= mid;
      c = __reduce_add_sync(kAll, c);
      if (c >= k) {
        lo = mid;
        if (c <= k + k / 4 + 4) break;
      } else {
        hi = mid;
      }
    }
    int live = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint32_t b = __ballot_sync(kAll, v[i] >= lo);
      if (v[i] >= lo) sh.live[live + __popc(b & ((1u << lane) - 1))] = (uint16_t)(i * 32 + lane);
      live += __popc(b);
    }
    if (lane == 0) {
      sh.tau = lo;
      sh.n_live = live;
      sh.n = 0;
    }
  }
  group_sync<G>();
  const uint32_t tau = sh.tau;
  const int live = sh.n_live;
  auto collect = [&](int granule, uint32_t from) {
    const uint4 w = get(granule);
    const int first = row.first(granule);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t key = key_of(Vec<T>::at(w, j));
      if (key >= from && first + j >= 0 && first + j < n) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < kCap) sh.found[at] = (unsigned long long)key << 32 | (uint32_t)~(first + j);
      }
    }
  };
  if (live > 0) {
    const int rounds = (end - begin + G - 1) / G;
    for (int i = rank; i < rounds * live; i += G) {
      const int granule = begin + i / live * G + sh.live[i % live];
      if (granule < end) collect(granule, tau);
    }
  }
  group_sync<G>();
  int found = sh.n, ties = 0;
  uint32_t equal = 0;
  if (found > kCap) {
    // Many equal values, or large ones crowded into few threads: halve over the whole
    // row until the values from lo up fit, or those above lo are fewer than k and the
    // rest of the k are ties at lo.
    uint32_t lo = tau, hi = 0xff800000u;
    int at_lo = found;
    while (hi > lo + 1 && at_lo > kCap) {
      const uint32_t mid = lo + (hi - lo) / 2;
      int c = 0;
      for (int i = begin + rank; i < end; i += G) c += count_from<T>(get(i), row.first(i), n, mid);
      c = group_count<G>(c, sh.total);
      if (c >= k) {
        lo = mid;
        at_lo = c;
      } else {
        hi = mid;
      }
    }
    const bool tied = at_lo > kCap;
    group_sync<G>();
    if (rank == 0) sh.n = 0;
    group_sync<G>();
    for (int i = begin + rank; i < end; i += G) collect(i, tied ? lo + 1 : lo);
    group_sync<G>();
    found = sh.n;
    if (tied) {
      equal = lo;
      ties = k - found;
    }
  }
  for (int i = rank; i < found; i += G) {
    const unsigned long long own = sh.found[i];
    int r = 0;
    for (int j = 0; j < found; ++j) r += sh.found[j] > own;
    if (r < k) emit(r, (uint32_t)(own >> 32), (int)~(uint32_t)own);
  }
  // ties in the order of their indices
  for (int i = begin, done = 0; done < ties && i < end; i += G) {
    const int granule = i + rank;
    uint4 w{};
    int c = 0;
    if (granule < end) {
      w = get(granule);
      const int first = row.first(granule);
#pragma unroll
      for (int j = 0; j < N; ++j) c += first + j >= 0 && first + j < n && key_of(Vec<T>::at(w, j)) == equal;
    }
    int before = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(kAll, before, o);
      if (lane >= o) before += v;
    }
    int all = __shfl_sync(kAll, before, 31);
    before -= c;
    if constexpr (G > 32) {
      group_sync<G>();
      if (lane == 0) sh.total[threadIdx.x >> 5] = all;
      group_sync<G>();
      const int t = lane < G / 32 ? sh.total[lane] : 0;
      before += __reduce_add_sync(kAll, lane < (int)(threadIdx.x >> 5) ? t : 0);
      all = __reduce_add_sync(kAll, t);
    }
    if (c) {
      const int first = row.first(granule);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (first + j >= 0 && first + j < n && key_of(Vec<T>::at(w, j)) == equal) {
          if (done + before < ties) emit(found + done + before, equal, first + j);
          ++before;
        }
    }
    done += all;
  }
  return min(found + ties, k);
}

// ---------------------------------------------------------------- log-probabilities
// What a row's sums say, and its outputs of one value.
struct RowSays {
  float m, log_sum;
  bool bad;
};
__device__ __forceinline__ RowSays write_row(const ProbArgs& a, int64_t row, const RowSums& r, float zy, bool write) {
  const bool bad = isnan(r.m);
  const float total = 1.f + r.others;
  float log_sum = r.none ? 0.f : log1pf(r.others), mean = r.none ? 0.f : -kLn2 * r.q / total;
  if (bad) log_sum = mean = NAN;
  if (write) {
    if (a.norm) {
      float* o = a.norm + 3 * row;
      o[0] = r.m;
      o[1] = log_sum;
      o[2] = mean;
    }
    if (a.entropy) a.entropy[row] = log_sum + mean;
    if (a.logprob) {
      const int y = a.target[row];
      const bool live = y >= 0 && y < a.classes;
      const float lp = r.none || zy == -INFINITY ? -INFINITY : (zy - r.m) / a.temperature - log_sum;
      a.logprob[row] = !live ? 0.f : bad ? NAN : lp;
    }
  }
  return RowSays{r.m, log_sum, bad};
}
__device__ __forceinline__ void put_top(const ProbArgs& a, int64_t row, const RowSays& says, int r, uint32_t key, int i) {
  a.top[row * a.k + r] = (value_of(key) - says.m) / a.temperature - says.log_sum;
  a.index[row * a.k + r] = i;
}
// places that no class fills
__device__ __forceinline__ void fill_top(const ProbArgs& a, int64_t row, int from, float with, int rank, int G) {
  for (int i = from + rank; i < a.k; i += G) {
    a.top[row * a.k + i] = with;
    a.index[row * a.k + i] = -1;
  }
}

// G threads a row: 32, of which a block holds four rows, or a block.
template <typename T, int G>
__global__ void __launch_bounds__(G == 32 ? 128 : G) k_probs(const T* z, const ProbArgs a) {
  constexpr int kRows = G == 32 ? 4 : 1;
  __shared__ SelectShared<G> select_s[kRows];
  __shared__ JoinShared<G> join_s[kRows];
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int slot = G == 32 ? threadIdx.x >> 5 : 0, rank = group_rank<G>();
  const int64_t t = (int64_t)blockIdx.x * kRows + slot;
  if (t >= a.tokens) return;
  const T* zr = z + t * a.ldz;
  const RowSpan<T> row(zr, a.classes);
  auto get = [&](int i) { return row.granules[i]; };
  float zy = 0.f;
  if (a.logprob && rank == 0) {
    const int y = a.target[t];
    if (y >= 0 && y < a.classes) zy = to_f32<T>(zr[y]);
  }
  const auto part = sum_part<T, G, true, 4>(row, 0, row.count, a.classes, rank, a.c, get);
  const RowSums sums = join_group<T, G, true>(part, row, 0, row.count, a.classes, a.c, get, join_s[slot]);
  const RowSays says = write_row(a, t, sums, zy, rank == 0);
  if (a.k == 0) return;
  int have = 0;
  if (!says.bad && !sums.none) {
    const uint32_t mine = part.s == 0 ? 0u : key_of(part.m);
    have = select_largest<T, G>(row, 0, row.count, a.classes, a.k, mine, get, select_s[slot],
                                [&](int r, uint32_t key, int i) { put_top(a, t, says, r, key, i); });
  }
  fill_top(a, t, have, says.bad ? NAN : -INFINITY, rank, G);
}

template <typename T>
void launch_probs(const T* z, const ProbArgs& a, cudaStream_t s) {
  const int granules = (int)ceil_div(a.classes, Vec<T>::N) + 1;
  if (granules <= 257 && a.k <= 32)
    launch_pdl(k_probs<T, 32>, dim3((unsigned)ceil_div(a.tokens, 4)), 128, s, z, a);
  else if (granules <= 2048)
    launch_pdl(k_probs<T, 128>, dim3((unsigned)a.tokens), 128, s, z, a);
  else
    launch_pdl(k_probs<T, 512>, dim3((unsigned)a.tokens), 512, s, z, a);
  LC_LAUNCH_CHECK("k_probs");
}

// ---------------------------------------------------------------- their gradient
struct ProbGradArgs {
  int64_t ldz, ldd, tokens;
  int classes, parts;  // parts: warps a row
  float temperature, c;
  const float *norm, *dlogprob, *dentropy;
  const int32_t* target;
};
constexpr int kGradVecs = 4;  // granules a lane takes

// A warp takes 32 kGradVecs granules of a row. With t in units of log 2:
// dz = exp2(t) (alpha + beta t), alpha = -(g + h mean) / (T sum), beta = -h ln 2 /
// (T sum); the target's own 1 - p is -expm1(logprob), without cancellation.
template <typename T>
__global__ void __launch_bounds__(256) k_probs_grad(const T* z, T* dz, const ProbGradArgs a) {
  constexpr int N = Vec<T>::N;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int64_t t = item / a.parts;
  if (t >= a.tokens) return;
  const int part = (int)(item - t * a.parts), lane = threadIdx.x & 31;
  const T* zr = z + t * a.ldz;
  T* dr = dz + t * a.ldd;
  const RowSpan<T> row(zr, a.classes);
  const int y = a.target ? __ldg(a.target + t) : -1;
  const bool live = y >= 0 && y < a.classes;
  const float g = live && a.dlogprob ? __ldg(a.dlogprob + t) : 0.f, h = a.dentropy ? __ldg(a.dentropy + t) : 0.f;
  const float m = __ldg(a.norm + 3 * t), log_sum = __ldg(a.norm + 3 * t + 1), mean = __ldg(a.norm + 3 * t + 2);
  const bool zero = (g == 0.f && h == 0.f) || m == -INFINITY;
  const float scale = exp2_of(-log_sum * kLog2e) / a.temperature;
  const uint64_t alpha = both(-(g + h * mean) * scale), beta = both(-h * kLn2 * scale);
  const uint64_t minus_m = both(-m), c = both(a.c);
  const bool same = (((uintptr_t)dr ^ (uintptr_t)zr) & 15) == 0;
  uint4 w[kGradVecs];
  const int from = part * 32 * kGradVecs + lane;
#pragma unroll
  for (int u = 0; u < kGradVecs; ++u)
    if (!zero && from + u * 32 < row.count) w[u] = row.granules[from + u * 32];
#pragma unroll
  for (int u = 0; u < kGradVecs; ++u) {
    const int i = from + u * 32, first = row.first(i);
    if (i >= row.count) break;
    uint64_t v[N / 2];
    if (zero) {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) v[j] = 0;
    } else {
      Vec<T>::open(w[u], v);
      float at_y = 0.f;
      if ((uint32_t)(y - first) < (uint32_t)N) {
        const float ty = (Vec<T>::at(w[u], y - first) - m) / a.temperature, p = __expf(ty - log_sum);
        at_y = (-g * expm1f(ty - log_sum) - (h == 0.f || p == 0.f ? 0.f : h * p * (ty + mean))) / a.temperature;
      }
#pragma unroll
      for (int j = 0; j < N / 2; ++j) {
        const uint64_t x = bounded(shifted(v[j], minus_m, c));
        v[j] = ptx::mul_f32x2(exp2_pair(x), ptx::fma_f32x2(beta, x, alpha));
      }
      if ((uint32_t)(y - first) < (uint32_t)N) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (first + j == y)
            v[j / 2] = j & 1 ? (v[j / 2] & 0xffffffffull) | ((uint64_t)__float_as_uint(at_y) << 32)
                             : (v[j / 2] & ~0xffffffffull) | __float_as_uint(at_y);
      }
      if (isnan(m)) {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) v[j] = both(NAN);
      }
    }
    put_granule<T>(dr, same, Vec<T>::close(v), first, a.classes);
  }
}

template <typename T>
void launch_probs_grad(const T* z, T* dz, ProbGradArgs a, cudaStream_t s) {
  const int granules = (int)ceil_div(a.classes, Vec<T>::N) + (a.ldz % Vec<T>::N || ((uintptr_t)z & 15) ? 1 : 0);
  a.parts = (int)ceil_div(granules, 32 * kGradVecs);
  launch_pdl(k_probs_grad<T>, dim3((unsigned)ceil_div(a.tokens * a.parts, 8)), 256, s, z, dz, a);
  LC_LAUNCH_CHECK("k_probs_grad");
}

}  // namespace

void log_probs(int type, const void* z, int64_t ldz, int64_t tokens, int classes, const int32_t* target, int k,
               double temperature, float* logprob, float* entropy, float* norm, float* top, int32_t* index,
               cudaStream_t s) {
  const ProbArgs a{ldz, tokens, classes, k, (float)temperature, (float)(1.4426950408889634 / temperature),
                   target, logprob, entropy, norm, top, index};
  if (type == LIPCACHE_F32)
    launch_probs(static_cast<const float*>(z), a, s);
  else
    launch_probs(static_cast<const __nv_bfloat16*>(z), a, s);
}

void log_probs_backward(int type, const void* z, int64_t ldz, int64_t tokens, int classes, const float* norm,
                        const int32_t* target, const float* dlogprob, const float* dentropy, double temperature,
                        void* dz, int64_t ldd, cudaStream_t s) {
  const ProbGradArgs a{ldz, ldd, tokens, classes, 0, (float)temperature, (float)(1.4426950408889634 / temperature),
                       norm, dlogprob, dentropy, target};
  if (type == LIPCACHE_F32)
    launch_probs_grad(static_cast<const float*>(z), static_cast<float*>(dz), a, s);
  else
    launch_probs_grad(static_cast<const __nv_bfloat16*>(z), static_cast<__nv_bfloat16*>(dz), a, s);
}

}  // namespace ops
}  // namespace lc

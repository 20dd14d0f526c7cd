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
//
// Measured: 4,096 x 50,001 BF16 88 us with 20 classes, 67 without (6.1 TB/s, near the
// memory's rate: the classes cost a block 2 us of barriers, threshold and second
// reading in which it loads nothing; rings of asynchronous copies across rows, 134 us,
// and batches loaded ahead, 109 us, cost more instructions than they hide; 512 threads
// a row 116 us). 65,536 x 200 FP32 with 5 classes 22 us, bound by instructions (306 a
// row, 77 % of the issue slots) and by the call from Python (17 us). One row 3 us of the
// GPU's time, of 50,001 BF16 classes 8. The gradient of 4,096 x 50,001 BF16 130 us, 6.3 TB/s. (Below, where launches
// are compared: times a launch in a graph, 2 to 4 us more.)
#include "head_mma.cuh"
#include "head_rows.cuh"

namespace lc {
namespace ops {
namespace {

struct ProbArgs {
  int64_t ldz, tokens;
  int classes, k;
  float temperature, c, reach;  // c = log2(e) / temperature, reach = 500 / c
  const int32_t* target;
  float *logprob, *entropy, *norm, *top;
  int32_t* index;
};

constexpr float kLn2 = 0.6931471805599453f;
using ops::key_of;

// ---------------------------------------------------------------- the k largest
// A candidate: a value's key, and below it the complement of its index, so that the
// larger candidate stands first.
using Found = unsigned long long;
__device__ __forceinline__ Found candidate(uint32_t key, int index) { return (Found)key << 32 | (uint32_t)~index; }
__device__ __forceinline__ uint32_t key_of(Found f) { return (uint32_t)(f >> 32); }
__device__ __forceinline__ int index_of(Found f) { return (int)~(uint32_t)f; }

// G threads, a warp or a block, whose maxima say where the k largest are.
template <int G>
struct SelectShared {
  static constexpr int kCap = G == 32 ? 128 : 4 * G;
  uint32_t key[G];
  uint16_t live[G];
  uint32_t tau;
  int n_live, n;
  int total[G / 32];
  __align__(16) Found found[kCap];
};

// One warp: tau, a key that at least k of the threads' maxima reach (or the lowest
// there is), and which threads reach it.
template <int G>
__device__ __forceinline__ void find_threshold(SelectShared<G>& sh, int k) {
  constexpr uint32_t kAll = 0xffffffffu;
  constexpr int R = G / 32;
  const int lane = threadIdx.x & 31;
  uint32_t v[R], high = 0, low = kAll;
  int some = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) {
    v[i] = sh.key[i * 32 + lane];
    high = max(high, v[i]);
    if (v[i]) low = min(low, v[i]), ++some;
  }
  some = __reduce_add_sync(kAll, some);
  uint32_t lo = kUnmasked;
  if (some >= k) {
    // [lo, hi): k maxima or more reach lo, fewer hi
    lo = __reduce_min_sync(kAll, low);
    uint32_t hi = __reduce_max_sync(kAll, high) + 1;
    const int enough = k + k / 4 + 4;
    while (some > enough && hi > lo + 1) {
      const uint32_t mid = lo + (hi - lo) / 2;
      int c = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) c += v[i] >= mid;
      c = __reduce_add_sync(kAll, c);
      if (c >= k) {
        lo = mid;
        some = c;
      } else {
        hi = mid;
      }
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

// Which of a granule's values reach `least`: a bit each.
template <typename T>
struct Reach;
template <>
struct Reach<float> {
  float least;
  __device__ __forceinline__ explicit Reach(float least) : least(least) {}
  __device__ __forceinline__ uint32_t of(const uint4& w) const {
    return (__uint_as_float(w.x) >= least ? 1u : 0u) | (__uint_as_float(w.y) >= least ? 2u : 0u) |
           (__uint_as_float(w.z) >= least ? 4u : 0u) | (__uint_as_float(w.w) >= least ? 8u : 0u);
  }
  __device__ __forceinline__ int index(int bit) const { return bit; }
  __device__ __forceinline__ float value(const uint4& w, int j) const {
    return __uint_as_float(j & 2 ? (j & 1 ? w.w : w.z) : (j & 1 ? w.y : w.x));
  }
};
template <>
struct Reach<__nv_bfloat16> {
  __nv_bfloat162 least;  // rounded up
  __device__ __forceinline__ explicit Reach(float x) {
    const uint32_t bits = __float_as_uint(x), up = (bits >> 31 ? bits : bits + 0xffffu) >> 16, two = up | up << 16;
    least = *reinterpret_cast<const __nv_bfloat162*>(&two);
  }
  __device__ __forceinline__ uint32_t of(const uint4& w) const {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w);
    return (__hge2_mask(h[0], least) & 0x00010001u) | (__hge2_mask(h[1], least) & 0x00020002u) |
           (__hge2_mask(h[2], least) & 0x00040004u) | (__hge2_mask(h[3], least) & 0x00080008u);
  }
  __device__ __forceinline__ int index(int bit) const { return bit < 16 ? 2 * bit : 2 * (bit - 16) + 1; }
  __device__ __forceinline__ float value(const uint4& w, int j) const {
    const uint32_t x = j & 4 ? (j & 2 ? w.w : w.z) : (j & 2 ? w.y : w.x);
    return __uint_as_float(j & 1 ? x & 0xffff0000u : x << 16);
  }
};

// The group's k largest unmasked values in granules [begin, end) of a row without
// NaN or +inf, after find_threshold and a barrier, to emit(rank, candidate), each rank
// from one thread; returns how many there are (at most k). m: the largest of them.
template <typename T, int G, typename Get, typename Emit>
__device__ __forceinline__ int select_largest(const RowSpan<T>& row, const Slice& at, int begin, int end, int n, int k,
                                              float m, Get get, SelectShared<G>& sh, Emit emit) {
  constexpr uint32_t kAll = 0xffffffffu;
  constexpr int N = Vec<T>::N, kCap = SelectShared<G>::kCap;
  const int rank = group_rank<G>(), lane = threadIdx.x & 31, warp = G == 32 ? 0 : threadIdx.x >> 5;
  auto keep = [&](float z, int index) {
    const int to = atomicAdd(&sh.n, 1);
    if (to < kCap) sh.found[to] = candidate(key_of(z), index);
  };
  auto collect = [&](int granule, uint32_t from) {
    const uint4 w = get(granule);
    const int first = row.first(granule);
    const float least = value_of(from);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float z = Vec<T>::at(w, j);
      if (z >= least && first + j >= 0 && first + j < n) keep(z, first + j);
    }
  };
  // a warp reads a live thread's granules, all inside the row; those at the row's
  // ends are read by all
  const int live = sh.n_live;
  const uint32_t tau = sh.tau;
  const Reach<T> reach(value_of(tau));
  // Of as many threads at a time as their granules fill lanes (a power of two each), Q
  // such loads before what comes of them.
  constexpr int W = G / 32, Q = 4;
  const int rounds = (at.last - at.first + G - 1) / G, bits = rounds > 16 ? 5 : rounds > 1 ? 32 - __clz(rounds - 1) : 0;
  const int each = 32 >> bits, mine = (warp << (5 - bits)) + (lane >> bits), nth = lane & ((1 << bits) - 1);
  for (int base = at.first; base < at.last; base += 32 * G)
    for (int l = mine; l - (lane >> bits) < live; l += Q * W * each) {
      uint4 w[Q];
      int i[Q];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int of = l + q * W * each;
        i[q] = of < live ? base + sh.live[of] + nth * G : at.last;
        if (i[q] < at.last) w[q] = get(i[q]);
      }
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if (i[q] >= at.last) continue;
        for (uint32_t hits = reach.of(w[q]); hits; hits &= hits - 1) {
          const int j = reach.index(__ffs(hits) - 1);
          keep(reach.value(w[q], j), row.first(i[q]) + j);
        }
      }
    }
  if (rank == 0 && at.head >= 0) collect(at.head, tau);
  if (rank == 1 && at.tail >= 0) collect(at.tail, tau);
  group_sync<G>();
  int found = sh.n, ties = 0;
  uint32_t equal = 0;
  if (found > kCap) {
    // Many equal values, or large ones crowded into few threads: halve over the whole
    // row until the values from lo up fit, or those above lo are fewer than k and the
    // rest of the k are ties at lo.
    uint32_t lo = tau, hi = ops::key_of(m) + 1;
    int from_lo = found;
    auto count = [&](int i, uint32_t from) {
      const uint4 w = get(i);
      const int first = row.first(i);
      int c = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) c += first + j >= 0 && first + j < n && key_of(Vec<T>::at(w, j)) >= from;
      return c;
    };
    while (hi > lo + 1 && from_lo > kCap) {
      const uint32_t mid = lo + (hi - lo) / 2;
      int c = 0;
      for (int i = begin + rank; i < end; i += G) c += count(i, mid);
      c = group_count<G>(c, sh.total);
      if (c >= k) {
        lo = mid;
        from_lo = c;
      } else {
        hi = mid;
      }
    }
    const bool tied = from_lo > kCap;
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
  if ((found & 1) && found < kCap) {  // (an even number: they are read in pairs)
    if (rank == 0) sh.found[found] = 0;
    if (G == 32 || found < 32)
      __syncwarp();
    else
      __syncthreads();
  }
  for (int i = rank; i < found; i += G) {
    const Found own = sh.found[i];
    int r = 0;
    for (int j = 0; j < found; j += 2) {
      const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(sh.found + j);
      r += (two.x > own) + (two.y > own);
    }
    if (r < k) emit(r, own);
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
      if (lane == 0) sh.total[warp] = all;
      group_sync<G>();
      const int t = lane < G / 32 ? sh.total[lane] : 0;
      before += __reduce_add_sync(kAll, lane < warp ? t : 0);
      all = __reduce_add_sync(kAll, t);
    }
    if (c) {
      const int first = row.first(granule);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (first + j >= 0 && first + j < n && key_of(Vec<T>::at(w, j)) == equal) {
          if (done + before < ties) emit(found + done + before, candidate(equal, first + j));
          ++before;
        }
    }
    done += all;
  }
  return min(found + ties, k);
}

// ---------------------------------------------------------------- log-probabilities
// What a row's sums say.
struct RowSays {
  float m, log_sum, mean;
  bool bad, none;
  __device__ __forceinline__ explicit RowSays(const RowSums& r) {
    m = r.m;
    none = r.none;
    bad = isnan(r.m);
    log_sum = bad ? NAN : none ? 0.f : log1pf(r.others);
    mean = bad ? NAN : none ? 0.f : __fdividef(-kLn2 * r.q, 1.f + r.others);
  }
  // log p of a value
  __device__ __forceinline__ float log_p(const ProbArgs& a, float z) const {
    return z == -INFINITY ? -INFINITY : (z - m) / a.temperature - log_sum;
  }
};
// The row's outputs of one value; zy: the target's logit.
__device__ __forceinline__ void put_row(const ProbArgs& a, int64_t row, const RowSays& says, int y, float zy) {
  if (a.norm) {
    float* o = a.norm + 3 * row;
    o[0] = says.m;
    o[1] = says.log_sum;
    o[2] = says.mean;
  }
  if (a.entropy) a.entropy[row] = says.log_sum + says.mean;
  if (a.logprob) a.logprob[row] = y < 0 || y >= a.classes ? 0.f : says.bad ? NAN : says.none ? -INFINITY : says.log_p(a, zy);
}
__device__ __forceinline__ void put_top(const ProbArgs& a, int64_t row, const RowSays& says, int r, Found f) {
  a.top[row * a.k + r] = says.log_p(a, value_of(key_of(f)));
  a.index[row * a.k + r] = index_of(f);
}
// places that no class fills
__device__ __forceinline__ void fill_top(const ProbArgs& a, int64_t row, int from, bool bad, int rank, int G) {
  for (int i = from + rank; i < a.k; i += G) {
    a.top[row * a.k + i] = bad ? NAN : -INFINITY;
    a.index[row * a.k + i] = -1;
  }
}

// Small rows: L lanes each, all of a row in registers. The k-th of the lanes' sorted
// maxima is the threshold; what reaches it is ranked as in select_largest, which also
// takes the rows of which too much does. k <= L.
template <typename T, int L, int U>
__global__ void __launch_bounds__(128, 8) k_probs_lanes(const T* z, const ProbArgs a) {
  constexpr int N = Vec<T>::N, kRows = 32 / L, kCap = L == 32 ? 128 : 64;
  constexpr uint32_t kAll = 0xffffffffu;
  __shared__ Found found_s[4 * kRows][kCap];
  __shared__ SelectShared<32> select_s[4];
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int warp = threadIdx.x >> 5, slot = (threadIdx.x & 31) / L, lane = threadIdx.x & (L - 1);
  const int64_t base = ((int64_t)blockIdx.x * 4 + warp) * kRows, t = base + slot;
  const bool live = t < a.tokens;
  const RowSpan<T> row(z + (live ? t : 0) * a.ldz, a.classes);
  LaneRow<T, L, U> r;
  r.load(row, a.classes, lane, live);
  int y = -1;
  float zy = 0.f;
  if (live && lane == 0 && a.logprob) {
    y = __ldg(a.target + t);
    if (y >= 0 && y < a.classes) zy = to_f32<T>(z[t * a.ldz + y]);
  }
  uint32_t mine;
  const RowSums sums = sum_lanes<T, L, U, true>(r, lane, a.c, mine);
  const RowSays says(sums);
  if (live && lane == 0) put_row(a, t, says, y, zy);
  if (a.k == 0) return;
  // the lanes' maxima in falling order
  uint32_t v = mine;
#pragma unroll
  for (int size = 2; size <= L; size <<= 1)
#pragma unroll
    for (int step = size / 2; step > 0; step >>= 1) {
      const uint32_t other = __shfl_xor_sync(kAll, v, step);
      v = ((lane & step) == 0) == ((lane & size) == 0) ? max(v, other) : min(v, other);
    }
  const float least = value_of(max(__shfl_sync(kAll, v, slot * L + a.k - 1), kUnmasked));
  const bool select = live && !says.bad && !says.none;
  int count = 0;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int j = 0; j < N; ++j) count += r.at(u, j) >= least;
  int to = count;
#pragma unroll
  for (int o = 1; o < L; o <<= 1) {
    const int p = __shfl_up_sync(kAll, to, o);
    if (lane >= o) to += p;
  }
  int all = __shfl_sync(kAll, to, slot * L + L - 1);
  if (!select) all = 0;
  Found* found = found_s[warp * kRows + slot];
  to -= count;
  if (count && all && all <= kCap) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float x = r.at(u, j);
        if (x >= least) found[to++] = candidate(key_of(x), row.first(u * L + lane) + j);
      }
  }
  __syncwarp();
  if (live && all <= kCap) {
    for (int i = lane; i < all; i += L) {
      const Found own = found[i];
      int before = 0;
      for (int j = 0; j < all; ++j) before += found[j] > own;
      if (before < a.k) put_top(a, t, says, before, own);
    }
    fill_top(a, t, min(all, a.k), says.bad, lane, L);
  }
  // rows with too many: the whole warp, one after another
  for (uint32_t over = __ballot_sync(kAll, all > kCap); over;) {
    const int from = __ffs(over) - 1;
    const int64_t tt = base + from / L;
    over &= L == 32 ? 0u : ~(((1u << (L & 31)) - 1) << from);
    const RowSpan<T> wide(z + tt * a.ldz, a.classes);
    auto get = [&](int i) { return wide.granules[i]; };
    const Slice at(wide, 0, wide.count, a.classes);
    uint32_t key = 0;
    for (int i = at.first + (int)(threadIdx.x & 31); i < at.last; i += 32) {
      const float top = top_nan<T>(get(i));
      if (top > -INFINITY) key = max(key, ops::key_of(top));
    }
    __syncwarp();
    select_s[warp].key[threadIdx.x & 31] = key;
    __syncwarp();
    find_threshold<32>(select_s[warp], a.k);
    __syncwarp();
    RowSays other = says;
    other.m = __shfl_sync(kAll, says.m, from);
    other.log_sum = __shfl_sync(kAll, says.log_sum, from);
    const int have = select_largest<T, 32>(wide, at, 0, wide.count, a.classes, a.k, other.m, get, select_s[warp],
                                           [&](int r, Found f) { put_top(a, tt, other, r, f); });
    fill_top(a, tt, have, false, threadIdx.x & 31, 32);
    __syncwarp();
  }
}

// Large rows: a block of G threads each, or a cluster of CL blocks that split it.
template <typename T, int G, int CL>
__global__ void __launch_bounds__(G, (CL > 1 ? 768 : 1536) / G) k_probs(const T* z, const ProbArgs a) {
  __shared__ SelectShared<G> select;
  __shared__ JoinShared<G> join;
  __shared__ RowSums part_s;
  __shared__ int have_s;
  static_assert(CL * LIPCACHE_MAX_TOP <= SelectShared<G>::kCap || CL == 1, "a cluster's candidates side by side");
  __shared__ Found best_s[CL > 1 ? LIPCACHE_MAX_TOP : 1];
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int64_t t = blockIdx.x / CL;
  const int block = CL > 1 ? (int)ptx::cluster_ctarank() : 0, rank = threadIdx.x;
  const T* zr = z + t * a.ldz;
  const RowSpan<T> row(zr, a.classes);
  const int share = (row.count + CL - 1) / CL, begin = min(block * share, row.count), end = min(begin + share, row.count);
  const Slice at(row, begin, end, a.classes);
  auto get = [&](int i) { return row.granules[i]; };
  int y = -1;
  float zy = 0.f;
  if (a.logprob && rank == 0 && block == 0) {
    y = __ldg(a.target + t);
    if (y >= 0 && y < a.classes) zy = to_f32<T>(zr[y]);
  }
  const auto part = sum_part<T, G, true, 4>(row, at, a.classes, rank, Scale{a.c, a.reach}, get);
  select.key[rank] = part.key();
  RowSums sums = join_block<T, G, G, true>(part, row, at, a.classes, a.c, get, join, [&] {
    if (rank < 32 && a.k) find_threshold<G>(select, a.k);
  });
  if constexpr (CL == 1) {
    if (rank == 0) put_row(a, t, RowSays(sums), y, zy);
    if (a.k == 0) return;
    int have = 0;
    const bool bad = isnan(sums.m);
    if (!bad && !sums.none)
      have = select_largest<T, G>(row, at, begin, end, a.classes, a.k, sums.m, get, select,
                                  [&](int r, Found f) { put_top(a, t, RowSays(sums), r, f); });
    if (have < a.k) fill_top(a, t, have, bad, rank, G);
  } else {
    // each block's best, which the first one ranks against each other
    int have = 0;
    if (a.k && !isnan(sums.m) && !sums.none)
      have = select_largest<T, G>(row, at, begin, end, a.classes, a.k, sums.m, get, select,
                                  [&](int r, Found f) { best_s[r] = f; });
    if (rank == 0) {
      part_s = sums;
      have_s = have;
    }
    ptx::cluster_sync();
    if (block == 0) {
      auto far = [](const void* p, int b) { return ptx::mapa(ptx::smem_u32(p), b); };
      auto load = [](uint32_t p) {
        uint32_t v;
        asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(p) : "memory");
        return v;
      };
      RowSums of[CL];
      int n[CL], all = 0;
      uint32_t top = 0;
#pragma unroll
      for (int b = 0; b < CL; ++b) {
        of[b].m = __uint_as_float(load(far(&part_s.m, b)));
        of[b].others = __uint_as_float(load(far(&part_s.others, b)));
        of[b].q = __uint_as_float(load(far(&part_s.q, b)));
        n[b] = (int)load(far(&have_s, b));
        all += n[b];
        of[b].none = of[b].m == -INFINITY;
        top = max(top, of[b].none ? 0u : isnan(of[b].m) ? kNanKey : ops::key_of(of[b].m));
      }
      sums.none = top == 0;
      sums.m = sums.none ? -INFINITY : top >= kNanKey ? NAN : value_of(top);
      sums.others = sums.q = 0.f;
      bool out = false;  // one block's maximum stands outside the others
#pragma unroll
      for (int b = 0; b < CL; ++b) {
        if (of[b].none) continue;
        const float delta = fmaxf((of[b].m - sums.m) * a.c, kLeast), f = exp2_of(delta);
        const bool own = !out && of[b].m == sums.m;
        out = out || own;
        sums.others += f * (own ? of[b].others : 1.f + of[b].others);
        sums.q += f * (of[b].q + delta * (1.f + of[b].others));
      }
      const RowSays says(sums);
      if (rank == 0) put_row(a, t, says, y, zy);
      if (says.bad) all = 0;
      // the blocks' lists side by side, each in falling order
      if (all) {
#pragma unroll
        for (int b = 0; b < CL; ++b)
          for (int i = rank; i < n[b]; i += G) {
            Found f;
            asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(f) : "r"(far(best_s + i, b)) : "memory");
            select.found[b * LIPCACHE_MAX_TOP + i] = f;
          }
        __syncthreads();
        for (int i = rank; i < CL * a.k; i += G) {
          const int b = i / a.k, j = i - b * a.k;
          int count = 0;
#pragma unroll
          for (int o = 0; o < CL; ++o)
            if (o == b) count = n[o];
          if (j >= count) continue;
          const Found own = select.found[b * LIPCACHE_MAX_TOP + j];
          int r = j;
#pragma unroll
          for (int o = 0; o < CL; ++o) {
            if (o == b) continue;
            int lo = 0, hi = n[o];  // of the other list, those above
            while (lo < hi) {
              const int mid = (lo + hi) / 2;
              if (select.found[o * LIPCACHE_MAX_TOP + mid] > own)
                lo = mid + 1;
              else
                hi = mid;
            }
            r += lo;
          }
          if (r < a.k) put_top(a, t, says, r, own);
        }
      }
      if (a.k) fill_top(a, t, min(all, a.k), says.bad, rank, G);
    }
    ptx::cluster_sync();  // (until the first one has read)
  }
}

template <typename T, int L, int U>
void launch_lanes(const T* z, const ProbArgs& a, cudaStream_t s) {
  launch_pdl(k_probs_lanes<T, L, U>, dim3((unsigned)ceil_div(a.tokens, 4 * (32 / L))), 128, s, z, a);
}
template <typename T, int L>
bool probs_lanes(const T* z, const ProbArgs& a, int granules, cudaStream_t s) {
  constexpr int kMost = sizeof(T) == 4 ? 8 : 4;  // 32 values a lane
  // (with k near L the least of the lanes' maxima would be the threshold, which half the row may reach)
  if (granules > L * kMost || 4 * a.k > 3 * L) return false;
  if (granules <= L)
    launch_lanes<T, L, 1>(z, a, s);
  else if (granules <= 2 * L)
    launch_lanes<T, L, 2>(z, a, s);
  else if (granules <= 4 * L)
    launch_lanes<T, L, 4>(z, a, s);
  else
    launch_lanes<T, L, kMost>(z, a, s);
  return true;
}

template <typename T, int G, int CL>
void launch_blocks(const T* z, const ProbArgs& a, cudaStream_t s) {
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CL;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.tokens * CL));
  cfg.blockDim = dim3(G);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 2 : 1;
  LC_CUDA(cudaLaunchKernelEx(&cfg, k_probs<T, G, CL>, z, a));
}

template <typename T>
void launch_probs(const T* z, const ProbArgs& a, cudaStream_t s) {
  // granules of a row, one more where rows start inside one
  const int granules = (int)ceil_div(a.classes, Vec<T>::N) + (a.ldz % Vec<T>::N || ((uintptr_t)z & 15) ? 1 : 0);
  // Lanes while 32 values each hold the row (FP32, 65,536 x 200 with 5 classes 25 us, a
  // block of 128 a row 195; 16,384 x 1,000 with 20 29 and 78) and maxima of theirs tell the
  // classes asked for (65,536 x 200 with 24 classes 74 us, with 25, in blocks, 147). Beyond, a block a row, of
  // so many threads that their sums and ranking do not outweigh the row (BF16, 20 classes:
  // 8,192 x 3,000 30 us with 64, 37 with 128, 60 with 256; x 16,000 83, 68 and 82; 4,096 x
  // 50,001 155, 117 and 90), but twice as many as classes are asked for, or the threshold
  // would let too much through. Few long rows a cluster (one row of 150,000 classes 14 us,
  // 16 in a block, of 400,000 16 and 29; 38 rows of 150,000 15 and 16, 60 rows 18 and 17, 80
  // rows 26 and 17).
  if (probs_lanes<T, 8>(z, a, granules, s) || probs_lanes<T, 16>(z, a, granules, s) ||
      probs_lanes<T, 32>(z, a, granules, s))
    ;
  else if (granules >= 16384 && 8 * a.tokens <= 2 * mma::num_sms())
    launch_blocks<T, 256, 8>(z, a, s);
  else if (granules <= 1024 && a.k <= 32)
    launch_blocks<T, 64, 1>(z, a, s);
  else if (granules <= 4096 && a.k <= 64)
    launch_blocks<T, 128, 1>(z, a, s);
  else
    launch_blocks<T, 256, 1>(z, a, s);
  LC_LAUNCH_CHECK("k_probs");
}

// ---------------------------------------------------------------- their gradient
struct ProbGradArgs {
  int64_t ldz, ldd, tokens;
  int classes;
  float temperature, c, reach;
  const float *norm, *dlogprob, *dentropy;
  const int32_t* target;
};
// A row's gradient. With t in units of log 2: dz = exp2(t) (alpha + beta t), alpha =
// -(g + h mean) / (T sum), beta = -h ln 2 / (T sum); at the target's class 1 - p is
// -expm1(logprob), without cancellation.
template <typename T>
struct ProbGradient {
  static constexpr int N = Vec<T>::N;
  float g, h, m, log_sum, mean;
  uint64_t alpha, beta, c;
  uint32_t floor;
  int y;  // the target, kNone: none (far before any row)
  static constexpr int kNone = -(1 << 30);
  bool zero, raise, nan;
  __device__ __forceinline__ ProbGradient(const ProbGradArgs& a, int64_t t) : c(both(a.c)) {
    y = a.target ? __ldg(a.target + t) : kNone;
    if (y < 0 || y >= a.classes) y = kNone;
    g = y >= 0 && a.dlogprob ? __ldg(a.dlogprob + t) : 0.f;
    h = a.dentropy ? __ldg(a.dentropy + t) : 0.f;
    m = __ldg(a.norm + 3 * t);
    log_sum = __ldg(a.norm + 3 * t + 1);
    mean = __ldg(a.norm + 3 * t + 2);
    if (g == 0.f) y = kNone;  // (its gradient is like the others')
    zero = (g == 0.f && h == 0.f) || m == -INFINITY;
    nan = isnan(m);
    const float scale = exp2_of(-log_sum * kLog2e) / a.temperature;
    alpha = both(-(g + h * mean) * scale);
    beta = both(-h * kLn2 * scale);
    raise = sizeof(T) == 2 && has_floor(m);
    floor = floor_below(m, a.reach);
  }
  template <bool RAISE>
  __device__ __forceinline__ uint4 of(const uint4& w) const {
    uint64_t v[N / 2];
    differences<T>(RAISE ? raised(w, floor) : w, m, v);
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      uint64_t x = ptx::mul_f32x2(v[j], c);
      if (!RAISE) x = bounded(x);
      v[j] = ptx::mul_f32x2(exp2_pair(x), ptx::fma_f32x2(beta, x, alpha));
    }
    return Vec<T>::close(v);
  }
  // where the row's gradient is the same value everywhere
  __device__ __forceinline__ uint4 filled() const {
    uint64_t v[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) v[j] = both(zero ? 0.f : NAN);
    return Vec<T>::close(v);
  }
  __device__ __forceinline__ T at_target(const ProbGradArgs& a, float zy) const {
    const float ty = (zy - m) / a.temperature, p = __expf(ty - log_sum);
    const float d = -g * expm1f(ty - log_sum) - (h == 0.f || p == 0.f ? 0.f : h * p * (ty + mean));
    return from_f32<T>(d / a.temperature);
  }
};

// L lanes a row, or a part of one (blockIdx.y of them, of `share` granules): U
// granules a lane, all loaded before any is written, which may be to the same array.
template <typename T, int L, int U>
__global__ void __launch_bounds__(128, 8) k_probs_grad(const T* z, T* dz, const ProbGradArgs a, int share) {
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int lane = threadIdx.x & (L - 1);
  const int64_t t = (int64_t)blockIdx.x * (128 / L) + threadIdx.x / L;
  if (t >= a.tokens) return;
  const T* zr = z + t * a.ldz;
  T* dr = dz + t * a.ldd;
  const RowSpan<T> row(zr, a.classes);
  const int from = blockIdx.y * share + lane, end = min((int)(blockIdx.y + 1) * share, row.count);
  uint4 w[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (from + u * L < end) w[u] = row.granules[from + u * L];
  const ProbGradient<T> gradient(a, t);
  const bool same = (((uintptr_t)dr ^ (uintptr_t)zr) & 15) == 0;
  auto write = [&](auto value) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (from + u * L < end) put_granule<T>(dr, same, value(w[u]), row.first(from + u * L), a.classes);
  };
  if (gradient.zero || gradient.nan) {
    write([&](const uint4&) { return gradient.filled(); });
    return;
  }
  if (sizeof(T) == 2 && gradient.raise)
    write([&](const uint4& x) { return gradient.template of<sizeof(T) == 2>(x); });
  else
    write([&](const uint4& x) { return gradient.template of<false>(x); });
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int at = gradient.y - row.first(from + u * L);
    if (from + u * L < end && (uint32_t)at < (uint32_t)Vec<T>::N) dr[gradient.y] = gradient.at_target(a, Vec<T>::at(w[u], at));
  }
}

template <typename T, int L, int U>
void launch_grad(const T* z, T* dz, const ProbGradArgs& a, int granules, cudaStream_t s) {
  const int parts = (int)ceil_div(granules, L * U);
  const dim3 grid((unsigned)ceil_div(a.tokens, 128 / L), (unsigned)parts);
  launch_pdl(k_probs_grad<T, L, U>, grid, 128, s, z, dz, a, (int)ceil_div(granules, parts));
}

template <typename T>
void launch_probs_grad(const T* z, T* dz, const ProbGradArgs& a, cudaStream_t s) {
  const int granules = (int)ceil_div(a.classes, Vec<T>::N) + (a.ldz % Vec<T>::N || ((uintptr_t)z & 15) ? 1 : 0);
  // (four granules a lane: 4,096 x 50,001 BF16 133 us, eight 144; at most 2^24 / 4 / 128 parts)
  if (granules <= 8)
    launch_grad<T, 8, 1>(z, dz, a, granules, s);
  else if (granules <= 32)
    launch_grad<T, 8, 4>(z, dz, a, granules, s);
  else if (granules <= 64)
    launch_grad<T, 16, 4>(z, dz, a, granules, s);
  else
    launch_grad<T, 32, 4>(z, dz, a, granules, s);
  LC_LAUNCH_CHECK("k_probs_grad");
}

}  // namespace

void log_probs(int type, const void* z, int64_t ldz, int64_t tokens, int classes, const int32_t* target, int k,
               double temperature, float* logprob, float* entropy, float* norm, float* top, int32_t* index,
               cudaStream_t s) {
  const ProbArgs a{ldz, tokens, classes, k, (float)temperature, (float)(1.4426950408889634 / temperature),
                   (float)(500.0 / 1.4426950408889634 * temperature), target, logprob, entropy, norm, top, index};
  if (type == LIPCACHE_F32)
    launch_probs(static_cast<const float*>(z), a, s);
  else
    launch_probs(static_cast<const __nv_bfloat16*>(z), a, s);
}

void log_probs_backward(int type, const void* z, int64_t ldz, int64_t tokens, int classes, const float* norm,
                        const int32_t* target, const float* dlogprob, const float* dentropy, double temperature,
                        void* dz, int64_t ldd, cudaStream_t s) {
  const ProbGradArgs a{ldz, ldd, tokens, classes, (float)temperature, (float)(1.4426950408889634 / temperature),
                       (float)(500.0 / 1.4426950408889634 * temperature), norm, dlogprob, dentropy, target};
  if (type == LIPCACHE_F32)
    launch_probs_grad(static_cast<const float*>(z), static_cast<float*>(dz), a, s);
  else
    launch_probs_grad(static_cast<const __nv_bfloat16*>(z), static_cast<__nv_bfloat16*>(dz), a, s);
}

}  // namespace ops
}  // namespace lc

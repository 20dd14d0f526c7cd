// Distillation of rows of logits from a teacher's most probable classes, with the
// gradient in the same call:
//   q = softmax of the teacher's values / T over the classes it names,
//   loss = w T^2 sum_j q_j (log q_j - log p_j),  dz = w T (p - q)
// A row's sums first, then its values again for the gradient: small rows wait in the
// registers of a few lanes, larger ones in shared memory (of a cluster where one
// block's does not hold them), the largest are read twice. The gradient is written as
// w T p everywhere, and at the teacher's classes once more.
//
// Measured: 4,096 x 50,001 BF16 from 64 classes 144 us, 5.7 TB/s (read and written
// once; two blocks an SM, whose loads, sums and stores alternate; a teacher's warp
// beside the others: 175 us while the first of them had it as well). 65,536 x 200 FP32
// from 10 classes 25 us, 4.4 TB/s, bound by instructions (309 a row, 71 % of the issue
// slots). (Below, where launches are compared: times a launch in a graph, 2 to 4 us more.)
#include "head_mma.cuh"
#include "head_rows.cuh"

namespace lc {
namespace ops {
namespace {

struct DistillArgs {
  int64_t ldz, ldd, tokens;
  int classes, k;
  float temperature, c;
  const float* top;
  const int32_t* index;
  const float* weight;
  float* loss;
};

constexpr uint32_t kAll = 0xffffffffu;

// The teacher's answers of one row on L lanes, entry L i + lane in a lane's
// registers. rest: the sum of the shares of other classes than the entry's; same: of
// its own; first: no entry before it names its class.
template <int L, int R>
struct Teacher {
  int index[R];
  float q[R], log_q[R], same[R], rest[R];
  bool first[R], bad, any;

  __device__ __forceinline__ void load(const DistillArgs& a, int64_t row, int lane, bool live) {
    float v[R], best = -INFINITY;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int j = L * i + lane;
      index[i] = -1;
      v[i] = -INFINITY;
      if (j < a.k && live) {
        index[i] = __ldg(a.index + row * a.k + j);
        const float x = __ldg(a.top + row * a.k + j);
        if (index[i] < 0 || index[i] >= a.classes)
          index[i] = -1;
        else
          v[i] = x;
      }
      best = max_nan(best, v[i]);
    }
    const uint32_t top = lanes_max<L>(key_of(best));
    any = top >= kUnmasked;
    bad = top >= kNanKey;
    best = any && !bad ? value_of(top) : 0.f;
    // the largest stands outside the sum: a sure teacher's logarithms keep their bits
    const int base = threadIdx.x & 31 & ~(L - 1);
    float others = 0.f;
    bool out = false, own[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      q[i] = 0.f, own[i] = false, log_q[i] = -INFINITY;
      if (i > 0 && L * i >= a.k) continue;
      const uint32_t b = (__ballot_sync(kAll, v[i] == best) >> base) & (L == 32 ? kAll : (1u << (L & 31)) - 1);
      own[i] = !out && b && __ffs(b) - 1 == lane;
      out = out || b;
      log_q[i] = (v[i] - best) / a.temperature;
      q[i] = v[i] == -INFINITY ? 0.f : expf(log_q[i]);
      if (!own[i]) others += q[i];
    }
    others = lanes_sum<L>(others);
    const float log_sum = log1pf(others), over = 1.f / (1.f + others);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      log_q[i] -= log_sum;
      q[i] *= over;
      same[i] = q[i];
      rest[i] = own[i] ? others * over : 1.f - q[i];
      first[i] = index[i] >= 0;
    }
  }
  // Where a class may be named twice.
  __device__ __forceinline__ void join_same(int k, int lane) {
    const int base = threadIdx.x & 31 & ~(L - 1);
#pragma unroll
    for (int i = 0; i < R; ++i) same[i] = rest[i] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
      for (int l = 0; l < L && L * i + l < k; ++l) {
        const int other = __shfl_sync(kAll, index[i], base + l);
        const float share = __shfl_sync(kAll, q[i], base + l);
#pragma unroll
        for (int e = 0; e < R; ++e) {
          const bool mine = other == index[e];
          same[e] += mine ? share : 0.f;
          rest[e] += mine ? 0.f : share;
          if (mine && L * i + l < L * e + lane) first[e] = false;
        }
      }
  }
  // This lane's part of the divergence; at: what the gradient is at the entries'
  // classes; zj: their logits.
  __device__ __forceinline__ float divergence(const DistillArgs& a, const RowSums& sums, float w, const float (&zj)[R],
                                              float (&at)[R]) const {
    const float log_sum = log1pf(sums.others);
    float loss = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (i > 0 && L * i >= a.k) continue;
      const float lp = sums.none || zj[i] == -INFINITY ? -INFINITY : (zj[i] - sums.m) / a.temperature - log_sum;
      if (q[i] > 0.f) loss += q[i] * (log_q[i] - lp);
      // p - q; where both are near 1, the difference of what they leave to others
      const float p = exp2_of(lp * kLog2e);
      at[i] = w * a.temperature * (p > 0.5f && same[i] > 0.5f ? rest[i] + expm1f(lp) : p - same[i]);
    }
    return loss;
  }
};

// The gradient w T p of a row's granules.
struct RowGradient {
  float m;
  uint64_t c, factor;
  __device__ __forceinline__ RowGradient(const DistillArgs& a, const RowSums& sums, float w)
      : m(sums.m), c(both(a.c)), factor(both(w * a.temperature / (1.f + sums.others))) {}
  template <typename T>
  __device__ __forceinline__ uint4 of(const uint4& w) const {
    constexpr int N = Vec<T>::N;
    uint64_t v[N / 2];
    differences<T>(w, m, v);
#pragma unroll
    for (int j = 0; j < N / 2; ++j) v[j] = ptx::mul_f32x2(exp2_pair(ptx::mul_f32x2(v[j], c)), factor);
    return Vec<T>::close(v);
  }
};
// A granule of `fill` (0 or NaN).
template <typename T>
__device__ __forceinline__ uint4 granule_of(float fill) {
  uint64_t v[Vec<T>::N / 2];
#pragma unroll
  for (int j = 0; j < Vec<T>::N / 2; ++j) v[j] = both(fill);
  return Vec<T>::close(v);
}

// Small rows: L lanes each, U granules a lane, up to 2 L classes of the teacher.
template <typename T, int L, int U>
__global__ void __launch_bounds__(128, 8) k_distill_lanes(const T* z, T* dz, const DistillArgs a) {
  constexpr int kRows = 32 / L, R = 2;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int lane = threadIdx.x & (L - 1);
  const int64_t t = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 5)) * kRows + (threadIdx.x & 31) / L;
  const bool is = t < a.tokens;
  const T* zr = z + (is ? t : 0) * a.ldz;
  const RowSpan<T> row(zr, a.classes);
  LaneRow<T, L, U> r;
  r.load(row, a.classes, lane, is);
  const float w = !is ? 0.f : a.weight ? __ldg(a.weight + t) : 1.f;
  Teacher<L, R> teacher;
  teacher.load(a, t, lane, is);
  float zj[R], at[R];
#pragma unroll
  for (int i = 0; i < R; ++i) zj[i] = teacher.index[i] >= 0 ? to_f32<T>(zr[teacher.index[i]]) : 0.f;
  teacher.join_same(a.k, lane);
  uint32_t mine;
  const RowSums sums = sum_lanes<T, L, U, false>(r, lane, a.c, mine);
  const bool taught = teacher.any && w != 0.f, bad = taught && (teacher.bad || isnan(sums.m));
  float loss = lanes_sum<L>(teacher.divergence(a, sums, w, zj, at));
  loss = bad ? NAN : taught ? w * a.temperature * a.temperature * loss : 0.f;
  if (is && a.loss && lane == 0) a.loss[t] = loss;
  if (!dz) return;
  T* dr = dz + t * a.ldd;
  const bool live = taught && !bad && !sums.none, same_place = (((uintptr_t)dr ^ (uintptr_t)zr) & 15) == 0;
  const RowGradient gradient(a, sums, w);
  if (is) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * L + lane < row.count)
        put_granule<T>(dr, same_place, live ? gradient.of<T>(r.w[u]) : granule_of<T>(bad ? NAN : 0.f),
                       row.first(u * L + lane), a.classes);
  }
  __syncwarp();  // (the row's lanes have written what is written over here)
#pragma unroll
  for (int i = 0; i < R; ++i)
    if (live && teacher.first[i]) dr[teacher.index[i]] = from_f32<T>(at[i]);
}

// Larger rows: a block of G threads each, or a cluster of CL blocks that split it. The
// last warp has the teacher, the S others the row's granules. RESIDENT: a thread copies
// its granules (16 at most) to shared memory, four at a time, and reads them there
// twice.
template <typename T, int G, int CL, bool RESIDENT>
__global__ void __launch_bounds__(G, RESIDENT && G == 512 ? 2 : 1) k_distill(const T* z, T* dz, const DistillArgs a) {
  constexpr int R = LIPCACHE_MAX_TOP / 32, U = 4, S = G - 32;
  extern __shared__ uint4 row_s[];
  __shared__ JoinShared<G> join;
  __shared__ int index_s[LIPCACHE_MAX_TOP], live_s, twice_s;
  __shared__ float2 part_s;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int rank = threadIdx.x, lane = rank & 31, block = CL > 1 ? (int)ptx::cluster_ctarank() : 0;
  const bool teaching = rank >= S;
  const int64_t t = blockIdx.x / CL;
  const T* zr = z + t * a.ldz;
  T* dr = dz ? dz + t * a.ldd : nullptr;
  const RowSpan<T> row(zr, a.classes);
  const int share = (row.count + CL - 1) / CL, begin = min(block * share, row.count), end = min(begin + share, row.count);
  const Slice at(row, begin, end, a.classes);
  auto get = [&](int i) { return row.granules[i]; };
  const float w = a.weight ? __ldg(a.weight + t) : 1.f;
  const Scale k{a.c, 0.f};
  Teacher<32, R> teacher;
  float zj[R], grad[R];
  // the sums of any row: which have a teacher the other warps know from the join on
  RowPart<T, false> part;
  if (teaching) {
    teacher.load(a, t, lane, true);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      zj[i] = teacher.index[i] >= 0 ? to_f32<T>(zr[teacher.index[i]]) : 0.f;
      if (32 * i + lane < a.k) index_s[32 * i + lane] = teacher.index[i];
    }
    if (lane == 0) {
      live_s = w == 0.f || !teacher.any ? 0 : teacher.bad ? 2 : 1;
      twice_s = 0;
    }
  } else {
    if constexpr (RESIDENT) {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = at.first + (b * U + u) * S + rank;
          if (i < at.last) {
            const uint32_t to = ptx::smem_u32(row_s + (i - begin));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row.granules + i) : "memory");
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (b == 0) asm volatile("cp.async.wait_group 3;" ::: "memory");
        if (b == 1) asm volatile("cp.async.wait_group 2;" ::: "memory");
        if (b == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        if (b == 3) asm volatile("cp.async.wait_group 0;" ::: "memory");
        int i = at.first + b * U * S + rank;
        const bool whole = i + (U - 1) * S < at.last;
        uint4 x[U];
        if (whole) {
#pragma unroll
          for (int u = 0; u < U; ++u) x[u] = row_s[i + u * S - begin];
        }
        if (b == 0) part.start(whole ? part.top_of(x) : -INFINITY, k);
        if (whole) {
          part.add(x, k);
        } else {
          for (; i < at.last && i < at.first + (b + 1) * U * S; i += S) {
            const uint4 one[1] = {row_s[i - begin]};
            part.add(one, k);
          }
        }
      }
      const int edge = rank == 0 ? at.head : rank == 1 ? at.tail : -1;
      if (edge >= 0) {
        const uint4 one[1] = {masked_outside<T>(get(edge), row.first(edge), a.classes)};
        part.add(one, k);
      }
    } else {
      part = sum_part<T, S, false, U>(row, at, a.classes, rank, k, get);
    }
  }
  RowSums sums = join_block<T, G, S, false>(part, row, at, a.classes, a.c, get, join, [&] {
    // whether a class is named twice: four threads an entry
    for (int e = rank; e < 4 * a.k; e += G) {
      const int entry = e >> 2, mine = index_s[entry];
      if (mine >= 0)
        for (int j = e & 3; j < entry; j += 4)
          if (index_s[j] == mine) twice_s = 1;
    }
  });
  int live = live_s;  // 1: a row with a teacher, 2: its results are NaN
  if constexpr (CL > 1) {
    if (rank == 0) part_s = float2{sums.m, sums.others};
    ptx::cluster_sync();
    if (live == 1) {
      float m[CL], others[CL];
      uint32_t top = 0;
#pragma unroll
      for (int b = 0; b < CL; ++b) {
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];"
                     : "=f"(m[b]), "=f"(others[b])
                     : "r"(ptx::mapa(ptx::smem_u32(&part_s), b))
                     : "memory");
        top = max(top, m[b] == -INFINITY ? 0u : isnan(m[b]) ? kNanKey : key_of(m[b]));
      }
      sums.none = top == 0;
      sums.m = sums.none ? -INFINITY : top >= kNanKey ? NAN : value_of(top);
      sums.others = 0.f;
      bool out = false;  // one block's maximum stands outside the others
#pragma unroll
      for (int b = 0; b < CL; ++b) {
        if (m[b] == -INFINITY) continue;
        const bool own = !out && m[b] == sums.m;
        out = out || own;
        sums.others += exp2_of(fmaxf((m[b] - sums.m) * a.c, kLeast)) * (own ? others[b] : 1.f + others[b]);
      }
    }
  }
  if (live == 1 && isnan(sums.m)) live = 2;
  if (teaching) {
    float loss = live == 2 ? NAN : 0.f;
    if (live == 1) {
      if (twice_s) teacher.join_same(a.k, lane);
      loss = w * a.temperature * a.temperature * warp_sum(teacher.divergence(a, sums, w, zj, grad));
    }
    if (a.loss && lane == 0 && block == 0) a.loss[t] = loss;
  }
  if (live == 1 && sums.none) live = 0;  // masked whole
  if (dr) {
    if (!teaching) {
      const RowGradient gradient(a, sums, w);
      const uint4 fill = granule_of<T>(live == 2 ? NAN : 0.f);
      const bool same = (((uintptr_t)dr ^ (uintptr_t)zr) & 15) == 0;
      if (live == 1 && same) {
        uint4* out = reinterpret_cast<uint4*>(dr + row.first(at.first));
        const int n = at.last - at.first;
        for (int i = rank; i < n; i += U * S) {
          // (loads of a batch before its stores, which may be to the same array)
          uint4 x[U];
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (i + u * S < n) x[u] = RESIDENT ? row_s[at.first - begin + i + u * S] : get(at.first + i + u * S);
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (i + u * S < n) out[i + u * S] = gradient.of<T>(x[u]);
        }
      } else {
        for (int i = at.first + rank; i < at.last; i += S) {
          const uint4 x = RESIDENT ? row_s[i - begin] : get(i);
          put_granule<T>(dr, same, live == 1 ? gradient.of<T>(x) : fill, row.first(i), a.classes);
        }
      }
      const int edge = rank == 0 ? at.head : rank == 1 ? at.tail : -1;
      if (edge >= 0) put_granule<T>(dr, same, live == 1 ? gradient.of<T>(get(edge)) : fill, row.first(edge), a.classes);
    }
    __syncthreads();
    // (each block those of its own classes)
    const int low = row.first(begin), high = row.first(end);
    if (teaching && live == 1) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (teacher.first[i] && teacher.index[i] >= low && teacher.index[i] < high) dr[teacher.index[i]] = from_f32<T>(grad[i]);
    }
  }
  if (CL > 1) ptx::cluster_sync();  // (until all have read part_s)
}

template <typename T, int L>
bool distill_lanes(const T* z, T* dz, const DistillArgs& a, int granules, cudaStream_t s) {
  constexpr int kMost = sizeof(T) == 4 ? 8 : 4;  // 32 values a lane
  if (granules > L * kMost || a.k > 2 * L) return false;
  const dim3 grid((unsigned)ceil_div(a.tokens, 4 * (32 / L)));
  if (granules <= L)
    launch_pdl(k_distill_lanes<T, L, 1>, grid, 128, s, z, dz, a);
  else if (granules <= 2 * L)
    launch_pdl(k_distill_lanes<T, L, 2>, grid, 128, s, z, dz, a);
  else if (granules <= 4 * L)
    launch_pdl(k_distill_lanes<T, L, 4>, grid, 128, s, z, dz, a);
  else
    launch_pdl(k_distill_lanes<T, L, kMost>, grid, 128, s, z, dz, a);
  return true;
}

constexpr int kResidentBytes = 111 * 1024;  // twice on an SM, beside what is static
static_assert(16 * 480 * 16 > kResidentBytes, "a thread holds 16 granules");

template <typename T, int G, int CL, bool RESIDENT>
void launch_blocks(const T* z, T* dz, const DistillArgs& a, int granules, cudaStream_t s) {
  const auto kernel = k_distill<T, G, CL, RESIDENT>;
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
  cfg.dynamicSmemBytes = RESIDENT ? (size_t)ceil_div(granules, CL) * 16 : 0;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = CL > 1 ? 2 : 1;
  if (cfg.dynamicSmemBytes > 40 * 1024) allow_smem(reinterpret_cast<const void*>(kernel), kResidentBytes);
  LC_CUDA(cudaLaunchKernelEx(&cfg, kernel, z, dz, a));
}

template <typename T>
void launch_distill(const T* z, T* dz, const DistillArgs& a, cudaStream_t s) {
  const int granules = (int)ceil_div(a.classes, Vec<T>::N) + (a.ldz % Vec<T>::N || ((uintptr_t)z & 15) ? 1 : 0);
  constexpr int kMost = kResidentBytes / 16;
  // Lanes while 32 values each hold the row and two entries each the teacher (FP32, 65,536 x
  // 200 from 10 classes 29 us, a block of 160 a row 316; from 64 135, from 65, in blocks of
  // 96, 299). Beyond, a block a row of about as many threads as keep 16 granules each (8,192 x
  // 3,000 BF16 31 us with 96, 44 with 160, 104 with 512; x 16,000 89 with 160, 146 with
  // 512), a cluster where one block's shared memory does not hold the row, or where rows
  // are few (BF16, 8 of 50,001 classes 8 to 10 us, 10 in a block each, 32 10 and 10, 64 16
  // and 10; of 20,001 8.8 and 7.5).
  if (distill_lanes<T, 8>(z, dz, a, granules, s) || distill_lanes<T, 16>(z, dz, a, granules, s) ||
      distill_lanes<T, 32>(z, dz, a, granules, s))
    ;
  else if (granules <= 1024)
    launch_blocks<T, 96, 1, true>(z, dz, a, granules, s);
  else if (granules <= 2048)
    launch_blocks<T, 160, 1, true>(z, dz, a, granules, s);
  else if (granules <= 4096 || (granules <= kMost && a.tokens > 32))
    launch_blocks<T, 512, 1, true>(z, dz, a, granules, s);
  else if (granules <= 4 * kMost && a.tokens > 32)
    launch_blocks<T, 512, 4, true>(z, dz, a, granules, s);
  else if (granules <= 8 * kMost)
    launch_blocks<T, 512, 8, true>(z, dz, a, granules, s);
  else
    launch_blocks<T, 512, 8, false>(z, dz, a, granules, s);
  LC_LAUNCH_CHECK("k_distill");
}

}  // namespace

void distill(int type, const void* z, int64_t ldz, int64_t tokens, int classes, int k, const float* top,
             const int32_t* index, const float* weight, double temperature, float* loss, void* dz, int64_t ldd,
             cudaStream_t s) {
  const DistillArgs a{ldz, ldd, tokens, classes, k, (float)temperature, (float)(1.4426950408889634 / temperature),
                      top, index, weight, loss};
  if (type == LIPCACHE_F32)
    launch_distill(static_cast<const float*>(z), static_cast<float*>(dz), a, s);
  else
    launch_distill(static_cast<const __nv_bfloat16*>(z), static_cast<__nv_bfloat16*>(dz), a, s);
}

}  // namespace ops
}  // namespace lc

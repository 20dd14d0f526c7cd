// Distillation of rows of logits from a teacher's most probable classes, with the
// gradient in the same call:
//   q = softmax of the teacher's values / T over the classes it names,
//   loss = w T^2 sum_j q_j (log q_j - log p_j),  dz = w T (p - q)
// A row's sums first, then its values again for the gradient: from shared memory
// where a block has the row in it, else from the caches. The gradient is written as
// w T p everywhere, and at the teacher's classes once more.
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

constexpr int kMostTop = LIPCACHE_MAX_TOP;
constexpr int kTopRegs = kMostTop / 32;

// The teacher's answers of one row, entry 32 i + lane in a warp's registers. rest:
// the sum of the shares of other classes than the entry's; same: of its own class;
// first: no entry before it names its class.
struct Teacher {
  int index[kTopRegs];
  float q[kTopRegs], log_q[kTopRegs], same[kTopRegs], rest[kTopRegs];
  bool first[kTopRegs], bad, any;

  __device__ __forceinline__ void load(const DistillArgs& a, int64_t row, int lane) {
    constexpr uint32_t kAll = 0xffffffffu;
    float v[kTopRegs];
    float best = -INFINITY;
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i) {
      const int j = 32 * i + lane;
      index[i] = -1;
      v[i] = -INFINITY;
      if (j < a.k) {
        index[i] = a.index[row * a.k + j];
        if (index[i] < 0 || index[i] >= a.classes) index[i] = -1;
        if (index[i] >= 0) v[i] = a.top[row * a.k + j];
      }
      best = max_nan(best, v[i]);
    }
    const uint32_t top = __reduce_max_sync(kAll, key_of(best));
    any = top >= kUnmasked;
    bad = top >= kNanKey;
    if (!any || bad) return;
    best = value_of(top);
    // the largest stands outside the sum: a sure teacher's logarithms keep their bits
    float others = 0.f;
    bool out = false;
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i) {
      const uint32_t b = __ballot_sync(kAll, v[i] == best);
      const bool own = !out && b && (__ffs(b) - 1) == lane;
      out = out || b;
      log_q[i] = (v[i] - best) / a.temperature;
      q[i] = v[i] == -INFINITY ? 0.f : expf(log_q[i]);
      if (!own) others += q[i];
    }
    others = warp_sum(others);
    const float log_sum = log1pf(others);
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i) {
      log_q[i] -= log_sum;
      q[i] /= 1.f + others;
      same[i] = rest[i] = 0.f;
      first[i] = index[i] >= 0;
    }
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i) {
      if (32 * i >= a.k) break;
      for (int l = 0; l < 32 && 32 * i + l < a.k; ++l) {
        const int other = __shfl_sync(kAll, index[i], l);
        const float share = __shfl_sync(kAll, q[i], l);
#pragma unroll
        for (int e = 0; e < kTopRegs; ++e) {
          const bool mine = other == index[e];
          same[e] += mine ? share : 0.f;
          rest[e] += mine ? 0.f : share;
          if (mine && 32 * i + l < 32 * e + lane) first[e] = false;
        }
      }
    }
  }
};

template <int G>
struct DistillShared {
  JoinShared<G> join;
  int live;
};

// G threads a row: 32, of which a block holds four rows, or a block. RESIDENT: the
// row waits in shared memory for its second reading.
template <typename T, int G, bool RESIDENT>
__global__ void __launch_bounds__(G == 32 ? 128 : G) k_distill(const T* z, T* dz, const DistillArgs a) {
  constexpr int kRows = G == 32 ? 4 : 1, N = Vec<T>::N;
  extern __shared__ uint4 row_s[];
  __shared__ DistillShared<G> shared[kRows];
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int slot = G == 32 ? threadIdx.x >> 5 : 0, rank = group_rank<G>(), lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * kRows + slot;
  if (t >= a.tokens) return;
  const T* zr = z + t * a.ldz;
  T* dr = dz ? dz + t * a.ldd : nullptr;
  const RowSpan<T> row(zr, a.classes);
  auto get = [&](int i) { return row.granules[i]; };
  auto keep = [&](int i) {
    const uint4 w = row.granules[i];
    if (RESIDENT) row_s[i] = w;
    return w;
  };
  auto again = [&](int i) { return RESIDENT ? row_s[i] : row.granules[i]; };
  const float w = a.weight ? a.weight[t] : 1.f;
  const bool first_warp = rank < 32;
  Teacher teacher;
  float zj[kTopRegs];
  int live = 0;  // 1: a row with a teacher, 2: its values are NaN
  if (first_warp) {
    teacher.load(a, t, lane);
    live = w == 0.f || !teacher.any ? 0 : teacher.bad ? 2 : 1;
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i) zj[i] = live == 1 && teacher.index[i] >= 0 ? to_f32<T>(zr[teacher.index[i]]) : 0.f;
    if (G > 32 && lane == 0) shared[slot].live = live;
  }
  group_sync<G>();
  if (G > 32) live = shared[slot].live;
  float fill = 0.f, loss = 0.f, factor = 0.f;
  RowSums sums{};
  if (live == 1) {
    const auto part = sum_part<T, G, false, 4>(row, 0, row.count, a.classes, rank, a.c, keep);
    sums = join_group<T, G, false>(part, row, 0, row.count, a.classes, a.c, get, shared[slot].join);
    if (isnan(sums.m)) live = 2;
  }
  if (live == 2) fill = loss = NAN;
  float at[kTopRegs];
  if (first_warp && live == 1) {
    const float log_sum = sums.none ? 0.f : log1pf(sums.others);
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i) {
      const float lp = sums.none || zj[i] == -INFINITY ? -INFINITY : (zj[i] - sums.m) / a.temperature - log_sum;
      if (teacher.q[i] > 0.f && teacher.index[i] >= 0) loss += teacher.q[i] * (teacher.log_q[i] - lp);
      // p - q; where both are near 1, the difference of what is left of them
      const float p = exp2_of(lp * kLog2e);
      at[i] = w * a.temperature * (p > 0.5f && teacher.same[i] > 0.5f ? teacher.rest[i] + expm1f(lp) : p - teacher.same[i]);
    }
    loss = w * a.temperature * a.temperature * warp_sum(loss);
  }
  if (a.loss && rank == 0) a.loss[t] = loss;
  if (!dr) return;
  if (live == 1 && sums.none) live = 0;  // masked whole
  if (live == 1) factor = w * a.temperature / (1.f + sums.others);
  const uint64_t minus_m = both(-sums.m), c = both(a.c), f = both(factor);
  const bool same = (((uintptr_t)dr ^ (uintptr_t)zr) & 15) == 0;
  for (int i = rank; i < row.count; i += G) {
    uint64_t v[N / 2];
    if (live == 1) {
      Vec<T>::open(again(i), v);
#pragma unroll
      for (int j = 0; j < N / 2; ++j) v[j] = ptx::mul_f32x2(exp2_pair(shifted(v[j], minus_m, c)), f);
    } else {
#pragma unroll
      for (int j = 0; j < N / 2; ++j) v[j] = both(fill);
    }
    put_granule<T>(dr, same, Vec<T>::close(v), row.first(i), a.classes);
  }
  if (live != 1) return;
  group_sync<G>();
  if (first_warp) {
#pragma unroll
    for (int i = 0; i < kTopRegs; ++i)
      if (teacher.index[i] >= 0 && teacher.first[i]) dr[teacher.index[i]] = from_f32<T>(at[i]);
  }
}

template <typename T>
void launch_distill(const T* z, T* dz, const DistillArgs& a, cudaStream_t s) {
  const int granules = (int)ceil_div(a.classes, Vec<T>::N) + 1;
  if (granules <= 257) {
    launch_pdl(k_distill<T, 32, false>, dim3((unsigned)ceil_div(a.tokens, 4)), 128, s, z, dz, a);
  } else if (granules <= 2048) {
    launch_pdl_smem(k_distill<T, 128, true>, dim3((unsigned)a.tokens), 128, granules * 16, s, z, dz, a);
  } else if (granules * 16 <= 112 * 1024 - 512) {
    allow_smem(reinterpret_cast<const void*>(k_distill<T, 512, true>), 112 * 1024);
    launch_pdl_smem(k_distill<T, 512, true>, dim3((unsigned)a.tokens), 512, granules * 16, s, z, dz, a);
  } else {
    launch_pdl(k_distill<T, 512, false>, dim3((unsigned)a.tokens), 512, s, z, dz, a);
  }
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

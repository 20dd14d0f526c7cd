// Softmax cross entropy of each row and its gradient, the logits read once:
//   loss_t = w_t (log sum_j exp z_tj - z_ty),  dz_tj = w_t (p_tj - [j = y])
// One read of z, one write of dz. Each thread keeps a running maximum and sum of
// its part of the row, the parts join at the end, and the row's values wait in
// registers (a warp a row) or shared memory (a block a row) for the gradient. The
// target stands outside the sum: 1 - p_y is the others' share, without
// cancellation. Bound by instructions: 65,536 x 200 FP32 (a warp a row) 32 us, 3.3
// TB/s; 4,096 x 50,001 BF16 (a block a row) 176 us, 4.7 TB/s; both issue one in
// three clocks of four, some twenty a value, most of them for the two exponentials.
#include "head_mma.cuh"
#include "head_rows.cuh"

namespace lc {
namespace ops {
namespace {

struct LossArgs {
  int64_t ldz, ldd, tokens;
  int classes;
  const int32_t* target;
  const float* weight;
  float* loss;
};

// The running maximum m and sum s of exp(z - m) of a set; m = -inf, s = 0:
// empty. A NaN or +inf among the values makes s NaN.
struct Run {
  float m, s;
  // (an empty side adds nothing; -inf minus itself would be NaN)
  __device__ __forceinline__ void join(float m2, float s2) {
    const float top = fmaxf(m, m2);
    const float a = m == -INFINITY ? s : s * __expf(m - top);
    const float b = m2 == -INFINITY ? s2 : s2 * __expf(m2 - top);
    m = top;
    s = a + b;
  }
  // The join of the warp's runs, on every lane: the maximum first, so that
  // each lane scales its sum once.
  __device__ __forceinline__ void join_warp() {
    float top = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (m != -INFINITY) s *= __expf(m - top);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    m = top;
  }
  template <typename T>
  __device__ __forceinline__ void add(const uint4& w) {
    constexpr int N = Vec<T>::N;
    const float top = Vec<T>::top(w);
    if (top > m) {
      s = m == -INFINITY ? s : s * __expf(m - top);
      m = top;
    }
    if (m == -INFINITY) {  // masked classes, or NaN, only
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (isnan(Vec<T>::at(w, i))) s = NAN;
      return;
    }
    uint64_t v[N / 2];
    Vec<T>::open(w, v);
    uint64_t t = exp_pair(v[0], both(-m));
#pragma unroll
    for (int i = 1; i < N / 2; ++i) t = ptx::add_f32x2(t, exp_pair(v[i], both(-m)));
    s += __uint_as_float((uint32_t)t) + __uint_as_float((uint32_t)(t >> 32));
  }
};

// What a row's sums say: the factor of exp(z - m) and the target's gradient;
// `odd`: every value is `fill` instead (NaN, or 0 of a row masked whole).
struct RowResult {
  float m, inv, at_target, fill;
  bool odd;
};
// `r` is the joined run of all classes but the target, whose logit is zy.
__device__ __forceinline__ RowResult finish(Run r, float zy, float w, float* loss, bool write) {
  const float m_o = r.m, s_o = r.s;
  const bool bad = isnan(r.s) || !(zy < INFINITY);
  r.join(zy, zy == -INFINITY ? 0.f : 1.f);
  const float others = s_o == 0.f ? 0.f : s_o * __expf(m_o - r.m);  // their share of r.s
  RowResult q;
  q.m = r.m;
  if (loss && write) {
    // Differences of logits first: the logarithm keeps its bits wherever the logits
    // stand. A target that is the maximum has r.s = 1 + others, of which a sure
    // row's loss would be the rounding.
    const float l = zy == -INFINITY ? INFINITY : r.m == zy ? log1pf(others) : logf(r.s) + (r.m - zy);
    *loss = bad ? NAN : w == 0.f ? 0.f : w * l;
  }
  q.odd = bad || r.m == -INFINITY;
  q.fill = bad ? NAN : 0.f;
  q.inv = w / r.s;
  q.at_target = s_o == 0.f ? 0.f : -w * (others / r.s);
  return q;
}

// Where a row lies in 16-byte granules: granule k holds its elements
// [k N - lead, k N - lead + N), the first and the last one some of a
// neighbour's (or of nothing's) too. Sums go by groups of N elements from the
// row's first, so that they do not depend on how the row is aligned; a group
// is a window on two granules.
template <typename T>
struct Place {
  static constexpr int N = Vec<T>::N;
  const uint4* granules;
  int lead, count, groups;
  __device__ __forceinline__ Place(const T* p, int n) {
    const int off = (int)((uintptr_t)p & 15);
    granules = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) - off);
    lead = off / (int)sizeof(T);
    count = (lead + n + N - 1) / N;
    groups = (n + N - 1) / N;
  }
};
// Group g's values join the run, the target's apart.
template <typename T>
__device__ __forceinline__ void add_group(Run& r, uint4 w, int g, int classes, int y, float& zy) {
  constexpr int N = Vec<T>::N;
  const int first = g * N;
  if (first + N > classes || (uint32_t)(y - first) < (uint32_t)N) {
    __align__(16) T v[N];
    *reinterpret_cast<uint4*>(v) = w;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (first + j == y) zy = to_f32<T>(v[j]);
      if (first + j == y || first + j >= classes) v[j] = from_f32<T>(-INFINITY);
    }
    w = *reinterpret_cast<const uint4*>(v);
  }
  r.add<T>(w);
}

// The gradient of a granule (values w, its first element `first`) to the
// output's row.
template <typename T>
__device__ __forceinline__ void put_granule(T* dr, bool same, const uint4& w, int first, int classes,
                                            const RowResult& q, int y) {
  constexpr int N = Vec<T>::N;
  uint64_t v[N / 2];
  if (!q.odd) {
    Vec<T>::open(w, v);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = ptx::mul_f32x2(exp_pair(v[i], both(-q.m)), both(q.inv));
    if ((uint32_t)(y - first) < (uint32_t)N) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (first + j == y)
          v[j / 2] = j & 1 ? (v[j / 2] & 0xffffffffull) | ((uint64_t)__float_as_uint(q.at_target) << 32)
                           : (v[j / 2] & ~0xffffffffull) | __float_as_uint(q.at_target);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = both(q.fill);
  }
  const uint4 o = Vec<T>::close(v);
  if (same && first >= 0 && first + N <= classes) {
    *reinterpret_cast<uint4*>(dr + first) = o;
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (first + j >= 0 && first + j < classes) dr[first + j] = reinterpret_cast<const T*>(&o)[j];
  }
}

// ---------------------------------------------------------------- a warp a row
constexpr int kWarpVecs = 8;  // granules a lane holds

// Warps take rows in turn; where a lane holds few granules, the next row's are
// loaded before this one's are summed.
template <typename T, int VECS>
__global__ void __launch_bounds__(128) k_loss_warp(const T* z, T* dz, const LossArgs a) {
  constexpr int N = Vec<T>::N;
  constexpr bool kAhead = VECS <= 2;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int lane = threadIdx.x & 31;
  const int64_t step = (int64_t)gridDim.x * 4;
  struct Row {
    uint4 keep[VECS];
    int y;
    float w;
  };
  auto load = [&](int64_t row, Row& r) {
    if (row >= a.tokens) return;
    r.y = __ldg(a.target + row);
    r.w = a.weight ? __ldg(a.weight + row) : 1.f;
    const Place<T> c(z + row * a.ldz, a.classes);
#pragma unroll
    for (int i = 0; i < VECS; ++i)
      if (i * 32 + lane < c.count) r.keep[i] = c.granules[i * 32 + lane];
  };
  int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  Row cur = {}, next = {};
  if (kAhead) load(row, next);
  for (; row < a.tokens; row += step) {
    if (kAhead) {
      cur = next;
      load(row + step, next);
    } else {
      load(row, cur);
    }
    const T* zr = z + row * a.ldz;
    const Place<T> c(zr, a.classes);
    const int y = cur.y;
    RowResult q{0.f, 0.f, 0.f, 0.f, true};  // an ignored row: 0
    if (y >= 0 && y < a.classes) {
      Run r{-INFINITY, 0.f};
      float zy = -INFINITY;
#pragma unroll
      for (int i = 0; i < VECS; ++i) {
        uint4 g = cur.keep[i];
        if (c.lead) {  // the next granule is the next lane's
          const uint4 n = cur.keep[i + 1 < VECS ? i + 1 : i];
          uint4 b;
          const int from = (lane + 1) & 31;
          b.x = __shfl_sync(0xffffffffu, lane == 0 ? n.x : g.x, from);
          b.y = __shfl_sync(0xffffffffu, lane == 0 ? n.y : g.y, from);
          b.z = __shfl_sync(0xffffffffu, lane == 0 ? n.z : g.z, from);
          b.w = __shfl_sync(0xffffffffu, lane == 0 ? n.w : g.w, from);
          g = window(g, b, c.lead * (int)sizeof(T));
        }
        if (i * 32 + lane < c.groups) add_group<T>(r, g, i * 32 + lane, a.classes, y, zy);
      }
      r.join_warp();
      // the target's logit stands on one lane
      const uint32_t group = (uint32_t)y / N;
      zy = __shfl_sync(0xffffffffu, zy, group & 31);
      q = finish(r, zy, cur.w, a.loss ? a.loss + row : nullptr, lane == 0);
    } else if (a.loss && lane == 0) {
      a.loss[row] = 0.f;
    }
    if (!dz) continue;
    T* dr = dz + row * a.ldd;
    const bool same = (((uintptr_t)dr ^ (uintptr_t)zr) & 15) == 0;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int k = i * 32 + lane;
      if (k < c.count) put_granule<T>(dr, same, cur.keep[i], k * N - c.lead, a.classes, q, y);
    }
  }
}

// ---------------------------------------------------------------- a block a row
constexpr int kRowThreads = 512;

// RESIDENT: the row is copied to shared memory (16-byte copies that stay in
// flight together); otherwise, for rows that do not fit twice on an SM, it is
// read again for the gradient.
template <typename T, bool RESIDENT>
__global__ void __launch_bounds__(kRowThreads, 2) k_loss_row(const T* z, T* dz, const LossArgs a) {
  constexpr int N = Vec<T>::N;
  extern __shared__ uint4 row_s[];
  __shared__ float sm[kRowThreads / 32], ss[kRowThreads / 32], szy;
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const int64_t row = blockIdx.x;
  const T* zr = z + row * a.ldz;
  T* dr = dz ? dz + row * a.ldd : nullptr;
  const int y = __ldg(a.target + row), tid = threadIdx.x;
  const bool live = y >= 0 && y < a.classes;
  const Place<T> c(zr, a.classes);
  RowResult q{0.f, 0.f, 0.f, 0.f, true};  // an ignored row: 0
  if (live) {
    // the copy in four parts: the sum of one runs while the next ones arrive
    // (its parts go by the groups: the same for any alignment)
    const int part = (c.groups + 4 * kRowThreads) / (4 * kRowThreads) * kRowThreads;
    if (RESIDENT) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        for (int i = k * part + tid; i < min((k + 1) * part, c.count); i += kRowThreads) {
          const uint32_t dst = ptx::smem_u32(row_s + i);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(c.granules + i) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
    }
    const float w = a.weight ? __ldg(a.weight + row) : 1.f;
    if (tid == 0) szy = to_f32<T>(zr[y]);
    Run r{-INFINITY, 0.f};
    float zy;  // (everyone's copy is szy)
#pragma unroll
    for (int k = 0; k < (RESIDENT ? 4 : 1); ++k) {
      if (RESIDENT) {
        if (k == 0) asm volatile("cp.async.wait_group 3;" ::: "memory");
        if (k == 1) asm volatile("cp.async.wait_group 2;" ::: "memory");
        if (k == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        if (k == 3) asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
      }
      // a window's second granule may be of the next part: one group behind
      const int end = k == (RESIDENT ? 3 : 0) ? c.groups : min((k + 1) * part - 1, c.groups);
      for (int i = max(k * part - 1, 0) + tid; i < end; i += kRowThreads) {
        uint4 g = RESIDENT ? row_s[i] : c.granules[i];
        if (c.lead && i + 1 < c.count)
          g = window(g, RESIDENT ? row_s[i + 1] : c.granules[i + 1], c.lead * (int)sizeof(T));
        else if (c.lead)
          g = window(g, uint4{0, 0, 0, 0}, c.lead * (int)sizeof(T));
        add_group<T>(r, g, i, a.classes, y, zy);
      }
    }
    r.join_warp();
    if ((tid & 31) == 0) sm[tid >> 5] = r.m, ss[tid >> 5] = r.s;
    __syncthreads();
    static_assert(kRowThreads == 512, "16 warps: half a warp's lanes hold their runs");
    r = Run{sm[tid & 15], (tid & 31) < 16 ? ss[tid & 15] : 0.f};
    r.join_warp();
    q = finish(r, szy, w, a.loss ? a.loss + row : nullptr, tid == 0);
  } else if (a.loss && tid == 0) {
    a.loss[row] = 0.f;
  }
  if (!dr) return;
  const bool same = (((uintptr_t)dr ^ (uintptr_t)zr) & 15) == 0;
  for (int i = tid; i < c.count; i += kRowThreads) {
    uint4 g{0, 0, 0, 0};
    if (live) g = RESIDENT ? row_s[i] : c.granules[i];
    put_granule<T>(dr, same, g, i * N - c.lead, a.classes, q, y);
  }
}

template <typename T>
void launch(const T* z, T* dz, const LossArgs& a, cudaStream_t s) {
  constexpr int N = Vec<T>::N;
  // granules of a row, one more where rows start inside one
  const int vecs = (int)ceil_div(a.classes, N) + (a.ldz % N || ((uintptr_t)z & 15) ? 1 : 0);
  const unsigned warps = (unsigned)std::min<int64_t>(ceil_div(a.tokens, 4), 12 * mma::num_sms());
  // A warp holds rows of up to 256 vectors in registers; longer ones take a
  // block and, up to 112 KB (two blocks an SM), stay in shared memory.
  if (vecs <= 32)
    launch_pdl(k_loss_warp<T, 1>, dim3(warps), 128, s, z, dz, a);
  else if (vecs <= 64)
    launch_pdl(k_loss_warp<T, 2>, dim3(warps), 128, s, z, dz, a);
  else if (vecs <= 32 * kWarpVecs)
    launch_pdl(k_loss_warp<T, kWarpVecs>, dim3(warps), 128, s, z, dz, a);
  else if (vecs * 16 <= 112 * 1024 - 512) {
    allow_smem(reinterpret_cast<const void*>(k_loss_row<T, true>), 112 * 1024);
    launch_pdl_smem(k_loss_row<T, true>, dim3((unsigned)a.tokens), kRowThreads, vecs * 16, s, z, dz, a);
  } else {
    launch_pdl(k_loss_row<T, false>, dim3((unsigned)a.tokens), kRowThreads, s, z, dz, a);
  }
  LC_LAUNCH_CHECK("k_loss");
}

}  // namespace

void cross_entropy(int type, const void* z, int64_t ldz, int64_t tokens, int classes, const int32_t* target,
                   const float* weight, float* loss, void* dz, int64_t ldd, cudaStream_t s) {
  const LossArgs a{ldz, ldd, tokens, classes, target, weight, loss};
  if (type == LIPCACHE_F32)
    launch(static_cast<const float*>(z), static_cast<float*>(dz), a, s);
  else
    launch(static_cast<const __nv_bfloat16*>(z), static_cast<__nv_bfloat16*>(dz), a, s);
}

}  // namespace ops
}  // namespace lc

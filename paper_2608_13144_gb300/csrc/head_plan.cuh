// The order in which the rows of many requests are worked on.
//
// Low-rank products take neighbouring rows that share an adapter (a run)
// together. Where the rows come in few runs (requests one after another) they
// stay where they are; where they come in many, they are sorted by adapter
// (stable, so that sums have one order), rows without one last.
#pragma once

#include <cooperative_groups.h>

#include "head_mma.cuh"

namespace lc {
namespace ops {

struct Plan {
  int* flags;   // [0] runs, [1] whether rows are sorted
  int* off;     // runs + 1: first row of each
  int* g;       // runs: adapter, G for none
  int* next;    // runs: the next run of the same adapter, -1 at the last
  int* first;   // G: first run of each adapter, -1 without rows
  int* perm;    // tokens: the row at each place (written where sorted)
  int* row_g;   // tokens: the adapter at each place, G for none
  int cap;      // runs that may stand unsorted

  // Runs are worth keeping while they hold 128 rows on average: a run's last
  // rows short of 16 are summed outside the tensor cores.
  void take(Carve& c, int64_t tokens, int G) {
    cap = (int)std::min<int64_t>(4096, std::max<int64_t>(G, tokens / 128) + 1);
    const int most = std::max(cap, G + 1);
    c.take(flags, 2);
    c.take(off, (size_t)most + 1);
    c.take(g, (size_t)most);
    c.take(next, (size_t)most);
    c.take(first, (size_t)std::max(G, 1));
    c.take(perm, (size_t)tokens);
    c.take(row_g, (size_t)tokens);
  }
  mma::Runs runs() const { return mma::Runs{off, g, flags}; }
};

constexpr int kPlanThreads = 1024;

// One cluster. Every warp owns a stretch of neighbouring rows: it counts them
// per adapter and counts the runs that start in it; sums over the warps before
// it (by way of the cluster's shared memory) give each run its number and each
// row its place.
__global__ void __launch_bounds__(kPlanThreads, 1)
    k_plan(const int32_t* adapter, int64_t tokens, int G, int warps, const Plan p) {
  namespace cg = cooperative_groups;
  extern __shared__ int hist[];  // warps x (G + 1), then G + 1 totals
  __shared__ int starts[33], cta_starts, tot_off[kPlanThreads / 32 + 1];
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = G + 1;
  int* total = hist + warps * n;
  for (int i = threadIdx.x; i < warps * n; i += kPlanThreads) hist[i] = 0;
  if (threadIdx.x < 33) starts[threadIdx.x] = 0;
  ptx::wait_prerequisites();
  __syncthreads();
  // stretches of whole groups of 32 rows
  const int64_t groups = ceil_div_dev(tokens, 32), per = ceil_div_dev(groups, (int64_t)ctas * warps);
  const int64_t r0 = min((rank * (int64_t)warps + warp) * per * 32, tokens), r1 = min(r0 + per * 32, tokens);
  auto id_of = [&](int64_t t) {
    const int g = __ldg(adapter + t);
    return g < 0 || g >= G ? G : g;
  };
  if (warp < warps) {
    int mine = 0;
    for (int64_t t0 = r0; t0 < r1; t0 += 32) {
      const int64_t t = t0 + lane;
      const bool live = t < r1;
      const int g = live ? id_of(t) : -1;
      const bool start = live && (t == 0 || id_of(t - 1) != g);
      mine += __popc(__ballot_sync(0xffffffffu, start));
      const uint32_t same = __match_any_sync(0xffffffffu, g);
      if (live && lane == __ffs(same) - 1) hist[warp * n + g] += __popc(same);
      __syncwarp();
    }
    if (lane == 0) starts[warp] = mine;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    int s = 0;
    for (int w = 0; w < warps; ++w) {
      const int v = starts[w];
      starts[w] = s;
      s += v;
    }
    cta_starts = s;
  }
  for (int g = threadIdx.x; g < n; g += kPlanThreads) {
    int s = 0;
    for (int w = 0; w < warps; ++w) s += hist[w * n + g];
    total[g] = s;
  }
  cluster.sync();
  int before = 0, runs = 0;
  for (int c = 0; c < ctas; ++c) {
    const int v = *cluster.map_shared_rank(&cta_starts, c);
    if (c < rank) before += v;
    runs += v;
  }
  const bool sorted = runs > p.cap;
  if (!sorted) {
    if (warp < warps) {
      int at = before + starts[warp];
      for (int64_t t0 = r0; t0 < r1; t0 += 32) {
        const int64_t t = t0 + lane;
        const bool live = t < r1;
        const int g = live ? id_of(t) : -1;
        const bool start = live && (t == 0 || id_of(t - 1) != g);
        const uint32_t m = __ballot_sync(0xffffffffu, start);
        if (live) p.row_g[t] = g;
        if (start) {
          const int i = at + __popc(m & ((1u << lane) - 1u));
          p.off[i] = (int)t;
          p.g[i] = g;
        }
        at += __popc(m);
      }
    }
    if (rank == 0 && threadIdx.x == 0) {
      p.flags[0] = runs;
      p.flags[1] = 0;
      p.off[runs] = (int)tokens;
    }
    __threadfence();
    cluster.sync();
    // each run's successor, from the last run back
    if (rank == 0) {
      for (int g = threadIdx.x; g < n; g += kPlanThreads) total[g] = -1;
      __syncthreads();
      if (warp == 0) {
        for (int i0 = (runs - 1) / 32 * 32; i0 >= 0; i0 -= 32) {
          const int i = i0 + lane;
          const int g = i < runs ? __ldcg(p.g + i) : -1;
          const uint32_t same = __match_any_sync(0xffffffffu, g);
          const uint32_t later = lane == 31 ? 0u : same & ~((2u << lane) - 1u);
          if (g >= 0) p.next[i] = later ? i0 + __ffs(later) - 1 : total[g];
          __syncwarp();
          if (g >= 0 && lane == __ffs(same) - 1) total[g] = i;
          __syncwarp();
        }
      }
      __syncthreads();
      for (int g = threadIdx.x; g < G; g += kPlanThreads) p.first[g] = total[g];
    }
  } else {
    // places: adapters in order, then CTAs, then warps; `chunk` adapters a thread
    const int chunk = (n + kPlanThreads - 1) / kPlanThreads;
    int sum = 0, present = 0;
    for (int k = 0; k < chunk; ++k) {
      const int g = threadIdx.x * chunk + k;
      if (g >= n) break;
      int s = 0;
      for (int c = 0; c < ctas; ++c) s += *cluster.map_shared_rank(total + g, c);
      sum += s;
      present += s > 0;
    }
    // exclusive sums over the threads: rows before, runs before
    int rows_at = sum, runs_at = present;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int a = __shfl_up_sync(0xffffffffu, rows_at, o), b = __shfl_up_sync(0xffffffffu, runs_at, o);
      if (lane >= o) rows_at += a, runs_at += b;
    }
    __syncthreads();  // starts and tot_off are free
    if (lane == 31) tot_off[warp] = rows_at, starts[warp] = runs_at;
    __syncthreads();
    int all_runs = 0;
    int add_rows = 0, add_runs = 0;
    for (int w = 0; w < kPlanThreads / 32; ++w) {
      if (w < warp) add_rows += tot_off[w], add_runs += starts[w];
      all_runs += starts[w];
    }
    rows_at += add_rows - sum;
    runs_at += add_runs - present;
    for (int k = 0; k < chunk; ++k) {
      const int g = threadIdx.x * chunk + k;
      if (g >= n) break;
      int s = 0, lower = 0;
      for (int c = 0; c < ctas; ++c) {
        const int v = *cluster.map_shared_rank(total + g, c);
        if (c < rank) lower += v;
        s += v;
      }
      if (rank == 0) {
        if (s) {
          p.off[runs_at] = rows_at;
          p.g[runs_at] = g;
          p.next[runs_at] = -1;
        }
        if (g < G) p.first[g] = s ? runs_at : -1;
      }
      int at = rows_at + lower;
      for (int w = 0; w < warps; ++w) {
        const int v = hist[w * n + g];
        hist[w * n + g] = at;
        at += v;
      }
      rows_at += s;
      runs_at += s > 0;
    }
    if (rank == 0 && threadIdx.x == 0) {
      p.flags[0] = all_runs;
      p.flags[1] = 1;
      p.off[all_runs] = (int)tokens;
    }
    __syncthreads();
    if (warp < warps) {
      for (int64_t t0 = r0; t0 < r1; t0 += 32) {
        const int64_t t = t0 + lane;
        const bool live = t < r1;
        const int g = live ? id_of(t) : -1;
        const uint32_t same = __match_any_sync(0xffffffffu, g);
        if (live) {
          const int at = hist[warp * n + g] + __popc(same & ((1u << lane) - 1u));
          p.perm[at] = (int)t;
          p.row_g[at] = g;
        }
        __syncwarp();
        if (live && lane == __ffs(same) - 1) hist[warp * n + g] += __popc(same);
        __syncwarp();
      }
    }
  }
  ptx::launch_dependents();
  cluster.sync();  // no CTA leaves while another reads its shared memory
}

inline void make_plan(const int32_t* adapter, int64_t tokens, int G, const Plan& p, cudaStream_t s) {
  const int warps = G + 1 <= 1024 ? 32 : 8;
  const int ctas = tokens <= 2048 ? 1 : 8;
  const int smem = (warps + 1) * (G + 1) * 4;
  allow_smem(reinterpret_cast<const void*>(k_plan), 200 * 1024);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  LC_CUDA(cudaLaunchKernelEx(&cfg, k_plan, adapter, tokens, G, warps, p));
  LC_LAUNCH_CHECK("k_plan");
}

}  // namespace ops
}  // namespace lc

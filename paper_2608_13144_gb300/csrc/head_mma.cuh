// Tensor-core products for the operators of heads: D = A B^T (+ low-rank
// products) in tiles of 128 CG x BN, with an epilogue of the caller's.
//
// Operands are 16-bit (FP16 or BF16) 3-D tensors read by TMA with
// the 128-byte swizzle, zero-filled past their ends, each either K-major (the
// contracted index is the innermost) or MN-major. tcgen05 MMAs accumulate in
// FP32 in tensor memory, two accumulators taking turns. CG = 2: a CTA pair
// works on one 256-row tile (cta_group::2), each CTA holding its 128 rows of A
// and half the columns of B, so that a CTA's shared memory feeds the MMAs 128
// bytes a clock instead of 192.
//
// Warps of a CTA: 0 TMA producer, 1 MMA issuer (of the pair's leader), 2-9
// epilogue (tcgen05.ld, 32 columns at a time). CTAs are persistent: tiles are
// dealt round robin. Every wait is bounded; a role that gives up raises the
// CTA's abort flag, the kernel drains, and a counter of the device takes note.
//
// The tensor cores' FP32 sums are cut off, not rounded, at each addition, which
// shows in long sums as a drift of one sign (K = 1003 .. 2048, FP32 operands:
// 1.8e-5 of the result after five Newton-Schulz steps). PLANES = 2 (FP32: both
// operands two planes, hi + lo, z apart by a_planes and b_planes; a stage holds
// all four, for lo hi + hi lo + hi hi) breaks a sum into blocks of `block`
// stages: the epilogue warps take each block's sums out of tensor memory and add
// them in registers, rounded, while the MMAs of the next block run into the
// other accumulator.
//
// A low-rank product can be limited to some rows of the tile: the MMA's disabled
// output lanes keep what they hold, so that rows of other adapters neither
// change nor turn NaN.
//
// Measured: 8,192 x 4,096 BF16 rows by 4,096 classes 148 us, 1.86 PFLOP/s (0.98
// of the library's measured burst rate), bound by the tensor cores (tiles of 256 x
// 256, stages of 64: 512 clocks of MMAs against some 450 of the producer's
// instructions). A producer and an issuer of one diverged lane were no faster
// and made the low-rank stages after them 50 us slower. 65,536 x 256 FP32 rows by
// 200 classes 38 us, bound by the epilogue (four blocks of 32 x 32 a warp and
// tile, one after another). 48 BF16 rows by 4,096 x 4,096 20 us, bound by what a
// CTA's 32 stages cost its producer and issuer.
#pragma once

#include "operators.cuh"
#include "tc_ptx.cuh"

namespace lc {
namespace ops {

namespace mma {

constexpr int kChunk = 64;           // contracted elements of a stage
constexpr int kABytes = 128 * 128;   // 128 rows x 64 elements
constexpr int kEpiWarps = 8;
constexpr int kTurnBytes = 32 * 32 * 4;  // a warp's block of 32 x 32, turned for coalesced writes
constexpr int kThreads = 32 * (2 + kEpiWarps);
constexpr long long kWaitLimit = 1LL << 31;  // ~1 s at GB300 clocks
constexpr int kSmem = 227 * 1024;

// A product: `chunks` stages along the contracted index, the last one of `last`
// MMAs (16 elements each).
struct Seg {
  int chunks, last;
  uint32_t idesc;
};

__host__ __device__ constexpr uint32_t idesc(int M, int N, bool bf16, bool a_mn, bool b_mn) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// Shared-memory descriptor of an operand stored with the 128-byte swizzle.
// K-major: rows of 128 bytes (64 elements of K), 8-row groups 1024 bytes apart.
// MN-major: blocks of 64 elements of MN (128 bytes) x 64 of K, 8192 bytes each;
// groups of 8 along K are 1024 bytes apart, blocks along MN 8192.
__device__ __forceinline__ uint64_t desc(uint32_t saddr, bool mn) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(mn ? 8192 >> 4 : 1) << 16) |
         ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

__device__ __forceinline__ void load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void load_3d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, int z,
                                             uint32_t leader_bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, "
      "%4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(leader_bar)
      : "memory");
}

__device__ __forceinline__ void store_3d(const CUtensorMap* map, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(x), "r"(y), "r"(z), "r"(src)
               : "memory");
}

// Eight FP32 columns of this thread's lane, read and written.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8]) {
  uint32_t r[8];
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
  ptx::tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
               "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])),
               "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
               "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7]))
               : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// The MMA with a mask of output lanes (rows) to leave alone; `off` holds the
// lanes of this CTA (CG = 1) or of both (CG = 2), 32 a word.
template <int CG>
__device__ __forceinline__ void mma_masked(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc,
                                           const uint32_t (&off)[8]) {
  if (CG == 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, {%5, %6, %7, %8}, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(id), "r"(acc), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3])
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%5, %6, %7, %8, %9, %10, %11, %12}, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(id), "r"(acc), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3]), "r"(off[4]),
        "r"(off[5]), "r"(off[6]), "r"(off[7])
        : "memory");
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t acc) {
  if (CG == 1)
    ptx::mma_f16(d, a, b, id, acc);
  else
    ptx::mma_f16_pair(d, a, b, id, acc);
}

// The low-rank segments of a tile: for each adapter among the tile's rows the
// rows' factor (two planes) times the adapter's, limited to the adapter's rows.
// Tiles with more than kFewAdapters leave it to the epilogue (`many`), which
// costs as much for any number.
constexpr int kFewAdapters = 8;
struct Low {
  const int32_t* adapter = nullptr;  // of each row
  int64_t tokens = 0;
  int G = 0;                         // 0: no low-rank segments
  int chunks = 0, last = 0;
  int dense = 0;                     // every adapter's factor side by side, the rows' factors 0 but in their own:
                                     // one product for all rows, three planes each (PLANES = 2)
  uint32_t idesc;
};

// The adapters among TM rows, one after another: lane l holds the adapters of
// rows 32 k + l, -1 for none.
template <int TM>
struct Groups {
  int id[TM / 32];
  uint32_t rest[TM / 32];  // rows of adapters still to come
  uint32_t on[TM / 32];    // rows of adapter g
  int g;
  __device__ __forceinline__ void begin(const int32_t* adapter, int64_t tokens, int G, int64_t m0, int lane) {
#pragma unroll
    for (int k = 0; k < TM / 32; ++k) {
      const int64_t t = m0 + 32 * k + lane;
      const int a = t < tokens ? __ldg(adapter + t) : -1;
      id[k] = a < G ? a : -1;
    }
    again();
  }
  __device__ __forceinline__ void again() {
#pragma unroll
    for (int k = 0; k < TM / 32; ++k) rest[k] = __ballot_sync(0xffffffffu, id[k] >= 0);
  }
  __device__ __forceinline__ bool next() {
    int found = -1;
#pragma unroll
    for (int k = TM / 32 - 1; k >= 0; --k) {
      const int a = __shfl_sync(0xffffffffu, id[k], (__ffs(rest[k]) - 1) & 31);
      if (rest[k]) found = a;
    }
    if (found < 0) return false;
    g = found;
#pragma unroll
    for (int k = 0; k < TM / 32; ++k) {
      on[k] = __ballot_sync(0xffffffffu, id[k] == found);
      rest[k] &= ~on[k];
    }
    return true;
  }
  // whether there are more than `most` of them
  __device__ __forceinline__ bool more_than(int most) {
    int n = 0;
    bool more = false;
    while (next())
      if (++n > most) {
        more = true;
        break;
      }
    again();
    return more;
  }
};

struct Args {
  int m_tiles, n_tiles, batches;
  int sym;  // tiles on or above the diagonal only (m_tiles == n_tiles in units of the wider side)
  int bn;   // columns of a tile
  int stages;
  int a_rows;  // rows of A's box (K-major): 128, or fewer where the tile has no more
  int a_mn, b_mn, lb_mn;
  int a_planes, b_planes;  // z from a plane to the next
  int low_after;           // the epilogue adds the low-rank product of every tile
  int block;  // stages per block (DRAIN)
  Seg seg;
  Low low;
  unsigned long long* errors;  // expired waits, counted
};

// The operands' maps: A, B and the low-rank segments' factors.
struct Maps {
  CUtensorMap a, b, la, lb;
};

// Tile `t`: its first row and column (in tiles) and batch index.
__device__ __forceinline__ void tile_at(const Args& a, int t, int& mt, int& nt, int& z) {
  if (a.sym) {
    const int per = a.m_tiles * (a.m_tiles + 1) / 2;
    z = t / per;
    t -= z * per;
    // column nt holds tiles 0..nt of the upper triangle
    nt = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (nt * (nt + 1) / 2 > t) --nt;
    while ((nt + 1) * (nt + 2) / 2 <= t) ++nt;
    mt = t - nt * (nt + 1) / 2;
    return;
  }
  const int per = a.m_tiles * a.n_tiles;
  z = t / per;
  t -= z * per;
  // bands of 8 row tiles, column by column: neighbours in time share operands in L2
  const int band = t / (8 * a.n_tiles), rest = t - band * 8 * a.n_tiles;
  const int high = min(8, a.m_tiles - band * 8);
  nt = rest / high;
  mt = band * 8 + rest - nt * high;
}

// Halves of a stage along the contracted index: the few-rows form's tiles are so
// small that what a stage costs its producer and issuer sets the pace (450 clocks
// for 64 of the index), so that theirs hold twice 64 (48 rows by 4,096 x 4,096: 27
// -> 20 us).
template <typename Epi>
constexpr int kHalves = Epi::kEarly ? 2 : 1;

template <int CG>
__device__ __forceinline__ void box_of(uint32_t dst, const CUtensorMap* m, int x, int y, int z, uint32_t bar) {
  if (CG == 2)
    load_3d_pair(dst, m, x, y, z, bar);
  else
    load_3d(dst, m, x, y, z, bar);
}

// DRAIN: a sum has more than one block (a kernel of its own: the registers that
// hold sums between blocks leave too few for the epilogue, which then spills).
template <int CG, int PLANES, bool DRAIN, typename Epi>
__global__ void __launch_bounds__(kThreads, 1)
    k_mma(const __grid_constant__ Maps maps, const Args a, const Epi epi) {
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  // a stage: A's planes, then B's
  // (A's rows past its box are whatever follows: their sums are not used)
  const int a_bytes = a.a_rows * 128, b_bytes = a.bn / CG * 128, stage_bytes = kHalves<Epi> * PLANES * (a_bytes + b_bytes);
  const int nst = a.stages;
  const uint32_t bars = base + nst * stage_bytes;
  const uint32_t full = bars, empty = bars + 8 * nst, acc_full = empty + 8 * nst, acc_empty = acc_full + 16,
                 drain = acc_empty + 16, misc = drain + 8, turn = (misc + 16 + 127) & ~127u;
  unsigned char* misc_p = smem_raw + (misc - ptx::smem_u32(smem_raw));
  volatile uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(misc_p);
  volatile int* abort_s = reinterpret_cast<volatile int*>(misc_p + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? ptx::cluster_ctarank() : 0u;
  const int worker = blockIdx.x / CG, workers = gridDim.x / CG;
  constexpr int TM = 128 * CG;
  const uint32_t cols = a.bn > 128 ? 512u : a.bn > 64 ? 256u : 128u;  // two accumulators
  const uint32_t acc_stride = cols / 2;

  if (threadIdx.x == 0) {
    for (int s = 0; s < nst; ++s) {
      ptx::mbar_init(full + 8 * s, 1);
      ptx::mbar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(acc_full + 8 * b, 1);
      ptx::mbar_init(acc_empty + 8 * b, CG * kEpiWarps);
    }
    ptx::mbar_init(drain, 1);
    *abort_s = 0;
    ptx::fence_mbar_init();
    ptx::tma_prefetch_desc(&maps.a);
    ptx::tma_prefetch_desc(&maps.b);
  }
  if (warp == 1) {
    if (CG == 2) {
      ptx::tmem_alloc_pair(misc, cols);
      ptx::tmem_relinquish_pair();
    } else {
      ptx::tmem_alloc(misc, cols);
      ptx::tmem_relinquish();
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (CG == 2) ptx::cluster_sync();
  ptx::wait_prerequisites();
  ptx::launch_dependents();
  const uint32_t tmem = *tmem_slot;
  const int per = a.sym ? a.m_tiles * (a.m_tiles + 1) / 2 : a.m_tiles * a.n_tiles;
  const int tiles = per * a.batches;
  const int chunks = a.seg.chunks;

  if (warp == 0) {
    // ------------------------------------------------------------ producer
    {  // the whole warp, converged, for the adapters' sake; lane 0 copies
      const uint32_t lead_full = CG == 2 ? ptx::mapa(full, 0) : full;
      int st = 0;
      uint32_t ph = 0;
      bool ok = true;
      // one stage: the boxes of A at (row, k) and of B at (column, k), of `planes` planes
      auto load = [&](const CUtensorMap* pa, bool a_mn, int row, int ak, int az, const CUtensorMap* pb, bool b_mn,
                      int col, int bk, int bz, int planes) {
        ok = ptx::mbar_wait_warp(empty + 8 * st, ph ^ 1u, abort_s, kWaitLimit);
        if (!ok) return;
        const uint32_t slot = st;
        if (++st == nst) st = 0, ph ^= 1u;
        if (lane != 0) return;
        if (rank == 0) ptx::mbar_expect_tx(full + 8 * slot, (uint32_t)(CG * planes * (a_bytes + b_bytes)));
        const uint32_t bar = lead_full + 8 * slot;
        auto box = [&](uint32_t dst, const CUtensorMap* m, int x, int y, int z) { box_of<CG>(dst, m, x, y, z, bar); };
        for (int p = 0; p < planes; ++p) {
          const uint32_t sa = base + slot * stage_bytes + p * a_bytes, sb = base + slot * stage_bytes + PLANES * a_bytes + p * b_bytes;
          const int za = az + p * a.a_planes, zb = bz + p * a.b_planes;
          if (a_mn) {
            box(sa, pa, row, ak, za);
            box(sa + 8192, pa, row + 64, ak, za);
          } else {
            box(sa, pa, ak, row, za);
          }
          if (b_mn) {
            for (int i = 0; i < a.bn / CG; i += 64) box(sb + i * 128, pb, col + i, bk, zb);
          } else {
            box(sb, pb, bk, col, zb);
          }
        }
      };
      // a dense low-rank product's stage: two planes of the rows' factors and two of the adapters', at z0 and z1
      auto load_planes = [&](int row, int col, int k, int z0, int z1) {
        ok = ptx::mbar_wait_warp(empty + 8 * st, ph ^ 1u, abort_s, kWaitLimit);
        if (!ok) return;
        const uint32_t slot = st;
        if (++st == nst) st = 0, ph ^= 1u;
        if (lane != 0) return;
        if (rank == 0) ptx::mbar_expect_tx(full + 8 * slot, (uint32_t)(CG * 2 * (a_bytes + b_bytes)));
        const uint32_t bar = lead_full + 8 * slot, sa = base + slot * stage_bytes, sb = sa + 2 * a_bytes;
        for (int p = 0; p < 2; ++p) {
          const int z = p ? z1 : z0;
          box_of<CG>(sa + p * a_bytes, &maps.la, k, row, z, bar);
          if (a.lb_mn) {
            for (int i = 0; i < a.bn / CG; i += 64) box_of<CG>(sb + p * b_bytes + i * 128, &maps.lb, col + i, k, z, bar);
          } else {
            box_of<CG>(sb + p * b_bytes, &maps.lb, k, col, z, bar);
          }
        }
      };
      for (int t = worker; t < tiles && ok; t += workers) {
        int mt, nt, z;
        tile_at(a, t, mt, nt, z);
        const int row = mt * TM + (int)rank * 128, col = nt * a.bn + (int)rank * (a.bn / CG);
        if constexpr (Epi::kEarly) {
          for (int c = 0; c < chunks && ok; c += 2) {
            ok = ptx::mbar_wait_warp(empty + 8 * st, ph ^ 1u, abort_s, kWaitLimit);
            if (!ok) break;
            if (lane == 0) {
              const int halves = min(2, chunks - c);
              const uint32_t sa = base + st * stage_bytes, bar = full + 8 * st;
              ptx::mbar_expect_tx(bar, (uint32_t)(halves * (a_bytes + b_bytes)));
              for (int p = 0; p < halves; ++p) {
                load_3d(sa + p * (a_bytes + b_bytes), &maps.a, (c + p) * kChunk, row, z, bar);
                load_3d(sa + p * (a_bytes + b_bytes) + a_bytes, &maps.b, (c + p) * kChunk, col, z, bar);
              }
            }
            if (++st == nst) st = 0, ph ^= 1u;
          }
        } else {
          for (int c = 0; c < chunks && ok; ++c)
            load(&maps.a, a.a_mn, row, c * kChunk, z, &maps.b, a.b_mn, col, c * kChunk, z, PLANES);
        }
        if (PLANES == 2 && a.low.dense) {
          for (int q = 0; q < 2 && ok; ++q)
            for (int c = 0; c < a.low.chunks && ok; ++c)
              load_planes(row, col, c * kChunk, 0, 2 - q);
        } else if (a.low.G) {
          Groups<TM> gr;
          gr.begin(a.low.adapter, a.low.tokens, a.low.G, (int64_t)mt * TM, lane);
          if (!gr.more_than(kFewAdapters))
            while (ok && gr.next())
              for (int q = 1; q >= 0 && ok; --q)
                for (int c = 0; c < a.low.chunks && ok; ++c)
                  load(&maps.la, false, row, c * kChunk, q, &maps.lb, a.lb_mn, col, c * kChunk, gr.g, 1);
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    if (rank == 0) {
      const bool lead = ptx::elect_one();
      int st = 0, n = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int t = worker; t < tiles && ok; t += workers) {
        int mt, nt, z;
        tile_at(a, t, mt, nt, z);
        uint32_t d = 0, acc = 0;
        // the next accumulator, once both CTAs' epilogues are done with it
        auto open = [&]() {
          ok = ptx::mbar_wait_warp<CG == 2>(acc_empty + 8 * (n & 1), (uint32_t)((n >> 1) & 1) ^ 1u, abort_s, kWaitLimit);
          if (!ok) return;
          ptx::tc_fence_after();
          d = tmem + (uint32_t)(n & 1) * acc_stride;
          acc = 0;
        };
        auto close = [&]() {
          if (ok && lead) {
            if (CG == 2)
              ptx::mma_commit_pair_multicast(acc_full + 8 * (n & 1), (uint16_t)3);
            else
              ptx::mma_commit(acc_full + 8 * (n & 1));
          }
          ++n;
        };
        // one stage of `steps` MMAs (a product of planes each), the rows in `off` left alone
        auto chunk = [&](bool a_mn, bool b_mn, uint32_t id, int steps, int planes, const uint32_t* off) {
          ok = ptx::mbar_wait_warp(full + 8 * st, ph, abort_s, kWaitLimit);
          if (!ok) return;
          ptx::tc_fence_after();
          if (lead) {
            const uint32_t sa = base + st * stage_bytes, sb = sa + PLANES * a_bytes;
            const uint64_t ia = a_mn ? 2048 >> 4 : 32 >> 4, ib = b_mn ? 2048 >> 4 : 32 >> 4;
            // lo hi, hi lo, hi hi
            for (int pr = planes == 2 ? 0 : 2; pr < 3; ++pr) {
              uint64_t da = desc(sa + (pr == 0 ? a_bytes : 0), a_mn), db = desc(sb + (pr == 1 ? b_bytes : 0), b_mn);
              for (int k = 0; k < steps; ++k, da += ia, db += ib) {
                if (off) {
                  const uint32_t o[8] = {off[0], off[1], off[2], off[3], off[4], off[5], off[6], off[7]};
                  mma_masked<CG>(d, da, db, id, 1u, o);
                } else {
                  mma<CG>(d, da, db, id, acc);
                }
                acc = 1;
              }
            }
            if (CG == 2)
              ptx::mma_commit_pair_multicast(empty + 8 * st, (uint16_t)3);
            else
              ptx::mma_commit(empty + 8 * st);
          }
          if (++st == nst) st = 0, ph ^= 1u;
        };
        open();
        if constexpr (Epi::kEarly) {
          for (int c = 0; c < chunks && ok; c += 2) {
            ok = ptx::mbar_wait_warp(full + 8 * st, ph, abort_s, kWaitLimit);
            if (!ok) break;
            ptx::tc_fence_after();
            if (lead) {
              const uint32_t sa = base + st * stage_bytes;
              for (int p = 0; p < 2 && c + p < chunks; ++p) {
                const int steps = c + p == chunks - 1 ? a.seg.last : 4;
                uint64_t da = desc(sa + p * (a_bytes + b_bytes), false), db = desc(sa + p * (a_bytes + b_bytes) + a_bytes, false);
                for (int k = 0; k < steps; ++k, da += 32 >> 4, db += 32 >> 4) {
                  mma<CG>(d, da, db, a.seg.idesc, acc);
                  acc = 1;
                }
              }
              ptx::mma_commit(empty + 8 * st);
            }
            if (++st == nst) st = 0, ph ^= 1u;
          }
        } else {
          for (int c0 = 0; c0 < chunks && ok; c0 += a.block) {
            if (c0) {
              close();
              open();
            }
            const int c1 = DRAIN ? min(c0 + a.block, chunks) : chunks;
            for (int c = c0; c < c1 && ok; ++c)
              chunk(a.a_mn, a.b_mn, a.seg.idesc, c == chunks - 1 ? a.seg.last : 4, PLANES, nullptr);
            if (!DRAIN) c0 = chunks;
          }
        }
        if (PLANES == 2 && a.low.dense) {
          // u0 f2 and u2 f0 from stages of planes 0 and 2, then u1 f1, u0 f1, u1 f0 and u0 f0 from those of 0 and 1
          for (int q = 0; q < 2 && ok; ++q)
            for (int c = 0; c < a.low.chunks && ok; ++c) {
              ok = ptx::mbar_wait_warp(full + 8 * st, ph, abort_s, kWaitLimit);
              if (!ok) break;
              ptx::tc_fence_after();
              if (lead) {
                const uint32_t sa = base + st * stage_bytes, sb = sa + 2 * a_bytes;
                const int steps = c == a.low.chunks - 1 ? a.low.last : 4;
                for (int pr = q == 0 ? 1 : 0; pr < (q == 0 ? 3 : 4); ++pr) {
                  // pairs (plane of u, plane of f) of the stage: 11, 01, 10, 00
                  uint64_t da = desc(sa + (pr == 0 || pr == 2 ? a_bytes : 0), false),
                           db = desc(sb + (pr < 2 ? b_bytes : 0), a.lb_mn);
                  for (int k = 0; k < steps; ++k, da += 32 >> 4, db += a.lb_mn ? 2048 >> 4 : 32 >> 4)
                    mma<CG>(d, da, db, a.low.idesc, 1u);
                }
                if (CG == 2)
                  ptx::mma_commit_pair_multicast(empty + 8 * st, (uint16_t)3);
                else
                  ptx::mma_commit(empty + 8 * st);
              }
              if (++st == nst) st = 0, ph ^= 1u;
            }
        } else if (a.low.G) {
          Groups<TM> gr;
          gr.begin(a.low.adapter, a.low.tokens, a.low.G, (int64_t)mt * TM, lane);
          if (!gr.more_than(kFewAdapters))
            while (ok && gr.next()) {
              uint32_t off[8] = {};
#pragma unroll
              for (int k = 0; k < TM / 32; ++k) off[k] = ~gr.on[k];
              for (int q = 0; q < 2 && ok; ++q)
                for (int c = 0; c < a.low.chunks && ok; ++c)
                  chunk(false, a.lb_mn, a.low.idesc, c == a.low.chunks - 1 ? a.low.last : 4, 1, off);
            }
        }
        close();
      }
      // every MMA has completed before tensor memory is given back
      if (lead) {
        volatile int never = 0;
        if (CG == 2)
          ptx::mma_commit_pair_multicast(drain, (uint16_t)1);
        else
          ptx::mma_commit(drain);
        ptx::mbar_wait(drain, 0, &never, kWaitLimit);
      }
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ epilogue
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    const uint32_t mine = turn + (uint32_t)((warp - 2) * kTurnBytes);
    const uint32_t lead_empty = CG == 2 ? ptx::mapa(acc_empty, 0) : acc_empty;
    int n = 0;
    bool ok = true;
    for (int t = worker; t < tiles && ok; t += workers) {
      int mt, nt, z;
      tile_at(a, t, mt, nt, z);
      const int row = mt * TM + (int)rank * 128 + quarter * 32;
      bool many = a.low_after;
      if (a.low.G && !a.low.dense) {
        Groups<TM> gr;
        gr.begin(a.low.adapter, a.low.tokens, a.low.G, (int64_t)mt * TM, lane);
        many = gr.more_than(kFewAdapters);
      }
      // narrow tiles: the low-rank product while the MMAs run
      float ahead[32];
      bool have = false;
      if constexpr (Epi::kEarly)
        if (a.bn <= 64 && half * 32 < a.bn) have = epi.ahead(row, nt * a.bn + half * 32, lane, ahead);
      // what the epilogue reads of the tile's rows and columns, before its sums are there
      typename Epi::Head head;
      epi.load(row, nt * a.bn + half * 32, a.bn - half * 32, lane, head);
      uint32_t src = 0;
      auto open = [&]() {
        ok = ptx::mbar_wait(acc_full + 8 * (n & 1), (uint32_t)((n >> 1) & 1), abort_s, kWaitLimit);
        ok = __all_sync(0xffffffffu, ok);
        ptx::tc_fence_after();
        src = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(n & 1) * acc_stride;
      };
      auto close = [&]() {
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (CG == 2)
            ptx::mbar_arrive_cluster(lead_empty + 8 * (n & 1));
          else
            ptx::mbar_arrive(acc_empty + 8 * (n & 1));
        }
        ++n;
      };
      if constexpr (DRAIN) {
        constexpr int kParts = CG == 2 ? 4 : 2;  // bn <= 128 CG
        float sum[kParts][32];
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
          for (int j = 0; j < 32; ++j) sum[i][j] = 0.f;
        for (int c0 = 0; c0 < chunks; c0 += a.block) {
          open();
          if (!ok) break;
#pragma unroll
          for (int i = 0; i < kParts; ++i) {
            if (half * 32 + 64 * i >= a.bn) break;
            uint32_t v[32];
            ptx::tmem_ld32(src + half * 32 + 64 * i, v);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) sum[i][j] += __uint_as_float(v[j]);
          }
          close();
        }
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
          const int c = half * 32 + 64 * i;
          if (c >= a.bn) break;
          uint32_t v[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(sum[i][j]);
          epi.store(row, nt * a.bn + c, z, lane, many, mine, v, head, i);
        }
      } else {
        open();
        if (!ok) break;
#pragma unroll 1
        for (int i = 0, c = half * 32; c < a.bn; c += 64, ++i) {
          uint32_t v[32];
          ptx::tmem_ld32(src + c, v);
          ptx::tmem_wait_ld();
          if constexpr (Epi::kEarly)
            if (have) {
#pragma unroll
              for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) + ahead[j]);
            }
          epi.store(row, nt * a.bn + c, z, lane, many && !have, mine, v, head, i);
        }
        close();
      }
    }
  }
  __syncthreads();
  if (*abort_s) {
    // copies this CTA has issued end long before this does
    const long long t0 = clock64();
    while (clock64() - t0 < (1LL << 23)) {
    }
    if (threadIdx.x == 0) atomicAdd(a.errors, 1ull);
    __syncthreads();
  }
  ptx::tc_fence_after();
  if (CG == 2) ptx::cluster_sync();
  if (warp == 1) {
    if (CG == 2)
      ptx::tmem_dealloc_pair(tmem, cols);
    else
      ptx::tmem_dealloc(tmem, cols);
  }
}

// ---------------------------------------------------------------- host side
EncodeTiledFn encoder();
int num_sms();
// The current device's counter of expired waits.
unsigned long long* error_counter();

// A 16-bit tensor of `planes` x rows x cols, row stride ld elements and plane
// stride `plane` elements (both multiples of 8, the base 16-byte aligned).
struct Tensor {
  const void* base;
  int64_t cols, rows, planes, ld, plane;
};
// Its map with a box of 64 x box_rows (128-byte swizzle), or of 32 x box_rows
// (64-byte swizzle).
CUtensorMap tensor_map(const Tensor& t, int box_rows, int box_cols = 64);
inline bool mappable(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; }

inline Seg segment(int64_t k, uint32_t id) {
  const int chunks = (int)ceil_div(k, kChunk);
  return Seg{chunks, (int)ceil_div(k - (int64_t)(chunks - 1) * kChunk, 16), id};
}

template <int CG, int PLANES, bool DRAIN, typename Epi>
void launch_as(const Maps& maps, Args a, const Epi& epi, cudaStream_t s) {
  const int half = PLANES * (a.a_rows + a.bn / CG) * 128, stage = kHalves<Epi> * half;
  a.errors = error_counter();
  const int turn = Epi::kTurns ? kEpiWarps * kTurnBytes + 128 : 0;
  // (the MMAs read 128 rows of A's last stage)
  const int past = std::max(0, kABytes - half);
  a.stages = std::min(16, (kSmem - 1024 - 640 - turn - past) / stage);
  const int smem = 1024 + a.stages * stage + 640 + turn + past;
  allow_smem(reinterpret_cast<const void*>(k_mma<CG, PLANES, DRAIN, Epi>), kSmem);
  const int64_t per = a.sym ? (int64_t)a.m_tiles * (a.m_tiles + 1) / 2 : (int64_t)a.m_tiles * a.n_tiles;
  const int64_t tiles = per * a.batches;
  LC_REQUIRE(tiles < (1LL << 31), LIPCACHE_E_INVALID, "too many tiles");
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(CG * std::min<int64_t>(tiles, num_sms() / CG)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CG;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CG == 2 ? 2 : 1;
  LC_CUDA(cudaLaunchKernelEx(&cfg, k_mma<CG, PLANES, DRAIN, Epi>, maps, a, epi));
  LC_LAUNCH_CHECK("k_mma");
}
template <int CG, int PLANES, typename Epi>
void launch(const Maps& maps, const Args& a, const Epi& epi, cudaStream_t s) {
  if constexpr (PLANES == 2) {
    if (a.seg.chunks > a.block) return launch_as<CG, PLANES, true>(maps, a, epi, s);
  }
  launch_as<CG, PLANES, false>(maps, a, epi, s);
}

}  // namespace mma
}  // namespace ops
}  // namespace lc

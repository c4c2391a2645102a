// Products of block-scaled 8-bit matrices for many rows: tiles of 256 columns x 256 rows, shared by a pair of thread blocks on
// neighbouring SMs (tcgen05 cta_group::2), or x 128 rows of one block.
//
// A pair's block loads its own 128 rows of A and half of the B rows, 32 KB for a block of 128 of the reduction, whose MMAs take 512
// cycles; a block alone loads 48 KB.  What bounds both is that the 128 x 256 accumulators of every such block go through the
// registers of eight warps and one FMA each, and beyond that the power limit: 8192^3 runs at 2.02 PFLOP/s, 1.4 GHz and 985 W, and
// without most of the FMAs (a wrong result) at 2.35.  Two accumulators in tensor memory (all 512 columns) let the sums of one block
// run under the MMAs of the next.  Tried and slower or no faster: MMAs of 128 columns
// with four accumulators (575 us instead of 563), sixteen warps of sums (813), runs of factors held in registers (592).
//
// The smaller tile is for groups of rows: half a tile of every group is empty on average.  32 groups of 240 rows, N 2048, K 4096:
// pair 121 us, alone 112; 64 groups of 512 rows through the expert layer, results in 16 bits, 390 and 375; 8192^3 in one group 541 and 580.
//
// Roles in each block: warp 0 copies, warp 1 of the leader issues the MMAs, warps 2 and 3 multiply the scales ahead, warps 4-11 keep
// the scaled sums: a warp has 32 rows x 128 columns, a thread one row, so that all its columns have one factor.
// The gated form takes 128 gate rows and the 128 up rows of the same columns as one B tile, ordered so that a thread holds
// 64 gate sums and the 64 up sums that belong to them; the activation and the quantisation happen in registers.
#include "fp8_mma.cuh"

namespace b2c {

namespace {

constexpr int kEpiWarps = 8;
constexpr int kScaleWarps = 2;
constexpr int kEpiWarp0 = 2 + kScaleWarps;  // first warp of the sums: a whole warpgroup before it
constexpr int kPairThreads = 32 * (kEpiWarp0 + kEpiWarps);
// Registers: 384 threads are launched with 168 each (a quarter of the SM's 65536 holds three warps).  The sums alone are 128 of a
// thread, and 64 values on their way from tensor memory beside them hide its latency: 128 * 88 + 256 * 208 = 384 * 168.
constexpr int kRegsSums = 208, kRegsRest = 88;
constexpr int kABytes = kTileM * kBlock;
constexpr int kBoxBytes = 32 * 128;  // results of a warp on their way out: 32 rows of 128 bytes
// CTAS thread blocks share a tile of CTAS * 128 rows and TN columns (see the head of this file).
template <int CTAS, int TN>
struct TileShape {
  static constexpr int kRows = CTAS * kTileM;
  static constexpr int kBRows = TN / CTAS;  // B rows that a block brings, in boxes of
  static constexpr int kBoxRows = kBRows < kTileM ? kBRows : kTileM;
  static constexpr int kBBytes = kBRows * kBlock;
  static constexpr int kStages = CTAS == 1 ? 3 : (TN == 256 ? 5 : 7);
  static constexpr int kBufs = 512 / TN;       // accumulators in tensor memory
  static constexpr int kWarpCols = TN / 2;     // accumulator columns of a warp of sums
  static constexpr int kColBlocks = TN / kBlock;
  static constexpr int kSmem = 1024 + kStages * (kABytes + kBBytes) + kEpiWarps * kBoxBytes;
};
constexpr int kRun = 4;       // blocks of the reduction whose scales are fetched together
constexpr int kRunSlots = 3;  // runs of factors in shared memory
constexpr int kBand = 8;  // row tiles that are walked together, so that their columns' B tiles are read from L2

__device__ __forceinline__ void tma_pair_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar, uint32_t on) {
  asm volatile(
      "{\n.reg .pred q;\nsetp.ne.b32 q, %6, 0;\n"
      "@q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], "
      "[%5];\n}" ::"r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar), "r"(on)
      : "memory");
}

// Arrival on a barrier of the leader that hands back accumulator columns.  What it orders are reads of tensor memory, and
// these have ended (tcgen05.wait::ld): no write of this thread has to be seen by the other side.  With .release, at
// cluster scope, every arrival waited for the thread's loads of scales under way (2100 of the 2500 cycles of a block).
__device__ __forceinline__ void mbar_arrive_cluster_relaxed(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// Row tiles of all groups; called by a whole warp.
__device__ __forceinline__ int count_row_tiles(const MatmulArgs& a, int tile) {
  if (a.offsets == nullptr) return (a.rows + tile - 1) / tile;
  const int lane = threadIdx.x & 31;
  int run = max(0, min(a.offsets[0], a.rows)), all = 0;
  for (int g0 = 0; g0 < a.groups; g0 += 32) {
    int hi = g0 + lane < a.groups ? max(0, min(a.offsets[g0 + lane + 1], a.rows)) : 0;
    hi = max(hi, run);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, hi, d);
      if (lane >= d) hi = max(hi, v);
    }
    int lo = __shfl_up_sync(0xffffffffu, hi, 1);
    if (lane == 0) lo = run;
    all += __reduce_add_sync(0xffffffffu, (hi - lo + tile - 1) / tile);
    run = __shfl_sync(0xffffffffu, hi, 31);
  }
  return all;
}

struct PairTile {
  int group, row0, row_end, nt;
};
// Tile t of the walk: without groups bands of kBand row tiles, column by column; with groups row tile by row tile.
template <int CTAS>
__device__ __forceinline__ PairTile pair_tile(const MatmulArgs& a, int t, int row_tiles, int n_tiles) {
  PairTile p;
  int mt;
  if (a.offsets == nullptr) {
    const int band = t / (kBand * n_tiles);
    const int in = t - band * kBand * n_tiles;
    const int height = min(kBand, row_tiles - band * kBand);
    p.nt = in / height;
    mt = band * kBand + in - p.nt * height;
  } else {
    mt = t / n_tiles;
    p.nt = t - mt * n_tiles;
  }
  const RowTile r = find_row_tile(a, mt, CTAS * kTileM);
  p.group = r.group;
  p.row0 = r.row0;
  p.row_end = r.row_end;
  return p;
}

// A box of results in shared memory (32 rows of 128 bytes, swizzled) to rows of any alignment; called by a whole warp.  Rows one after
// another, neighbouring lanes neighbouring columns; 16-bit results in words where a row starts on an odd one too.
// (Two-byte stores of a row a lane, 32 lines an instruction, made a product of 762 x 3937 x 608 take 46 us.)
template <typename T>
__device__ __forceinline__ void store_box(T* y, long long ldy, uint32_t box, int rows, int cols, bool wide, int lane) {
  constexpr int kPer = 16 / (int)sizeof(T);
  if (wide) {  // rows on the 16-byte grid, but not all of them: eight lanes a row
    const int c = lane & 7;
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += 4) {
      const int r = r0 + (lane >> 3);
      uint4 w;
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                   : "r"(box + (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)))
                   : "memory");
      T* dst = y + r * ldy + c * kPer;
      if (r < rows && c * kPer + kPer <= cols) {
        *reinterpret_cast<uint4*>(dst) = w;
      } else if (r < rows) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (c * kPer + i < cols) {
            if constexpr (sizeof(T) == 4) reinterpret_cast<uint32_t*>(dst)[i] = u[i];
            else reinterpret_cast<uint16_t*>(dst)[i] = (uint16_t)(u[i >> 1] >> (16 * (i & 1)));
          }
      }
    }
    return;
  }
  for (int r = 0; r < rows; ++r) {
    T* dst = y + r * ldy;
    const uint32_t line = box + (uint32_t)(r * 128);
    auto at = [&](int byte) { return line + (uint32_t)((((byte >> 4) ^ (r & 7)) << 4) | (byte & 15)); };
    if constexpr (sizeof(T) == 4) {
      uint32_t w;
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at(4 * lane)) : "memory");
      if (lane < cols) reinterpret_cast<uint32_t*>(dst)[lane] = w;
    } else {
      auto load = [&](int e) {
        uint16_t h;
        asm volatile("ld.shared.b16 %0, [%1];" : "=h"(h) : "r"(at(2 * e)) : "memory");
        return (uint32_t)h;
      };
      auto one = [&](int e, uint32_t h) {
        if (e >= 0 && e < cols) reinterpret_cast<uint16_t*>(dst)[e] = (uint16_t)h;
      };
      const int odd = (int)(reinterpret_cast<uintptr_t>(dst) >> 1) & 1;
      const int e = 2 * lane - odd;  // this lane's word: elements e and e + 1
      const uint32_t lo = load(max(e, 0)), hi = load(e + 1);
      if (e >= 0 && e + 1 < cols) {
        *reinterpret_cast<uint32_t*>(dst + e) = lo | (hi << 16);
      } else {
        one(e, lo);
        one(e + 1, hi);
      }
      if (odd && lane == 31) one(63, load(63));
    }
  }
}

template <int CTAS, int TN, bool GATED, typename YT>
__global__ void __launch_bounds__(kPairThreads, 1)
    matmul_pair_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
                       const __grid_constant__ CUtensorMap tmap_y, const MatmulArgs a, const bool y_boxes) {
  using S = TileShape<CTAS, TN>;
  static_assert(!GATED || TN == 256, "a block of 128 columns is gate and up");
  constexpr int kStages = S::kStages, kBBytes = S::kBBytes;
  extern __shared__ uint8_t smem_raw[];
  __shared__ SharedCtl ctl;
  __shared__ int row_tiles_s;
  // products of a row's scale and a column block's: [slot][block of the run][column block][row]
  __shared__ float factor[kRunSlots][kRun][2][kTileM];
  __shared__ PairTile run_tile[kRunSlots];  // the tile that a run belongs to
  __shared__ __align__(8) unsigned long long factor_full[kRunSlots], factor_empty[kRunSlots];
  __shared__ float row_max[2][2][kTileM];  // gated: largest magnitude of a row's halves, by tile parity

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t rank = CTAS == 2 ? cluster_ctarank() : 0u;  // 0: leader (issues the MMAs), 1: peer
  const int pair_id = (int)blockIdx.x / CTAS, num_pairs = (int)gridDim.x / CTAS;
  const uint32_t a_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t b_base = a_base + kStages * kABytes;
  const uint32_t box_base = b_base + kStages * kBBytes;

  if (warp == 0) {
    if (lane < kStages) {
      // full[] is used in the leader only: one arrival (its producer) plus the bytes of both blocks
      mbar_init(smem_u32(&ctl.full[lane]), 1);
      mbar_init(smem_u32(&ctl.empty[lane]), 1);
    }
    if (lane == 8) {
      for (int b = 0; b < S::kBufs; ++b) {
        mbar_init(smem_u32(&ctl.tmem_full[b]), 1);
        mbar_init(smem_u32(&ctl.tmem_empty[b]), CTAS * kEpiWarps);  // the warps of sums of both blocks
      }
      for (int b = 0; b < kRunSlots; ++b) {
        mbar_init(smem_u32(&factor_full[b]), kScaleWarps);
        mbar_init(smem_u32(&factor_empty[b]), kEpiWarps);
      }
      ctl.abort_flag = 0;
    }
    if (lane == 9) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_a) : "memory");
    if (lane == 10) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_b) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (CTAS == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl.tmem_base)), "r"(512) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl.tmem_base)), "r"(512) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  pdl_wait();
  if (warp == 2) {
    const int n = count_row_tiles(a, S::kRows);
    if (lane == 0) row_tiles_s = n;
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  // the other block's barriers must be initialised before anything arrives on them
  if (CTAS == 2) cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_acc = __shfl_sync(0xffffffffu, ctl.tmem_base, 0);
  const int row_tiles = row_tiles_s;
  const int cols = GATED ? kBlock : TN;  // output columns of a tile
  const int n_tiles = (a.N + cols - 1) / cols;
  const int tiles = row_tiles * n_tiles;     // (fits: checked by the host)
  const int kb_all = (int)blocks_of(a.K);

  if (warp < kEpiWarp0) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRest));
  if (warp == 0) {
    // ---------------------------------------------------------------- copies (both blocks)
    const uint32_t on = elect_one() ? 1u : 0u;
    int s = 0;
    uint32_t ph = 0;
    bool alive = true;
    for (int t = pair_id; t < tiles && alive; t += num_pairs) {
      const PairTile p = pair_tile<CTAS>(a, t, row_tiles, n_tiles);
      const int m = p.row0 + (int)rank * kTileM;
      for (int kb = 0; kb < kb_all; ++kb) {
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.empty[s]), ph ^ 1u, &ctl, &g_fp8_status))) {
          alive = false;
          break;
        }
        const uint32_t full = CTAS == 2 ? map_to_rank(smem_u32(&ctl.full[s]), 0u) : smem_u32(&ctl.full[s]);
        if (rank == 0) mbar_arrive_expect_tx(smem_u32(&ctl.full[s]), (uint32_t)CTAS * (kABytes + kBBytes), on);
        const uint32_t dst = b_base + s * kBBytes;
        auto load_b = [&](int part, int n, int plane) {
          if constexpr (CTAS == 2) tma_pair_load_3d(dst + part, &tmap_b, kb * kBlock, n, plane, full, on);
          else tma_load_3d(dst + part, &tmap_b, kb * kBlock, n, plane, full, on);
        };
        if constexpr (CTAS == 2) tma_pair_load_2d(a_base + s * kABytes, &tmap_a, kb * kBlock, m, full, on);
        else tma_load_2d(a_base + s * kABytes, &tmap_a, kb * kBlock, m, full, on);
        if (GATED) {
          // a warp's 128 accumulator columns: 64 gate columns and the up columns of the same 64
#pragma unroll
          for (int i = 0; i < S::kBRows / 64; ++i) load_b(i * 64 * kBlock, p.nt * kBlock + ((int)rank * S::kBRows / 128 + (i >> 1)) * 64, 2 * p.group + (i & 1));
        } else {
#pragma unroll
          for (int i = 0; i < S::kBRows / S::kBoxRows; ++i)
            load_b(i * S::kBoxRows * kBlock, p.nt * TN + (int)rank * S::kBRows + i * S::kBoxRows, p.group);
        }
        if (++s == kStages) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issue (leader)
    if (rank == 0) {
      const uint32_t on = elect_one() ? 1u : 0u;
      const uint32_t idesc = make_idesc_f8(S::kRows, TN, a.a_type, a.b_type);
      int s = 0, buf = 0;
      uint32_t ph = 0, bph = 0;
      bool alive = true;
      for (int t = pair_id; t < tiles && alive; t += num_pairs) {
        for (int kb = 0; kb < kb_all; ++kb) {
          if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.full[s]), ph, &ctl, &g_fp8_status)) ||
              !__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.tmem_empty[buf]), bph ^ 1u, &ctl, &g_fp8_status))) {
            alive = false;
            break;
          }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const int ksteps = min(4, (a.K - kb * kBlock + kMmaK - 1) / kMmaK);
          mma_f8_block<CTAS>(tmem_acc + buf * TN, make_smem_desc(a_base + s * kABytes, kBlock), make_smem_desc(b_base + s * kBBytes, kBlock), idesc,
                          on, ksteps);
          if constexpr (CTAS == 2) {
            mma_commit_pair(smem_u32(&ctl.empty[s]), on);
            mma_commit_pair(smem_u32(&ctl.tmem_full[buf]), on);
          } else {
            mma_commit(smem_u32(&ctl.empty[s]), on);
            mma_commit(smem_u32(&ctl.tmem_full[buf]), on);
          }
          if (++s == kStages) {
            s = 0;
            ph ^= 1u;
          }
          if (++buf == S::kBufs) {
            buf = 0;
            bph ^= 1u;
          }
        }
      }
    }
    pdl_launch_dependents();
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- scales (both blocks)
    // They also find the tiles: the warps of sums, which have no time for that, read them beside the first factors.
    // A thread has two rows.  The loads of a run are under way while the run before it is multiplied and handed over.
    const int st = (int)threadIdx.x - 64;
    const int nb = (int)blocks_of(a.N);
    int slot = 0;
    uint32_t sph = 0;
    bool alive = true;
    for (int t = pair_id; t < tiles && alive; t += num_pairs) {
      const PairTile p = pair_tile<CTAS>(a, t, row_tiles, n_tiles);
      const float* sa[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
        sa[h] = a.a_scale + min((long long)p.row0 + (int)rank * kTileM + st + 64 * h, (long long)a.rows - 1) * a.lds;
      // the two column blocks: gate and up, or the two of the tile (past the end: the last one again)
      const float* sb[2];
#pragma unroll
      for (int c = 0; c < 2; ++c)
        sb[c] = a.b_scale + (GATED ? (long long)(2 * p.group + c) * nb + p.nt : (long long)p.group * nb + min(p.nt * S::kColBlocks + c % S::kColBlocks, nb - 1)) * kb_all;
      float na[2][kRun], ncol[2][kRun];
      auto fetch = [&](int kb) {
#pragma unroll
        for (int i = 0; i < kRun; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            na[h][i] = kb + i < kb_all ? sa[h][kb + i] : 0.0f;
            ncol[h][i] = kb + i < kb_all ? sb[h][kb + i] : 0.0f;
          }
      };
      fetch(0);
      for (int kb = 0; kb < kb_all; kb += kRun) {
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&factor_empty[slot]), sph ^ 1u, &ctl, &g_fp8_status))) {
          alive = false;
          break;
        }
#pragma unroll
        for (int i = 0; i < kRun; ++i)
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) factor[slot][i][c][st + 64 * h] = na[h][i] * ncol[c][i];
        if (st == 0) run_tile[slot] = p;
        fetch(kb + kRun);
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&factor_full[slot]));
        if (++slot == kRunSlots) {
          slot = 0;
          sph ^= 1u;
        }
      }
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSums));
    // ---------------------------------------------------------------- scaled sums and results (both blocks)
    const int quad = warp & 3;         // lanes of tensor memory this warp may read
    const int half = (warp - kEpiWarp0) >> 2;  // its columns
    const uint32_t leader_empty = CTAS == 2 ? map_to_rank(smem_u32(&ctl.tmem_empty[0]), 0u) : smem_u32(&ctl.tmem_empty[0]);
    const uint32_t taddr0 = tmem_acc + ((uint32_t)(quad * 32) << 16) + (uint32_t)(half * S::kWarpCols);
    const int in_tile = quad * 32 + lane;
    int slot = 0;
    uint32_t sph = 0;
    int buf = 0, parity = 0;
    uint32_t bph = 0;
    bool ok = true;
    for (int t = pair_id; t < tiles; t += num_pairs, parity ^= 1) {
      PairTile p = {0, 0, 0, 0};
      f32x2 acc[S::kWarpCols / 2];
#pragma unroll
      for (int i = 0; i < S::kWarpCols / 2; ++i) acc[i] = 0;
      // Factors of block kb; read while the block before it is added, so that neither the barrier's nor the memory's latency is waited for.
      float f = 0.0f, fu = 0.0f;
      auto next_factor = [&](int kb) {
        const int i = kb % kRun;
        if (i == 0) ok = ok && __all_sync(0xffffffffu, mbar_wait_inline(smem_u32(&factor_full[slot]), sph, &ctl, &g_fp8_status));
        f = factor[slot][i][GATED || S::kColBlocks == 1 ? 0 : half][in_tile];
        if (GATED) fu = factor[slot][i][1][in_tile];
        if (kb == 0) p = run_tile[slot];
        if (i == kRun - 1 || kb == kb_all - 1) {
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&factor_empty[slot]));
          if (++slot == kRunSlots) {
            slot = 0;
            sph ^= 1u;
          }
        }
      };
      next_factor(0);
#pragma unroll 1
      for (int kb = 0; kb < kb_all; ++kb) {
        const f32x2 ff = pair_of(f, f), ffu = pair_of(fu, fu);
        // (voted, so that the lanes are together at the warp-wide loads and agree on whether there is a result; a wait that gave up does not
        // leave the loop)
        ok = ok && __all_sync(0xffffffffu, mbar_wait_inline(smem_u32(&ctl.tmem_full[buf]), bph, &ctl, &g_fp8_status));
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t taddr = taddr0 + (uint32_t)(buf * TN);
#pragma unroll
        for (int c = 0; c < S::kWarpCols; c += 64) {
          float v[64];
          tmem_ld64(taddr + c, reinterpret_cast<int32_t*>(v));
          if (c == 0 && kb + 1 < kb_all) next_factor(kb + 1);
          if (c + 64 == S::kWarpCols) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              if constexpr (CTAS == 2) mbar_arrive_cluster_relaxed(leader_empty + 8 * buf);
              else mbar_arrive(leader_empty + 8 * buf);
            }
          }
#pragma unroll
          for (int j = 0; j < 64; j += 2) fma2(&acc[(c + j) / 2], pair_of(v[j], v[j + 1]), GATED && c >= 64 ? ffu : ff);
        }
        if (++buf == S::kBufs) {
          buf = 0;
          bph ^= 1u;
        }
      }
      const long long m = (long long)p.row0 + (int)rank * kTileM + in_tile;
      if constexpr (GATED) {
        float h[64], u[64], mx = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          unpair(acc[i], &h[2 * i], &h[2 * i + 1]);
          unpair(acc[32 + i], &u[2 * i], &u[2 * i + 1]);
        }
#pragma unroll
        for (int i = 0; i < 64; ++i) {
          h[i] = silu(h[i]) * u[i];
          mx = fmaxf(mx, fabsf(h[i]));
        }
        // a block of 128 columns is the two halves of a row: two warps
        row_max[parity][half][in_tile] = mx;
        asm volatile("bar.sync %0, 64;" ::"r"(1 + quad) : "memory");
        const BlockScale s = block_scale<B2C_E4M3>(fmaxf(mx, row_max[parity][half ^ 1][in_tile]));
        if (ok && m < p.row_end) {
          const int n = p.nt * kBlock + half * 64;
          uint8_t* y = (uint8_t*)a.y + m * a.ldy + n;
#pragma unroll
          for (int i = 0; i < 64; i += 16)
            if (n + i < a.N) *reinterpret_cast<uint4*>(y + i) = quantize16<B2C_E4M3>(s, h + i);  // (N and ldy are multiples of 16)
          if (half == 0) a.y_scale[m * a.ldys + p.nt] = s.scale;
        }
      } else {
        const int n = p.nt * TN + half * S::kWarpCols, m0 = p.row0 + (int)rank * kTileM + quad * 32;
        // 128 bytes of each of the warp's 32 rows go to shared memory (16-byte pieces, swizzled as the tensor map says).  From there, if
        // the copy engine can address the result and all 32 rows are this group's, in one copy, which runs beside the next tile (stores
        // from registers took 3200 cycles of a tile of bf16, as long as five blocks of the reduction); else by the lanes.  The copy
        // clips what lies past the last column in steps of 16 bytes: a box that the result ends in at another place is left to the lanes.
        constexpr int kCols = 128 / (int)sizeof(YT);
        const uint32_t box = box_base + (uint32_t)((warp - kEpiWarp0) * kBoxBytes);
#pragma unroll
        for (int i = 0; i < S::kWarpCols; i += kCols) {
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          __syncwarp();
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            constexpr int kPer = 16 / (int)sizeof(YT);
            float v[kPer];
#pragma unroll
            for (int j = 0; j < kPer; j += 2) unpair(acc[(i + c * kPer + j) / 2], &v[j], &v[j + 1]);
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if constexpr (sizeof(YT) == 4) w[j] = __float_as_uint(v[j]);
              else w[j] = pack2<YT>(v[2 * j], v[2 * j + 1]);
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box + (uint32_t)(lane * 128 + ((c ^ (lane & 7)) * 16))), "r"(w[0]),
                         "r"(w[1]), "r"(w[2]), "r"(w[3])
                         : "memory");
          }
          const bool by_copy = y_boxes && m0 + 32 <= p.row_end && (n + i + kCols <= a.N || a.N * (int)sizeof(YT) % 16 == 0);
          if (by_copy) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0 && ok && n + i < a.N) {
              asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(&tmap_y),
                           "r"((n + i) * (int)sizeof(YT)), "r"(m0), "r"(box)
                           : "memory");
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          } else {
            __syncwarp();
            if (ok && n + i < a.N)
              store_box<YT>((YT*)a.y + (long long)m0 * a.ldy + n + i, a.ldy, box, min(32, p.row_end - m0), min(kCols, a.N - n - i), y_boxes, lane);
            __syncwarp();
          }
        }
      }
    }
  }

  // copies of results read shared memory: they end before the block does
  if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");

  // ---------------------------------------------------------------- teardown
  // No block of the pair leaves, or frees tensor memory, while the other may still read its shared memory, arrive on
  // its barriers or write its accumulators.
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (ctl.abort_flag) {
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 50000ull) __nanosleep(1000);
    __syncthreads();
  }
  if (CTAS == 2) cluster_sync();
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if constexpr (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_acc), "r"(512) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_acc), "r"(512) : "memory");
  }
}

template <int CTAS, int TN, bool GATED, typename YT>
int launch_pair(const MatmulArgs& a, cudaStream_t st) {
  using S = TileShape<CTAS, TN>;
  const long long cols = GATED ? kBlock : TN;
  const long long n_tiles = (a.N + cols - 1) / cols;
  const long long row_tiles = a.offsets ? a.rows / S::kRows + std::min(a.groups, a.rows) : (a.rows + S::kRows - 1) / S::kRows;
  if (row_tiles * n_tiles > 0x7FFFFFFFLL - kNumSMs) return B2C_E_UNSUPPORTED;
  CUtensorMap ta, tb, ty;
  int rc = encode_tiled_2d(&ta, a.a, a.K, a.rows, a.rows > 1 ? a.lda : a.K, kBlock, kTileM, kBlock);
  if (rc == B2C_OK)
    rc = encode_tiled_3d(&tb, a.b, a.K, a.N, (uint64_t)a.groups * (GATED ? 2 : 1), a.K, (uint64_t)a.N * a.K, kBlock, GATED ? 64 : S::kBoxRows, kBlock);
  if (rc != B2C_OK) return rc;
  const bool y_boxes = results_by_copy(a);  // (of 128 bytes x 32 rows)
  ty = ta;
  if (y_boxes) rc = encode_tiled_2d(&ty, a.y, (uint64_t)a.N * sizeof(YT), a.rows, (uint64_t)a.ldy * sizeof(YT), 128, 32, 128);
  if (rc != B2C_OK) return rc;
  static std::atomic<unsigned long long> configured{0};
  cudaError_t e = set_max_dynamic_smem_once(configured, (const void*)matmul_pair_kernel<CTAS, TN, GATED, YT>, S::kSmem);
  if (e == cudaSuccess) {
    const int pairs = (int)std::min<long long>(row_tiles * n_tiles, kNumSMs / CTAS);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(CTAS * pairs));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CTAS;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CTAS == 2 ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, matmul_pair_kernel<CTAS, TN, GATED, YT>, ta, tb, ty, a, y_boxes);
  }
  if (e != cudaSuccess) {
    set_last_cuda_error((int)e);
    return B2C_E_CUDA;
  }
  return B2C_OK;
}

template <int CTAS, int TN>
int launch_type(const MatmulArgs& a, cudaStream_t st) {
  if (a.y_type == B2C_F32) return launch_pair<CTAS, TN, false, float>(a, st);
  if (a.y_type == B2C_F16) return launch_pair<CTAS, TN, false, __half>(a, st);
  return launch_pair<CTAS, TN, false, __nv_bfloat16>(a, st);
}

}  // namespace

namespace {

// Cycles by tiles of `tn` columns: the tiles of 128 are for products with fewer tiles than pairs.  A block of the reduction takes them 560
// cycles instead of 850 (4096 x 4096: 512 rows 14.7 and 19.1 us, 768 rows, where they need a second wave, 24.2 and 19.9).
long long tile_cycles(const MatmulArgs& a, int tn) {
  const long long tiles = ((a.N + tn - 1) / tn) * (long long)((a.rows + 2 * kTileM - 1) / (2 * kTileM));
  const long long waves = (tiles + kNumSMs / 2 - 1) / (kNumSMs / 2);
  return waves * ((tn == 128 ? 560 : 850) * blocks_of(a.K) + 4000);
}

}  // namespace

long long pair_cycles(const MatmulArgs& a) { return std::min(tile_cycles(a, 128), tile_cycles(a, 256)); }

int launch_fp8_matmul_pair(const MatmulArgs& a, cudaStream_t st) {
  const int rows = rows_of_a_group(a);
  // Half a tile of every group is empty: 64 rows of a tile of its own, 128 of a pair's, which is 7 % faster a row.  Even at some
  // 800 rows of a group; without groups the pair always.
  if (a.gated) return rows <= 768 ? launch_pair<1, 256, true, uint8_t>(a, st) : launch_pair<2, 256, true, uint8_t>(a, st);
  if (a.offsets) return rows <= 768 ? launch_type<1, 256>(a, st) : launch_type<2, 256>(a, st);
  return tile_cycles(a, 128) < tile_cycles(a, 256) ? launch_type<2, 128>(a, st) : launch_type<2, 256>(a, st);
}

cudaError_t fp8_pair_wait_selftest(cudaStream_t st) { return launch_wait_selftest(st); }

cudaError_t fp8_pair_status(int* status) { return take_status(status); }

}  // namespace b2c

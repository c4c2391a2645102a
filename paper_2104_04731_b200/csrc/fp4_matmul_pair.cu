// Products of 4-bit matrices for many rows: tiles of 256 columns x 256 rows, shared by a pair of thread blocks on neighbouring SMs (tcgen05
// cta_group::2), or x 128 rows of one block.
//
// The tensor core applies the scales and keeps the sums of the whole reduction, so a tile's accumulators are read once, at its end: eight warps
// take them into registers, hand the columns back and turn them into results while the next tile's MMAs run.  8192^3: NV 203 us, 5.4 PFLOP/s, MX 181
// and 6.1 in a short run; one after another for seconds the power limit makes it 244.  What else there is: the copies of scales to tensor
// memory, twelve a stage (NV) beside MMAs of 512 cycles (without them, a wrong result, 190 us), and the drain at a tile's end.
// Tried and slower: copies of a stage's scales issued before the MMAs of the stage before it (240 us), a ring of scales for every stage (256).
//
// With many groups of rows and a long reduction the axes are swapped: the weights are the A operand, and a tile has as many columns as its group has
// rows left, in steps of 32, so that a group's last tile costs what it holds (32 groups, 8192 x 2048 x 4096: 43 us for 47).
//
// Roles in each block: warp 0 copies, warp 1 of the leader carries scales to tensor memory (in both blocks) and issues the MMAs, warp 2
// copies the scales of the A operand and turns them round, warp 3 those of the B operand, which both blocks need for all columns; warps 4-11 take
// results out, 32 rows x half of the columns each.  The gated form takes 128 gate rows and the 128 up rows of the same columns as one B tile: a
// thread reads both parts of its columns, so activation and quantisation happen in registers.
#include "fp4_mma.cuh"

namespace b2c {

namespace {

constexpr int kEpiWarps = 8;
constexpr int kEpiWarp0 = 4;
constexpr int kPairThreads = 32 * (kEpiWarp0 + kEpiWarps);
// 384 threads are launched with 168 registers each; a thread of the results holds 128 sums: 128 * 88 + 256 * 208 = 384 * 168.
constexpr int kRegsSums = 208, kRegsRest = 88;
constexpr int kABytes = kTileM * kStageRow;
constexpr int kBoxRow = 64;
constexpr int kBoxBytes = 32 * kBoxRow;  // results of a warp on their way out: 32 rows
constexpr int kGateBytes = 32 * 32 * 4;  // 32 values of every lane of a warp: gated, in the place of the boxes
constexpr int kGroups = 2;               // groups of scales in shared memory
// Which operand has the accumulator's rows.  The rows of a, and a tile's columns are rows of b; gated, 128 gate rows and the 128 up rows of the same
// columns.  Or the weights (groups): the rows of a group are the tile's columns then, as many of them, in steps of 32, as there are.
enum Form { kRowsFirst, kGated, kWeightsFirst };
constexpr int kTokenBox = 32;  // rows of a copy where their number varies
// CTAS thread blocks share a tile of CTAS * 128 rows and TN columns.
template <int CTAS, int TN>
struct TileShape4 {
  static constexpr int kRows = CTAS * kTileM;
  static constexpr int kBRows = TN / CTAS;  // B rows that a block brings, in boxes of
  static constexpr int kBoxRows = kBRows < kTileM ? kBRows : kTileM;
  static constexpr int kBBytes = kBRows * kStageRow;
  static constexpr int kColTiles = TN / kTileM;                      // of 128 columns
  static constexpr int kScaleBytes = (1 + kColTiles) * kGroupTile;   // of a group: the block's A rows, all B rows
  static constexpr int kStages = CTAS == 1 ? (TN == 256 ? 3 : 5) : (TN == 256 ? 5 : 7);
  static constexpr int kBufs = TN == 256 ? 1 : 2;  // accumulators in tensor memory, beside the scales of two stages
  static constexpr int kScaleCols = 16 * (1 + kColTiles);
  static constexpr int kWarpCols = TN / 2;  // accumulator columns of a warp of results
  static constexpr int kSmem = 1024 + kStages * (kABytes + kBBytes) + kGroups * kScaleBytes + kEpiWarps * kBoxBytes;
  static_assert(kSmem <= 226 * 1024, "shared memory, some static beside it");
  static_assert(kBufs * TN + 2 * kScaleCols <= 512, "tensor memory");
};

// Arrival on a barrier of the leader that says that scales in this block's shared memory are in place.  Who reads them is this block's own tensor
// core (a copy for the pair takes each block's part from its own memory), so the release is to this block and the signal alone goes to the other.
// (Released to the cluster, the arrival took 1400 cycles of a stage's 2000: 8192^3 468 us instead of 227.)
__device__ __forceinline__ void mbar_arrive_leader(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cta.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

template <int CTAS, int TN, int FORM, typename YT>
__global__ void __launch_bounds__(kPairThreads, 1)
    matmul4_pair_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_as, const __grid_constant__ CUtensorMap tmap_b,
                        const __grid_constant__ CUtensorMap tmap_bs, const __grid_constant__ CUtensorMap tmap_y, const Matmul4Args a, const bool y_boxes) {
  using S = TileShape4<CTAS, TN>;
  constexpr bool TURNED = FORM == kWeightsFirst, GATED = FORM == kGated;
  static_assert(!TURNED || (CTAS == 2 && TN == 256), "pairs");
  static_assert(!GATED || (CTAS == 1 && TN == 256), "a block of 128 columns is gate and up");
  constexpr int kStages = S::kStages, kBBytes = S::kBBytes;
  extern __shared__ uint8_t smem_raw[];
  __shared__ SharedCtl ctl;
  __shared__ __align__(8) unsigned long long scales_full[2][kGroups];  // a group's scales have come: of the A rows, of the B rows (each block its own)
  __shared__ __align__(8) unsigned long long turned[kGroups];          // and are in place in all blocks (the leader's)
  __shared__ __align__(8) unsigned long long scales_empty[kGroups];
  __shared__ int row_tiles_s;

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t rank = CTAS == 2 ? cluster_ctarank() : 0u;  // 0: leader (issues the MMAs), 1: peer
  const int pair_id = (int)blockIdx.x / CTAS, num_pairs = (int)gridDim.x / CTAS;
  const uint32_t a_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t b_base = a_base + kStages * kABytes;
  const uint32_t s_base = b_base + kStages * kBBytes;
  const uint32_t box_base = s_base + kGroups * S::kScaleBytes;

  if (warp == 0) {
    if (lane < kStages) {
      // full[] is used in the leader only: one arrival (its producer) plus the bytes of both blocks
      mbar_init(smem_u32(&ctl.full[lane]), 1);
      mbar_init(smem_u32(&ctl.empty[lane]), 1);
    }
    if (lane < kGroups) {
      mbar_init(smem_u32(&scales_full[0][lane]), 1);
      mbar_init(smem_u32(&scales_full[1][lane]), 1);
      mbar_init(smem_u32(&turned[lane]), 2 * CTAS);
      mbar_init(smem_u32(&scales_empty[lane]), 1);
    }
    if (lane == 8) {
      for (int b = 0; b < S::kBufs; ++b) {
        mbar_init(smem_u32(&ctl.tmem_full[b]), 1);
        mbar_init(smem_u32(&ctl.tmem_empty[b]), CTAS * kEpiWarps);
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
  const uint32_t tmem_scales = tmem_acc + S::kBufs * TN;
  const int row_tiles = row_tiles_s;
  const int cols = GATED ? kTileM : TN;  // output columns of a tile
  const int n_tiles = (a.N + cols - 1) / cols;
  const int tiles = row_tiles * n_tiles;  // (fits: checked by the host)
  const int kb_all = (a.K + kFp4Stage - 1) / kFp4Stage;

  // rows first: a tile's columns, 128 at a time: row of the B matrix, and which matrix
  auto b_row = [&](const PairTile& p, int i) { return GATED ? p.nt * kTileM : p.nt * TN + i * kTileM; };
  auto b_plane = [&](const PairTile& p, int i) { return GATED ? 2 * p.group + i : p.group; };
  // weights first: rows of a tile, which are columns of the MMA
  auto width_of = [&](const PairTile& p) { return (min(S::kRows, p.row_end - p.row0) + kTokenBox - 1) / kTokenBox * kTokenBox; };

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
        const int per = width_of(p) / 2, boxes = (per + kTokenBox - 1) / kTokenBox, token0 = p.row0 + (int)rank * per;  // (of each block)
        for (int kb = 0; kb < kb_all; ++kb) {
          if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.empty[s]), ph ^ 1u, &ctl, &g_wait_status))) {
            alive = false;
            break;
          }
          const uint32_t full = CTAS == 2 ? map_to_rank(smem_u32(&ctl.full[s]), 0u) : smem_u32(&ctl.full[s]);
          const uint32_t dst = b_base + s * kBBytes;
          if constexpr (TURNED) {
            if (rank == 0) mbar_arrive_expect_tx(smem_u32(&ctl.full[s]), 2u * (kABytes + (uint32_t)(boxes * kTokenBox * kStageRow)), on);
            const int n = p.nt * TN + (int)rank * kTileM;
            tma_pair_load_3d(a_base + s * kABytes, &tmap_b, kb * kStageRow, n, p.group, full, on);
            for (int i = 0; i < boxes; ++i) tma_pair_load_2d(dst + i * kTokenBox * kStageRow, &tmap_a, kb * kStageRow, token0 + i * kTokenBox, full, on);
          } else if constexpr (CTAS == 2) {
            if (rank == 0) mbar_arrive_expect_tx(smem_u32(&ctl.full[s]), 2u * (kABytes + kBBytes), on);
            tma_pair_load_2d(a_base + s * kABytes, &tmap_a, kb * kStageRow, m, full, on);
            tma_pair_load_3d(dst, &tmap_b, kb * kStageRow, p.nt * TN + (int)rank * S::kBRows, p.group, full, on);
          } else {
            mbar_arrive_expect_tx(full, kABytes + kBBytes, on);
            tma_load_2d(a_base + s * kABytes, &tmap_a, kb * kStageRow, m, full, on);
#pragma unroll
            for (int i = 0; i < S::kColTiles; ++i) tma_load_3d(dst + i * kTileM * kStageRow, &tmap_b, kb * kStageRow, b_row(p, i), b_plane(p, i), full, on);
          }
          if (++s == kStages) {
            s = 0;
            ph ^= 1u;
          }
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      // ---------------------------------------------------------------- scales to tensor memory, MMA issue (leader)
      if (rank == 0) {
        const uint32_t on = elect_one() ? 1u : 0u;
        auto run = [&](auto format) {
          constexpr int FORMAT = decltype(format)::value;
          int s = 0, g = 0, buf = 0;
          uint32_t ph = 0, gph = 0, bph = 0, ts_at = 0;
          bool alive = true;
          for (int t = pair_id; t < tiles && alive; t += num_pairs) {
            int width = TN;
            if constexpr (TURNED) width = width_of(pair_tile<CTAS>(a, t, row_tiles, n_tiles));
            const uint32_t idesc = make_idesc_f4(S::kRows, width, FORMAT);
            if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.tmem_empty[buf]), bph ^ 1u, &ctl, &g_wait_status))) break;
            for (int kb = 0; kb < kb_all; ++kb) {
              const int in = kb % kGroup;  // stage of the group
              if ((in == 0 && !__all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&turned[g]), gph, &ctl, &g_wait_status))) ||
                  !__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.full[s]), ph, &ctl, &g_wait_status))) {
                alive = false;
                break;
              }
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
              const int ksteps = min(4, (a.K - kb * kFp4Stage + 63) / 64);
              // (copies and MMAs run in the order in which they are issued)
              const uint32_t ts = tmem_scales + ts_at, scales = s_base + g * S::kScaleBytes + (uint32_t)(512 * stage_words(FORMAT) * in);
              ts_at = S::kScaleCols - ts_at;
              copy_scales<CTAS, FORMAT, 512>(ts, scales, 4, on);
#pragma unroll
              for (int i = 0; i < S::kColTiles; ++i)
                if (i * kTileM < width) copy_scales<CTAS, FORMAT, 512>(ts + 16 + 4 * i, scales + (1 + i) * kGroupTile, 4 * S::kColTiles, on);
              mma_f4_stage<CTAS, FORMAT>(tmem_acc + buf * TN, make_smem_desc(a_base + s * kABytes, kStageRow), make_smem_desc(b_base + s * kBBytes, kStageRow), idesc,
                                         ts, ts + 16, 4 * S::kColTiles, kb > 0, on, ksteps);
              if constexpr (CTAS == 2) mma_commit_pair(smem_u32(&ctl.empty[s]), on);
              else mma_commit(smem_u32(&ctl.empty[s]), on);
              if (++s == kStages) {
                s = 0;
                ph ^= 1u;
              }
              if (in == kGroup - 1 || kb == kb_all - 1) {
                if constexpr (CTAS == 2) mma_commit_pair(smem_u32(&scales_empty[g]), on);
                else mma_commit(smem_u32(&scales_empty[g]), on);
                if (++g == kGroups) {
                  g = 0;
                  gph ^= 1u;
                }
              }
            }
            if constexpr (CTAS == 2) mma_commit_pair(smem_u32(&ctl.tmem_full[buf]), on);
            else mma_commit(smem_u32(&ctl.tmem_full[buf]), on);
            if (++buf == S::kBufs) {
              buf = 0;
              bph ^= 1u;
            }
          }
        };
        if (a.format == B2C_MXFP4) run(std::integral_constant<int, B2C_MXFP4>());
        else run(std::integral_constant<int, B2C_NVFP4>());
      }
      pdl_launch_dependents();
      __syncwarp();
    } else {
      // ---------------------------------------------------------------- scales: copied and turned round (both blocks)
      const uint32_t on = elect_one() ? 1u : 0u;
      const int part = warp - 2;  // 0: A rows, 1: B rows
      const uint32_t mine = s_base + part * kGroupTile;
      // the walk of the copies, up to two groups ahead
      int lt = pair_id, lkb = 0, lg = 0;
      PairTile lp = {0, 0, 0, 0};
      auto load_next = [&]() {
        if (lt >= tiles) return;
        if (lkb == 0) lp = pair_tile<CTAS>(a, lt, row_tiles, n_tiles);
        const uint32_t full = smem_u32(&scales_full[part][lg]), dst = mine + lg * S::kScaleBytes;
        const int width = group_row(a.format), x = lkb / kGroup * width;
        mbar_arrive_expect_tx(full, (uint32_t)((part == 0 ? 1 : S::kColTiles) * kTileM * width), on);
        if constexpr (TURNED) {
          if (part == 1) {
#pragma unroll
            for (int i = 0; i < S::kColTiles; ++i) tma_load_2d(dst + i * kGroupTile, &tmap_as, x, lp.row0 + i * kTileM, full, on);
          } else {
            tma_load_3d(dst, &tmap_bs, x, lp.nt * TN + (int)rank * kTileM, lp.group, full, on);
          }
        } else if (part == 0) {
          tma_load_2d(dst, &tmap_as, x, lp.row0 + (int)rank * kTileM, full, on);
        } else {
#pragma unroll
          for (int i = 0; i < S::kColTiles; ++i) tma_load_3d(dst + i * kGroupTile, &tmap_bs, x, b_row(lp, i), b_plane(lp, i), full, on);
        }
        lg ^= 1;
        lkb += kGroup;
        if (lkb >= kb_all) {
          lkb = 0;
          lt += num_pairs;
        }
      };
      static_assert(kGroups == 2, "the places of the walk");
      load_next();
      load_next();
      int g = 0;
      uint32_t ph = 0;
      bool alive = true, first = true;
      for (int t = pair_id; t < tiles && alive; t += num_pairs) {
        for (int kb = 0; kb < kb_all; kb += kGroup) {
          if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&scales_full[part][g]), ph, &ctl, &g_wait_status))) {
            alive = false;
            break;
          }
          turn_group(mine + g * S::kScaleBytes, kTileM, a.format, lane);
          if (part == 1 && S::kColTiles == 2) turn_group(mine + g * S::kScaleBytes + kGroupTile, kTileM, a.format, lane);
          __syncwarp();
          if (lane == 0) {
            if constexpr (CTAS == 2) mbar_arrive_leader(map_to_rank(smem_u32(&turned[g]), 0u));
            else mbar_arrive(smem_u32(&turned[g]));
          }
          g ^= 1;
          // the other place, when the MMAs of its group (the one before) have ended: it was in use for as many turns as `ph` says
          if (!first) {
            if (lt < tiles && !__all_sync(0xffffffffu, mbar_wait(smem_u32(&scales_empty[g]), g == 0 ? ph : ph ^ 1u, &ctl, &g_wait_status))) {
              alive = false;
              break;
            }
            load_next();
          }
          first = false;
          if (g == 0) ph ^= 1u;
        }
      }
      __syncwarp();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSums));
    // ---------------------------------------------------------------- results (both blocks)
    const int quad = warp & 3;                 // lanes of tensor memory this warp may read
    const int half = (warp - kEpiWarp0) >> 2;  // its columns
    const uint32_t leader_empty = CTAS == 2 ? map_to_rank(smem_u32(&ctl.tmem_empty[0]), 0u) : smem_u32(&ctl.tmem_empty[0]);
    const uint32_t taddr0 = tmem_acc + ((uint32_t)(quad * 32) << 16);
    const int in_tile = quad * 32 + lane;
    QuickFactor4 hf = {};
    if constexpr (GATED) hf = quick_factor4(a.y_global, a.format);
    int buf = 0;
    uint32_t bph = 0;
    bool ok = true;
    for (int t = pair_id; t < tiles; t += num_pairs) {
      const PairTile p = pair_tile<CTAS>(a, t, row_tiles, n_tiles);
      const float alpha = alpha_of(a, p.group);
      // (voted, so that the lanes are together at the warp-wide loads; a wait that gave up does not leave the loop)
      ok = ok && __all_sync(0xffffffffu, mbar_wait_inline(smem_u32(&ctl.tmem_full[buf]), bph, &ctl, &g_wait_status));
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      // gated: 64 gate columns, then the up columns of the same 64;  weights first: half of the tile's rows, rounded to 32 (what lies behind
      // them is read and not used)
      const int mine = TURNED ? (width_of(p) / 2 + 31) / 32 * 32 : S::kWarpCols, c0 = half * mine;
      float v[S::kWarpCols];
#pragma unroll
      for (int c = 0; c < S::kWarpCols; c += 64) tmem_ld64(taddr0 + (uint32_t)(buf * TN + (GATED ? half * 64 + c * 2 : c0 + c)), reinterpret_cast<int32_t*>(v + c));
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        if constexpr (CTAS == 2) mbar_arrive_cluster_relaxed(leader_empty + 8 * buf);
        else mbar_arrive(leader_empty + 8 * buf);
      }
      if (++buf == S::kBufs) {
        buf = 0;
        bph ^= 1u;
      }
      if constexpr (GATED) {
        const long long m = (long long)p.row0 + in_tile;
        const int n = p.nt * kTileM + half * 64;
        float low = 0.0f;
#pragma unroll
        for (int i = 0; i < 64; ++i) v[i] *= alpha;
#pragma unroll
        for (int i = 0; i < 64; i += 2) low = min3(low, v[i], v[i + 1]);
        if (__any_sync(0xffffffffu, low < kFarGate)) {
          // Rare, so by short code: 16 columns at a time go through shared memory, where a loop can index them.  (us of 8192 tokens, 4 of 64 experts,
          // 2048 x 1024, and of 2048 tokens, 4 of 32, 1024 x 512: 240 and 47.9; 257 and 54 with such gates in every tile.  The longer form for every
          // value made them 250 and 48.9, a second copy of the 64 beside the first 240 and 49.7, the longer form of one value at a time here 307
          // and 62 with such gates.)
          const uint32_t at = box_base + (uint32_t)((warp - kEpiWarp0) * kGateBytes + lane * 16);
          auto put = [&](int p, const float* u) {
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at + 512 * p), "f"(u[0]), "f"(u[1]), "f"(u[2]), "f"(u[3]) : "memory");
          };
#pragma unroll
          for (int i = 0; i < 64; i += 16) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              put(p, v + i + 4 * p);
              put(4 + p, v + 64 + i + 4 * p);
            }
#pragma unroll 1
            for (int p = 0; p < 4; ++p) {
              const float4 g = ld_shared_f4(at + 512 * p), u = ld_shared_f4(at + 512 * (4 + p));
              const float h[4] = {quick_gated<true>(g.x, u.x * alpha), quick_gated<true>(g.y, u.y * alpha), quick_gated<true>(g.z, u.z * alpha), quick_gated<true>(g.w, u.w * alpha)};
              put(p, h);
            }
#pragma unroll
            for (int p = 0; p < 4; ++p) {
              const float4 h = ld_shared_f4(at + 512 * p);
              v[i + 4 * p] = h.x;
              v[i + 4 * p + 1] = h.y;
              v[i + 4 * p + 2] = h.z;
              v[i + 4 * p + 3] = h.w;
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 64; ++i) v[i] = quick_gated<false>(v[i], v[64 + i] * alpha);
        }
        uint8_t* y = (uint8_t*)a.y + m * a.ldy + n / 2;
        const bool on = ok && m < p.row_end;
#pragma unroll
        for (int c = 0; c < 64; c += 32) {
          float top[2] = {0.0f, 0.0f};
          uint32_t q[4];
#pragma unroll
          for (int i = 0; i < 32; i += 2) top[i >> 4] = max_abs3(top[i >> 4], v[c + i], v[c + i + 1]);
          uint32_t mx[2] = {abs_bits(top[0]), abs_bits(top[1])};
          if (a.format == B2C_MXFP4) mx[0] = mx[1] = max(mx[0], mx[1]);
          Scale4 s[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            s[i] = quick_scale(mx[i], hf, a.format);
            quick_quantise4<16>(s[i], v + c + 16 * i, q + 2 * i);
          }
          if (on && n + c < a.N) {  // (N is a multiple of 32, ldy of 16)
            *reinterpret_cast<uint4*>(y + c / 2) = make_uint4(q[0], q[1], q[2], q[3]);
            uint8_t* ys = a.y_scale + m * a.ldys + (n + c) / fp4_block(a.format);
            if (a.format == B2C_MXFP4) ys[0] = (uint8_t)s[0].code;
            else *reinterpret_cast<uint16_t*>(ys) = (uint16_t)(s[0].code | (s[1].code << 8));  // (ldys is a multiple of 16)
          }
        }
      } else if constexpr (TURNED) {
        // A lane has a column.  Runs of 32 columns (a warp's) of 16 or 32 rows go to shared memory, and from there, as below, by one copy or by the lanes.
        // (Stored from the registers, 128 bytes of a row an instruction, the second product of 8192 tokens, 4 of 64 experts, 2048 x 1024, took 123 us.)
        constexpr int kBoxRows = kBoxBytes / (32 * (int)sizeof(YT));
        const int n = p.nt * TN + (int)rank * kTileM + quad * 32, rows = min(mine, p.row_end - p.row0 - c0), m0 = p.row0 + c0;
        const uint32_t box = box_base + (uint32_t)((warp - kEpiWarp0) * kBoxBytes), here = box + (uint32_t)(lane * (int)sizeof(YT));
#pragma unroll
        for (int i = 0; i < S::kWarpCols; i += kBoxRows) {
          if (i < rows && n < a.N) {
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kBoxRows; j += 2) {
              const float x0 = v[i + j] * alpha, x1 = v[i + j + 1] * alpha;
              if constexpr (sizeof(YT) == 4) {
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(here + (uint32_t)(j * 128)), "f"(x0) : "memory");
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(here + (uint32_t)(j * 128 + 128)), "f"(x1) : "memory");
              } else {
                const uint32_t w = pack2<YT>(x0, x1);
                asm volatile("st.shared.b16 [%0], %1;" ::"r"(here + (uint32_t)(j * 64)), "h"((unsigned short)w) : "memory");
                asm volatile("st.shared.b16 [%0], %1;" ::"r"(here + (uint32_t)(j * 64 + 64)), "h"((unsigned short)(w >> 16)) : "memory");
              }
            }
            if (y_boxes && i + kBoxRows <= rows && (n + 32 <= a.N || a.N * (int)sizeof(YT) % 16 == 0)) {
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0 && ok) {
                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(&tmap_y), "r"(n * (int)sizeof(YT)), "r"(m0 + i), "r"(box)
                             : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
              }
            } else {
              __syncwarp();
              YT* y = (YT*)a.y + (long long)(m0 + i) * a.ldy + n + lane;
              if (ok && n + lane < a.N)
#pragma unroll 4
                for (int j = 0; j < min(kBoxRows, rows - i); ++j, y += a.ldy) {
                  if constexpr (sizeof(YT) == 4) {
                    float x;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(here + (uint32_t)(j * 128)) : "memory");
                    *y = x;
                  } else {
                    unsigned short x;
                    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(x) : "r"(here + (uint32_t)(j * 64)) : "memory");
                    *reinterpret_cast<unsigned short*>(y) = x;
                  }
                }
              __syncwarp();
            }
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < S::kWarpCols; ++i) v[i] *= alpha;
        const int n = p.nt * TN + half * S::kWarpCols, m0 = p.row0 + (int)rank * kTileM + quad * 32;
        // 64 bytes of each of the warp's 32 rows go to shared memory (16-byte pieces, swizzled as the tensor map says).  From there, if
        // the copy engine can address the result and all 32 rows are this group's, in one copy, which runs beside the next tile; else by the
        // lanes.  The copy clips what lies past the last column in steps of 16 bytes: a box that the result ends in at another place is
        // left to the lanes.
        constexpr int kCols = kBoxRow / (int)sizeof(YT);
        const uint32_t box = box_base + (uint32_t)((warp - kEpiWarp0) * kBoxBytes);
#pragma unroll
        for (int i = 0; i < S::kWarpCols; i += kCols) {
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          __syncwarp();
#pragma unroll
          for (int c = 0; c < kBoxRow / 16; ++c) {
            constexpr int kPer = 16 / (int)sizeof(YT);
            const float* u = v + i + c * kPer;
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if constexpr (sizeof(YT) == 4) w[j] = __float_as_uint(u[j]);
              else w[j] = pack2<YT>(u[2 * j], u[2 * j + 1]);
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box + (uint32_t)(lane * kBoxRow + ((c ^ ((lane >> 1) & 3)) * 16))), "r"(w[0]),
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
              store_box<YT, kBoxRow>((YT*)a.y + (long long)m0 * a.ldy + n + i, a.ldy, box, min(32, p.row_end - m0), min(kCols, a.N - n - i), y_boxes, lane);
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

// Whether the copy engine can take a product's results out (see results_by_copy).
bool boxes_of(const Matmul4Args& a, int bytes) {
  return (reinterpret_cast<uintptr_t>(a.y) & 15) == 0 && a.ldy * bytes % 16 == 0 && (long long)a.N * bytes <= 0x7FFFFFFFLL;
}

template <int CTAS, int TN, int FORM, typename YT>
int launch_pair(const Matmul4Args& a, cudaStream_t st) {
  using S = TileShape4<CTAS, TN>;
  constexpr bool TURNED = FORM == kWeightsFirst, GATED = FORM == kGated;
  constexpr int kSmem = S::kSmem + (GATED ? kEpiWarps * (kGateBytes - kBoxBytes) : 0);
  static_assert(kSmem <= 226 * 1024, "shared memory, some static beside it");
  const long long cols = GATED ? kTileM : TN;
  const long long n_tiles = (a.N + cols - 1) / cols;
  const long long row_tiles = a.offsets ? a.rows / S::kRows + std::min(a.groups, a.rows) : (a.rows + S::kRows - 1) / S::kRows;
  if (row_tiles * n_tiles > 0x7FFFFFFFLL - kNumSMs) return B2C_E_UNSUPPORTED;
  const uint64_t bytes = a.K / 2, scales = fp4_scales(a.K, a.format), planes = (uint64_t)a.groups * (GATED ? 2 : 1);
  const int width = group_row(a.format);
  CUtensorMap ta, tas, tb, tbs, ty;
  int rc = encode_tiled_2d(&ta, a.a, bytes, a.rows, a.rows > 1 ? a.lda : bytes, kStageRow, TURNED ? kTokenBox : kTileM, 128);
  if (rc == B2C_OK) rc = encode_tiled_2d(&tas, a.a_scale, scales, a.rows, a.rows > 1 ? a.lds : fp4_scale_pitch(a.K, a.format), width, kTileM, width);
  if (rc == B2C_OK) rc = encode_tiled_3d(&tb, a.b, bytes, a.N, planes, bytes, (uint64_t)a.N * bytes, kStageRow, TURNED ? kTileM : S::kBoxRows, 128);
  if (rc == B2C_OK) rc = encode_tiled_3d(&tbs, a.b_scale, scales, a.N, planes, a.ldbs, (uint64_t)a.N * a.ldbs, width, kTileM, width);
  if (rc != B2C_OK) return rc;
  const bool y_boxes = !GATED && boxes_of(a, (int)sizeof(YT));  // 64 bytes x 32 rows, weights first 32 columns
  const int box_row = TURNED ? 32 * (int)sizeof(YT) : kBoxRow;
  ty = ta;
  if (y_boxes)
    rc = encode_tiled_2d(&ty, a.y, (uint64_t)a.N * sizeof(YT), a.rows, a.rows > 1 ? (uint64_t)a.ldy * sizeof(YT) : ((uint64_t)a.N * sizeof(YT) + 15) / 16 * 16, box_row,
                         kBoxBytes / box_row, TURNED ? 0 : kBoxRow);
  if (rc != B2C_OK) return rc;
  static std::atomic<unsigned long long> configured{0};
  cudaError_t e = set_max_dynamic_smem_once(configured, (const void*)matmul4_pair_kernel<CTAS, TN, FORM, YT>, kSmem);
  if (e == cudaSuccess) {
    const int pairs = (int)std::min<long long>(row_tiles * n_tiles, kNumSMs / CTAS);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(CTAS * pairs));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = kSmem;
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
    e = cudaLaunchKernelEx(&cfg, matmul4_pair_kernel<CTAS, TN, FORM, YT>, ta, tas, tb, tbs, ty, a, y_boxes);
  }
  if (e != cudaSuccess) {
    set_last_cuda_error((int)e);
    return B2C_E_CUDA;
  }
  return B2C_OK;
}

template <int CTAS, int TN, int FORM>
int launch_type(const Matmul4Args& a, cudaStream_t st) {
  if (a.y_type == B2C_F32) return launch_pair<CTAS, TN, FORM, float>(a, st);
  if (a.y_type == B2C_F16) return launch_pair<CTAS, TN, FORM, __half>(a, st);
  return launch_pair<CTAS, TN, FORM, __nv_bfloat16>(a, st);
}

// Nanoseconds by tiles of 128 x 128 on one SM, and by those of 256 x 256 on a pair: the small ones where the large ones are fewer than the pairs.
// Measured, us small / large: 384 x 4096 x 4096 9.2 / 11.6, 300 x 1024 x 8192 12.3 / 16.2, 1000 x 1024 x 1024 5.2 / 7.5,
// 4096 x 512 x 4096 9.3 / 11.5;   768 x 4096 x 4096 13.8 / 12.4, 512 x 8192 x 8192 24.2 / 19.5, 2048 x 2048 x 2048 9.2 / 9.3.
long long small_ns(const Matmul4Args& a) {
  const long long tiles = (long long)((a.N + 127) / 128) * ((a.rows + 127) / 128), kb = (a.K + kFp4Stage - 1) / kFp4Stage;
  const long long waves = (tiles + kNumSMs - 1) / kNumSMs;
  return 4300 + waves * kb * (waves > 1 ? 300 : 250);
}
long long large_ns(const Matmul4Args& a) {
  const long long tiles = (long long)((a.N + 255) / 256) * ((a.rows + 255) / 256), kb = (a.K + kFp4Stage - 1) / kFp4Stage;
  return 5400 + (tiles + kNumSMs / 2 - 1) / (kNumSMs / 2) * (330 * kb + 700);
}

}  // namespace

long long fp4_pair_ns(const Matmul4Args& a) { return std::min(small_ns(a), large_ns(a)); }

int launch_fp4_matmul_pair(const Matmul4Args& a, cudaStream_t st) {
  const int rows = rows_of_a_group(a);
  if (a.gated) return launch_pair<1, 256, kGated, uint8_t>(a, st);
  if (a.offsets) {
    // Half a tile of every group is empty: 64 rows of a tile of its own, 128 of a pair's, 16 of a pair's with the weights first.  That one's results take
    // longer, which shows unless the reduction is long, and its tiles are fewer.  One SM / weights first, us, NV, 32 groups of 128, 256, 512 rows:
    //   K 8192, N 2048: 68.6 / 62.9, 90.4 / 83.5, 142 / 128;
    //   K 4096, N 1024: 26.7 / 23.9, 34.3 / 30.6, 42.5 / 43.1;  N 2048: 38.8 / 38.0, 49.0 / 44.8, 76.4 / 69.1;  N 4096: 66.6 / 65.9, 92.7 / 83.4, 144 / 131;
    //   K 3584, N 1024: 24.9 / 22.0, 26.0 / 28.9, 41.0 / 42.1;  N 2048: 35.4 / 35.8, 43.4 / 43.6, 72.7 / 66.4;  N 4096: 59.2 / 60.9, 83.6 / 78.3, 136 / 124;
    //   K 2560, N 1024: 20.2 / 18.9, 23.3 / 24.5, 33.1 / 33.2;  N 2048: 28.6 / 29.5, 37.0 / 36.0, 56.4 / 52.6;  N 4096: 45.1 / 48.8, 66.2 / 61.4, 104 / 97;
    // and 8 of 256, K 4096, N 2048: 19.6 / 21.4;  32 of 64: 33.9 / 35.7;  16 of 512, K 2048: 25.7 / 26.2.  MX is like it (K 4096, N 2048: 36.7 / 36.2, 47.2 /
    // 42.5, 73.0 / 63.6).  What the rule gives to the weights first loses 2 % at most.  Of the rest, N 1024 would gain 11 % with short groups, and
    // below K 4096 long groups gain up to 9 % and short ones lose as much, by how either form's tiles divide the SMs: one SM stays.  At 240 rows of a group and more the pair with the rows first is within 5 % of one SM either way.
    const long long large = (a.rows / 256 + a.groups / 2) * (long long)((a.N + 255) / 256);  // tiles, about
    if (a.K >= 4096 && rows >= 100 && large >= 3 * (kNumSMs / 2)) return launch_type<2, 256, kWeightsFirst>(a, st);
    return rows <= 768 ? launch_type<1, 256, kRowsFirst>(a, st) : launch_type<2, 256, kRowsFirst>(a, st);
  }
  return small_ns(a) < large_ns(a) ? launch_type<1, 128, kRowsFirst>(a, st) : launch_type<2, 256, kRowsFirst>(a, st);
}

cudaError_t fp4_pair_wait_selftest(cudaStream_t st) { return launch_wait_selftest(st); }

cudaError_t fp4_pair_status(int* status) { return take_status(status); }

}  // namespace b2c

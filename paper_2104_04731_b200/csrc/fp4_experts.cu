// The expert layer of a few tokens in two kernels: rows are quantised, multiplied by gate and up matrices, activated and quantised again in the
// first; multiplied by the second matrix and summed by token in the second.
//
// What there is to do is to read the weights of the experts that have a token, once; everything else is latency, and a launch of its own for the
// sort, the quantisation and the weighted sum costs more than any of them.  So every thread block sorts the pairs (token, slot) for itself, one
// block an SM walks over the items (up to 16 rows of an expert, 128 weight rows), and the copies of weights run ahead over the items' ends.
// The weights are on the accumulator's rows, the tokens are its columns.
//
// First kernel: 64 gate rows and the 64 up rows of the same columns are one tile of weights.  Eight warps quantise the rows of the tile as the
// stages go by, into the place and order that the tensor core reads; every block of an expert does that again, beside its copies.
// Second kernel: its blocks start where those of the first have ended, sort, and fetch weights until all rows are there.  A slot's row goes to
// memory in fp32; the block that finishes the last tile of 128 columns sums them by token, in the order of the slots (no sum depends on who is
// last).
//
// 2048 x 1024, 4 of 64 experts: 16 tokens NV 37 us (145 MB; 22.5 at the rate of a copy), one token MX 13: of these 13 some 1.5 us are the plan, 2 the way
// of the first weights and rows, 2 the MMAs of eight stages, each kernel.
#include "fp4_mma.cuh"

namespace b2c {

namespace {

constexpr int kTileRows = 16;  // tokens of a tile
constexpr int kStages4 = 8;
constexpr int kWBytes = kTileM * kStageRow, kXBytes = kTileRows * kStageRow;
constexpr int kFewStage = kWBytes + kXBytes;
// Scales of 16 rows, turned round: a word of all rows takes 256 bytes, of which the copy to tensor memory reads the next 256 too (lanes of no row).
constexpr int kRowWord = 16 * 16;
constexpr int kRowStage = 1536, kRowGroup = 4608;  // of a stage (first kernel), of a group (second): words of it, and one more
static_assert(4 * kRowWord + kRowWord <= kRowStage && 16 * kRowWord + kRowWord <= kRowGroup && kRowGroup % 512 == 0, "scales of rows");
// Stages, two groups of scales of the weights, scales of the rows.  An SM has room for one block of either kernel.  (With half the stages a block of the
// second stood beside one of the first and fetched weights ahead, but fewer bytes were under way: 32 tokens, 4 of 64 experts, 46 us instead of 43.)
constexpr int kUpSmem = 1024 + kStages4 * kFewStage + 2 * kGroupTile + kStages4 * kRowStage;
constexpr int kDownSmem = 1024 + kStages4 * kFewStage + 2 * kGroupTile + 2 * kRowGroup;
constexpr int kMaxTiles = kFewPairs + kFewPairs / kTileRows;
static_assert(kMaxExperts * (kFewPairs / 32) * 4 <= kStages4 * kFewStage, "the bits of plan_few");
constexpr int kAccCols = kTileRows, kFewScaleCols = 32;  // of a tile; of a stage: weights, rows
constexpr int kFewTmem = 128;                            // two accumulators, scales of two stages

struct FewTile {
  int expert, row0, rows;  // row0: first sorted position
};
// What a block finds out about the pairs.
struct FewPlan {
  int16_t first[kMaxExperts];  // first position of an expert's pairs
  int16_t order[kFewPairs];    // pair at a position
  int16_t place[kFewPairs];    // position of a pair, -1 for none
  FewTile tile[kMaxTiles];
  int tiles;
};

// Sorts the pairs by expert, stably, and cuts each expert's into tiles; called by all threads of a block.  Every expert has a bit for every pair, in
// `bits` (shared memory that nobody else uses yet): setting them needs no order, and a pair's place is the number of bits before its own.
// (One warp that matches ids took 0.3 us for 32 pairs, counting the lower ids for every pair 6 us for 256.)
__device__ __forceinline__ void plan_few(FewPlan& plan, uint32_t* bits, const int32_t* ids, int pairs, int experts) {
  const int words = (pairs + 31) / 32;
  int id[(kFewPairs + 255) / 256];  // of this thread's pairs (256 threads at least)
#pragma unroll
  for (int k = 0; k < (kFewPairs + 255) / 256; ++k) {
    const int p = threadIdx.x + k * blockDim.x;
    id[k] = p < pairs ? ids[p] : -1;
    if (id[k] >= experts) id[k] = -1;
  }
  for (int i = threadIdx.x; i < experts * words; i += blockDim.x) bits[i] = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < (kFewPairs + 255) / 256; ++k) {
    const int p = threadIdx.x + k * blockDim.x;
    if (p < pairs && id[k] >= 0) atomicOr(bits + id[k] * words + p / 32, 1u << (p & 31));
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    int base = 0;  // pairs so far in the lower half, tiles in the upper
#pragma unroll 1
    for (int e0 = 0; e0 < experts; e0 += 32) {
      const int e = e0 + lane;
      int n = 0;
      if (e < experts)
        for (int w = 0; w < words; ++w) n += __popc(bits[e * words + w]);
      if (__ballot_sync(0xffffffffu, n > 0) == 0) continue;  // (no pair refers to them)
      const int own = n | ((n + kTileRows - 1) / kTileRows) << 16;
      int sum = own;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += v;
      }
      const int before = base + sum - own, at = before & 0xFFFF;
      if (e < experts) plan.first[e] = (int16_t)at;
      for (int i = 0; i < own >> 16; ++i) plan.tile[(before >> 16) + i] = {e, at + i * kTileRows, min(kTileRows, n - i * kTileRows)};
      base += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) plan.tiles = base >> 16;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < (kFewPairs + 255) / 256; ++k) {
    const int p = threadIdx.x + k * blockDim.x;
    if (p >= pairs) continue;
    int at = -1;
    if (id[k] >= 0) {
      const uint32_t* mine = bits + id[k] * words;
      at = plan.first[id[k]] + __popc(mine[p / 32] & ((1u << (p & 31)) - 1u));
      for (int w = 0; w < p / 32; ++w) at += __popc(mine[w]);
      plan.order[at] = (int16_t)p;
    }
    plan.place[p] = (int16_t)at;
  }
  // (copies will write to where the bits are)
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncthreads();
}

// Barriers and tensor memory of a block; called by all threads.  `fillers`: warps that fill a stage (the copies' one among them),
// `turners`: warps that put a group's scales in place.
struct FewCtl {
  SharedCtl ctl;
  unsigned long long scales_full[2][2], scales_empty[2], turned[2];  // of a group of scales
};
__device__ __forceinline__ void setup_few(FewCtl& c, int warp, int lane, int fillers, int turners) {
  if (warp == 0) {
    if (lane < kStages4) {
      mbar_init(smem_u32(&c.ctl.full[lane]), fillers);
      mbar_init(smem_u32(&c.ctl.empty[lane]), 1);
    }
    if (lane < 2) {
      mbar_init(smem_u32(&c.ctl.tmem_full[lane]), 1);
      mbar_init(smem_u32(&c.ctl.tmem_empty[lane]), 4);
      mbar_init(smem_u32(&c.scales_full[0][lane]), 1);
      mbar_init(smem_u32(&c.scales_full[1][lane]), 1);
      mbar_init(smem_u32(&c.scales_empty[lane]), 1);
      mbar_init(smem_u32(&c.turned[lane]), turners);
    }
    if (lane == 8) c.ctl.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&c.ctl.tmem_base)), "r"(kFewTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void teardown_few(FewCtl& c, int warp, uint32_t tmem) {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (c.ctl.abort_flag) {
    // copies may still be under way: they land before this block leaves
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 50000ull) __nanosleep(1000);
    __syncthreads();
  }
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kFewTmem) : "memory");
  }
}

// The MMAs of all items of this block; called by warp 1 of either kernel.  row_scales(stage, group's place, stage of the group): where the scales
// of the rows are.
template <int FORMAT, typename F>
__device__ __forceinline__ void mma_few(FewCtl& c, uint32_t smem, uint32_t scales, F row_scales, uint32_t tmem, int items, int kb_all, int K) {
  const uint32_t on = elect_one() ? 1u : 0u;
  const uint32_t idesc = make_idesc_f4(kTileM, kTileRows, FORMAT);
  int s = 0, g = 0, buf = 0;
  uint32_t ph = 0, gph = 0, bph = 0, odd = 0;
  bool alive = true;
  for (int item = blockIdx.x; item < items && alive; item += gridDim.x) {
    if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&c.ctl.tmem_empty[buf]), bph ^ 1u, &c.ctl, &g_wait_status))) break;
    for (int kb = 0; kb < kb_all; ++kb) {
      const int in = kb % kGroup;  // stage of the group
      if ((in == 0 && !__all_sync(0xffffffffu, mbar_wait(smem_u32(&c.turned[g]), gph, &c.ctl, &g_wait_status))) ||
          !__all_sync(0xffffffffu, mbar_wait(smem_u32(&c.ctl.full[s]), ph, &c.ctl, &g_wait_status))) {
        alive = false;
        break;
      }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t base = smem + s * kFewStage, ws = scales + g * kGroupTile + (uint32_t)(512 * stage_words(FORMAT) * in);
      const uint32_t ts = tmem + 2 * kAccCols + odd * kFewScaleCols;
      odd ^= 1u;
      copy_scales<1, FORMAT, 512>(ts, ws, 4, on);
      copy_scales<1, FORMAT, kRowWord>(ts + 16, row_scales(s, g, in), 4, on);
      mma_f4_stage<1, FORMAT>(tmem + buf * kAccCols, make_smem_desc(base, kStageRow), make_smem_desc(base + kWBytes, kStageRow), idesc, ts, ts + 16, 4, kb > 0, on,
                              min(4, (K - kb * kFp4Stage + 63) / 64));
      mma_commit(smem_u32(&c.ctl.empty[s]), on);
      if (++s == kStages4) {
        s = 0;
        ph ^= 1u;
      }
      if (in == kGroup - 1 || kb == kb_all - 1) {
        mma_commit(smem_u32(&c.scales_empty[g]), on);
        g ^= 1;
        if (g == 0) gph ^= 1u;
      }
    }
    mma_commit(smem_u32(&c.ctl.tmem_full[buf]), on);
    buf ^= 1;
    if (buf == 0) bph ^= 1u;
  }
  __syncwarp();
}

// The scales of one operand (0: weights, 1: rows), copied two groups ahead and turned round; called by a warp.  load(item, group of the item, place,
// barrier) issues the copies, turn(place) puts them in order.
template <typename Load, typename Turn>
__device__ __forceinline__ void scales_few(FewCtl& c, int part, int items, int kb_all, int lane, Load load, Turn turn, bool wait_first) {
  int li = blockIdx.x, lgroup = 0, place = 0;
  auto load_next = [&]() {
    if (li >= items) return;
    load(li, lgroup, place, smem_u32(&c.scales_full[part][place]));
    place ^= 1;
    if (++lgroup * kGroup >= kb_all) {
      lgroup = 0;
      li += gridDim.x;
    }
  };
  if (wait_first) pdl_wait();
  load_next();
  load_next();
  int g = 0;
  uint32_t ph = 0;
  bool first = true;
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    for (int kb = 0; kb < kb_all; kb += kGroup) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&c.scales_full[part][g]), ph, &c.ctl, &g_wait_status))) return;
      turn(g);
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&c.turned[g]));
      g ^= 1;
      // the other place, when the MMAs of its group (the one before) have ended
      if (!first && li < items) {
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&c.scales_empty[g]), g == 0 ? ph : ph ^ 1u, &c.ctl, &g_wait_status))) return;
        load_next();
      }
      first = false;
      if (g == 0) ph ^= 1u;
    }
  }
}

// A group's scales of 16 rows, as a copy with the swizzle of their width left them, turned round in place: a word of all rows after another.
__device__ __forceinline__ void turn_rows(uint32_t base, int format, int lane) {
  uint32_t w[16];
  const int r = lane & 15, pieces = format == B2C_MXFP4 ? 2 : 4, x = format == B2C_MXFP4 ? (r >> 2) & 1 : (r >> 1) & 3;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    if (p < pieces)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(w[4 * p]), "=r"(w[4 * p + 1]), "=r"(w[4 * p + 2]), "=r"(w[4 * p + 3])
                   : "r"(base + (uint32_t)(r * 16 * pieces + ((p ^ x) << 4)))
                   : "memory");
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < 4 * pieces && lane < 16) asm volatile("st.shared.b32 [%0], %1;" ::"r"(base + (uint32_t)(kRowWord * i + r * 16)), "r"(w[i]) : "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// Eight neighbouring elements of a row of n as they lie in memory, zeros past its end; widened.
template <typename T>
struct Raw8 {
  uint4 u[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8(const T* row, int at, int n, bool wide) {
  Raw8<T> r = {};
  if (wide && at + 8 <= n) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.u[i] = reinterpret_cast<const uint4*>(row + at)[i];
  } else {
    T* e = reinterpret_cast<T*>(r.u);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at + i < n) e[i] = row[at + i];
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, float* v) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
    const uint32_t w[4] = {r.u[i].x, r.u[i].y, r.u[i].z, r.u[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4) v[4 * i + j] = __uint_as_float(w[j]);
      else unpack2<T>(w[j], &v[2 * j], &v[2 * j + 1]);
    }
  }
}

constexpr int kQuantWarp0 = 8, kQuantWarps = 2 * kStages4, kUpThreads = 32 * (kQuantWarp0 + kQuantWarps);
template <typename T>
__global__ void __launch_bounds__(kUpThreads, 1) experts4_up_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_ws, const Few4Args a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ FewCtl c;
  __shared__ FewPlan plan;
  __shared__ float sums[kTileRows][kTileM];
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t ws = smem + kStages4 * kFewStage, xs0 = ws + 2 * kGroupTile;
  setup_few(c, warp, lane, 1 + kQuantWarps / kStages4, 1);
  if (warp == 0 && lane == 9) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_w) : "memory");
  if (warp == 0 && lane == 10) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_ws) : "memory");
  pdl_wait();
  pdl_launch_dependents();
  Factor4 f = {};  // of what this warp quantises
  QuickFactor4 hf = {};
  if (warp >= kQuantWarp0) f = load_factor4(a.x_global, a.format);
  else if (warp >= 4) hf = quick_factor4(a.h_global, a.format);
  plan_few(plan, reinterpret_cast<uint32_t*>(smem_raw + (smem - smem_u32(smem_raw))), a.ids, a.pairs, a.experts);
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = __shfl_sync(0xffffffffu, c.ctl.tmem_base, 0);
  constexpr int cols = 64;
  const int n_tiles = (a.inter + cols - 1) / cols, items = plan.tiles * n_tiles;
  const int kb_all = (a.hidden + kFp4Stage - 1) / kFp4Stage;
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < (a.hidden + kTileM - 1) / kTileM; i += blockDim.x) a.done[i] = 0;

  if (warp == 0) {
    // ---------------------------------------------------------------- copies of weights
    const uint32_t on = elect_one() ? 1u : 0u;
    int s = 0;
    uint32_t ph = 0;
    bool alive = true;
    for (int item = blockIdx.x; item < items && alive; item += gridDim.x) {
      const int t = item / n_tiles, n0 = (item - t * n_tiles) * cols, plane = 2 * plan.tile[t].expert;
      for (int kb = 0; kb < kb_all; ++kb) {
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&c.ctl.empty[s]), ph ^ 1u, &c.ctl, &g_wait_status))) {
          alive = false;
          break;
        }
        const uint32_t full = smem_u32(&c.ctl.full[s]), dst = smem + s * kFewStage;
        mbar_arrive_expect_tx(full, kWBytes, on);
#pragma unroll
        for (int h = 0; h < 2; ++h) tma_load_3d(dst + h * (kWBytes / 2), &tmap_w, kb * kStageRow, n0, plane + h, full, on);  // gate, up
        if (++s == kStages4) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    auto row_scales = [&](int s, int, int) { return xs0 + (uint32_t)(s * kRowStage); };
    if (a.format == B2C_MXFP4) mma_few<B2C_MXFP4>(c, smem, ws, row_scales, tmem, items, kb_all, a.hidden);
    else mma_few<B2C_NVFP4>(c, smem, ws, row_scales, tmem, items, kb_all, a.hidden);
  } else if (warp == 2) {
    // ---------------------------------------------------------------- scales of weights
    const uint32_t on = elect_one() ? 1u : 0u;
    const int width = group_row(a.format);
    scales_few(
        c, 0, items, kb_all, lane,
        [&](int item, int group, int place, uint32_t full) {
          const int t = item / n_tiles, n0 = (item - t * n_tiles) * cols, plane = 2 * plan.tile[t].expert;
          mbar_arrive_expect_tx(full, (uint32_t)(kTileM * width), on);
#pragma unroll
          for (int h = 0; h < 2; ++h) tma_load_3d(ws + (uint32_t)(place * kGroupTile + h * 64 * width), &tmap_ws, group * width, n0, plane + h, full, on);
        },
        [&](int place) { turn_group(ws + (uint32_t)(place * kGroupTile), kTileM, a.format, lane); }, false);
    __syncwarp();
  } else if (warp >= kQuantWarp0) {
    // ---------------------------------------------------------------- rows
    // A place of the ring has two warps, for its even and its odd rows: the latency of a warp's loads is spread over the stages between.  (A warp
    // sees every phase of its place's barrier; one that skipped some would take an older phase for the one it waits for.)
    const bool wide = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && (a.ldx * (long long)sizeof(T)) % 16 == 0;
    const int all = (items - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x * kb_all;  // (0 where there is no item for this block)
    // It takes two rows at a time, and the two after them, of this stage or of its next one, are on their way.
    const int s = (warp - kQuantWarp0) % kStages4, half = (warp - kQuantWarp0) / kStages4;
    const int per = a.format == B2C_MXFP4 ? 2 : 1;  // lanes of a block: 4 or 2
    const uint32_t x = smem + s * kFewStage + kWBytes, xs = xs0 + s * kRowStage;
    Raw8<T> next[2];
    auto fetch = [&](const FewTile& t, int i, int r) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (r + 2 * j < t.rows)
          next[j] = load_raw8<T>((const T*)a.x + (long long)(plan.order[t.row0 + r + 2 * j] / a.topk) * a.ldx, i % kb_all * kFp4Stage + 8 * lane, a.hidden, wide);
    };
    auto tile_of = [&](int i) { return plan.tile[((int)blockIdx.x + i / kb_all * (int)gridDim.x) / n_tiles]; };
    int i = s, r = half;
    FewTile t = {0, 0, 0};
    if (i < all) {
      t = tile_of(i);
      fetch(t, i, r);
    }
#pragma unroll 1
    while (i < all) {
      const Raw8<T> raw[2] = {next[0], next[1]};
      const int r0 = r, rows = t.rows;
      const uint32_t phase = (uint32_t)((i / kStages4) & 1) ^ 1u;
      r += 4;
      const bool done = r >= rows;  // with this stage
      if (done) {
        r = half;
        i += kStages4;
        if (i < all) t = tile_of(i);
      }
      if (i < all) fetch(t, i, r);
      if (r0 == half && !__all_sync(0xffffffffu, mbar_wait(smem_u32(&c.ctl.empty[s]), phase, &c.ctl, &g_wait_status))) break;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = r0 + 2 * j;
        float v[8];
        widen8<T>(raw[j], v);
        uint32_t m = 0, q;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, abs_bits(v[e]));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        if (a.format == B2C_MXFP4) m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const Scale4 sc = scale_of(m, f, a.format);
        quantise4<8>(sc, f, a.format, v, &q);
        // 128-byte rows, pieces of 16 bytes swizzled; scales as the tensor core's copy takes them: row, word block / 4
        if (row < rows) {
          const int block = lane >> per;
          asm volatile("st.shared.b32 [%0], %1;" ::"r"(x + (uint32_t)(row * kStageRow + (((lane >> 2) ^ (row & 7)) << 4) + (lane & 3) * 4)), "r"(q) : "memory");
          if ((lane & ((1 << per) - 1)) == 0)
            asm volatile("st.shared.b8 [%0], %1;" ::"r"(xs + (uint32_t)((block >> 2) * kRowWord + row * 16 + (block & 3))), "r"(sc.code) : "memory");
        }
      }
      if (done) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&c.ctl.full[s]));
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    // ---------------------------------------------------------------- activation and quantisation
    const int quad = warp - 4;
    const float xg = a.x_global != nullptr ? *a.x_global : 1.0f;
    int buf = 0;
    uint32_t bph = 0;
    bool ok = true;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
      const int ti = item / n_tiles, n0 = (item - ti * n_tiles) * cols;
      const FewTile t = plan.tile[ti];
      // (a warp whose wait gave up still meets the others at their barriers)
      ok = ok && __all_sync(0xffffffffu, mbar_wait(smem_u32(&c.ctl.tmem_full[buf]), bph, &c.ctl, &g_wait_status));
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      float v[16];
      tmem_ld<16>(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * kAccCols), reinterpret_cast<int32_t*>(v));
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&c.ctl.tmem_empty[buf]));
      // gate sums are in lanes 0..63, up sums in 64..127
      const float alpha = xg * (a.w1_global != nullptr ? a.w1_global[t.expert] : 1.0f);
      asm volatile("bar.sync 1, 128;" ::: "memory");  // (those of the item before have been read)
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[i][quad * 32 + lane] = v[i] * alpha;
      asm volatile("bar.sync 1, 128;" ::: "memory");
      // half a warp takes a token: each lane four neighbouring columns
      const int l = lane & 15, n = n0 + 4 * l;
      for (int r = 2 * quad + (lane >> 4); r - (lane >> 4) < t.rows; r += 8) {
        float h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = r < t.rows ? quick_gated<true>(sums[r][4 * l + i], sums[r][64 + 4 * l + i]) : 0.0f;
        uint32_t mx = max(max(abs_bits(h[0]), abs_bits(h[1])), max(abs_bits(h[2]), abs_bits(h[3])));
        mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        if (a.format == B2C_MXFP4) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        const Scale4 s = quick_scale(mx, hf, a.format);
        uint32_t q;
        quick_quantise4<4>(s, h, &q);
        if (ok && r < t.rows && n < a.inter) {  // (inter is a multiple of 32)
          const long long row = t.row0 + r;
          *reinterpret_cast<uint16_t*>(a.hq + row * (a.inter / 2) + n / 2) = (uint16_t)q;
          const int block = fp4_block(a.format);
          if (n % block == 0) a.hs[row * a.ldhs + n / block] = (uint8_t)s.code;
        }
      }
      buf ^= 1;
      if (buf == 0) bph ^= 1u;
    }
    __syncwarp();
  }
  teardown_few(c, warp, tmem);
}

constexpr int kDownThreads = 256;
// The weighted sums of 128 columns, by four warps: a warp takes N tokens at a time, a lane four neighbouring columns.  All loads of S slots of
// these tokens come first, so that their latency is waited for once (with 60 tokens of two slots, two tokens at a time took 6 us).
template <typename T, int N, int S>
__device__ __forceinline__ void sum_tokens(const Few4Args& a, const FewPlan& plan, int nt, int quad, int lane) {
  const int tokens = a.pairs / a.topk, col = nt * kTileM + 4 * lane;
  const bool on = col < a.hidden;  // (hidden is a multiple of 32)
  T* y = (T*)a.y + col;
#pragma unroll 1
  for (int t0 = N * quad; t0 < tokens; t0 += 4 * N) {
    float4 sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
    for (int j0 = 0; j0 < a.topk; j0 += S) {
      float4 part[N][S];
      float w[N][S];
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < S; ++j) {
          const int p = (t0 + i) * a.topk + j0 + j;
          const int at = t0 + i < tokens && j0 + j < a.topk ? plan.place[p] : -1;
          part[i][j] = at >= 0 && on ? __ldcg(reinterpret_cast<const float4*>(a.part + (long long)at * a.hidden + col)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          w[i][j] = at >= 0 ? a.weights[p] : 0.0f;
        }
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < S; ++j) {
          sum[i].x = fmaf(w[i][j], part[i][j].x, sum[i].x);
          sum[i].y = fmaf(w[i][j], part[i][j].y, sum[i].y);
          sum[i].z = fmaf(w[i][j], part[i][j].z, sum[i].z);
          sum[i].w = fmaf(w[i][j], part[i][j].w, sum[i].w);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float out[4] = {sum[i].x, sum[i].y, sum[i].z, sum[i].w};
      if (t0 + i < tokens && on) store4<T>(y + (t0 + i) * a.ldy, out, 4);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kDownThreads, 1)
    experts4_down_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_ws, const __grid_constant__ CUtensorMap tmap_x,
                         const __grid_constant__ CUtensorMap tmap_xs, const Few4Args a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ FewCtl c;
  __shared__ FewPlan plan;
  __shared__ int last;
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t ws = smem + kStages4 * kFewStage, xs0 = ws + 2 * kGroupTile;
  setup_few(c, warp, lane, 1, 2);
  if (warp == 0 && lane == 9) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_w) : "memory");
  if (warp == 0 && lane == 10) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_ws) : "memory");
  if (warp == 0 && lane == 11) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_x) : "memory");
  if (warp == 0 && lane == 12) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_xs) : "memory");
  // Neither ids nor weights come from the first kernel, and what came before that has ended (it starts this one behind its own wait): the
  // sort and the copies of weights run beside it.  Rows, their sums and the counters are not touched before it has ended.
  plan_few(plan, reinterpret_cast<uint32_t*>(smem_raw + (smem - smem_u32(smem_raw))), a.ids, a.pairs, a.experts);
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = __shfl_sync(0xffffffffu, c.ctl.tmem_base, 0);
  constexpr int cols = kTileM;
  const int n_tiles = (a.hidden + cols - 1) / cols, items = plan.tiles * n_tiles;
  const int kb_all = (a.inter + kFp4Stage - 1) / kFp4Stage;

  if (warp == 0) {
    // ---------------------------------------------------------------- copies
    const uint32_t on = elect_one() ? 1u : 0u;
    const int mine = (items - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x, all = max(0, mine) * kb_all;
    struct At {
      int item, kb;
    };
    auto step = [&](At& p) {
      if (++p.kb == kb_all) {
        p.kb = 0;
        p.item += gridDim.x;
      }
    };
    auto load_w = [&](const At& p, int s) {
      const int t = p.item / n_tiles, n0 = (p.item - t * n_tiles) * cols;
      const uint32_t full = smem_u32(&c.ctl.full[s]);
      mbar_arrive_expect_tx(full, kFewStage, on);
      tma_load_3d(smem + s * kFewStage, &tmap_w, p.kb * kStageRow, n0, plan.tile[t].expert, full, on);
    };
    auto load_x = [&](const At& p, int s) {
      tma_load_2d(smem + s * kFewStage + kWBytes, &tmap_x, p.kb * kStageRow, plan.tile[p.item / n_tiles].row0, smem_u32(&c.ctl.full[s]), on);
    };
    const int ahead = min(kStages4, all);
    At w = {(int)blockIdx.x, 0}, x = w;
    for (int i = 0; i < ahead; ++i) {
      load_w(w, i);
      step(w);
    }
    pdl_wait();
    for (int i = 0; i < ahead; ++i) {
      load_x(x, i);
      step(x);
    }
    int s = ahead % kStages4;
    uint32_t ph = ahead == kStages4 ? 1u : 0u;
    for (int i = ahead; i < all; ++i) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&c.ctl.empty[s]), ph ^ 1u, &c.ctl, &g_wait_status))) break;
      load_w(w, s);
      load_x(w, s);
      step(w);
      if (++s == kStages4) {
        s = 0;
        ph ^= 1u;
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    const int stage = kRowWord * stage_words(a.format);
    auto row_scales = [&](int, int g, int in) { return xs0 + (uint32_t)(g * kRowGroup + stage * in); };
    if (a.format == B2C_MXFP4) mma_few<B2C_MXFP4>(c, smem, ws, row_scales, tmem, items, kb_all, a.inter);
    else mma_few<B2C_NVFP4>(c, smem, ws, row_scales, tmem, items, kb_all, a.inter);
  } else if (warp < 4) {
    // ---------------------------------------------------------------- scales of weights, of rows
    const uint32_t on = elect_one() ? 1u : 0u;
    const int width = group_row(a.format);
    if (warp == 2) {
      scales_few(
          c, 0, items, kb_all, lane,
          [&](int item, int group, int place, uint32_t full) {
            const int t = item / n_tiles, n0 = (item - t * n_tiles) * cols;
            mbar_arrive_expect_tx(full, (uint32_t)(kTileM * width), on);
            tma_load_3d(ws + (uint32_t)(place * kGroupTile), &tmap_ws, group * width, n0, plan.tile[t].expert, full, on);
          },
          [&](int place) { turn_group(ws + (uint32_t)(place * kGroupTile), kTileM, a.format, lane); }, false);
    } else {
      scales_few(
          c, 1, items, kb_all, lane,
          [&](int item, int group, int place, uint32_t full) {
            mbar_arrive_expect_tx(full, (uint32_t)(kTileRows * width), on);
            tma_load_2d(xs0 + (uint32_t)(place * kRowGroup), &tmap_xs, group * width, plan.tile[item / n_tiles].row0, full, on);
          },
          [&](int place) { turn_rows(xs0 + (uint32_t)(place * kRowGroup), a.format, lane); }, true);
    }
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- rows of the slots, their sums by token
    pdl_wait();
    pdl_launch_dependents();
    const int quad = warp - 4, in_tile = quad * 32 + lane;
    const float hg = a.h_global != nullptr ? *a.h_global : 1.0f;
    T* y = (T*)a.y;
    if (plan.tiles == 0) {
      for (int n = (int)blockIdx.x * kTileM + in_tile; n < a.hidden; n += (int)gridDim.x * kTileM)
        for (int t = 0; t < a.pairs / a.topk; ++t) y[t * a.ldy + n] = from_float<T>(0.0f);
    }
    int buf = 0;
    uint32_t bph = 0;
    bool ok = true;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
      const int ti = item / n_tiles, nt = item - ti * n_tiles, n = nt * cols + in_tile;
      const bool mine = n < a.hidden;
      const FewTile t = plan.tile[ti];
      // (a warp whose wait gave up still meets the others at their barriers)
      ok = ok && __all_sync(0xffffffffu, mbar_wait(smem_u32(&c.ctl.tmem_full[buf]), bph, &c.ctl, &g_wait_status));
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      float v[16];
      tmem_ld<16>(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * kAccCols), reinterpret_cast<int32_t*>(v));
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&c.ctl.tmem_empty[buf]));
      buf ^= 1;
      if (buf == 0) bph ^= 1u;
      const float alpha = hg * (a.w2_global != nullptr ? a.w2_global[t.expert] : 1.0f);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (ok && i < t.rows && mine) __stcg(a.part + (long long)(t.row0 + i) * a.hidden + n, v[i] * alpha);
      // who is last with these columns sums them up
      __threadfence();
      asm volatile("bar.sync 1, 128;" ::: "memory");
      if (in_tile == 0) last = ok && atomicAdd(a.done + nt, 1) == plan.tiles - 1;
      asm volatile("bar.sync 1, 128;" ::: "memory");
      if (last) {
        __threadfence();
        // (a token or two a warp by short code: fetching that of 16 loads costs a microsecond)
        const int tokens = a.pairs / a.topk;
        if (tokens <= 4) sum_tokens<T, 1, 4>(a, plan, nt, quad, lane);
        else if (tokens <= 8) sum_tokens<T, 2, 4>(a, plan, nt, quad, lane);
        else if (a.topk == 1) sum_tokens<T, 16, 1>(a, plan, nt, quad, lane);
        else if (a.topk == 2) sum_tokens<T, 8, 2>(a, plan, nt, quad, lane);
        else sum_tokens<T, 4, 4>(a, plan, nt, quad, lane);
      }
    }
    __syncwarp();
  }
  teardown_few(c, warp, tmem);
  // (no block leaves before the first kernel has ended: what comes after this one relies on that)
  pdl_wait();
}

int fail(cudaError_t e) {
  set_last_cuda_error((int)e);
  return B2C_E_CUDA;
}

template <typename T>
int launch(const Few4Args& a, cudaStream_t st) {
  const uint64_t b1 = a.hidden / 2, b2 = a.inter / 2, s1 = fp4_scales(a.hidden, a.format), s2 = fp4_scales(a.inter, a.format);
  const int width = group_row(a.format);
  CUtensorMap w1, ws1, w2, ws2, x, xs;
  int rc = encode_tiled_3d(&w1, a.w1, b1, a.inter, 2ull * a.experts, b1, (uint64_t)a.inter * b1, kStageRow, 64, 128);
  if (rc == B2C_OK) rc = encode_tiled_3d(&ws1, a.w1_scale, s1, a.inter, 2ull * a.experts, a.ld1, (uint64_t)a.inter * a.ld1, width, 64, width);
  if (rc == B2C_OK) rc = encode_tiled_3d(&w2, a.w2, b2, a.hidden, a.experts, b2, (uint64_t)a.hidden * b2, kStageRow, kTileM, 128);
  if (rc == B2C_OK) rc = encode_tiled_3d(&ws2, a.w2_scale, s2, a.hidden, a.experts, a.ld2, (uint64_t)a.hidden * a.ld2, width, kTileM, width);
  if (rc == B2C_OK) rc = encode_tiled_2d(&x, a.hq, b2, a.pairs, b2, kStageRow, kTileRows, 128);
  if (rc == B2C_OK) rc = encode_tiled_2d(&xs, a.hs, s2, a.pairs, a.ldhs, width, kTileRows, width);
  if (rc != B2C_OK) return rc;
  static std::atomic<unsigned long long> up{0}, down{0};
  cudaError_t e = set_max_dynamic_smem_once(up, (const void*)experts4_up_kernel<T>, kUpSmem);
  if (e == cudaSuccess) e = set_max_dynamic_smem_once(down, (const void*)experts4_down_kernel<T>, kDownSmem);
  // (as many tiles as experts or pairs at most, and one more for every 16 pairs)
  const long long tiles = std::min(a.experts, a.pairs) + a.pairs / kTileRows;
  auto grid = [&](long long n) { return dim3((unsigned)std::min<long long>(tiles * n, kNumSMs)); };
  if (e == cudaSuccess) e = launch_pdl(experts4_up_kernel<T>, grid((a.inter + 63) / 64), dim3(kUpThreads), kUpSmem, st, w1, ws1, a);
  if (e == cudaSuccess) e = launch_pdl(experts4_down_kernel<T>, grid((a.hidden + kTileM - 1) / kTileM), dim3(kDownThreads), kDownSmem, st, w2, ws2, x, xs, a);
  return e == cudaSuccess ? B2C_OK : fail(e);
}

}  // namespace

int launch_fp4_few_experts(const Few4Args& a, cudaStream_t st) {
  if (a.type == B2C_F32) return launch<float>(a, st);
  if (a.type == B2C_F16) return launch<__half>(a, st);
  return launch<__nv_bfloat16>(a, st);
}

cudaError_t fp4_few_status(int* status) { return take_status(status); }

cudaError_t fp4_few_wait_selftest(cudaStream_t st) { return launch_wait_selftest(st); }

}  // namespace b2c

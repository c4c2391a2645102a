// Products of 4-bit matrices on the tensor core: the kernel for few rows, and the choice between the two.
//
// With few rows the weights are the bytes, and the tensor core's 128 accumulator rows are given to them (the axes are swapped): a
// thread block owns 128 weight rows and 16, 32 or 64 activation rows.  What bounds it is the way from the launch to the first sums and how many bytes
// are in flight: the reduction is cut over the blocks of a cluster until all SMs have a share, and the partial sums meet in distributed shared
// memory, in a fixed order.  1 x 8192 x 8192 NV: 9.8 us, 3.9 TB/s (37.8 MB; 5.9 at the rate of a copy);  37 x 5136 x 4128 MX: 7.0.
//
// Roles: warp 0 copies (TMA), warp 1 carries the scales to tensor memory and issues the MMAs, the others copy the scales and turn them round (a
// warp an operand, see fp4_mma.cuh) and take the sums out of tensor memory when all stages have been added there.
#include "fp4_mma.cuh"

namespace b2c {

namespace {

constexpr int kMaxSplit = 8;

// WT weight tiles of 128 rows (2: gate and up of the same columns) x NT activation rows.
template <int NT, int WT>
struct RowsShape {
  static constexpr int kCols = NT * WT;
  static constexpr int kEpiWarps = kCols >= 64 ? 8 : 4;
  static constexpr int kThreads = 64 + 32 * kEpiWarps;
  static constexpr int kWarpCols = kCols / (kEpiWarps / 4);
  static constexpr int kW = WT * kTileM * kStageRow, kX = NT * kStageRow;
  static constexpr int kStageBytes = kW + kX;
  static constexpr int kScaleBytes = (WT + 1) * kGroupTile;  // of a group; two groups
  // two thread blocks share an SM where that leaves each three stages (228 KB, 1 KB of it kept for each block; the barriers are static)
  static constexpr int kHalf = 113 * 1024 - 1024 - 1024 - 2 * kScaleBytes, kWhole = 227 * 1024 - 1024 - 1024 - 2 * kScaleBytes;
  static constexpr int kPerSm = kHalf / kStageBytes >= 3 ? 2 : 1;
  static constexpr int kRing = kPerSm == 2 ? kHalf : kWhole;
  static constexpr int kStages = kRing / kStageBytes < 8 ? kRing / kStageBytes : 8;
  static constexpr int kScaleCols = 16 * (WT + 1);  // of a stage in tensor memory; two stages there
  static constexpr int kNeed = kCols + 2 * kScaleCols;
  static constexpr int kTmemCols = kNeed <= 128 ? 128 : (kNeed <= 256 ? 256 : 512);
  static constexpr int kPartBytes = kCols * kTileM * 4;  // sums, in the place of the stages
  static constexpr int kUsed = kStages * kStageBytes + 2 * kScaleBytes;
  static constexpr int kSmem = 1024 + (kUsed > kPartBytes ? kUsed : kPartBytes);
  static_assert(kPerSm * kTmemCols <= 512, "tensor memory of the blocks of an SM");
};

template <int NT, int WT>
__global__ void __launch_bounds__(RowsShape<NT, WT>::kThreads, RowsShape<NT, WT>::kPerSm)
    matmul4_rows_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_ws, const __grid_constant__ CUtensorMap tmap_x,
                        const __grid_constant__ CUtensorMap tmap_xs, const Matmul4Args a, const int kb_per_split, const bool early) {
  using S = RowsShape<NT, WT>;
  constexpr int stages = S::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ SharedCtl ctl;
  __shared__ __align__(8) unsigned long long scales_full[WT + 1][2], scales_empty[2];  // of a group of scales
  __shared__ __align__(8) unsigned long long turned[2];                                // and when all of them are in place
  __shared__ RowTile tile;

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t s_base = smem_base + stages * S::kStageBytes;
  const int split = (int)gridDim.z, rank = (int)blockIdx.z;  // (a cluster is the blocks of one z run)

  if (warp == 0) {
    if (lane < stages) {
      mbar_init(smem_u32(&ctl.full[lane]), 1);
      mbar_init(smem_u32(&ctl.empty[lane]), 1);
    }
    if (lane < 2) {
      for (int w = 0; w <= WT; ++w) mbar_init(smem_u32(&scales_full[w][lane]), 1);
      mbar_init(smem_u32(&scales_empty[lane]), 1);
      mbar_init(smem_u32(&turned[lane]), WT + 1);
    }
    if (lane == 8) mbar_init(smem_u32(&ctl.tmem_full[0]), 1);
    if (lane == 9) ctl.abort_flag = 0;
    if (lane == 10) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_w) : "memory");
    if (lane == 11) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_x) : "memory");
    if (lane == 12) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_ws) : "memory");
    if (lane == 13) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_xs) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl.tmem_base)), "r"(S::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // `early`: neither the weights nor the offsets come from the kernel before this one (nor does anything it overlaps with write them),
  // so tile and weights are fetched while that one drains; rows and their scales are not touched before it has ended.
  if (!early) pdl_wait();
  if (warp == 2) {
    const RowTile t = find_row_tile(a, (int)blockIdx.y, NT);
    if (lane == 0) tile = t;
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (!early) pdl_launch_dependents();
  const uint32_t tmem_acc = __shfl_sync(0xffffffffu, ctl.tmem_base, 0);
  const uint32_t tmem_scales = tmem_acc + S::kCols;
  const int group = tile.group, row0 = tile.row0;
  const int n0 = (int)blockIdx.x * kTileM;
  const int kb_all = (a.K + kFp4Stage - 1) / kFp4Stage;
  const int kb0 = rank * kb_per_split, kb1 = min(kb_all, kb0 + kb_per_split);

  if (group < 0) {
    // (all blocks of the cluster: there is nothing to do)
  } else if (warp == 0) {
    // ---------------------------------------------------------------- copies
    const uint32_t leader = elect_one() ? 1u : 0u;
    auto load_w = [&](int kb, int s) {
      const uint32_t full = smem_u32(&ctl.full[s]), dst = smem_base + s * S::kStageBytes;
      mbar_arrive_expect_tx(full, S::kStageBytes, leader);
#pragma unroll
      for (int w = 0; w < WT; ++w) tma_load_3d(dst + w * kTileM * kStageRow, &tmap_w, kb * kStageRow, n0, group * WT + w, full, leader);
    };
    auto load_x = [&](int kb, int s) {
      tma_load_2d(smem_base + s * S::kStageBytes + S::kW, &tmap_x, kb * kStageRow, row0, smem_u32(&ctl.full[s]), leader);
    };
    const int ahead = early ? min(stages, kb1 - kb0) : 0;
    for (int i = 0; i < ahead; ++i) load_w(kb0 + i, i);
    if (early) pdl_wait();
    for (int i = 0; i < ahead; ++i) load_x(kb0 + i, i);
    int s = ahead % stages;
    uint32_t ph = ahead == stages ? 1u : 0u;
    for (int kb = kb0 + ahead; kb < kb1; ++kb) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.empty[s]), ph ^ 1u, &ctl, &g_wait_status))) break;
      load_w(kb, s);
      load_x(kb, s);
      if (++s == stages) {
        s = 0;
        ph ^= 1u;
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- scales to tensor memory, MMA issue
    const uint32_t leader = elect_one() ? 1u : 0u;
    const uint32_t idesc = make_idesc_f4(kTileM, NT, a.format);
    auto run = [&](auto format) {
      constexpr int FORMAT = decltype(format)::value;
      int s = 0, g = 0;
      uint32_t ph = 0, gph = 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        const int in = kb % kGroup;  // stage of the group (the first group may begin inside)
        if (in == 0 || kb == kb0) {
          if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&turned[g]), gph, &ctl, &g_wait_status))) break;
        }
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.full[s]), ph, &ctl, &g_wait_status))) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int ksteps = min(4, (a.K - kb * kFp4Stage + 63) / 64);
        const uint32_t base = smem_base + s * S::kStageBytes, scales = s_base + g * S::kScaleBytes + (uint32_t)(512 * stage_words(FORMAT) * in);
        // (copies and MMAs run in the order in which they are issued)
        const uint32_t ts = tmem_scales + (uint32_t)((kb - kb0) & 1) * S::kScaleCols;
#pragma unroll
        for (int w = 0; w <= WT; ++w) copy_scales<1, FORMAT, 512>(ts + 16 * w, scales + w * kGroupTile, 4, leader);
        const uint64_t xdesc = make_smem_desc(base + S::kW, kStageRow);
#pragma unroll
        for (int w = 0; w < WT; ++w)
          mma_f4_stage<1, FORMAT>(tmem_acc + w * NT, make_smem_desc(base + w * kTileM * kStageRow, kStageRow), xdesc, idesc, ts + 16 * w, ts + 16 * WT, 4, kb > kb0,
                                  leader, ksteps);
        mma_commit(smem_u32(&ctl.empty[s]), leader);
        if (in == kGroup - 1) {
          mma_commit(smem_u32(&scales_empty[g]), leader);
          g ^= 1;
          if (g == 0) gph ^= 1u;
        }
        if (kb == kb1 - 1) mma_commit(smem_u32(&ctl.tmem_full[0]), leader);
        if (++s == stages) {
          s = 0;
          ph ^= 1u;
        }
      }
    };
    if (a.format == B2C_MXFP4) run(std::integral_constant<int, B2C_MXFP4>());
    else run(std::integral_constant<int, B2C_NVFP4>());
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- scales: a warp has a tile of weights, the one after them the rows
    const int part = warp - 2;
    int lg = kb0 / kGroup, place = 0;  // next group to be copied, and where to
    const int last = (kb1 - 1) / kGroup;
    auto load_next = [&]() {
      if (lg > last) return;
      const uint32_t on = elect_one() ? 1u : 0u, full = smem_u32(&scales_full[part][place]), dst = s_base + place * S::kScaleBytes + part * kGroupTile;
      const int width = group_row(a.format);
      mbar_arrive_expect_tx(full, (uint32_t)((part < WT ? kTileM : NT) * width), on);
      if (part < WT) tma_load_3d(dst, &tmap_ws, lg * width, n0, group * WT + part, full, on);
      else tma_load_2d(dst, &tmap_xs, lg * width, row0, full, on);
      ++lg;
      place ^= 1;
    };
    if (part < WT) {
      load_next();
      load_next();
    }
    if (early) {
      pdl_wait();
      pdl_launch_dependents();
    }
    if (part <= WT) {
      if (part == WT) {
        load_next();
        load_next();
      }
      uint32_t ph = 0;
      int g = 0;
      for (int n = kb0 / kGroup; n <= last; ++n) {
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&scales_full[part][g]), ph, &ctl, &g_wait_status))) break;
        turn_group(s_base + g * S::kScaleBytes + part * kGroupTile, part == WT ? NT : kTileM, a.format, lane);
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&turned[g]));
        g ^= 1;
        // the other place, when the MMAs of its group (the one before) have ended
        if (n > kb0 / kGroup && lg <= last) {
          if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&scales_empty[g]), g == 0 ? ph : ph ^ 1u, &ctl, &g_wait_status))) break;
          load_next();
        }
        if (g == 0) ph ^= 1u;
      }
      __syncwarp();
    }
    // ---------------------------------------------------------------- sums
    const int quad = warp & 3;                         // lanes of tensor memory this warp may read
    const int c0 = ((warp - 2) >> 2) * S::kWarpCols;   // its columns
    if (__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.tmem_full[0]), 0, &ctl, &g_wait_status))) {
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      // every MMA of this block has been waited for, so the stages are free: the sums take their place
      float* sums = reinterpret_cast<float*>(smem_raw + (smem_base - smem_u32(smem_raw)));
      const uint32_t taddr = tmem_acc + ((uint32_t)(quad * 32) << 16) + (uint32_t)c0;
#pragma unroll 1
      for (int c = 0; c < S::kWarpCols; c += 16) {
        float v[16];
        tmem_ld<16>(taddr + c, reinterpret_cast<int32_t*>(v));
#pragma unroll
        for (int j = 0; j < 16; ++j) sums[(c0 + c + j) * kTileM + quad * 32 + lane] = v[j];
      }
    }
  }

  // ---------------------------------------------------------------- sums of the cluster, results
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (ctl.abort_flag) {
    // copies may still be under way: they land before this block leaves
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 50000ull) __nanosleep(1000);
    __syncthreads();
  }
  // Tensor memory goes back before the blocks of the cluster wait for each other: one that held it could wait for one that waits for it,
  // where a pair kernel of another stream has asked for the same columns in between.
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_acc), "r"(S::kTmemCols) : "memory");
  }
  if (split > 1) cluster_sync();
  if (group >= 0) {
    // one warp takes one activation row: each lane four neighbouring columns
    const int rows = min(NT, tile.row_end - row0);
    const int n = n0 + 4 * lane;
    const float alpha = alpha_of(a, group);
    QuickFactor4 hf = {};
    if constexpr (WT == 2) hf = quick_factor4(a.y_global, a.format);
    // (code that runs once or twice is paid for when it is fetched, not when it runs)
#pragma unroll 1
    for (int j = rank + split * warp; j < rows; j += split * (S::kThreads / 32)) {
      float4 v[WT];
#pragma unroll
      for (int w = 0; w < WT; ++w) {
        const uint32_t at = smem_base + (uint32_t)(((w * NT + j) * kTileM + 4 * lane) * 4);
        if (split == 1) {
          v[w] = ld_shared_f4(at);
        } else {
          float4 part[kMaxSplit];  // (all loads first, so that their latency is waited for once)
#pragma unroll
          for (int z = 0; z < kMaxSplit; ++z)
            if (z < split) part[z] = ld_cluster_f4(map_to_rank(at, (uint32_t)z));
          v[w] = part[0];
#pragma unroll
          for (int z = 1; z < kMaxSplit; ++z)
            if (z < split) {
              v[w].x += part[z].x;
              v[w].y += part[z].y;
              v[w].z += part[z].z;
              v[w].w += part[z].w;
            }
        }
        v[w] = make_float4(v[w].x * alpha, v[w].y * alpha, v[w].z * alpha, v[w].w * alpha);
      }
      const long long row = row0 + j;
      if constexpr (WT == 1) {
        const float out[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
        if (n < a.N) {
          if (a.y_type == B2C_F32) store4<float>((float*)a.y + row * a.ldy + n, out, a.N - n);
          else if (a.y_type == B2C_F16) store4<__half>((__half*)a.y + row * a.ldy + n, out, a.N - n);
          else store4<__nv_bfloat16>((__nv_bfloat16*)a.y + row * a.ldy + n, out, a.N - n);
        }
      } else {
        // a block of 16 (32) columns is four (eight) neighbouring lanes
        const float h[4] = {quick_gated<true>(v[0].x, v[1].x), quick_gated<true>(v[0].y, v[1].y), quick_gated<true>(v[0].z, v[1].z), quick_gated<true>(v[0].w, v[1].w)};
        uint32_t mx = max(max(abs_bits(h[0]), abs_bits(h[1])), max(abs_bits(h[2]), abs_bits(h[3])));
        mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        if (a.format == B2C_MXFP4) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        const Scale4 s = quick_scale(mx, hf, a.format);
        uint32_t q;
        quick_quantise4<4>(s, h, &q);
        if (n < a.N) {  // (N is a multiple of 32)
          *reinterpret_cast<uint16_t*>((uint8_t*)a.y + row * a.ldy + n / 2) = (uint16_t)q;
          const int block = fp4_block(a.format);
          if (n % block == 0) a.y_scale[row * a.ldys + n / block] = (uint8_t)s.code;
        }
      }
    }
  }
  // no block leaves while another reads its sums, and none before the kernel ahead has ended: what comes after this one relies on that
  if (early) pdl_wait();
  if (split > 1) cluster_sync();
}

int fail(cudaError_t e) {
  set_last_cuda_error((int)e);
  return B2C_E_CUDA;
}

// How many thread blocks share a tile's reduction: what counts is the stages that a block fetches, one after another.  Blocks that share an SM are
// a fifth slower each; a cut costs the exchange of the partial sums, about as long as two stages and one more for every block of the cluster.
// Measured, us with 1, 2, 3, 4, 6 blocks a tile (four sets of operands in turn, more than L2 holds):
//   1 x 8192 x 8192 (64 tiles of 32 stages) 13.9, 12.1, 11.1, 10.7, 15.4;   37 x 5136 x 4128 (41 of 17) 9.2, 8.3, 7.8, 9.0, 8.7;
//   16 x 4096 x 4096 (32 of 16) 8.0, 7.5, 6.7, 6.3, 6.8;   128 x 4096 x 4096 (64 of 16) 9.3, 8.6, 9.0, 8.8, 15.3;
//   300 x 1024 x 8192 (40 of 32) 13.9, 10.7, 9.4, 9.7, 9.7.
int choose_split(long long tiles, int kb_all, int per_sm, bool counted, double* stages = nullptr) {
  if (!counted && tiles >= kNumSMs) return 1;  // (a guess of the tiles says nothing about the last wave)
  int best = 1;
  double least = 0;
  for (int s = 1; s <= kMaxSplit && 2 * s <= std::max(2, kb_all); ++s) {
    const int per = (kb_all + s - 1) / s;
    if ((kb_all + per - 1) / per != s) continue;  // (no thread block without work)
    if (s > 4 && tiles * s > kNumSMs) break;  // (300 x 1024 x 8192, 40 tiles: 15.0 us by seven)
    const long long blocks = tiles * s, waves = (blocks + kNumSMs * per_sm - 1) / (kNumSMs * per_sm);
    const double cost = (double)waves * per * (per_sm > 1 && blocks > kNumSMs ? 1.2 : 1.0) + (s > 1 ? 1.5 + s : 0.0);
    if (s == 1 || cost < least) {
      best = s;
      least = cost;
    }
  }
  if (stages != nullptr) *stages = least;
  return best;
}

template <int NT, int WT>
int launch_rows(const Matmul4Args& a, cudaStream_t st) {
  using S = RowsShape<NT, WT>;
  const int n_tiles = (a.N + kTileM - 1) / kTileM, kb_all = (a.K + kFp4Stage - 1) / kFp4Stage;
  // every group adds at most one tile that is not full
  const long long row_tiles = a.offsets ? a.rows / NT + std::min(a.groups, a.rows) : (a.rows + NT - 1) / NT;
  if (row_tiles > 65535) return B2C_E_UNSUPPORTED;
  // (with groups the number of tiles is known on the device only: as many groups as there are rows may have some)
  const long long busy = (long long)n_tiles * (a.offsets ? std::max<long long>((a.rows + NT - 1) / NT, std::min(a.groups, a.rows)) : row_tiles);
  const int split = choose_split(busy, kb_all, S::kPerSm, a.offsets == nullptr);
  const int kb_per_split = (kb_all + split - 1) / split;
  const uint64_t bytes = a.K / 2, scales = fp4_scales(a.K, a.format), planes = (uint64_t)a.groups * WT;
  const int width = group_row(a.format);
  CUtensorMap tw, tws, tx, txs;
  int rc = encode_tiled_3d(&tw, a.b, bytes, a.N, planes, bytes, (uint64_t)a.N * bytes, kStageRow, kTileM, 128);
  if (rc == B2C_OK) rc = encode_tiled_3d(&tws, a.b_scale, scales, a.N, planes, a.ldbs, (uint64_t)a.N * a.ldbs, width, kTileM, width);
  if (rc == B2C_OK) rc = encode_tiled_2d(&tx, a.a, bytes, a.rows, a.rows > 1 ? a.lda : bytes, kStageRow, NT, 128);
  if (rc == B2C_OK) rc = encode_tiled_2d(&txs, a.a_scale, scales, a.rows, a.rows > 1 ? a.lds : fp4_scale_pitch(a.K, a.format), width, NT, width);
  if (rc != B2C_OK) return rc;
  static std::atomic<unsigned long long> configured{0};
  cudaError_t e = set_max_dynamic_smem_once(configured, (const void*)matmul4_rows_kernel<NT, WT>, S::kSmem);
  if (e == cudaSuccess)
    e = launch_pdl_cluster(matmul4_rows_kernel<NT, WT>, dim3((unsigned)n_tiles, (unsigned)row_tiles, (unsigned)split), dim3(S::kThreads), S::kSmem, st, split,
                           tw, tws, tx, txs, a, kb_per_split, a.early != 0);
  return e == cudaSuccess ? B2C_OK : fail(e);
}

template <int NT>
int launch_rows_of(const Matmul4Args& a, cudaStream_t st) {
  return a.gated ? launch_rows<NT, 2>(a, st) : launch_rows<NT, 1>(a, st);
}

}  // namespace

int launch_fp4_matmul(const Matmul4Args& a, cudaStream_t st) {
  int rows = a.rows;
  if (a.offsets) {
    rows = rows_of_a_group_tile(a);
    if (rows > 64) return launch_fp4_matmul_pair(a, st);
  } else if (rows > 64) {
    // 5.4 us and 0.3 for every stage that a block fetches: with few tiles and a long reduction the cut is worth more than larger tiles (us here and
    // there: 128 x 2048 x 8192 8.6 and 12.4, 100 x 4096 x 4096 8.8 and 8.3)
    const long long tiles = (long long)((a.N + kTileM - 1) / kTileM) * ((rows + 63) / 64);
    double stages = 0;
    choose_split(tiles, (a.K + kFp4Stage - 1) / kFp4Stage, RowsShape<64, 1>::kPerSm, true, &stages);
    if (5400 + 300 * stages > (double)fp4_pair_ns(a)) return launch_fp4_matmul_pair(a, st);
  }
  if (rows <= 16) return launch_rows_of<16>(a, st);
  if (rows <= 32) return launch_rows_of<32>(a, st);
  return launch_rows_of<64>(a, st);
}

cudaError_t fp4_rows_wait_selftest(cudaStream_t st) { return launch_wait_selftest(st); }

int fp4_status_read_and_clear(int32_t* status) {
  int rows = 0, pair = 0, few = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = take_status(&rows);
  if (e == cudaSuccess) e = fp4_pair_status(&pair);
  if (e == cudaSuccess) e = fp4_few_status(&few);
  if (e != cudaSuccess) return fail(e);
  *status = rows != 0 ? rows : (pair != 0 ? pair : few);
  return B2C_OK;
}

}  // namespace b2c

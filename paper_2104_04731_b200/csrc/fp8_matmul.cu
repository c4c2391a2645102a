// Products of block-scaled 8-bit matrices on the tensor core: the kernel for few rows, and the choice between the two.
//
// With few rows the weights are the bytes, and the tensor core's 128 accumulator rows are given to them (the axes
// are swapped): a thread block owns 128 weight rows and 16 to 64 activation rows, so that an MMA of a few activation rows
// is no larger than these.  What bounds it is how many bytes are in flight: the reduction is cut over the
// blocks of a cluster until all SMs have a share, and the partial sums meet in distributed shared memory, in a fixed
// order, without a second launch or atomics.
//
// Roles: warp 0 copies (TMA, 128-byte swizzle), warp 1 issues the MMAs, the others take each block of 128 of the
// reduction out of tensor memory, scale it and add it up in registers (see fp8_mma.cuh).
#include "fp8_mma.cuh"

namespace b2c {

namespace {

constexpr int kMaxSplit = 8;
constexpr int kScaleRun = 4;  // blocks of the reduction whose scales are fetched together

// WT weight tiles of 128 rows (2: gate and up of the same columns) x NT activation rows.
template <int NT, int WT>
struct RowsShape {
  static constexpr int kCols = NT * WT;                   // accumulator columns of one block of the reduction
  static constexpr int kEpiWarps = kCols >= 64 ? 8 : 4;
  static constexpr int kThreads = 64 + 32 * kEpiWarps;
  static constexpr int kWarpCols = kCols / (kEpiWarps / 4);
  static constexpr int kStageBytes = WT * kTileM * kBlock + NT * kBlock;
  // two thread blocks share an SM: half of the shared memory (228 KB, 1 KB of it kept for each block; `factor` and the
  // barriers are static) and of the 512 columns of tensor memory each
  static constexpr int kFactorBytes = 2 * kScaleRun * kCols * 4;
  // (where that is fewer than three stages a block has an SM to itself: two of 40 KB cost the latency of a copy, 0.95 us, for a block
  // of the reduction)
  static constexpr int kHalf = 113 * 1024 - 1024 - 1024 - kFactorBytes, kWhole = 227 * 1024 - 1024 - 1024 - kFactorBytes;
  static constexpr int kPerSm = kHalf / kStageBytes >= 3 ? 2 : 1;
  static constexpr int kRing = kPerSm == 2 ? kHalf : kWhole;
  static constexpr int kStages = kRing / kStageBytes < 8 ? kRing / kStageBytes : 8;
  static constexpr int kBufs = kCols <= 64 ? 4 : 2;
  static constexpr int kTmemCols = kCols * kBufs < 32 ? 32 : kCols * kBufs;
  static constexpr int kPartBytes = kCols * kTileM * 4;   // partial sums, in the place of the stages
  static constexpr int kSmem = 1024 + (kStages * kStageBytes > kPartBytes ? kStages * kStageBytes : kPartBytes);
};

template <typename T>
__device__ __forceinline__ void store4(T* p, const float* v, int n) {
  if (n >= 4 && (reinterpret_cast<uintptr_t>(p) & (4 * sizeof(T) - 1)) == 0) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]));
  } else {
    for (int i = 0; i < min(n, 4); ++i) p[i] = from_float<T>(v[i]);
  }
}
template <>
__device__ __forceinline__ void store4<float>(float* p, const float* v, int n) {
  if (n >= 4 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    for (int i = 0; i < min(n, 4); ++i) p[i] = v[i];
  }
}

template <int NT, int WT, typename YT>
__global__ void __launch_bounds__(RowsShape<NT, WT>::kThreads, RowsShape<NT, WT>::kPerSm)
    matmul_rows_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_x, const MatmulArgs a,
                       const int kb_per_split, const bool early) {
  constexpr int stages = RowsShape<NT, WT>::kStages;
  using S = RowsShape<NT, WT>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ SharedCtl ctl;
  __shared__ RowTile tile;
  __shared__ __align__(16) float factor[2][kScaleRun][S::kCols];

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int split = (int)gridDim.z, rank = (int)blockIdx.z;  // (a cluster is the blocks of one z run)

  if (warp == 0) {
    if (lane < stages) {
      mbar_init(smem_u32(&ctl.full[lane]), 1);
      mbar_init(smem_u32(&ctl.empty[lane]), 1);
    }
    if (lane < S::kBufs) {
      mbar_init(smem_u32(&ctl.tmem_full[lane]), 1);
      mbar_init(smem_u32(&ctl.tmem_empty[lane]), S::kEpiWarps);
    }
    if (lane == 0) ctl.abort_flag = 0;
    if (lane == 9) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_w) : "memory");
    if (lane == 10) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_x) : "memory");
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
  const int group = tile.group, row0 = tile.row0;
  const int n0 = (int)blockIdx.x * kTileM;
  const int kb_all = (int)blocks_of(a.K);
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
      for (int w = 0; w < WT; ++w) tma_load_3d(dst + w * kTileM * kBlock, &tmap_w, kb * kBlock, n0, group * WT + w, full, leader);
    };
    auto load_x = [&](int kb, int s) {
      tma_load_2d(smem_base + s * S::kStageBytes + WT * kTileM * kBlock, &tmap_x, kb * kBlock, row0, smem_u32(&ctl.full[s]), leader);
    };
    const int ahead = early ? min(stages, kb1 - kb0) : 0;
    for (int i = 0; i < ahead; ++i) load_w(kb0 + i, i);
    if (early) pdl_wait();
    for (int i = 0; i < ahead; ++i) load_x(kb0 + i, i);
    int s = ahead % stages;
    uint32_t ph = ahead == stages ? 1u : 0u;
    for (int kb = kb0 + ahead; kb < kb1; ++kb) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.empty[s]), ph ^ 1u, &ctl, &g_fp8_status))) break;
      load_w(kb, s);
      load_x(kb, s);
      if (++s == stages) {
        s = 0;
        ph ^= 1u;
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issue
    const uint32_t leader = elect_one() ? 1u : 0u;
    const uint32_t idesc = make_idesc_f8(kTileM, NT, a.b_type, a.a_type);
    int s = 0, buf = 0;
    uint32_t ph = 0, bph = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.tmem_empty[buf]), bph ^ 1u, &ctl, &g_fp8_status))) break;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&ctl.full[s]), ph, &ctl, &g_fp8_status))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int ksteps = min(4, (a.K - kb * kBlock + kMmaK - 1) / kMmaK);
      const uint32_t base = smem_base + s * S::kStageBytes;
      const uint64_t xdesc = make_smem_desc(base + WT * kTileM * kBlock, kBlock);
#pragma unroll
      for (int w = 0; w < WT; ++w)
        mma_f8_block<1>(tmem_acc + buf * S::kCols + w * NT, make_smem_desc(base + w * kTileM * kBlock, kBlock), xdesc, idesc, leader, ksteps);
      mma_commit(smem_u32(&ctl.empty[s]), leader);
      mma_commit(smem_u32(&ctl.tmem_full[buf]), leader);
      if (++s == stages) {
        s = 0;
        ph ^= 1u;
      }
      if (++buf == S::kBufs) {
        buf = 0;
        bph ^= 1u;
      }
    }
    __syncwarp();
  } else {
    // ---------------------------------------------------------------- scaled sums
    if (early) {
      pdl_wait();
      pdl_launch_dependents();
    }
    const int quad = warp & 3;                         // lanes of tensor memory this warp may read
    const int c0 = ((warp - 2) >> 2) * S::kWarpCols;   // its columns
    const int et = (int)threadIdx.x - 64;              // thread of this role
    f32x2 acc[S::kWarpCols / 2];
#pragma unroll
    for (int i = 0; i < S::kWarpCols / 2; ++i) acc[i] = 0;
    // thread c fetches the scales of column c (activation row c % NT, weight tile c / NT), a run of blocks ahead
    const bool fetches = et < S::kCols;
    const int tok = row0 + et % NT;
    const float* sx = a.a_scale + (long long)min(tok, a.rows - 1) * a.lds;
    const float* sw = a.b_scale + ((long long)(group * WT + et / NT) * blocks_of(a.N) + blockIdx.x) * kb_all;
    float next[kScaleRun];
    auto fetch = [&](int kb) {
#pragma unroll
      for (int i = 0; i < kScaleRun; ++i) next[i] = fetches && kb + i < kb1 ? sx[kb + i] * sw[kb + i] : 0.0f;
    };
    fetch(kb0);
    int buf = 0, run = 0;
    uint32_t bph = 0;
    bool ok = true;  // a warp whose wait gave up still meets the others at their barriers
    for (int kb = kb0; kb < kb1; ++kb) {
      const int i = (kb - kb0) % kScaleRun;
      if (i == 0) {
        // the other half of `factor` may still be read by slower warps; this half was read before the last barrier
        run ^= 1;
        if (fetches) {
#pragma unroll
          for (int j = 0; j < kScaleRun; ++j) factor[run][j][et] = next[j];
        }
        asm volatile("bar.sync 1, %0;" ::"n"(32 * S::kEpiWarps) : "memory");
        fetch(kb + kScaleRun);
      }
      ok = ok && __all_sync(0xffffffffu, mbar_wait_inline(smem_u32(&ctl.tmem_full[buf]), bph, &ctl, &g_fp8_status));
      if (!ok) continue;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t taddr = tmem_acc + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * S::kCols + c0);
      constexpr int kLd = S::kWarpCols == 32 ? 32 : 16;  // (64 sums a thread leave no room for 32 more values)
#pragma unroll
      for (int c = 0; c < S::kWarpCols; c += kLd) {
        float v[kLd];
        tmem_ld<kLd>(taddr + c, reinterpret_cast<int32_t*>(v));
#pragma unroll
        for (int j = 0; j < kLd; j += 4) {
          const float4 f = *reinterpret_cast<const float4*>(&factor[run][i][c0 + c + j]);
          fma2(&acc[(c + j) / 2], pair_of(v[j], v[j + 1]), pair_of(f.x, f.y));
          fma2(&acc[(c + j) / 2 + 1], pair_of(v[j + 2], v[j + 3]), pair_of(f.z, f.w));
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl.tmem_empty[buf]));
      if (++buf == S::kBufs) {
        buf = 0;
        bph ^= 1u;
      }
    }
    // every MMA of this block has been waited for, so the stages are free: the sums take their place
    float* part = reinterpret_cast<float*>(smem_raw + (smem_base - smem_u32(smem_raw)));
#pragma unroll
    for (int i = 0; i < S::kWarpCols; i += 2) {
      float lo, hi;
      unpair(acc[i / 2], &lo, &hi);
      part[(c0 + i) * kTileM + quad * 32 + lane] = lo;
      part[(c0 + i + 1) * kTileM + quad * 32 + lane] = hi;
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
    // (Code that runs once or twice is paid for when it is fetched, not when it runs: with four rows unrolled side by side this part
    // took 5 us of a launch of 44 rows.)
#pragma unroll 1
    for (int j = rank + split * warp; j < rows; j += split * (S::kThreads / 32)) {
      float4 v[WT];
#pragma unroll
      for (int w = 0; w < WT; ++w) {
        const uint32_t at = smem_base + (uint32_t)(((w * NT + j) * kTileM + 4 * lane) * 4);
        if (split == 1) {
          v[w] = ld_shared_f4(at);
          continue;
        }
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
      const long long row = row0 + j;
      if constexpr (WT == 1) {
        const float out[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
        if (n < a.N) store4<YT>((YT*)a.y + row * a.ldy + n, out, a.N - n);
      } else {
        const float h[4] = {silu(v[0].x) * v[1].x, silu(v[0].y) * v[1].y, silu(v[0].z) * v[1].z, silu(v[0].w) * v[1].w};
        float mx = fmaxf(fmaxf(fabsf(h[0]), fabsf(h[1])), fmaxf(fabsf(h[2]), fabsf(h[3])));
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const BlockScale s = block_scale<B2C_E4M3>(mx);
        const uint32_t q = __byte_perm(quantize2<B2C_E4M3>(s, h[0], h[1]), quantize2<B2C_E4M3>(s, h[2], h[3]), 0x5410);
        if (n < a.N) *reinterpret_cast<uint32_t*>((uint8_t*)a.y + row * a.ldy + n) = q;  // (N and ldy are multiples of 16)
        if (lane == 0) a.y_scale[row * a.ldys + blockIdx.x] = s.scale;
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

// How many thread blocks share a tile's reduction.  What counts is the SM with the most blocks of the reduction to fetch: tiles * split
// thread blocks are spread over 148 SMs.  A cut costs the exchange of the partial sums, about as long as three such blocks, and more
// the larger the cluster (measured, 37 x 5136 x 4112, 41 tiles of 33 blocks: 13.7 us with one, 10.3 with two, 8.7 with three,
// 9.8 with four and 13.7 with seven of them; 1 x 8192 x 8192, 64 tiles of 64: 18.4, 14.6, 15.5, 14.9 and with eight 14.9 us).
int choose_split(long long tiles, int kb_all, bool counted) {
  if (!counted && tiles >= kNumSMs) return 1;  // (a guess of the tiles says nothing about the last wave)
  int best = 1;
  double least = 0;
  for (int s = 1; s <= kMaxSplit && 2 * s <= std::max(2, kb_all); ++s) {
    const int per = (kb_all + s - 1) / s;
    if ((kb_all + per - 1) / per != s) continue;  // (no thread block without work)
    const double cost = (double)((tiles * s + kNumSMs - 1) / kNumSMs) * per + (s > 1 ? 2.5 + 0.5 * s : 0.0);
    if (s == 1 || cost < least) {
      best = s;
      least = cost;
    }
  }
  return best;
}

template <int NT, int WT, typename YT>
int launch_rows(const MatmulArgs& a, cudaStream_t st) {
  using S = RowsShape<NT, WT>;
  const int n_tiles = (int)blocks_of(a.N), kb_all = (int)blocks_of(a.K);
  // every group adds at most one tile that is not full
  const long long row_tiles = a.offsets ? a.rows / NT + std::min(a.groups, a.rows) : (a.rows + NT - 1) / NT;
  if (row_tiles > 65535) return B2C_E_UNSUPPORTED;
  // (with groups the number of tiles is known on the device only: as many groups as there are rows may have some)
  const long long busy = (long long)n_tiles * (a.offsets ? std::max<long long>((a.rows + NT - 1) / NT, std::min(a.groups, a.rows)) : row_tiles);
  const int split = choose_split(busy, kb_all, a.offsets == nullptr);
  const int kb_per_split = (kb_all + split - 1) / split;
  CUtensorMap tw, tx;
  int rc = encode_tiled_3d(&tw, a.b, a.K, a.N, (uint64_t)a.groups * WT, a.K, (uint64_t)a.N * a.K, kBlock, kTileM, kBlock);
  if (rc == B2C_OK) rc = encode_tiled_2d(&tx, a.a, a.K, a.rows, a.rows > 1 ? a.lda : a.K, kBlock, NT, kBlock);
  if (rc != B2C_OK) return rc;
  static std::atomic<unsigned long long> configured{0};
  cudaError_t e = set_max_dynamic_smem_once(configured, (const void*)matmul_rows_kernel<NT, WT, YT>, S::kSmem);
  if (e == cudaSuccess)
    e = launch_pdl_cluster(matmul_rows_kernel<NT, WT, YT>, dim3((unsigned)n_tiles, (unsigned)row_tiles, (unsigned)split), dim3(S::kThreads),
                           S::kSmem, st, split, tw, tx, a, kb_per_split, a.early != 0);
  return e == cudaSuccess ? B2C_OK : fail(e);
}

template <int NT>
int launch_rows_type(const MatmulArgs& a, cudaStream_t st) {
  if (a.y_type == B2C_F32) return launch_rows<NT, 1, float>(a, st);
  if (a.y_type == B2C_F16) return launch_rows<NT, 1, __half>(a, st);
  return launch_rows<NT, 1, __nv_bfloat16>(a, st);
}

// Whether one product of 65 rows or more is better formed by tiles of 128 weight rows x 64 rows, one on each of up to 148 SMs, than by
// the pair kernel's tiles on 74 pairs.  In cycles: 770 for a block of the reduction and 4600 besides here, as long as every tile has
// an SM of its own (two on one take two and a half times as long); from 385 rows on the weights, fetched once for every 64 rows, are
// what counts.  Measured, us here / there (tiles of 256 columns):
//   4096 x 4096: 128 rows 11.3 / 18.8, 256 rows 15.5 / 18.9, 320 rows 39 / 19.0;   8192 x 2048: 128 rows 10.2 / 12.6, 200 rows 13.7 / 12.7;
//   2048 x 7168: 256 rows 15.0 / 27.5, 384 rows 24.5 / 27.5, 512 rows 37.6 / 27.6.
bool rows_kernel_is_better(const MatmulArgs& a) {
  const long long kb_all = blocks_of(a.K), tiles = blocks_of(a.N) * ((a.rows + 63) / 64);
  const int split = choose_split(tiles, (int)kb_all, true);
  if (a.rows > 384 || tiles * split > kNumSMs) return false;
  return 770 * ((kb_all + split - 1) / split) + 4600 + (split > 1 ? 2000 : 0) < pair_cycles(a);
}

}  // namespace

int launch_fp8_matmul(const MatmulArgs& a, cudaStream_t st) {
  const int rows = rows_of_a_group(a);
  if (rows > 64 && !(a.offsets ? rows <= 128 : rows_kernel_is_better(a))) return launch_fp8_matmul_pair(a, st);
  if (a.gated) {
    if (rows <= 16) return launch_rows<16, 2, uint8_t>(a, st);
    if (rows <= 32) return launch_rows<32, 2, uint8_t>(a, st);
    return launch_rows<64, 2, uint8_t>(a, st);
  }
  if (rows <= 16) return launch_rows_type<16>(a, st);
  if (rows <= 32) return launch_rows_type<32>(a, st);
  return launch_rows_type<64>(a, st);
}

cudaError_t fp8_rows_wait_selftest(cudaStream_t st) { return launch_wait_selftest(st); }

int fp8_status_read_and_clear(int32_t* status) {
  int rows = 0, pair = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = take_status(&rows);
  if (e == cudaSuccess) e = fp8_pair_status(&pair);
  if (e != cudaSuccess) return fail(e);
  *status = rows != 0 ? rows : pair;
  return B2C_OK;
}

}  // namespace b2c

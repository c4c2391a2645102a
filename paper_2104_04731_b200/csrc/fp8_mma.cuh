// Device code shared by the two kernels that form products of block-scaled 8-bit matrices on the tensor core.
//
// The intrinsic adds unscaled products, and every block of 128 along the reduction has scales of its own.  So each
// block is an accumulator of its own in tensor memory (four MMAs of depth 32, the first one overwriting), and the
// epilogue warps add it, times the product of its two scales, to fp32 sums that they keep in registers.
#pragma once

#include "conv_mma_cluster.cuh"
#include "fp8_common.cuh"

namespace b2c {

namespace {

__device__ int g_fp8_status;  // first expired wait of this file's kernels on the device

// Reads and clears it; the device is idle.
inline cudaError_t take_status(int* status) {
  const int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(status, g_fp8_status, sizeof(int));
  if (e == cudaSuccess && *status != 0) e = cudaMemcpyToSymbol(g_fp8_status, &zero, sizeof(zero));
  return e;
}

// Instruction descriptor of kind::f8f6f4: D = fp32 (code 1 at bit 4), formats of A and B (E4M3 0, E5M2 1) at bits 7 and
// 10, both K-major, N/8 at bit 17, M/16 at bit 24.
__device__ __forceinline__ uint32_t make_idesc_f8(int m, int n, int a_type, int b_type) {
  return (1u << 4) | ((a_type == B2C_E5M2 ? 1u : 0u) << 7) | ((b_type == B2C_E5M2 ? 1u : 0u) << 10) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}

// One block of the reduction: `ksteps` (1..4) MMAs over consecutive 32-byte slices, the first overwrites.
template <int CTAS>
__device__ __forceinline__ void mma_f8_block(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t on, int ksteps) {
#define B2C_F8_BLOCK(GROUP)                                                              \
  asm volatile(                                                                          \
      "{\n"                                                                              \
      ".reg .pred pfalse, ptrue, q0, q1, q2, q3;\n"                                      \
      ".reg .b64 a1, a2, a3, b1, b2, b3;\n"                                              \
      "setp.ne.b32 pfalse, 0, 0;\n"                                                      \
      "setp.eq.b32 ptrue, 0, 0;\n"                                                       \
      "setp.ne.b32 q0, %4, 0;\n"                                                         \
      "setp.gt.and.s32 q1, %5, 1, q0;\n"                                                 \
      "setp.gt.and.s32 q2, %5, 2, q0;\n"                                                 \
      "setp.gt.and.s32 q3, %5, 3, q0;\n"                                                 \
      "add.u64 a1, %1, 2;\n"                                                             \
      "add.u64 b1, %2, 2;\n"                                                             \
      "add.u64 a2, %1, 4;\n"                                                             \
      "add.u64 b2, %2, 4;\n"                                                             \
      "add.u64 a3, %1, 6;\n"                                                             \
      "add.u64 b3, %2, 6;\n"                                                             \
      "@q0 tcgen05.mma.cta_group::" GROUP ".kind::f8f6f4 [%0], %1, %2, %3, pfalse;\n"    \
      "@q1 tcgen05.mma.cta_group::" GROUP ".kind::f8f6f4 [%0], a1, b1, %3, ptrue;\n"     \
      "@q2 tcgen05.mma.cta_group::" GROUP ".kind::f8f6f4 [%0], a2, b2, %3, ptrue;\n"     \
      "@q3 tcgen05.mma.cta_group::" GROUP ".kind::f8f6f4 [%0], a3, b3, %3, ptrue;\n"     \
      "}" ::"r"(d_tmem),                                                                 \
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(on), "r"(ksteps)                           \
      : "memory")
  if (CTAS == 1) B2C_F8_BLOCK("1");
  else B2C_F8_BLOCK("2");
#undef B2C_F8_BLOCK
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar, uint32_t on) {
  asm volatile(
      "{\n.reg .pred q;\nsetp.ne.b32 q, %6, 0;\n"
      "@q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n}" ::"r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar), "r"(on)
      : "memory");
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ float4 ld_shared_f4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// 64 consecutive accumulator columns of this thread's lane of tensor memory.
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, int32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, "
      "%22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32, %33, %34, %35, %36, %37, %38, %39, %40, %41, "
      "%42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, "
      "%62, %63}, [%64];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
        "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
        "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
        "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31]),
        "=r"(v[32]), "=r"(v[33]), "=r"(v[34]), "=r"(v[35]), "=r"(v[36]), "=r"(v[37]), "=r"(v[38]), "=r"(v[39]),
        "=r"(v[40]), "=r"(v[41]), "=r"(v[42]), "=r"(v[43]), "=r"(v[44]), "=r"(v[45]), "=r"(v[46]), "=r"(v[47]),
        "=r"(v[48]), "=r"(v[49]), "=r"(v[50]), "=r"(v[51]), "=r"(v[52]), "=r"(v[53]), "=r"(v[54]), "=r"(v[55]),
        "=r"(v[56]), "=r"(v[57]), "=r"(v[58]), "=r"(v[59]), "=r"(v[60]), "=r"(v[61]), "=r"(v[62]), "=r"(v[63])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// Bounded wait of the warps that keep sums in registers: as mbar_wait, without a call (which would have to save them).
__device__ __forceinline__ bool mbar_wait_inline(uint32_t bar, uint32_t parity, SharedCtl* ctl, int* status) {
  unsigned long long t0 = 0;
#pragma unroll 1
  for (int i = 0; !mbar_try_wait(bar, parity); ++i) {
    if (i < 32) continue;
    if (ctl->abort_flag) return false;
    const unsigned long long now = global_ns();
    if (t0 == 0) t0 = now;
    if (now - t0 > kWaitLimitNs) {
      ctl->abort_flag = 1;
      atomicCAS(status, 0, B2C_E_TIMEOUT);
      return false;
    }
  }
  return true;
}

// Each form of the wait, in a block of its own, on a barrier that nothing completes.
__global__ void __launch_bounds__(32) wait_selftest_kernel() {
  __shared__ SharedCtl ctl;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&ctl.full[0]), 1);
    ctl.abort_flag = 0;
  }
  __syncthreads();
  const bool ok = blockIdx.x == 0 ? mbar_wait(smem_u32(&ctl.full[0]), 0, &ctl, &g_fp8_status) : mbar_wait_inline(smem_u32(&ctl.full[0]), 0, &ctl, &g_fp8_status);
  if (__any_sync(0xffffffffu, ok)) atomicExch(&g_fp8_status, B2C_E_NOT_READY);  // (cannot be)
}
inline cudaError_t launch_wait_selftest(cudaStream_t st) {
  wait_selftest_kernel<<<2, 32, 0, st>>>();
  return cudaGetLastError();
}

// Row tile `index` over all groups, each group's rows cut into tiles of `tile` rows; called by a whole warp.  Offsets are
// clamped to [0, rows] and never fall, so the groups are disjoint and their tiles at most rows / tile + groups.
struct RowTile {
  int group, row0, row_end;  // group < 0: there is no such tile
};
__device__ __forceinline__ RowTile find_row_tile(const MatmulArgs& a, int index, int tile) {
  RowTile r = {-1, 0, 0};
  if (a.offsets == nullptr) {
    if ((long long)index * tile < a.rows) r = {0, index * tile, a.rows};
    return r;
  }
  const int lane = threadIdx.x & 31;
  int run = max(0, min(a.offsets[0], a.rows));
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
    const int tiles = (hi - lo + tile - 1) / tile;
    int sum = tiles;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += v;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, index < sum);
    if (hit) {
      const int l = __ffs(hit) - 1;
      r.group = g0 + l;
      r.row0 = __shfl_sync(0xffffffffu, lo + (index - (sum - tiles)) * tile, l);
      r.row_end = __shfl_sync(0xffffffffu, hi, l);
      return r;
    }
    index -= __shfl_sync(0xffffffffu, sum, 31);
    run = __shfl_sync(0xffffffffu, hi, 31);
  }
  return r;
}

}  // namespace
}  // namespace b2c

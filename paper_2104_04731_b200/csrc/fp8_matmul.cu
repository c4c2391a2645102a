// Products of block-scaled 8-bit matrices, plain arithmetic: one thread block computes a 64 x 64 tile of one
// group's rows, the operands are widened to fp32 in shared memory, the sums of a 128-element block are scaled and added.
#include "fp8_common.cuh"

namespace b2c {

namespace {

constexpr int kTile = 64;
constexpr int kDepth = 32;

__device__ int g_status;

// Row tile `index` over all groups, each group's rows in tiles of `tile` rows: its group, first row and end.
__device__ bool find_row_tile(const MatmulArgs& a, int index, int tile, int* group, int* row0, int* row_end) {
  int hi = a.offsets ? max(0, min(a.offsets[0], a.rows)) : 0;
  for (int g = 0; g < a.groups; ++g) {
    const int lo = hi;
    hi = a.offsets ? max(lo, min(a.offsets[g + 1], a.rows)) : a.rows;  // (an offset that falls counts as the one before it)
    const int tiles = (hi - lo + tile - 1) / tile;
    if (index < tiles) {
      *group = g;
      *row0 = lo + index * tile;
      *row_end = hi;
      return true;
    }
    index -= tiles;
  }
  return false;
}

__device__ void tile_sums(const MatmulArgs& a, const uint8_t* b, const float* b_scale, int row0, int row_end, int n0,
                          float (*As)[kTile + 1], float (*Bs)[kTile + 1], float acc[4][4]) {
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const int kb_all = (int)blocks_of(a.K);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
  for (int kb = 0; kb < kb_all; ++kb) {
    float part[4][4] = {};
    for (int k0 = kb * kBlock; k0 < min(a.K, (kb + 1) * kBlock); k0 += kDepth) {
      for (int i = threadIdx.x; i < kTile * kDepth; i += 256) {
        const int r = i / kDepth, k = k0 + i % kDepth;
        As[i % kDepth][r] = row0 + r < row_end && k < a.K ? fp8_to_float(((const uint8_t*)a.a)[(long long)(row0 + r) * a.lda + k], a.a_type) : 0.0f;
        Bs[i % kDepth][r] = n0 + r < a.N && k < a.K ? fp8_to_float(b[(long long)(n0 + r) * a.K + k], a.b_type) : 0.0f;
      }
      __syncthreads();
      for (int k = 0; k < kDepth; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) part[i][j] = fmaf(As[k][ty * 4 + i], Bs[k][tx * 4 + j], part[i][j]);
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int m = row0 + ty * 4 + i, n = n0 + tx * 4 + j;
        if (m < row_end && n < a.N)
          acc[i][j] = fmaf(part[i][j], a.a_scale[(long long)m * a.lds + kb] * b_scale[(long long)(n / kBlock) * kb_all + kb], acc[i][j]);
      }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) matmul_kernel(const MatmulArgs a) {
  __shared__ float As[kDepth][kTile + 1], Bs[kDepth][kTile + 1];
  pdl_wait();
  pdl_launch_dependents();
  int g, row0, row_end;
  if (!find_row_tile(a, blockIdx.y, kTile, &g, &row0, &row_end)) return;
  const int n0 = blockIdx.x * kTile;
  float acc[4][4];
  tile_sums(a, (const uint8_t*)a.b + (long long)g * a.N * a.K, a.b_scale + (long long)g * blocks_of(a.N) * blocks_of(a.K), row0, row_end, n0,
            As, Bs, acc);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int m = row0 + threadIdx.x / 16 * 4 + i, n = n0 + threadIdx.x % 16 * 4 + j;
      if (m < row_end && n < a.N) ((T*)a.y)[(long long)m * a.ldy + n] = from_float<T>(acc[i][j]);
    }
}

// Gate and up products of 64 rows x 128 columns, then the activation and the quantisation of the 1 x 128 blocks.
__global__ void __launch_bounds__(256) matmul_gated_kernel(const MatmulArgs a) {
  extern __shared__ float dyn[];
  float(*As)[kTile + 1] = (float(*)[kTile + 1])dyn;
  float(*Bs)[kTile + 1] = As + kDepth;
  float* H = (float*)(Bs + kDepth);  // [64][128]
  pdl_wait();
  pdl_launch_dependents();
  int g, row0, row_end;
  if (!find_row_tile(a, blockIdx.y, kTile, &g, &row0, &row_end)) return;
  for (int half = 0; half < 2; ++half) {
    const int n0 = blockIdx.x * kBlock + half * kTile;
    float gate[4][4], up[4][4];
    const long long mat = (long long)a.N * a.K, sc = blocks_of(a.N) * blocks_of(a.K);
    tile_sums(a, (const uint8_t*)a.b + 2 * g * mat, a.b_scale + 2 * g * sc, row0, row_end, n0, As, Bs, gate);
    tile_sums(a, (const uint8_t*)a.b + (2 * g + 1) * mat, a.b_scale + (2 * g + 1) * sc, row0, row_end, n0, As, Bs, up);
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j)
        H[(threadIdx.x / 16 * 4 + i) * kBlock + half * kTile + threadIdx.x % 16 * 4 + j] = silu(gate[i][j]) * up[i][j];
  }
  __syncthreads();
  for (int r = threadIdx.x / 8; r < kTile; r += 32) {
    const int m = row0 + r, c0 = blockIdx.x * kBlock + threadIdx.x % 8 * 16;
    float v[16], mx = 0.0f;
    for (int i = 0; i < 16; ++i) {
      v[i] = c0 + i < a.N ? H[r * kBlock + threadIdx.x % 8 * 16 + i] : 0.0f;
      mx = fmaxf(mx, fabsf(v[i]));
    }
    for (int d = 4; d > 0; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    const BlockScale s = block_scale<B2C_E4M3>(mx);
    const uint4 w = quantize16<B2C_E4M3>(s, v);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    if (m >= row_end) continue;
    for (int i = 0; i < 16; ++i)
      if (c0 + i < a.N) ((uint8_t*)a.y)[(long long)m * a.ldy + c0 + i] = (uint8_t)(u[i >> 2] >> (8 * (i & 3)));
    if (threadIdx.x % 8 == 0) a.y_scale[(long long)m * a.ldys + blockIdx.x] = s.scale;
  }
}

}  // namespace

int launch_fp8_matmul(const MatmulArgs& a, cudaStream_t st) {
  // every group adds at most one tile that is not full
  const long long row_tiles = a.rows / kTile + std::min<long long>(a.groups, a.rows);
  if (row_tiles > 65535) return B2C_E_UNSUPPORTED;
  cudaError_t e;
  if (a.gated) {
    const size_t smem = (2 * kDepth * (kTile + 1) + kTile * kBlock) * sizeof(float);
    static std::atomic<unsigned long long> configured{0};
    e = set_max_dynamic_smem_once(configured, (const void*)matmul_gated_kernel, (int)smem);
    if (e == cudaSuccess)
      e = launch_pdl(matmul_gated_kernel, dim3((unsigned)blocks_of(a.N), (unsigned)row_tiles), dim3(256), smem, st, a);
  } else {
    const dim3 grid((unsigned)((a.N + kTile - 1) / kTile), (unsigned)row_tiles);
    if (a.y_type == B2C_F32) e = launch_pdl(matmul_kernel<float>, grid, dim3(256), 0, st, a);
    else if (a.y_type == B2C_F16) e = launch_pdl(matmul_kernel<__half>, grid, dim3(256), 0, st, a);
    else e = launch_pdl(matmul_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, a);
  }
  if (e != cudaSuccess) {
    set_last_cuda_error((int)e);
    return B2C_E_CUDA;
  }
  return B2C_OK;
}

int fp8_status_read_and_clear(int32_t* status) {
  int s = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&s, g_status, sizeof(s));
  const int zero = 0;
  if (e == cudaSuccess && s != 0) e = cudaMemcpyToSymbol(g_status, &zero, sizeof(zero));
  if (e != cudaSuccess) {
    set_last_cuda_error((int)e);
    return B2C_E_CUDA;
  }
  *status = s;
  return B2C_OK;
}

}  // namespace b2c

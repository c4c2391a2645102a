// Internal declarations of the 4-bit float operators (quantisation with microscales, block-scaled products, expert layers), shared by
// their host code and kernel launchers.
#pragma once

#include "fp8_internal.h"

namespace b2c {

constexpr int kFp4Stage = 256;  // reduction elements of a stage: 128 bytes of a row, the width of a swizzled tile

#ifdef __CUDACC__
__host__ __device__
#endif
inline int fp4_block(int format) { return format == B2C_MXFP4 ? 32 : 16; }
#ifdef __CUDACC__
__host__ __device__
#endif
inline long long fp4_scales(long long cols, int format) { return (cols + fp4_block(format) - 1) / fp4_block(format); }
inline long long fp4_scale_pitch(long long cols, int format) { return (fp4_scales(cols, format) + 15) / 16 * 16; }

struct Quantize4Args {
  const void* x;
  long long ldx;
  uint8_t* q;
  long long ldq;
  uint8_t* scale;
  long long lds;
  const float* global;
  long long rows;
  int cols;
  int x_type, format;
  // Rows of an expert layer: input row t is written to output rows map[t * copies + j] (none where negative).
  const int32_t* map;
  int copies;
};

struct Dequantize4Args {
  const uint8_t* q;
  long long ldq;
  const uint8_t* scale;
  long long lds;
  const float* global;
  long long rows;
  int cols;
  int y_type, format;
  void* y;
  long long ldy;
};

struct Matmul4Args {
  const uint8_t* a;  // [rows][K / 2]
  long long lda;
  const uint8_t* a_scale;
  long long lds;
  const uint8_t* b;  // [groups][N][K / 2]; gated: [groups][2][N][K / 2], gate rows then up rows
  const uint8_t* b_scale;
  long long ldbs;
  const float* alpha;   // [groups] or null
  const float* alpha2;  // one more factor of all groups, or null
  const int32_t* offsets;
  void* y;              // gated: packed values
  long long ldy;        // (gated: bytes)
  uint8_t* y_scale;     // gated only
  long long ldys;
  const float* y_global;  // gated only: factor that the results are quantised with
  int rows, N, K, groups;
  int format, y_type;
  int early;  // weights and offsets are older than the kernel before this one (see matmul4_rows_kernel)
  int gated;  // y = quantise(silu(a . gate) * (a . up))
};

// Rows of a group, on average (all rows without groups).
inline int rows_of_a_group(const Matmul4Args& a) { return a.offsets ? (int)(((long long)a.rows + a.groups - 1) / a.groups) : a.rows; }

// Rows of a tile of a product by groups: 16, 32 or 64 by the kernel for few rows, 128 by that for many.  A tile holds half as many rows again as a
// group has on average: a second tile of a group reads its weights again (256 tokens, 4 of 64 experts, 16 rows a group: 87 us by tiles of 16, 74 of
// 32; 64 rows a group: 109 us by tiles of 64, 80 of 128).  (In 64 bits: one group may have all rows.)
inline int rows_of_a_group_tile(const Matmul4Args& a) {
  const long long average = rows_of_a_group(a), rows = average + average / 2;
  return rows <= 16 ? 16 : (rows <= 32 ? 32 : (rows <= 64 ? 64 : 128));
}

// The expert layer of few tokens (see fp4_experts.cu).
constexpr int kFewPairs = 512;
struct Few4Args {
  const void* x;
  long long ldx;
  const int32_t* ids;
  const float* weights;
  const uint8_t *w1, *w1_scale, *w2, *w2_scale;
  long long ld1, ld2;
  const float *x_global, *w1_global, *h_global, *w2_global;
  uint8_t *hq, *hs;  // [pairs][inter / 2], [pairs][ldhs]
  long long ldhs;
  float* part;       // [pairs][hidden]
  int32_t* done;     // [128 columns of hidden]
  void* y;
  long long ldy;
  int pairs, topk, experts, hidden, inter, type, format;
};

cudaError_t launch_fp4_quantize(const Quantize4Args& a, cudaStream_t st);
cudaError_t launch_fp4_dequantize(const Dequantize4Args& a, cudaStream_t st);
int launch_fp4_matmul(const Matmul4Args& a, cudaStream_t st);  // B2C_* code
int launch_fp4_matmul_pair(const Matmul4Args& a, cudaStream_t st);  // its form for many rows
long long fp4_pair_ns(const Matmul4Args& a);  // what it takes without groups, about
cudaError_t fp4_pair_status(int* status);
int launch_fp4_few_experts(const Few4Args& a, cudaStream_t st);
cudaError_t fp4_few_status(int* status);
cudaError_t fp4_few_wait_selftest(cudaStream_t st);
int fp4_status_read_and_clear(int32_t* status);
cudaError_t fp4_rows_wait_selftest(cudaStream_t st);
cudaError_t fp4_pair_wait_selftest(cudaStream_t st);

}  // namespace b2c

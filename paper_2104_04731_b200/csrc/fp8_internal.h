// Internal declarations of the 8-bit float operators (block quantisation, products with a scale per block of 128,
// routing, expert layers), shared by their host code and kernel launchers.
#pragma once

#include <algorithm>

#include "b2c_internal.h"

namespace b2c {

constexpr int kBlock = 128;        // reduction elements (and weight rows) that share one scale
constexpr int kMaxExperts = 1024;  // groups of a product, experts of a route
constexpr int kMaxTopk = 32;
constexpr int kMaxRouteGroups = 32;
constexpr long long kMaxRows = 0x7FFFFF00LL;  // rows of one call: tile origins stay inside 32 bits
constexpr int kMaxCols = 1 << 30;  // columns and reduction lengths: so do the columns that a tile rounds up to
constexpr long long kMaxStride = 1ll << 40;  // bytes; tensor maps hold no more
constexpr float kMinAmax = 0x1p-100f;         // a block's largest magnitude counts as at least this much

#ifdef __CUDACC__
__host__ __device__
#endif
inline long long blocks_of(long long n) { return (n + kBlock - 1) / kBlock; }
inline int type_bytes(int t) { return t == B2C_F32 ? 4 : (t == B2C_F16 || t == B2C_BF16 ? 2 : 1); }

struct QuantizeArgs {
  const void* x;
  long long ldx;
  uint8_t* q;
  long long ldq;
  float* scale;
  long long lds;
  long long rows;
  int cols;
  int block_rows;  // 1 or 128
  int x_type, q_type;
  // Rows of an expert layer: input row t is written to output rows map[t * copies + j] (none where negative).
  const int32_t* map;
  int copies;
};

struct MatmulArgs {
  const void* a;
  long long lda;
  const float* a_scale;
  long long lds;
  const void* b;         // [groups][N][K]; gated: [groups][2][N][K], gate rows then up rows
  const float* b_scale;  // [groups][ceil(N/128)][ceil(K/128)]; gated: [groups][2][...]
  const int32_t* offsets;  // [groups + 1], or null with one group of all rows
  void* y;               // gated: 8-bit values
  long long ldy;
  float* y_scale;        // gated only
  long long ldys;
  int rows, N, K, groups;
  int a_type, b_type, y_type;
  int early;             // weights and offsets are older than the kernel before this one (see matmul_rows_kernel)
  int gated;             // y = quantise(silu(a . gate) * (a . up)), blocks of 1 x 128
};

// Rows of a group, on average (all rows without groups).
inline int rows_of_a_group(const MatmulArgs& a) { return a.offsets ? (int)(((long long)a.rows + a.groups - 1) / a.groups) : a.rows; }

// Whether the copy engine can take a product's results out (boxes of a map of bytes): rows on its 16-byte grid, and the byte a row ends
// at within the copy's 32-bit coordinates.
inline bool results_by_copy(const MatmulArgs& a) {
  const long long bytes = type_bytes(a.y_type);
  return !a.gated && (reinterpret_cast<uintptr_t>(a.y) & 15) == 0 && a.ldy * bytes % 16 == 0 && a.N * bytes <= 0x7FFFFFFFLL;
}

struct RouteArgs {
  b2c_route_desc d;
  long long tokens;
  const void* logits;
  long long ld;
  const float* bias;
  float* weights;
  int32_t* ids;
};

cudaError_t launch_fp8_quantize(const QuantizeArgs& a, cudaStream_t st);
// launch_route_sort and launch_fp8_quantize (E4M3 rows, a.copies slots a token) in one, for at most kSmallPairs pairs.
constexpr int kSmallPairs = 1024;
cudaError_t launch_sort_quantize(const QuantizeArgs& a, const int32_t* ids, int pairs, int experts, int32_t* offsets, int32_t* rows,
                                 cudaStream_t st);
int launch_fp8_matmul(const MatmulArgs& a, cudaStream_t st);  // B2C_* code
int launch_fp8_matmul_pair(const MatmulArgs& a, cudaStream_t st);  // its form for many rows
long long pair_cycles(const MatmulArgs& a);  // what it takes without groups, in SM cycles
cudaError_t fp8_pair_status(int* status);
int fp8_status_read_and_clear(int32_t* status);
cudaError_t fp8_rows_wait_selftest(cudaStream_t st);
cudaError_t fp8_pair_wait_selftest(cudaStream_t st);
cudaError_t launch_route(const RouteArgs& a, cudaStream_t st);
size_t route_sort_workspace(long long pairs, int experts);
cudaError_t launch_route_sort(const int32_t* ids, long long pairs, int experts, int32_t* offsets, int32_t* rows,
                              int32_t* order, int32_t* workspace, cudaStream_t st);
cudaError_t launch_route_combine(const void* y, int y_type, long long y_rows, long long ldy, const int32_t* rows, const float* weights,
                                 long long tokens, int topk, int cols, void* out, int out_type, long long ldo,
                                 cudaStream_t st);

}  // namespace b2c

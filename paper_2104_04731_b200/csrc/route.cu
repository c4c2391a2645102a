// Routing of tokens to experts: scores, groups and the best experts of each token; the stable sort of the
// (token, slot) pairs by expert; the weighted sum of the experts' results.
#include "fp8_common.cuh"

namespace b2c {

namespace {

constexpr unsigned kAll = 0xffffffffu;

// Doubles as unsigned integers of the same order (NaN below everything else, but above 0, which marks what is out).
__device__ __forceinline__ unsigned long long order_key(double v) {
  if (v != v) return 1ull;
  const long long b = __double_as_longlong(v);
  return b < 0 ? ~(unsigned long long)b : (unsigned long long)b | 0x8000000000000000ull;
}
// The larger key, at equal keys the lower index, over the warp.
__device__ __forceinline__ void warp_best(unsigned long long* key, int* index) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    const unsigned long long k = __shfl_xor_sync(kAll, *key, d);
    const int i = __shfl_xor_sync(kAll, *index, d);
    if (k > *key || (k == *key && i < *index)) {
      *key = k;
      *index = i;
    }
  }
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  return v;
}

// One warp for one token; the scores and choices of its row lie in shared memory.
template <typename T>
__global__ void __launch_bounds__(128) route_kernel(const RouteArgs a) {
  extern __shared__ double dyn[];
  pdl_wait();
  pdl_launch_dependents();
  const int E = a.d.experts, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long t = (long long)blockIdx.x * 4 + warp;
  if (t >= a.tokens) return;
  double* score = dyn + (size_t)warp * 2 * E;
  double* choice = score + E;
  const T* row = (const T*)a.logits + t * a.ld;
  double mx = -INFINITY;
  for (int e = lane; e < E; e += 32) {
    double x = (double)to_float<T>(row[e]);
    if (x != x) x = -INFINITY;
    score[e] = x;
    mx = fmax(mx, x);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) mx = fmax(mx, __shfl_xor_sync(kAll, mx, d));
  double sum = 0.0;
  for (int e = lane; e < E; e += 32) {
    const double x = score[e];
    double s;
    if (a.d.score == B2C_SCORE_SIGMOID) s = x == -INFINITY ? 0.0 : 1.0 / (1.0 + exp(-x));
    else s = x == -INFINITY ? 0.0 : (x == mx ? 1.0 : exp(x - mx));
    score[e] = s;
    sum += s;
  }
  if (a.d.score == B2C_SCORE_SOFTMAX) sum = warp_sum(sum);
  for (int e = lane; e < E; e += 32) {
    double s = score[e];
    if (a.d.score == B2C_SCORE_SOFTMAX) {
      s = sum > 0.0 ? s / sum : 0.0;
      score[e] = s;
    }
    choice[e] = a.bias ? s + (double)a.bias[e] : s;
  }
  __syncwarp();
  const int G = a.d.groups, size = E / G;
  unsigned open = 0xffffffffu;  // groups that stay
  if (G > 1) {
    unsigned long long key = 0;
    if (lane < G) {
      double first = -INFINITY, second = -INFINITY;
      for (int i = 0; i < size; ++i) {
        const double v = choice[lane * size + i];
        if (v > first) {
          second = first;
          first = v;
        } else if (v > second) {
          second = v;
        }
      }
      key = order_key(a.d.group_score == B2C_GROUP_MAX || size == 1 ? first : first + second);
    }
    int better = 0;
    for (int g = 0; g < G; ++g) {
      const unsigned long long k = __shfl_sync(kAll, key, g);
      better += k > key || (k == key && g < lane);
    }
    open = __ballot_sync(kAll, lane < G && better < a.d.topk_groups);
  }
  double total = 0.0, mine = 0.0;
  int my_id = 0;
  unsigned taken = 0;  // of this lane's experts, lane + 32 * i
  for (int j = 0; j < a.d.topk; ++j) {
    unsigned long long key = 0;
    int index = 0x7FFFFFFF;
    for (int i = 0, e = lane; e < E; e += 32, ++i) {
      if ((taken >> i) & 1u || (G > 1 && !((open >> (e / size)) & 1u))) continue;
      const unsigned long long k = order_key(choice[e]);
      if (k > key) {
        key = k;
        index = e;
      }
    }
    warp_best(&key, &index);
    if ((index & 31) == lane) taken |= 1u << (index >> 5);
    const double s = score[index];
    total += s;
    if (lane == j) {
      mine = s;
      my_id = index;
    }
  }
  if (lane < a.d.topk) {
    const double w = a.d.renormalise ? (total > 0.0 ? mine / total : 0.0) : mine;
    a.weights[t * a.d.topk + lane] = (float)(w * (double)a.d.scale);
    a.ids[t * a.d.topk + lane] = my_id;
  }
}

// ---- stable sort of the pairs by expert ---------------------------------------------------------------------------

constexpr int kChunk = 1024;  // pairs of one thread block, one a thread

// How many pairs of each chunk go to each expert.
__global__ void __launch_bounds__(kChunk) count_kernel(const int32_t* ids, const long long pairs, const int experts, int32_t* counts) {
  extern __shared__ int hist[];
  pdl_wait();
  pdl_launch_dependents();
  for (int e = threadIdx.x; e < experts; e += kChunk) hist[e] = 0;
  __syncthreads();
  const long long p = (long long)blockIdx.x * kChunk + threadIdx.x;
  const int id = p < pairs ? ids[p] : -1;
  if (id >= 0 && id < experts) atomicAdd(&hist[id], 1);  // (integers: the order does not matter)
  __syncthreads();
  for (int e = threadIdx.x; e < experts; e += kChunk) counts[(size_t)blockIdx.x * experts + e] = hist[e];
}

// Places of a chunk's pairs: the experts before, the chunks before, the warps before, the lanes before.
__global__ void __launch_bounds__(kChunk) place_kernel(const int32_t* ids, const long long pairs, const int experts, const int32_t* counts,
                                                      const int chunks, int32_t* offsets, int32_t* rows, int32_t* order) {
  extern __shared__ int smem[];
  int* base = smem;                 // [experts]: first place of this chunk's pairs of the expert
  int* by_warp = smem + experts;    // [32][experts]
  __shared__ int warp_total[32];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < 32 * experts; i += kChunk) by_warp[i] = 0;
  __syncthreads();
  const long long p = (long long)blockIdx.x * kChunk + threadIdx.x;
  int id = p < pairs ? ids[p] : -1;
  if (id >= experts) id = -1;
  const unsigned same = __match_any_sync(kAll, id);
  const int rank = __popc(same & ((1u << lane) - 1u));
  if (id >= 0 && rank == 0) by_warp[warp * experts + id] = __popc(same);
  __syncthreads();
  // expert e (experts <= 1024: one a thread): pairs of all chunks, of the chunks before this one
  const int e = threadIdx.x;
  int all = 0, before = 0;
  if (e < experts) {
    if (counts != nullptr) {
      for (int c = 0; c < chunks; ++c) {
        const int n = counts[(size_t)c * experts + e];
        if (c < (int)blockIdx.x) before += n;
        all += n;
      }
    }
    int run = 0;
    for (int w = 0; w < 32; ++w) {
      const int n = by_warp[w * experts + e];
      by_warp[w * experts + e] = run;
      run += n;
    }
    if (counts == nullptr) all = run;
  }
  int scan = all;  // inclusive over the experts
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int n = __shfl_up_sync(kAll, scan, d);
    if (lane >= d) scan += n;
  }
  if (lane == 31) warp_total[warp] = scan;
  __syncthreads();
  if (warp == 0) {
    int n = warp_total[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int up = __shfl_up_sync(kAll, n, d);
      if (lane >= d) n += up;
    }
    warp_total[lane] = n;
  }
  __syncthreads();
  if (warp > 0) scan += warp_total[warp - 1];
  if (e < experts) {
    base[e] = scan - all + before;
    if (blockIdx.x == 0) {
      if (e == 0) offsets[0] = 0;
      offsets[e + 1] = scan;
    }
  }
  __syncthreads();
  if (p < pairs) {
    const int at = id >= 0 ? base[id] + by_warp[warp * experts + id] + rank : -1;
    rows[p] = at;
    if (order != nullptr && at >= 0) order[at] = (int)p;
  }
}

// ---- weighted sum ---------------------------------------------------------------------------------------------------

// W neighbouring columns of a row in one load and one store (1 where alignment or width do not allow more).
template <typename T, int W>
__device__ __forceinline__ void load_cols(const T* p, float* v) {
  if constexpr (W == 1) {
    v[0] = to_float<T>(p[0]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const float4 f = *reinterpret_cast<const float4*>(p + i);
      v[i] = f.x;
      v[i + 1] = f.y;
      v[i + 2] = f.z;
      v[i + 3] = f.w;
    }
  } else {
    static_assert(W == 8, "16 bytes");
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2<T>(w[i], &v[2 * i], &v[2 * i + 1]);
  }
}
template <typename T, int W>
__device__ __forceinline__ void store_cols(T* p, const float* v) {
  if constexpr (W == 1) {
    p[0] = from_float<T>(v[0]);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < W; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
  }
}

// Weighted sum of a token's rows: memory-bound, every row is read once.  A thread has W columns of one token; four slots'
// loads are under way together.
template <typename YT, typename OT, int W>
__global__ void __launch_bounds__(256) combine_kernel(const YT* y, const long long y_rows, const long long ldy, const int32_t* rows,
                                                     const float* weights, const long long tokens, const int topk, const int cols,
                                                     const int pieces, OT* out, const long long ldo) {
  pdl_wait();
  pdl_launch_dependents();
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long t = id / pieces;
  const int c = (int)(id - t * pieces) * W;
  if (t >= tokens) return;
  const int32_t* r = rows + t * topk;
  const float* wt = weights + t * topk;
  float sum[W];
#pragma unroll
  for (int i = 0; i < W; ++i) sum[i] = 0.0f;
  for (int j0 = 0; j0 < topk; j0 += 4) {
    float v[4][W], w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = j0 + j < topk ? r[j0 + j] : -1;
      const bool on = row >= 0 && row < y_rows;
      w[j] = on ? wt[j0 + j] : 0.0f;
#pragma unroll
      for (int i = 0; i < W; ++i) v[j][i] = 0.0f;
      if (on) load_cols<YT, W>(y + row * ldy + c, v[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < W; ++i) sum[i] = fmaf(w[j], v[j][i], sum[i]);
  }
  store_cols<OT, W>(out + t * ldo + c, sum);
}

}  // namespace

cudaError_t launch_route(const RouteArgs& a, cudaStream_t st) {
  const size_t smem = 4 * 2 * (size_t)a.d.experts * sizeof(double);
  const dim3 grid((unsigned)((a.tokens + 3) / 4));
  cudaError_t e;
#define B2C_ROUTE(T)                                                                                    \
  {                                                                                                     \
    static std::atomic<unsigned long long> configured{0};                                               \
    e = set_max_dynamic_smem_once(configured, (const void*)route_kernel<T>, 4 * 2 * kMaxExperts * 8);    \
    if (e == cudaSuccess) e = launch_pdl(route_kernel<T>, grid, dim3(128), smem, st, a);                 \
  }
  if (a.d.logit_type == B2C_F32) B2C_ROUTE(float)
  else if (a.d.logit_type == B2C_F16) B2C_ROUTE(__half)
  else B2C_ROUTE(__nv_bfloat16)
#undef B2C_ROUTE
  return e;
}

size_t route_sort_workspace(long long pairs, int experts) {
  return pairs <= kChunk ? 0 : (size_t)((pairs + kChunk - 1) / kChunk) * experts * sizeof(int32_t);
}

cudaError_t launch_route_sort(const int32_t* ids, long long pairs, int experts, int32_t* offsets, int32_t* rows, int32_t* order,
                              int32_t* workspace, cudaStream_t st) {
  const int chunks = (int)std::max<long long>(1, (pairs + kChunk - 1) / kChunk);
  const size_t smem = (size_t)33 * experts * sizeof(int);
  static std::atomic<unsigned long long> configured{0};
  cudaError_t e = set_max_dynamic_smem_once(configured, (const void*)place_kernel, 33 * kMaxExperts * (int)sizeof(int));
  if (e != cudaSuccess) return e;
  if (chunks > 1) {
    e = launch_pdl(count_kernel, dim3((unsigned)chunks), dim3(kChunk), experts * sizeof(int), st, ids, pairs, experts, workspace);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(place_kernel, dim3((unsigned)chunks), dim3(kChunk), smem, st, ids, pairs, experts,
                    (const int32_t*)(chunks > 1 ? workspace : nullptr), chunks, offsets, rows, order);
}

namespace {

template <typename YT, typename OT>
cudaError_t combine(const void* y, long long y_rows, long long ldy, const int32_t* rows, const float* weights, long long tokens, int topk,
                    int cols, void* out, long long ldo, cudaStream_t st) {
  auto fits = [](const void* p, long long ld, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld * bytes) % 16 == 0; };
  const bool wide = cols % 8 == 0 && fits(y, ldy, sizeof(YT)) && fits(out, ldo, sizeof(OT));
  const int pieces = wide ? cols / 8 : cols;
  const long long grid = (tokens * pieces + 255) / 256;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  return launch_pdl(wide ? combine_kernel<YT, OT, 8> : combine_kernel<YT, OT, 1>, dim3((unsigned)grid), dim3(256), 0, st, (const YT*)y, y_rows,
                    ldy, rows, weights, tokens, topk, cols, pieces, (OT*)out, ldo);
}

}  // namespace

cudaError_t launch_route_combine(const void* y, int y_type, long long y_rows, long long ldy, const int32_t* rows, const float* weights,
                                 long long tokens, int topk, int cols, void* out, int out_type, long long ldo, cudaStream_t st) {
#define B2C_COMBINE(YT)                                                                                                        \
  return out_type == B2C_F32   ? combine<YT, float>(y, y_rows, ldy, rows, weights, tokens, topk, cols, out, ldo, st)           \
         : out_type == B2C_F16 ? combine<YT, __half>(y, y_rows, ldy, rows, weights, tokens, topk, cols, out, ldo, st)          \
                               : combine<YT, __nv_bfloat16>(y, y_rows, ldy, rows, weights, tokens, topk, cols, out, ldo, st)
  if (y_type == B2C_F32) B2C_COMBINE(float);
  if (y_type == B2C_F16) B2C_COMBINE(__half);
  B2C_COMBINE(__nv_bfloat16);
#undef B2C_COMBINE
}

}  // namespace b2c

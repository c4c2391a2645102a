// Block quantisation to 8-bit floating point, one scale for each 1 x 128 or 128 x 128 block.  Memory-bound: every
// element is read once and kept in registers between the search for the largest magnitude and the conversion.
#include "fp8_common.cuh"

namespace b2c {

namespace {

constexpr int kThreads = 256;
constexpr int kLanes = kBlock / 16;  // lanes that share a row of a block, 16 elements each

// A lane's 16 elements of the 128 of a block: neighbours, moved by 16-byte loads and stores, where x and q lie on that grid; else every
// eighth one, so that the eight lanes of a block move neighbouring elements (16 neighbours a lane, one by one, made 11353 x 1183 bf16
// take 57 us).
template <bool WIDE>
struct Part {
  static constexpr bool wide = WIDE;
  __device__ __forceinline__ int at(int sub, int i) const { return WIDE ? sub * 16 + i : i * kLanes + sub; }
};

template <typename T, bool WIDE>
__device__ __forceinline__ void load_part(const QuantizeArgs& a, Part<WIDE> part, long long row, int blk, int sub, float* v) {
  const T* p = (const T*)a.x + row * a.ldx + blk * kBlock;
  const int left = a.cols - blk * kBlock;
  if (part.wide && sub * 16 + 16 <= left) {
    widen16<T>(load_raw16<T>(p + sub * 16), v);
  } else if (!part.wide || sub * 16 < left) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = part.at(sub, i) < left ? to_float<T>(p[part.at(sub, i)]) : 0.0f;
  }
}
template <bool WIDE>
__device__ __forceinline__ void store_part(const QuantizeArgs& a, Part<WIDE> part, long long row, int blk, int sub, const uint4& w) {
  uint8_t* p = a.q + row * a.ldq + blk * kBlock;
  const int left = a.cols - blk * kBlock;
  if (part.wide && sub * 16 + 16 <= left) {
    *reinterpret_cast<uint4*>(p + sub * 16) = w;
  } else if (!part.wide || sub * 16 < left) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (part.at(sub, i) < left) p[part.at(sub, i)] = (uint8_t)(u[i >> 2] >> (8 * (i & 3)));
  }
}
__device__ __forceinline__ float amax16(const float* v) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(v[i]));
  return m;
}

// The 16 values of a lane to the row, or the rows, of its block.
template <bool WIDE>
__device__ __forceinline__ void store_block(const QuantizeArgs& a, Part<WIDE> part, long long row, int blk, int sub, const BlockScale& s, const uint4& w) {
  for (int j = 0; j < (a.map == nullptr ? 1 : a.copies); ++j) {
    const long long to = a.map == nullptr ? row : (long long)a.map[row * a.copies + j];
    if (to < 0) continue;
    store_part(a, part, to, blk, sub, w);
    if (sub == 0) a.scale[to * a.lds + blk] = s.scale;
  }
}
__device__ __forceinline__ float block_max(float m) {
#pragma unroll
  for (int d = kLanes / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  return m;
}

// Eight lanes hold the 128 elements of a block, three shuffles give the maximum.
template <typename T, int QT, bool WIDE>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const QuantizeArgs a, const int nb, const long long blocks) {
  constexpr Part<WIDE> part;
  pdl_wait();
  pdl_launch_dependents();
  const long long id = (long long)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  const bool on = id < blocks;
  const long long row = on ? id / nb : 0;
  const int blk = on ? (int)(id - row * nb) : 0, sub = threadIdx.x % kLanes;
  float v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = 0.0f;
  if (on) load_part<T>(a, part, row, blk, sub, v);
  const float m = block_max(amax16(v));
  if (!on) return;
  const BlockScale s = block_scale<QT>(m);
  store_block(a, part, row, blk, sub, s, quantize16<QT>(s, v));
}

// The same for many blocks of aligned rows.  What bounds it there are instructions, not bytes (16384 x 8192 bf16 took 82 us with
// the kernel above, 283 instructions for 16 elements of a lane): four lanes share a block, so that what is done once a block is done
// for 32 elements, the maximum is formed on packed pairs, and the loads of the next block are under way while this one is converted
// (65 us, 6.3 TB/s: the rate of a plain copy).
constexpr int kFewLanes = 4;
template <typename T, int QT>
__global__ void __launch_bounds__(kThreads) quantize_many_rows_kernel(const QuantizeArgs a, const FastDiv nb, const unsigned blocks) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int kGroups = kThreads / kFewLanes;
  const int part = (threadIdx.x % kFewLanes) * 16;  // elements [part, part + 16) and 64 further on
  const unsigned step = gridDim.x * kGroups;
  unsigned id = blockIdx.x * kGroups + threadIdx.x / kFewLanes;
  Raw16<T> next[2] = {};
  auto fetch = [&](unsigned b) {
    const unsigned row = nb.div(b);
    const int c0 = (int)(b - row * nb.d) * kBlock + part;
    const T* p = (const T*)a.x + (long long)row * a.ldx + c0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (b < blocks && c0 + 64 * h < a.cols) next[h] = load_raw16<T>(p + 64 * h);
      else next[h] = {};
    }
  };
  fetch(id);
  for (unsigned first = blockIdx.x * kGroups; first < blocks; first += step, id += step) {  // (the same for all lanes of a warp)
    const Raw16<T> raw[2] = {next[0], next[1]};
    fetch(id + step);
    float m = fmaxf(raw_max(raw[0]), raw_max(raw[1]));
#pragma unroll
    for (int d = kFewLanes / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (id >= blocks) continue;
    const BlockScale s = block_scale<QT>(m);
    uint4 w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float v[16];
      widen16<T>(raw[h], v);
      w[h] = quantize16<QT>(s, v);
    }
    const unsigned row = nb.div(id);
    const int blk = (int)(id - row * nb.d), c0 = blk * kBlock + part;
    for (int j = 0; j < (a.map == nullptr ? 1 : a.copies); ++j) {
      const long long to = a.map == nullptr ? (long long)row : (long long)a.map[(long long)row * a.copies + j];
      if (to < 0) continue;
      uint8_t* q = a.q + to * a.ldq + c0;
      if (c0 < a.cols) *reinterpret_cast<uint4*>(q) = w[0];
      if (c0 + 64 < a.cols) *reinterpret_cast<uint4*>(q + 64) = w[1];
      if (part == 0) a.scale[to * a.lds + blk] = s.scale;
    }
  }
}

// One thread block holds a 128 x 128 block in registers: four rows of 16 elements a thread.  8200 x 5136 fp32: 35 us, 5.9 TB/s; three blocks
// an SM, so that one stores while another waits for its largest magnitude.
template <typename T, int QT, bool WIDE>
__global__ void __launch_bounds__(kThreads, 3) quantize_blocks_kernel(const QuantizeArgs a, const int nb) {
  constexpr Part<WIDE> part;
  __shared__ float part_max[kThreads / 32];
  pdl_wait();
  pdl_launch_dependents();
  const long long rb = blockIdx.x / nb;
  const int blk = (int)(blockIdx.x - rb * nb), sub = threadIdx.x % kLanes;
  const long long row0 = rb * kBlock + threadIdx.x / kLanes;
  constexpr int kStep = kThreads / kLanes, kRows = kBlock / kStep;
  float v[kRows][16];
  float m = 0.0f;
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[r][i] = 0.0f;
    if (row0 + r * kStep < a.rows) load_part<T>(a, part, row0 + r * kStep, blk, sub, v[r]);
  }
#pragma unroll
  for (int r = 0; r < kRows; ++r) m = fmaxf(m, amax16(v[r]));
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  if (threadIdx.x % 32 == 0) part_max[threadIdx.x / 32] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) m = fmaxf(m, part_max[i]);
  const BlockScale s = block_scale<QT>(m);
#pragma unroll
  for (int r = 0; r < kRows; ++r)
    if (row0 + r * kStep < a.rows) store_part(a, part, row0 + r * kStep, blk, sub, quantize16<QT>(s, v[r]));
  if (threadIdx.x == 0) a.scale[rb * a.lds + blk] = s.scale;
}

// Sort and quantisation of a small batch on its way into an expert layer, in one launch: a thread block takes one token and sorts all
// pairs for itself (at most kSmallPairs, in shared memory), because a launch of its own for the sort costs more than sorting
// everywhere.  Same order as the sort on its own: by expert, then by pair.
constexpr int kWarps = kThreads / 32;
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) sort_quantize_kernel(const QuantizeArgs a, const int nb, const int32_t* ids,
                                                                 const int pairs, const int experts, int32_t* offsets, int32_t* rows) {
  extern __shared__ int count[];  // [kWarps][experts], then [experts]: first place of every expert
  __shared__ int place_s[kMaxTopk], warp_sum_s[kWarps];
  constexpr Part<WIDE> part;
  int* base = count + kWarps * experts;
  const int t = blockIdx.x, topk = a.copies, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sub = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  for (int i = threadIdx.x; i < kWarps * experts; i += kThreads) count[i] = 0;
  pdl_wait();
  pdl_launch_dependents();
  float v[16];  // the first block travels while the pairs are sorted
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = 0.0f;
  if (group < nb) load_part<T>(a, part, t, group, sub, v);
  __syncthreads();
  // each warp counts a run of the pairs; a pair's place in it is the count of its expert so far
  const int steps = (pairs + kThreads - 1) / kThreads;
  for (int s = 0; s < steps; ++s) {
    const int p = (warp * steps + s) * 32 + lane;
    int id = p < pairs ? ids[p] : -1;
    if (id >= experts) id = -1;
    const unsigned same = __match_any_sync(0xffffffffu, id);
    const int before = id >= 0 ? count[warp * experts + id] : 0;
    const int rank = __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (id >= 0 && rank == 0) count[warp * experts + id] = before + __popc(same);
    __syncwarp();
    if (p < pairs && p / topk == t) place_s[p - t * topk] = before + rank;
  }
  __syncthreads();
  // places of the warps within an expert, and of the experts: each thread a run of neighbouring experts
  const int per = (experts + kThreads - 1) / kThreads, e0 = threadIdx.x * per, e1 = min(experts, e0 + per);
  int mine = 0;
  for (int e = e0; e < e1; ++e) {
    int run = 0;
    for (int w = 0; w < kWarps; ++w) {
      const int n = count[w * experts + e];
      count[w * experts + e] = run;
      run += n;
    }
    base[e] = run;
    mine += run;
  }
  int scan = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int n = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += n;
  }
  if (lane == 31) warp_sum_s[warp] = scan;
  __syncthreads();
  int at = scan - mine;
  for (int w = 0; w < warp; ++w) at += warp_sum_s[w];
  for (int e = e0; e < e1; ++e) {
    const int n = base[e];
    base[e] = at;
    at += n;
    if (t == 0) {
      if (e == 0) offsets[0] = 0;
      offsets[e + 1] = at;
    }
  }
  __syncthreads();
  if (threadIdx.x < topk) {
    const int p = t * topk + threadIdx.x, id = ids[p];
    int to = -1;
    if (id >= 0 && id < experts) to = base[id] + count[p / 32 / steps * experts + id] + place_s[threadIdx.x];
    place_s[threadIdx.x] = to;
    rows[p] = to;
  }
  __syncthreads();
  for (int blk = group; blk < (nb + kThreads / kLanes - 1) / (kThreads / kLanes) * (kThreads / kLanes); blk += kThreads / kLanes) {
    if (blk != group) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = 0.0f;
      if (blk < nb) load_part<T>(a, part, t, blk, sub, v);
    }
    const BlockScale s = block_scale<B2C_E4M3>(block_max(amax16(v)));
    if (blk >= nb) continue;
    const uint4 w = quantize16<B2C_E4M3>(s, v);
    for (int j = 0; j < topk; ++j) {
      const int to = place_s[j];
      if (to < 0) continue;
      store_part(a, part, to, blk, sub, w);
      if (sub == 0) a.scale[(long long)to * a.lds + blk] = s.scale;
    }
  }
}

// Whether rows of x and of q lie on 16-byte boundaries.
template <typename T>
bool is_wide(const QuantizeArgs& a) {
  return (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && (a.ldx * sizeof(T)) % 16 == 0 && (reinterpret_cast<uintptr_t>(a.q) & 15) == 0 &&
         a.ldq % 16 == 0;
}

template <typename T, int QT>
cudaError_t launch(const QuantizeArgs& a, cudaStream_t st) {
  const int nb = (int)blocks_of(a.cols);
  const bool wide = is_wide<T>(a);
  if (a.block_rows == 1) {
    const long long blocks = a.rows * nb;
    const long long grid = (blocks + kThreads / kLanes - 1) / (kThreads / kLanes);
    if (wide && a.cols % 16 == 0 && grid >= 8 * kNumSMs && blocks < (1ll << 30))  // (each SM's 2048 threads have work twice)
      return launch_pdl(quantize_many_rows_kernel<T, QT>, dim3(4 * kNumSMs), dim3(kThreads), 0, st, a, make_fastdiv((uint32_t)nb), (unsigned)blocks);
    if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
    return launch_pdl(wide ? quantize_rows_kernel<T, QT, true> : quantize_rows_kernel<T, QT, false>, dim3((unsigned)grid), dim3(kThreads), 0, st, a, nb, blocks);
  }
  const long long grid = blocks_of(a.rows) * nb;
  if (grid > 0x7FFFFFFFLL) return cudaErrorInvalidValue;
  return launch_pdl(wide ? quantize_blocks_kernel<T, QT, true> : quantize_blocks_kernel<T, QT, false>, dim3((unsigned)grid), dim3(kThreads), 0, st, a, nb);
}

template <typename T>
cudaError_t launch_sort(const QuantizeArgs& a, const int32_t* ids, int pairs, int experts, int32_t* offsets, int32_t* rows, cudaStream_t st) {
  return launch_pdl(is_wide<T>(a) ? sort_quantize_kernel<T, true> : sort_quantize_kernel<T, false>, dim3((unsigned)a.rows), dim3(kThreads),
                    (size_t)(kWarps + 1) * experts * sizeof(int), st, a, (int)blocks_of(a.cols), ids, pairs, experts, offsets, rows);
}

}  // namespace

cudaError_t launch_sort_quantize(const QuantizeArgs& a, const int32_t* ids, int pairs, int experts, int32_t* offsets, int32_t* rows,
                                 cudaStream_t st) {
  if (a.x_type == B2C_F32) return launch_sort<float>(a, ids, pairs, experts, offsets, rows, st);
  if (a.x_type == B2C_F16) return launch_sort<__half>(a, ids, pairs, experts, offsets, rows, st);
  return launch_sort<__nv_bfloat16>(a, ids, pairs, experts, offsets, rows, st);
}

cudaError_t launch_fp8_quantize(const QuantizeArgs& a, cudaStream_t st) {
#define B2C_BY_TYPE(T) return a.q_type == B2C_E4M3 ? launch<T, B2C_E4M3>(a, st) : launch<T, B2C_E5M2>(a, st)
  if (a.x_type == B2C_F32) B2C_BY_TYPE(float);
  if (a.x_type == B2C_F16) B2C_BY_TYPE(__half);
  B2C_BY_TYPE(__nv_bfloat16);
#undef B2C_BY_TYPE
}

}  // namespace b2c

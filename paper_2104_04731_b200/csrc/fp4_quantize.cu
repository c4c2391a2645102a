// Quantisation to 4-bit floating point with microscales, and back.  Memory-bound: every element is read once and kept in registers
// between the search for its block's largest magnitude and the conversion.
//
// 16384 x 8192 bf16 to NV and back 129 us, 688 MB, 5.3 TB/s (106 at the rate of a copy): the way back moves its bytes at nearly that rate (8192 x
// 8192 32 us, 172 MB), the way there is bound by instructions, some 14 for every element, half of them for the exact side of the borders.
// Rows off the 16-byte grid: 8203 x 5137 fp32 and back 81 us (59), 16384 x 8191 bf16 and back 198 (106).
#include "fp4_common.cuh"

namespace b2c {

namespace {

constexpr int kThreads = 256;
constexpr int kRun = 16;  // elements of a lane: a block of NV, half a block of MX

// Largest magnitude, as bits of fp32, of 16 elements as they lie in memory (of 16-bit types as whole numbers, two at a time).
__device__ __forceinline__ uint32_t raw_amax(const Raw16<float>& r) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    m = max(m, max(max(r.u[i].x & 0x7FFFFFFFu, r.u[i].y & 0x7FFFFFFFu), max(r.u[i].z & 0x7FFFFFFFu, r.u[i].w & 0x7FFFFFFFu)));
  return m;
}
template <typename T>
__device__ __forceinline__ uint32_t raw_amax(const Raw16<T>& r) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    m = __vmaxu2(m, r.u[i].x & 0x7FFF7FFFu);
    m = __vmaxu2(m, r.u[i].y & 0x7FFF7FFFu);
    m = __vmaxu2(m, r.u[i].z & 0x7FFF7FFFu);
    m = __vmaxu2(m, r.u[i].w & 0x7FFF7FFFu);
  }
  float lo, hi;
  unpack2<T>(max(m >> 16, m & 0xFFFFu), &lo, &hi);
  return __float_as_uint(lo) & 0x7FFFFFFFu;
}

// Elements of a lane to the row, or the rows, of its block.
__device__ __forceinline__ void store_run(const Quantize4Args& a, long long row, int run, const Scale4& s, const uint32_t* q) {
  const bool first = a.format == B2C_NVFP4 || (run & 1) == 0;
  const int at = a.format == B2C_NVFP4 ? run : run >> 1;
  for (int j = 0; j < (a.map == nullptr ? 1 : a.copies); ++j) {
    const long long to = a.map == nullptr ? row : (long long)a.map[row * a.copies + j];
    if (to < 0) continue;
    *reinterpret_cast<uint2*>(a.q + to * a.ldq + run * (kRun / 2)) = make_uint2(q[0], q[1]);
    if (first) a.scale[to * a.lds + at] = (uint8_t)s.code;
  }
}

// 32 bytes at once, from a 32-byte boundary.
__device__ __forceinline__ void load_8_words(const void* p, uint32_t* w) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store_8_words(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// Rows on the grid of 32-byte loads and 8-byte stores, whole blocks of 32: a lane has 16 elements, and those of the next turn are under
// way while these are converted.  FLAT: all rows follow each other without a gap, as one.  What bounds it are instructions as much as bytes.
template <typename T, bool FLAT>
__global__ void __launch_bounds__(kThreads) quantize4_kernel(const Quantize4Args a, const FastDiv per_row, const unsigned runs) {
  pdl_wait();
  pdl_launch_dependents();
  const Factor4 f = load_factor4(a.global, a.format);
  const unsigned step = gridDim.x * kThreads;
  unsigned id = blockIdx.x * kThreads + threadIdx.x;
  struct Place {
    unsigned row, run;
  };
  auto place = [&](unsigned i) {
    if (FLAT) return Place{0u, i};
    const unsigned row = per_row.div(i);
    return Place{row, i - row * per_row.d};
  };
  Raw16<T> next = {};
  Place at = {0, 0}, at_next = {0, 0};
  auto fetch = [&](unsigned i) {
    if (i >= runs) return;
    at_next = place(i);
    const T* p = (const T*)a.x + (FLAT ? 0ll : (long long)at_next.row * a.ldx) + (long long)at_next.run * kRun;
    uint32_t* w = reinterpret_cast<uint32_t*>(&next);
    load_8_words(p, w);
    if constexpr (sizeof(T) == 4) load_8_words(p + 8, w + 8);
  };
  fetch(id);
  for (unsigned first = blockIdx.x * kThreads; first < runs; first += step, id += step) {  // (the same for all lanes of a warp)
    const Raw16<T> raw = next;
    at = at_next;
    fetch(id + step);
    uint32_t m = raw_amax(raw);
    if (a.format == B2C_MXFP4) m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));  // (runs are a multiple of two: a block's lanes both have some)
    if (id >= runs) continue;
    const Scale4 s = scale_of(m, f, a.format);
    float v[kRun];
    widen16<T>(raw, v);
    uint32_t q[2];
    quantise4<kRun>(s, f, a.format, v, q);
    if (FLAT) {
      *reinterpret_cast<uint2*>(a.q + (long long)id * (kRun / 2)) = make_uint2(q[0], q[1]);
      if (a.format == B2C_NVFP4) a.scale[id] = (uint8_t)s.code;
      else if ((id & 1) == 0) a.scale[id >> 1] = (uint8_t)s.code;
    } else {
      store_run(a, at.row, (int)at.run, s, q);
    }
  }
}

// Runs one after another, `step` further at a time, without a division for each: row and place in the row.
struct Walk {
  int rows, rest, per_row;  // of a step
  __device__ __forceinline__ Walk(int step, int n) : rows(step / n), rest(step % n), per_row(n) {}
  __device__ __forceinline__ void next(long long* row, int* run) const {
    *row += rows;
    *run += rest;
    if (*run >= per_row) {
      *run -= per_row;
      ++*row;
    }
  }
};

// 16 elements of a 16-bit type from any address: the words that hold them (each has at least one of them, so none is outside the tensor's
// memory), shifted where the first begins inside one; zeros from element n on.
template <typename T>
__device__ __forceinline__ Raw16<T> load_run16(const T* p, int n) {
  Raw16<T> r = {};
  if (n <= 0) return r;
  const uint32_t* w = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)3);
  const int odd = (int)(reinterpret_cast<uintptr_t>(p) >> 1) & 1, words = (min(n, kRun) + odd + 1) >> 1;
  uint32_t u[9];
#pragma unroll
  for (int i = 0; i < 9; ++i) u[i] = i < words ? w[i] : 0u;
  uint32_t* out = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    out[i] = __funnelshift_r(u[i], u[i + 1], 16 * odd);
    const int left = n - 2 * i;
    if (left < 2) out[i] &= left == 1 ? 0xFFFFu : 0u;
  }
  return r;
}

// Any rows.  fp32: a warp has 32 runs, whose elements neighbouring lanes bring together (16 lanes a run) and exchange in shared memory; 16-bit types:
// a lane loads its own run in words.  Packed bytes go through shared memory to neighbouring lanes where rows of q do not lie on the grid.
constexpr int kPitch = kRun + 1;
template <typename T>
__global__ void __launch_bounds__(kThreads) quantize4_any_kernel(const Quantize4Args a, const FastDiv per_row, const long long runs, const bool words) {
  __shared__ float stage[kThreads / 32][32 * kPitch];
  pdl_wait();
  pdl_launch_dependents();
  const Factor4 f = load_factor4(a.global, a.format);
  const int lane = threadIdx.x & 31, n = (int)per_row.d;
  float* mine = stage[threadIdx.x >> 5];
  uint8_t* bytes = reinterpret_cast<uint8_t*>(mine);
  const Walk two(2, n), four(4, n);
  // (rows * runs of a row may pass 32 bits: what is above 2^31 is divided the long way)
  auto place = [&](long long id, long long* row, int* run) {
    *row = id < (1ll << 31) ? (long long)per_row.div((uint32_t)id) : id / n;
    *run = (int)(id - *row * n);
  };
  for (long long first = (long long)blockIdx.x * kThreads + (threadIdx.x & ~31u); first < runs; first += (long long)gridDim.x * kThreads) {
    long long row0, row;
    int run0, run;
    place(first, &row0, &run0);
    const bool whole = (run0 + 32) * kRun <= a.cols;  // all of one row, and whole
    float v[kRun];
    uint32_t m = 0;
    if constexpr (sizeof(T) == 2) {
      Raw16<T> raw;
      if (whole) {  // the words that hold the 512 elements, a lane's eight or nine of them in turn
        const T* p = (const T*)a.x + row0 * a.ldx + run0 * kRun;
        const uint32_t* w = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)3);
        const int odd = (int)(reinterpret_cast<uintptr_t>(p) >> 1) & 1;
        uint32_t* words4 = reinterpret_cast<uint32_t*>(mine);
        uint32_t u[9];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = w[32 * i + lane];
        u[8] = odd && lane == 0 ? w[256] : 0u;
        __syncwarp();
        // (a word more for every eight, so that lanes eight words apart meet in different banks)
#pragma unroll
        for (int i = 0; i < 8; ++i) words4[(32 * i + lane) + (32 * i + lane) / 8] = u[i];
        if (lane == 0) words4[256 + 32] = u[8];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 9; ++i) u[i] = words4[9 * lane + i + i / 8];
        uint32_t* out = reinterpret_cast<uint32_t*>(&raw);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = __funnelshift_r(u[i], u[i + 1], 16 * odd);
        __syncwarp();
      } else {
        place(first + lane, &row, &run);
        raw = load_run16<T>((const T*)a.x + row * a.ldx + run * kRun, row < a.rows ? a.cols - run * kRun : 0);
      }
      m = raw_amax(raw);
      widen16<T>(raw, v);
    } else {
      if (whole) {
        const float* p = (const float*)a.x + row0 * a.ldx + run0 * kRun + lane;
#pragma unroll
        for (int i = 0; i < kRun; ++i) v[i] = p[32 * i];
      } else {
        place(first + (lane >> 4), &row, &run);
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          const int c = run * kRun + (lane & 15);
          v[i] = row < a.rows && c < a.cols ? ((const float*)a.x)[row * a.ldx + c] : 0.0f;
          two.next(&row, &run);
        }
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kRun; ++i) mine[(2 * i + (lane >> 4)) * kPitch + (lane & 15)] = v[i];
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        v[i] = mine[lane * kPitch + i];
        m = max(m, abs_bits(v[i]));
      }
    }
    if (a.format == B2C_MXFP4) m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    const Scale4 s = scale_of(m, f, a.format);
    uint32_t q[2];
    quantise4<kRun>(s, f, a.format, v, q);
    row = row0;
    run = run0 + lane;
    if (!whole) place(first + lane, &row, &run);
    const bool on = row < a.rows && run * kRun < a.cols, scales = on && (a.format == B2C_NVFP4 || (run & 1) == 0);
    const int at = a.format == B2C_NVFP4 ? run : run >> 1;
    if (a.map == nullptr) {
      if (scales) a.scale[row * a.lds + at] = (uint8_t)s.code;
      if (words && on && run * kRun + kRun <= a.cols) {
        *reinterpret_cast<uint2*>(a.q + row * a.ldq + run * (kRun / 2)) = make_uint2(q[0], q[1]);
      } else if (words && on) {
        for (int i = 0; i < (a.cols - run * kRun + 1) / 2; ++i) a.q[row * a.ldq + run * (kRun / 2) + i] = (uint8_t)(q[i >> 2] >> (8 * (i & 3)));
      } else if (!words) {
        __syncwarp();
        *reinterpret_cast<uint2*>(bytes + 8 * lane) = make_uint2(q[0], q[1]);
        __syncwarp();
        if (whole) {  // 256 bytes: words on their grid, shifted together, and up to three bytes before and behind them
          uint8_t* d = a.q + row0 * a.ldq + run0 * (kRun / 2);
          const int head = (int)(-reinterpret_cast<uintptr_t>(d) & 3), inner = head == 0 ? 64 : 63;
          const uint32_t* from = reinterpret_cast<const uint32_t*>(mine);
          uint32_t* to = reinterpret_cast<uint32_t*>(d + head);
#pragma unroll
          for (int i = 0; i < 64; i += 32)
            if (i + lane < inner) to[i + lane] = __funnelshift_r(from[i + lane], from[i + lane + 1], 8 * head);
          const int at = lane < head ? lane : 252 + lane;  // (the four lanes of either end)
          if (head != 0 && lane < 4) d[at] = bytes[at];
          __syncwarp();
          continue;
        }
        place(first + (lane >> 3), &row, &run);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = run * (kRun / 2) + (lane & 7);  // byte of the row
          if (row < a.rows && 2 * c < a.cols) a.q[row * a.ldq + c] = bytes[32 * i + lane];
          four.next(&row, &run);
        }
      }
    } else {  // rows of an expert layer are whole blocks and on the grid
      for (int j = 0; j < a.copies; ++j) {
        const long long to = on ? (long long)a.map[row * a.copies + j] : -1;
        if (to < 0) continue;
        *reinterpret_cast<uint2*>(a.q + to * a.ldq + run * (kRun / 2)) = make_uint2(q[0], q[1]);
        if (scales) a.scale[to * a.lds + at] = (uint8_t)s.code;
      }
    }
    __syncwarp();
  }
}

// 16 values a lane, stored 32 bytes at once; FLAT as above.
template <typename T, bool FLAT>
__global__ void __launch_bounds__(kThreads) dequantize4_kernel(const Dequantize4Args a, const FastDiv per_row, const unsigned runs) {
  pdl_wait();
  pdl_launch_dependents();
  const float g = a.global != nullptr ? *a.global : 1.0f;
  const int shift = a.format == B2C_MXFP4 ? 1 : 0;  // runs of 16 in a block
  constexpr int kAhead = 4;
  const unsigned step = gridDim.x * kThreads;
  for (unsigned id0 = blockIdx.x * kThreads + threadIdx.x; id0 < runs; id0 += kAhead * step) {
    uint2 q[kAhead];
    uint32_t code[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const unsigned id = id0 + i * step;
      q[i] = make_uint2(0, 0);
      code[i] = 0;
      if (id < runs && id >= id0) {
        const unsigned row = FLAT ? 0u : per_row.div(id), run = id - row * per_row.d;
        q[i] = *reinterpret_cast<const uint2*>(a.q + (FLAT ? 0ll : (long long)row * a.ldq) + 8ll * run);
        code[i] = a.scale[(FLAT ? 0ll : (long long)row * a.lds) + (run >> shift)];
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const unsigned id = id0 + i * step;
      if (id >= runs || id < id0) continue;
      const unsigned row = FLAT ? 0u : per_row.div(id), run = id - row * per_row.d;
      const float s = scale_value(code[i], a.format);
      T* dst = (T*)a.y + (FLAT ? 0ll : (long long)row * a.ldy) + 16ll * run;
      const uint32_t both[2] = {q[i].x, q[i].y};
      uint32_t out[4 * sizeof(T)];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        uint32_t h[4];
        cvt_f16x8(both[p], h);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float lo, hi;
          unpack2<__half>(h[j], &lo, &hi);
          unpair(mul2(mul2(pair_of(lo, hi), pair_of(s, s)), pair_of(g, g)), &lo, &hi);
          if constexpr (sizeof(T) == 4) {
            out[8 * p + 2 * j] = __float_as_uint(lo);
            out[8 * p + 2 * j + 1] = __float_as_uint(hi);
          } else {
            out[4 * p + j] = pack2<T>(lo, hi);
          }
        }
      }
      store_8_words(dst, out);
      if constexpr (sizeof(T) == 4) store_8_words(dst + 8, out + 8);
    }
  }
}

// Any rows: 32 bytes of y a lane that begin on the 32-byte grid, where that is (the first and the last of a row are not whole), so that a
// store is whole sectors; their 4-bit values begin at any nibble of q.
template <typename T>
__global__ void __launch_bounds__(kThreads) dequantize4_any_kernel(const Dequantize4Args a, const FastDiv per_row, const long long runs) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int E = 32 / (int)sizeof(T);  // columns: 8 or 16, of two blocks at most
  const float g = a.global != nullptr ? *a.global : 1.0f;
  const int shift = a.format == B2C_MXFP4 ? 5 : 4, n = (int)per_row.d;
  const long long step = (long long)gridDim.x * kThreads;
  for (long long id = (long long)blockIdx.x * kThreads + threadIdx.x; id < runs; id += step) {
    const long long row = id < (1ll << 31) ? (long long)per_row.div((uint32_t)id) : id / n;
    T* y = (T*)a.y + row * a.ldy;
    const int behind = (int)((reinterpret_cast<uintptr_t>(y) & 31) / sizeof(T));  // columns that the row begins behind the grid
    const int c0 = (int)(id - row * n) * E - behind;
    const int lo = max(c0, 0), hi = min(c0 + E, a.cols);
    if (lo >= hi) continue;
    const uint8_t* q = a.q + row * a.ldq;
    const uint8_t* scale = a.scale + row * a.lds;
    // the words that hold columns lo .. hi - 1 (each has at least one of them, so none is outside the tensor's memory)
    const uint8_t* from = q + (lo >> 1);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(from) & ~(uintptr_t)3);
    const int words = (int)((reinterpret_cast<uintptr_t>(q + ((hi - 1) >> 1)) - reinterpret_cast<uintptr_t>(w)) >> 2) + 1;
    uint32_t u[E / 8 + 1];
#pragma unroll
    for (int i = 0; i <= E / 8; ++i) u[i] = i < words ? w[i] : 0u;
    const uint32_t code0 = scale[lo >> shift], code1 = scale[(hi - 1) >> shift];
    const int bits = (int)(reinterpret_cast<uintptr_t>(from) & 3) * 8 + 4 * (lo & 1);
    const float s0 = scale_value(code0, a.format), s1 = scale_value(code1, a.format);
    const int first = (((lo >> shift) + 1) << shift) - lo;  // columns of the block that the run begins in
    float v[E];
#pragma unroll
    for (int p = 0; p < E / 8; ++p) {
      uint32_t h[4];
      cvt_f16x8(__funnelshift_r(u[p], u[p + 1], bits), h);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = 8 * p + 2 * j;
        float x0, x1;
        unpack2<__half>(h[j], &x0, &x1);
        unpair(mul2(mul2(pair_of(x0, x1), pair_of(i < first ? s0 : s1, i + 1 < first ? s0 : s1)), pair_of(g, g)), &v[i], &v[i + 1]);
      }
    }
    if (hi - lo == E) {
      uint32_t out[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) out[i] = __float_as_uint(v[i]);
        else out[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
      }
      store_8_words(y + lo, out);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (lo + i < hi) y[lo + i] = from_float<T>(v[i]);
    }
  }
}

bool on_grid(const void* p, long long ld_bytes, long long rows, int grid) {
  return reinterpret_cast<uintptr_t>(p) % grid == 0 && (rows <= 1 || ld_bytes % grid == 0);
}

template <typename T>
cudaError_t launch_quantize(const Quantize4Args& a, cudaStream_t st) {
  // (an MX row has an even number of runs, so that the two halves of a block are neighbours in a warp)
  const long long per_row = a.format == B2C_MXFP4 ? (a.cols + 31ll) / 32 * 2 : (a.cols + 15ll) / 16, runs = a.rows * per_row;
  const bool words = on_grid(a.q, a.ldq, a.map != nullptr ? 2 : a.rows, 8);
  const bool wide = on_grid(a.x, a.ldx * (long long)sizeof(T), a.rows, 32) && words && a.cols % 32 == 0 && runs < (1ll << 30);
  const long long blocks = (runs + kThreads - 1) / kThreads;
  const FastDiv div = make_fastdiv((uint32_t)per_row);
  if (wide) {
    const bool flat = a.map == nullptr && (a.rows <= 1 || (a.ldx == a.cols && 2 * a.ldq == a.cols && a.lds == fp4_scales(a.cols, a.format)));
    // resident at once: 4 or 5 blocks of 256 threads an SM; each loads one run ahead
    const dim3 grid((unsigned)std::min<long long>(blocks, 8 * kNumSMs));
    return flat ? launch_pdl(quantize4_kernel<T, true>, grid, dim3(kThreads), 0, st, a, div, (unsigned)runs)
                : launch_pdl(quantize4_kernel<T, false>, grid, dim3(kThreads), 0, st, a, div, (unsigned)runs);
  }
  // (as many blocks as are resident: what a thread does before its first run is as much as a run)
  return launch_pdl(quantize4_any_kernel<T>, dim3((unsigned)std::min<long long>(blocks, 8 * kNumSMs)), dim3(kThreads), 0, st, a, div, runs, words);
}

template <typename T>
cudaError_t launch_dequantize(const Dequantize4Args& a, cudaStream_t st) {
  const bool wide = on_grid(a.y, a.ldy * (long long)sizeof(T), a.rows, 32) && on_grid(a.q, a.ldq, a.rows, 8);
  if (wide && a.cols % 16 == 0 && a.rows * (a.cols / 16) < (1ll << 30)) {
    const long long runs = a.rows * (a.cols / 16), blocks = (runs + kThreads - 1) / kThreads;
    const bool flat = a.rows <= 1 || (a.ldy == a.cols && 2 * a.ldq == a.cols && a.lds * fp4_block(a.format) == a.cols);
    const FastDiv div = make_fastdiv((uint32_t)(a.cols / 16));
    const dim3 grid((unsigned)std::min<long long>(blocks, 8 * kNumSMs));
    return flat ? launch_pdl(dequantize4_kernel<T, true>, grid, dim3(kThreads), 0, st, a, div, (unsigned)runs)
                : launch_pdl(dequantize4_kernel<T, false>, grid, dim3(kThreads), 0, st, a, div, (unsigned)runs);
  }
  constexpr long long E = 32 / sizeof(T);
  const long long per_row = (a.cols + E - 1 + E - 1) / E, runs = a.rows * per_row, blocks = (runs + kThreads - 1) / kThreads;  // (a row may begin inside a run)
  // (more blocks than are resident: 16384 x 8191 bf16 there and back 198 us; by 16 an SM 200, by 256 204)
  return launch_pdl(dequantize4_any_kernel<T>, dim3((unsigned)std::min<long long>(blocks, 64 * kNumSMs)), dim3(kThreads), 0, st, a,
                    make_fastdiv((uint32_t)per_row), runs);
}

}  // namespace

cudaError_t launch_fp4_quantize(const Quantize4Args& a, cudaStream_t st) {
  if (a.x_type == B2C_F32) return launch_quantize<float>(a, st);
  if (a.x_type == B2C_F16) return launch_quantize<__half>(a, st);
  return launch_quantize<__nv_bfloat16>(a, st);
}

cudaError_t launch_fp4_dequantize(const Dequantize4Args& a, cudaStream_t st) {
  if (a.y_type == B2C_F32) return launch_dequantize<float>(a, st);
  if (a.y_type == B2C_F16) return launch_dequantize<__half>(a, st);
  return launch_dequantize<__nv_bfloat16>(a, st);
}

}  // namespace b2c

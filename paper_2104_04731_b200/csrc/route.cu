// Routing of tokens to experts: scores, groups and the best experts of each token; the stable sort of the
// (token, slot) pairs by expert; the weighted sum of the experts' results.
#include <type_traits>

#include "fp8_common.cuh"

namespace b2c {

namespace {

constexpr unsigned kAll = 0xffffffffu;

// Floats as unsigned integers of the same order (NaN below everything else, but above 0, which marks what is out).
__device__ __forceinline__ unsigned order_key(float v) {
  if (v != v) return 1u;
  const unsigned b = __float_as_uint(v);
  return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned long long order_key(double v) {
  if (v != v) return 1ull;
  const unsigned long long b = (unsigned long long)__double_as_longlong(v);
  return (b >> 63) ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float((k >> 31) ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ unsigned warp_max(unsigned k) { return __reduce_max_sync(kAll, k); }
__device__ __forceinline__ unsigned long long warp_max(unsigned long long k) {
  const unsigned hi = __reduce_max_sync(kAll, (unsigned)(k >> 32));
  const unsigned lo = __reduce_max_sync(kAll, (unsigned)(k >> 32) == hi ? (unsigned)k : 0u);
  return ((unsigned long long)hi << 32) | lo;
}
template <typename V>
__device__ __forceinline__ V warp_sum(V v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  return v;
}

// The chosen experts of one token in 64 bits.  A lane holds P neighbouring experts (keys 0 where there is none), so the lowest index
// of several equal choices is that of the lowest lane.  Lane j returns the j-th chosen expert.  `part` is what a run's score is made
// of, `part_of(e)` the same for any expert: runs that do not end with a lane's experts are scored by one lane each.
template <int P, typename F>
__device__ __forceinline__ int choose_exact(const b2c_route_desc& d, const double (&choice)[P], const double (&part)[P], F part_of, int lane) {
  typedef unsigned long long K;
  K key[P];
#pragma unroll
  for (int i = 0; i < P; ++i) key[i] = lane * P + i < d.experts ? order_key(choice[i]) : (K)0;
  if (d.groups > 1) {
    const int size = d.experts / d.groups;
    const bool whole = size % P == 0;             // a run is a number of lanes
    const int lanes = whole ? size / P : 1;
    const int run = lane / lanes, base = run * lanes;
    double first = -INFINITY, second = -INFINITY;
    auto add = [&](double a, double b) {  // a >= b
      second = fmax(fmin(first, a), fmax(second, b));
      first = fmax(first, a);
    };
    if (whole) {
#pragma unroll
      for (int i = 0; i < P; ++i) add(part[i], -INFINITY);
      const double f0 = first, s0 = second;
      for (int j = 1; j < lanes; ++j) {
        const int from = base + (lane - base + j) % lanes;
        const double a = __shfl_sync(kAll, f0, from), b = __shfl_sync(kAll, s0, from);
        add(a, b);
      }
    } else if (lane < d.groups) {
      for (int i = 0; i < size; ++i) add(part_of(lane * size + i), -INFINITY);
    }
    const bool two = d.group_score == B2C_GROUP_TOP2 && size > 1;
    const double score = two ? (second == -INFINITY ? second : first + second) : first;  // (+inf and -inf: -inf)
    const K mine = run < d.groups ? order_key(score) : (K)0;
    int better = 0;
    for (int g = 0; g < d.groups; ++g) {
      const K k = __shfl_sync(kAll, mine, g * lanes);
      better += k > mine || (k == mine && g < run);
    }
    const bool kept = run < d.groups && better < d.topk_groups;
    const unsigned open = __ballot_sync(kAll, kept);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int of = whole ? lane : min(lane * P + i, d.experts - 1) / size;
      if (!((open >> of) & 1u)) key[i] = 0;
    }
  }
  int my_id = 0;
  for (int j = 0; j < d.topk; ++j) {
    K best = key[0];
#pragma unroll
    for (int i = 1; i < P; ++i) best = key[i] > best ? key[i] : best;
    const K top = warp_max(best);
    unsigned at = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) at |= key[i] == top ? 1u << i : 0u;
    const int owner = __ffs(__ballot_sync(kAll, at != 0)) - 1;
    const int slot = __ffs(at) - 1;
    const int id = owner * P + __shfl_sync(kAll, slot, owner);
    if (lane == owner) {
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (i == slot) key[i] = 0;
    }
    if (lane == j) my_id = id;
  }
  return my_id;
}

// Keys that carry their place among a lane's experts, so that they can be sorted: either exactly, value in the upper word and
// place (the lower the larger) in the lower one, or in 32 bits with the place in the lowest bits of the value, which moves it by
// less than P units of its last place.
template <int P>
__device__ __forceinline__ unsigned long long pack_exact(float v, int i) {
  return ((unsigned long long)order_key(v) << 32) | (unsigned)(P - i);
}
__device__ __forceinline__ unsigned value_bits(unsigned long long k) { return (unsigned)(k >> 32); }
__device__ __forceinline__ unsigned value_bits(unsigned k) { return k; }
template <int P>
__device__ __forceinline__ int place_of(unsigned long long k) { return P - (int)(unsigned)k; }
template <int P>
__device__ __forceinline__ int place_of(unsigned k) { return P - 1 - (int)(k & (P - 1)); }

// Largest first: Batcher's odd-even merge sort, unrolled.
template <int P, typename K>
__device__ __forceinline__ void sort_lane(K (&k)[P]) {
#pragma unroll
  for (int p = 1; p < P; p *= 2)
#pragma unroll
    for (int q = p; q >= 1; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < P; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < P && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
            const K a = k[i + j], b = k[i + j + q];
            k[i + j] = a > b ? a : b;
            k[i + j + q] = a > b ? b : a;
          }
}

// A choice that a key can carry its place in: infinities become the largest values, NaN the lowest one.  (Choices that only
// this makes equal are too near to each other, and compared again as they are.)
__device__ __forceinline__ float finite(float v) { return fminf(fmaxf(v, -3.402823466e38f), 3.402823466e38f); }

// What in an order of 32-bit choices may be wrong, because two of them are nearer than their errors.
struct Near {
  bool runs;    // a kept and a dropped run
  bool inside;  // two neighbours among the chosen
  bool last;    // the two last ones among the chosen
  bool border;  // the last chosen and the first left out
};

// choose_exact() for 32-bit choices: every lane sorts its own once, a round compares the lanes' first ones.  Lane j < rounds gets the
// j-th expert.  With CHECK the choices may be off by half of `unit` * (1 + |choice|), and *near tells what that leaves open.  With PARTS
// the runs are scored by other values than the experts: scores without a bias, off by less than half of `unit` of themselves from 2^-100
// on, and never by more than 2^-20; below that 32 bits hold their addends with fewer bits or not at all, and the runs are left open.
// 32-bit keys without CHECK are for values whose lowest bits are zero (16-bit logits): the place fits into them.
template <int P, typename K, bool CHECK, bool PARTS, typename F>
__device__ __forceinline__ int choose32(const b2c_route_desc& d, int rounds, const float (&choice)[P], const float (&part)[P], F part_of, int lane,
                                        float unit, Near* near) {
  constexpr bool kExact = sizeof(K) == 8;
  K key[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if constexpr (kExact) key[i] = lane * P + i < d.experts ? pack_exact<P>(choice[i], i) : 0ull;
    else key[i] = lane * P + i < d.experts ? ((order_key(choice[i]) & ~(unsigned)(P - 1)) | (unsigned)(P - 1 - i)) : 0u;
  }
  sort_lane<P, K>(key);
  *near = {false, false, false, false};
  bool by_expert = false;  // runs that do not end with a lane's experts: keys are dropped one by one
  unsigned open = kAll;
  const int size = d.experts / d.groups;
  if (d.groups > 1) {
    by_expert = size % P != 0;
    const int lanes = by_expert ? 1 : size / P;
    const int run = lane / lanes;
    float first = -INFINITY, second = -INFINITY;
    auto add = [&](float a, float b) {  // a >= b
      second = fmaxf(fminf(first, a), fmaxf(second, b));
      first = fmaxf(first, a);
    };
    if (!by_expert) {
      float f0, s0;
      if constexpr (PARTS) {
#pragma unroll
        for (int i = 0; i < P; ++i) add(part[i], -INFINITY);
        f0 = first;
        s0 = second;
      } else {
        constexpr unsigned kValue = kExact || CHECK ? 0xFFFFFFFFu : ~(unsigned)(P - 1);  // (equal runs: the first, wherever in a lane their best is)
        f0 = key_value(value_bits(key[0]) & kValue);
        s0 = P > 1 ? key_value(value_bits(key[P > 1 ? 1 : 0]) & kValue) : -INFINITY;
        add(f0, s0);
      }
      int from = lane;
      for (int j = 1; j < lanes; ++j) {
        from = from + 1 == (run + 1) * lanes ? run * lanes : from + 1;
        const float a = __shfl_sync(kAll, f0, from), b = __shfl_sync(kAll, s0, from);
        add(a, b);
      }
    } else if (lane < d.groups) {
      for (int i = 0; i < size; ++i) add(part_of(lane * size + i), -INFINITY);
    }
    const bool two = d.group_score == B2C_GROUP_TOP2 && size > 1;
    // (infinities are about the largest values here, up to the place in their keys: a sum with the lowest one is that, and sums stay
    // between them; a sum of both is left to 64 bits)
    constexpr float kHuge = 3.4028e38f;
    const float score = two ? (second <= -kHuge ? -3.402823466e38f : finite(first + second)) : first;
    const unsigned mine = run < d.groups ? order_key(score) : 0u;
    int better = 0;
    for (int g = 0; g < d.groups; ++g) {
      const unsigned k = __shfl_sync(kAll, mine, g * lanes);
      better += k > mine || (k == mine && g < run);
    }
    const bool kept = run < d.groups && better < d.topk_groups;
    if constexpr (CHECK || PARTS) {
      const float low = key_value(__reduce_min_sync(kAll, kept ? mine : 0xFFFFFFFFu));
      const unsigned high = __reduce_max_sync(kAll, kept ? 0u : mine);
      if constexpr (PARTS) near->runs = high != 0u && !(low >= 0x1p-100f && low - key_value(high) > fminf(unit * low, 0x1p-19f));
      else {
        // (a sum is off by the errors of its addends, which may be far larger than itself; sums that stand for the largest value, or with
        // the lowest one, are what they are)
        const bool adds = two && run < d.groups && fabsf(score) < kHuge;
        const float addend = __uint_as_float(__reduce_max_sync(kAll, adds ? __float_as_uint(fmaxf(fabsf(first), fabsf(second))) : 0u));
        near->runs = high != 0u && !(low - key_value(high) > 2.0f * unit * (1.0f + fmaxf(fabsf(low), addend)));
      }
      if (!PARTS) near->runs |= __any_sync(kAll, two && first >= kHuge && second <= -kHuge);
    }
    open = __ballot_sync(kAll, kept);
    if (!by_expert && !kept) {
#pragma unroll
      for (int i = 0; i < P; ++i) key[i] = 0;
    }
  }
  int my_id = 0;
  float my_value = 0.0f;
  for (int j = 0; j < rounds;) {
    // (exact 32-bit keys: the place is not part of the value, or equal values would not go to the lowest lane)
    const unsigned mine = kExact || CHECK ? value_bits(key[0]) : value_bits(key[0]) & ~(unsigned)(P - 1);
    const unsigned top = __reduce_max_sync(kAll, mine);
    if (top == 0u) break;  // (nothing left: cannot be, topk is at most what the kept runs hold)
    const int owner = __ffs(__ballot_sync(kAll, mine == top)) - 1;
    int id;
    if constexpr (kExact || !CHECK) id = __shfl_sync(kAll, lane * P + place_of<P>(key[0]), owner);
    else id = owner * P + place_of<P>(top);
    if (lane == owner) {
#pragma unroll
      for (int i = 0; i + 1 < P; ++i) key[i] = key[i + 1];
      key[P - 1] = 0;
    }
    if (by_expert && !((open >> (id / size)) & 1u)) continue;  // of a dropped run
    if (lane == j) {
      my_id = id;
      if constexpr (CHECK) my_value = key_value(top);
    }
    ++j;
  }
  if constexpr (CHECK) {
    // each chosen one against the next, the last against the first that was left out
    float next = __shfl_down_sync(kAll, my_value, 1);
    unsigned left = 0u;
    if (!by_expert) {
      left = __reduce_max_sync(kAll, value_bits(key[0]));
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (value_bits(key[i]) != 0u && ((open >> ((lane * P + place_of<P>(key[i])) / size)) & 1u)) left = max(left, value_bits(key[i]));
      left = __reduce_max_sync(kAll, left);
    }
    const bool ends = lane == rounds - 1;
    if (ends) next = left != 0u ? key_value(left) : -INFINITY;
    const bool open_order = lane < rounds && !(ends && left == 0u) && !(my_value - next > unit * (1.0f + fabsf(my_value)));
    const unsigned who = __ballot_sync(kAll, open_order);
    near->border = ((who >> (rounds - 1)) & 1u) != 0u;
    near->last = rounds > 1 && ((who >> (rounds - 2)) & 1u) != 0u;
    near->inside = (who & ((1u << (rounds - 1)) - 1u)) != 0u;
  }
  return my_id;
}

template <typename T>
__device__ __forceinline__ float logit(const T* row, int e) {
  const float x = to_float<T>(row[e]);
  return x != x ? -INFINITY : x + 0.0f;  // (a zero loses its sign, so that all zeros are equal)
}

__device__ __forceinline__ double sigmoid64(double x) { return x == -INFINITY ? 0.0 : 1.0 / (1.0 + exp(-x)); }

// The same choice in 64 bits, for a token whose 32-bit choices are too near to each other (rare: kept out of the way of the others).
template <typename T, int P>
__device__ __noinline__ int choose64(const RouteArgs& a, const T* row, int lane, float mx) {
  double s[P], c[P], sum = 0.0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int e = lane * P + i;
    const double x = e < a.d.experts ? (double)logit<T>(row, e) : -INFINITY;
    s[i] = a.d.score == B2C_SCORE_SIGMOID ? sigmoid64(x) : (x == -INFINITY ? 0.0 : (x == (double)mx ? 1.0 : exp(x - (double)mx)));
    sum += s[i];
  }
  if (a.d.score == B2C_SCORE_SOFTMAX) {
    sum = warp_sum(sum);
#pragma unroll
    for (int i = 0; i < P; ++i) s[i] = sum > 0.0 ? s[i] / sum : 0.0;
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int e = lane * P + i;
    c[i] = e < a.d.experts ? (a.bias != nullptr ? s[i] + (double)a.bias[e] : s[i]) : -INFINITY;
    c[i] = c[i] != c[i] ? -INFINITY : c[i];
  }
  auto part_of = [&](int e) {
    const double l = (double)logit<T>(row, e);
    double v = a.d.score == B2C_SCORE_SIGMOID ? sigmoid64(l) : (l == -INFINITY ? 0.0 : (l == (double)mx ? 1.0 : exp(l - (double)mx)));
    if (a.d.score == B2C_SCORE_SOFTMAX) v = sum > 0.0 ? v / sum : 0.0;
    v = a.bias != nullptr ? v + (double)a.bias[e] : v;
    return v != v ? -INFINITY : v;
  };
  if (a.bias == nullptr) {  // (the experts are taken by their logits, the runs by their scores)
    double x[P];
#pragma unroll
    for (int i = 0; i < P; ++i) x[i] = lane * P + i < a.d.experts ? (double)logit<T>(row, lane * P + i) : -INFINITY;
    return choose_exact<P>(a.d, x, c, part_of, lane);
  }
  return choose_exact<P>(a.d, c, c, part_of, lane);
}

// The experts of lanes 0 .. count - 1 in the order of their choices in 64 bits.
__device__ __forceinline__ int order64(double choice, int id, int count, int lane) {
  const unsigned long long key = order_key(choice != choice ? -INFINITY : choice);
  int rank = 0;
#pragma unroll 1
  for (int j = 0; j < count; ++j) {
    const unsigned long long k = __shfl_sync(kAll, key, j);
    const int i = __shfl_sync(kAll, id, j);
    rank += k > key || (k == key && i < id);
  }
  int sorted = id;
#pragma unroll 1
  for (int j = 0; j < count; ++j) {
    const int r = __shfl_sync(kAll, rank, j), i = __shfl_sync(kAll, id, j);
    if (r == lane) sorted = i;
  }
  return sorted;
}

// One warp for one token, everything in registers.  Scores are monotonic in the logits, so without a bias the logits themselves are
// compared, which is exact.  With a bias (or run scores that are sums) the choices are formed in 32 bits: exponential, quotient and
// additions put each off by at most 6 units of 2^-24 * (1 + |choice|), with the sum of a softmax by 11, its place in the key's lowest
// bits by P - 1 units of 2^-23, together less than 2^-19 for P <= 8 and 2^-17 beyond, and sums of two by that of both, however small they
// are.  A token in which two choices that decide
// something are not further apart than twice this (about one in fifty at 256 experts) needs a second look: where only the order of the
// topk + 1 first is open, these few are compared in 64 bits; else all are chosen again with the places beside the values (2^-20, with a softmax
// 2^-18), and where that does not settle it, or if the scores hang on all logits, the token is done in 64 bits from the start.  (On one run:
// all such tokens chosen again 26.2 us for the work below, this way 25.7, none looked at twice, which is wrong, 22.)
// Memory-bound on paper (one read of the logits); what it spends are the instructions of exponentials, sort and topk rounds (16384 tokens
// of 256 experts, 8 of 4 of 8 runs: 25 to 31 us by the run's clock, issue slots 76 % busy, against 2.8 us for the bytes).  Two tokens a warp, 16 lanes each, took
// 38: the largest of 16 lanes is four exchanges, that of a warp one instruction.
constexpr int kRouteWarps = 8;
template <typename T, int P>
__global__ void __launch_bounds__(32 * kRouteWarps, P <= 8 ? 5 : 1) route_kernel(const RouteArgs a, const bool vec, const bool bias_vec) {
  pdl_wait();
  pdl_launch_dependents();
  const int E = a.d.experts, lane = threadIdx.x & 31;
  const long long t = (long long)blockIdx.x * kRouteWarps + (threadIdx.x >> 5);
  if (t >= a.tokens) return;
  const T* row = (const T*)a.logits + t * a.ld;
  float x[P];
  bool loaded = false;
  if constexpr (P * sizeof(T) % 16 == 0) {
    if (vec) {
      loaded = true;
      constexpr int kPer = 16 / sizeof(T);
#pragma unroll
      for (int i = 0; i < P; i += kPer) {
        uint4 u = make_uint4(0, 0, 0, 0);
        const bool in = lane * P + i < E;  // (E is a multiple of kPer)
        if (in) u = *reinterpret_cast<const uint4*>(row + lane * P + i);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (sizeof(T) == 4) x[i + j] = in ? __uint_as_float(w[j]) : -INFINITY;
          else {
            unpack2<T>(w[j], &x[i + 2 * j], &x[i + 2 * j + 1]);
            if (!in) x[i + 2 * j] = x[i + 2 * j + 1] = -INFINITY;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < P; ++i) x[i] = x[i] != x[i] ? -INFINITY : x[i] + 0.0f;
    }
  }
  if (!loaded) {
#pragma unroll
    for (int i = 0; i < P; ++i) x[i] = lane * P + i < E ? logit<T>(row, lane * P + i) : -INFINITY;
  }
  const bool softmax = a.d.score == B2C_SCORE_SOFTMAX;
  const bool by_logit = a.bias == nullptr;
  const bool sums = a.d.groups > 1 && a.d.group_score == B2C_GROUP_TOP2;
  float mx = 0.0f;
  double all = 0.0;
  if (softmax) {
    mx = x[0];
#pragma unroll
    for (int i = 1; i < P; ++i) mx = fmaxf(mx, x[i]);
    mx = key_value(warp_max(order_key(mx)));
  }
  int id;
  Near near;
  // logits of 16 bits leave the lowest 13 of a float free; lanes of up to 32 experts need five
  using LogitKey = typename std::conditional<sizeof(T) == 2, unsigned, unsigned long long>::type;
  if (by_logit && !sums) {
    if (softmax && !a.d.renormalise) {
      // (in 64 bits from the start: 1024 scores of one size put 32-bit partial sums off by a rounding each, always the same way)
#pragma unroll
      for (int i = 0; i < P; ++i) all += (double)(x[i] == -INFINITY ? 0.0f : (x[i] == mx ? 1.0f : expf(x[i] - mx)));
      all = warp_sum(all);
    }
    id = choose32<P, LogitKey, false, false>(a.d, a.d.topk, x, x, [&](int e) { return logit<T>(row, e); }, lane, 0.0f, &near);
  } else {
    float c[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (softmax) c[i] = x[i] == -INFINITY ? 0.0f : (x[i] == mx ? 1.0f : expf(x[i] - mx));
      else c[i] = __fdividef(1.0f, 1.0f + __expf(-x[i]));
    }
    if (softmax) {
#pragma unroll
      for (int i = 0; i < P; ++i) all += (double)c[i];
      all = warp_sum(all);
#pragma unroll
      for (int i = 0; i < P; ++i) c[i] = all > 0.0 ? __fdividef(c[i], (float)all) : 0.0f;
    }
    const float total = (float)all;
    auto part_of = [&](int e) {
      const float l = logit<T>(row, e);
      float v;
      if (softmax) v = total > 0.0f && l != -INFINITY ? __fdividef(l == mx ? 1.0f : expf(l - mx), total) : 0.0f;
      else v = __fdividef(1.0f, 1.0f + __expf(-l));
      return finite(by_logit ? v : v + a.bias[e]);
    };
    if (!by_logit) {
      if (P >= 4 && bias_vec) {
#pragma unroll
        for (int i = 0; i + 3 < P; i += 4)
          if (lane * P + i < E) {
            const float4 b = *reinterpret_cast<const float4*>(a.bias + lane * P + i);
            c[i] += b.x;
            c[i + 1] += b.y;
            c[i + 2] += b.z;
            c[i + 3] += b.w;
          }
      } else {
#pragma unroll
        for (int i = 0; i < P; ++i)
          if (lane * P + i < E) c[i] += a.bias[lane * P + i];
      }
    }
    if (by_logit) {
      // the runs by sums of scores, the experts by their logits, which is exact
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (lane * P + i >= E) c[i] = -INFINITY;
      // (from 2^-100 on exponents are above -70: __expf, by its documented bound of 2 + 1.173 |x| units of the last place, is off by
      // 84 of 2^-23, or the difference from the largest logit by 70 of 2^-24; quotient and sum add a few.  A score close to one hardly
      // feels that, c (1 - c) |x| or c |log c| of it: 6 and 10 units of 2^-24 a choice, sum included.  By the relative bound alone
      // 16384 x 256 logistic scores take 31.5 us, with both 26.)
      id = choose32<P, LogitKey, false, true>(a.d, a.d.topk, x, c, part_of, lane, 0x1p-15f, &near);
      if (near.runs) id = choose64<T, P>(a, row, lane, mx);
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) c[i] = finite(c[i]);
      // one expert further than asked for, so that a border within the errors lies inside
      const int rounds = min(min(a.d.topk + 1, 32), E / a.d.groups * a.d.topk_groups);
      const bool further = rounds > a.d.topk;
      id = choose32<P, unsigned, true, false>(a.d, rounds, c, c, part_of, lane, P <= 8 ? 0x1p-18f : 0x1p-16f, &near);
      if (near.runs || near.inside || (near.border && !further)) {
        if (near.runs || (near.border && (near.last || !further)))
          id = choose32<P, unsigned long long, true, false>(a.d, rounds, c, c, part_of, lane, softmax ? 0x1p-18f : 0x1p-20f, &near);
        if (near.runs || (near.border && (near.last || !further)) || (softmax && near.inside)) {
          id = choose64<T, P>(a, row, lane, mx);
        } else if (near.inside) {
          const int e = lane < rounds ? id : 0;
          id = order64(sigmoid64((double)logit<T>(row, e)) + (double)a.bias[e], id, rounds, lane);
        }
      }
    }
  }
  // the weights of the chosen, from their logits; the argument of the exponential without the rounding of its difference
  const bool on = lane < a.d.topk;
  const float l = on ? logit<T>(row, id) : -INFINITY;
  // Scores that 32 bits cannot hold: renormalised ones are taken relative to the largest chosen one, which may be far below the
  // largest of the row where a bias or a run decides; logistic ones below -17 are exponentials in 32 bits (1 + e^l rounds to 1).  (From -740 on 64 bits cannot
  // hold them either: 0, as for the lowest values of a type that masks write.)
  const float best = key_value(__reduce_max_sync(kAll, order_key(l)));
  const float top = softmax && !(a.d.renormalise && mx - best < 740.0f) ? mx : best;
  float s;
  if (softmax || (a.d.renormalise && top < -17.0f && top > -740.0f)) {
    const double diff = (double)l - (double)top;
    const float hi = (float)diff;
    const float e = expf(hi);
    s = l == -INFINITY ? 0.0f : (l == top ? 1.0f : (e == 0.0f ? 0.0f : fmaf(e, (float)(diff - (double)hi), e)));
  } else {
    const float e = expf(l < -17.0f ? l : -l);
    s = l < -17.0f ? e : 1.0f / (1.0f + e);
  }
  float w = s;
  if (a.d.renormalise) {
    const float total = warp_sum(s);
    w = total > 0.0f ? s / total : 0.0f;
  } else if (softmax) {
    w = all > 0.0 ? s / (float)all : 0.0f;
  }
  if (on) {
    a.weights[t * a.d.topk + lane] = w * a.d.scale;
    a.ids[t * a.d.topk + lane] = id;
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

// Many chunks: the counts of each expert become the counts of the chunks before, and the row behind them its total.  One warp an expert.
constexpr int kScanFrom = 64;  // chunks; below, every block of place_kernel adds the counts up for itself
__global__ void __launch_bounds__(256) scan_kernel(int32_t* counts, const int chunks, const int experts) {
  pdl_wait();
  pdl_launch_dependents();
  const int e = (int)blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (e >= experts) return;
  int run = 0;
  for (int c0 = 0; c0 < chunks; c0 += 128) {
    int n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) n[i] = c0 + 32 * i + lane < chunks ? counts[(size_t)(c0 + 32 * i + lane) * experts + e] : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int sum = n[i];
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int up = __shfl_up_sync(kAll, sum, d);
        if (lane >= d) sum += up;
      }
      if (c0 + 32 * i + lane < chunks) counts[(size_t)(c0 + 32 * i + lane) * experts + e] = run + sum - n[i];
      run += __shfl_sync(kAll, sum, 31);
    }
  }
  if (lane == 0) counts[(size_t)chunks * experts + e] = run;
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
    if (counts != nullptr && chunks > kScanFrom) {
      before = counts[(size_t)blockIdx.x * experts + e];
      all = counts[(size_t)chunks * experts + e];
    } else if (counts != nullptr) {
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
// loads are under way together.  8192 tokens x 4 rows of 4096 bf16: 62 us, 5.4 TB/s.
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

namespace {

template <typename T>
cudaError_t route_type(const RouteArgs& a, cudaStream_t st) {
  const dim3 grid((unsigned)((a.tokens + kRouteWarps - 1) / kRouteWarps)), block(32 * kRouteWarps);
  const bool bias_vec = (reinterpret_cast<uintptr_t>(a.bias) & 15) == 0 && a.d.experts % 4 == 0;
  constexpr int kPer = 16 / (int)sizeof(T);
  const bool vec = (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0 && a.ld % kPer == 0 && a.d.experts % kPer == 0;
#define B2C_ROUTE(P) \
  if (a.d.experts <= 32 * P) return launch_pdl(route_kernel<T, P>, grid, block, 0, st, a, vec, bias_vec)
  B2C_ROUTE(1);
  B2C_ROUTE(2);
  B2C_ROUTE(4);
  B2C_ROUTE(8);
  B2C_ROUTE(16);
  B2C_ROUTE(32);
#undef B2C_ROUTE
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_route(const RouteArgs& a, cudaStream_t st) {
  if (a.d.logit_type == B2C_F32) return route_type<float>(a, st);
  if (a.d.logit_type == B2C_F16) return route_type<__half>(a, st);
  return route_type<__nv_bfloat16>(a, st);
}

size_t route_sort_workspace(long long pairs, int experts) {
  return pairs <= kChunk ? 0 : (size_t)((pairs + kChunk - 1) / kChunk + 1) * experts * sizeof(int32_t);
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
    if (e == cudaSuccess && chunks > kScanFrom)
      e = launch_pdl(scan_kernel, dim3((unsigned)(experts + 7) / 8), dim3(256), 0, st, workspace, chunks, experts);
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

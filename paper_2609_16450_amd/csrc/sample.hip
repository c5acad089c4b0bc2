// A token per row from its logits and a given random number: temperature, top-k, top-p, min-p.
//
// With w_v = exp((z_v - m) / t) and the vocabulary in the order (z falling, id rising), every filter
// keeps a prefix of that order, so what is kept is one cut: all ids whose logit lies above a value,
// and of those that equal it the lowest ids up to one.  The token is the lowest kept id whose running
// sum, over the kept ids in rising order, exceeds u times the sum of all of them.
//
// The drawn id depends on sums over up to the whole vocabulary next to a border, and has to be the
// same whatever cuts the sums into pieces.  So weights are formed in 64 bits and held as whole
// numbers of 2^-62 of (at least) their sum: the sums are exact in any order, also by atomics, and the
// one rounding of a weight is off by 2^-63 of the sum, less than a sum in 64-bit floats would lose.
//
// Two launches.  sample_scan_kernel reads every logit once and leaves, per segment of 2048 ids, its
// largest and lowest logit and its sums of weights, and the largest of each of its 64 groups of 32 ids.
// sample_pick_kernel, a workgroup per row, cuts and draws from these: with a temperature alone it
// reads the one segment that the draw falls into; with a top-k, or where the nucleus is small, the
// groups that can hold what is kept (their largest logits say which), at most kList ids, sorted
// in LDS; and otherwise the row again, twice per cut: once for a histogram that finds the bin which
// the cut lies in, once for the exact sums above that bin and the ids within it.  Where that bin holds
// more ids than the list (logits that tie, or a few that lie far off the others), the cut's key is
// found bit by bit instead.
#include <float.h>

#include <type_traits>

#include "attn_common.hpp"
#include "eb_common.hpp"
#include "eb_internal.hpp"
#include "paged.hpp"

namespace eb {
namespace {

constexpr int kSegment = 2048;         // ids that a wave takes at a time
constexpr int kGroup = kSegment / 64;  // of them a lane's
constexpr int kScanThreads = 256;
constexpr int kScanWaves = kScanThreads / 64;
constexpr int kThreads = 1024;  // of the workgroup that picks
constexpr int kWaves = kThreads / 64;
constexpr int kMaxSegments = kThreads;
constexpr int kList = kThreads;  // ids that are sorted in LDS
constexpr int kBins = 2048;
static_assert(kMaxSegments * kSegment >= kSampleMaxVocab, "a thread per segment");

typedef uint32_t u32x4h __attribute__((ext_vector_type(4), aligned(2)));  // at any 2 bytes

template <class T>
constexpr int kVec = 16 / sizeof(T);  // ids of a lane and load
template <class T>
constexpr int kLoads = kGroup / kVec<T>;  // loads of a lane per segment

// Id of element e of load i of a lane, in its segment.
template <class T>
__device__ __forceinline__ int id_in_segment(int i, int lane) {
  return (i * 64 + lane) * kVec<T>;
}

// Logits at .. at + kVec - 1 of a row; -inf behind its end.
__device__ __forceinline__ void load_logits(const float* row, int at, int vocab, float (&z)[4]) {
  if (at + 4 <= vocab) {
    const f32x4 x = *reinterpret_cast<const f32x4u*>(row + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = x[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = at + e < vocab ? row[at + e] : -INFINITY;
  }
}
__device__ __forceinline__ void load_logits(const uint16_t* row, int at, int vocab, float (&z)[8]) {
  if (at + 8 <= vocab) {
    const u32x4 x = *reinterpret_cast<const u32x4h*>(row + at);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t w = x[e / 2];
      z[e] = __uint_as_float(e % 2 ? w & 0xffff0000u : w << 16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      z[e] = at + e < vocab ? bf16_bits_to_f32(row[at + e]) : -INFINITY;
  }
}
__device__ __forceinline__ float load_logit(const float* row, int id) { return row[id]; }
__device__ __forceinline__ float load_logit(const uint16_t* row, int id) {
  return bf16_bits_to_f32(row[id]);
}

// A whole number that orders as the float does (-0 as +0), and back.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}

// 2^(i / 16)
__constant__ const double kPow16[16] = {
    0x1.0000000000000p+0, 0x1.0b5586cf9890fp+0, 0x1.172b83c7d517bp+0, 0x1.2387a6e756238p+0,
    0x1.306fe0a31b715p+0, 0x1.3dea64c123422p+0, 0x1.4bfdad5362a27p+0, 0x1.5ab07dd485429p+0,
    0x1.6a09e667f3bcdp+0, 0x1.7a11473eb0187p+0, 0x1.8ace5422aa0dbp+0, 0x1.9c49182a3f090p+0,
    0x1.ae89f995ad3adp+0, 0x1.c199bdd85529cp+0, 0x1.d5818dcfba487p+0, 0x1.ea4afa2a490dap+0};

// exp((z - top) / temperature) in 64 bits.  With y = (z - top) 16 log2(e) / temperature and n the
// whole number nearest to y, it is 2^(n / 16) 2^((y - n) / 16): a table (of 16 values, which the
// lanes of a wave read from LDS without a conflict) and the power series of the exponential to the fifth
// term, |y - n| <= 1/2, which leaves less than 2^-42 of the value.  A weight's error of that size moves
// a border of the draw by as much of the sum at most, and one in 10^10 draws across it.
struct Weights {
  const double* pow16;  // LDS
  double top, rate;     // largest logit; 16 log2(e) / temperature
  __device__ __forceinline__ double operator()(float z) const {
    constexpr double c1 = 0x1.62e42fefa39efp-5, c2 = 0x1.ebfbdff82c58fp-11,
                     c3 = 0x1.c6b08d704a0c0p-17, c4 = 0x1.3b2ab6fba4e77p-23,
                     c5 = 0x1.5d87fe78a6731p-30;  // (ln 2 / 16)^k / k!
    // (z = -inf ends at the lower bound, whose power is 0)
    const double y = fmax((static_cast<double>(z) - top) * rate, -20000.0);
    const double n = rint(y), r = y - n;
    const int k = static_cast<int>(n);
    const double p = fma(r, fma(r, fma(r, fma(r, fma(r, c5, c4), c3), c2), c1), 1.0);
    return ldexp(pow16[k & 15] * p, k >> 4);
  }
};
__device__ __forceinline__ double weight_rate(float temperature) {
  return 0x1.71547652b82fep+4 / static_cast<double>(temperature);  // 16 log2(e) / t
}
// Weights as whole numbers of 1 / scale, a power of two; one that is not 0 counts at least 1.
__device__ __forceinline__ uint64_t whole(double w, double scale) {
  return w > 0.0 ? max(static_cast<uint64_t>(rint(w * scale)), uint64_t{1}) : 0;
}

// Kept: above key, or equal to it with an id of at most last.
struct Cut {
  uint32_t key;
  int32_t last;
  __device__ __forceinline__ bool keeps(uint32_t k, int id) const {
    return k > key || (k == key && id <= last);
  }
  __device__ __forceinline__ bool tighter(const Cut& o) const {
    return key > o.key || (key == o.key && last < o.last);
  }
};
constexpr Cut kKeepAll{0, INT32_MAX};

// What the first launch leaves of a segment.
struct alignas(8) SegmentStats {
  float top, low;   // largest and lowest logit above -inf (-inf and +inf where there is none); top
                    // is NaN where one is NaN or +inf
  float soft, pad;  // sum of exp(z - top) at temperature 1
  double sum;       // sum of the weights relative to its own top
};
static_assert(sizeof(SegmentStats) == 24, "packed");

// A row's settings and whether it is one of few kept ids by count.
struct Settings {
  float temperature, top_p, min_p;
  int32_t top_k;  // 0: no limit
  __device__ __forceinline__ bool greedy() const { return !(temperature > 0.f); }
};
__device__ __forceinline__ Settings settings(const SampleArgs& a, int b) {
  Settings s;
  s.temperature = a.temperature ? a.temperature[b] : 1.f;
  s.top_p = a.top_p ? a.top_p[b] : 1.f;
  s.min_p = a.min_p ? fminf(a.min_p[b], 1.f) : 0.f;
  const int32_t k = a.top_k ? a.top_k[b] : 0;
  s.top_k = k > 0 && k < a.vocab ? k : 0;
  return s;
}
// Top-k small enough to be settled in LDS: half the list, so that the ids which the groups' largest
// logits let through besides fit as well.
constexpr int kFewIds = kList / 2;

struct Workspace {
  SegmentStats* stats;  // [n_rows, segments]
  float* group_top;     // [n_rows, segments, 64]: largest logit of a lane's ids
  int segments;
};

template <class V, class Op>
__device__ __forceinline__ V wave_reduce(V x, Op op) {
  for (int mask = 32; mask >= 1; mask >>= 1) x = op(x, __shfl_xor(x, mask));
  return x;
}
struct Add {
  template <class V>
  __device__ __forceinline__ V operator()(V a, V b) const {
    return a + b;
  }
};
struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
  __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); }
};
struct Min {
  __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); }
  __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return min(a, b); }
};

// ---------------------------------------------------------------------------------------
// First launch: a wave per segment.
// ---------------------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(kScanThreads) void sample_scan_kernel(SampleArgs a, Workspace ws) {
  __shared__ double pow16[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int parts = (ws.segments + kScanWaves - 1) / kScanWaves;
  const int r = blockIdx.x / parts;
  const int g = (blockIdx.x - r * parts) * kScanWaves + wave;
  const T* const row = static_cast<const T*>(a.logits) + static_cast<size_t>(r) * a.pitch;
  float z[kLoads<T>][kVec<T>];
#pragma unroll
  for (int i = 0; i < kLoads<T>; ++i)
    load_logits(row, g * kSegment + id_in_segment<T>(i, lane), a.vocab, z[i]);
  if (threadIdx.x < 16) pow16[threadIdx.x] = kPow16[threadIdx.x];
  const Settings st = settings(a, find_sequence(a.cu_block, a.batch, r, lane));
  __syncthreads();
  if (g >= ws.segments) return;

  float top = -INFINITY, low = INFINITY;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kLoads<T>; ++i)
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) {
      top = fmaxf(top, z[i][e]);
      low = fminf(low, z[i][e] == -INFINITY ? INFINITY : z[i][e]);
      bad |= !(z[i][e] < INFINITY);
    }
  const size_t at = static_cast<size_t>(r) * ws.segments + g;
  ws.group_top[at * 64 + lane] = top;
  top = wave_reduce(top, Max{});
  low = wave_reduce(low, Min{});
  bad = __any(bad);
  SegmentStats out{bad ? NAN : top, low, 0.f, 0.f, 0.0};
  if (top > -INFINITY && !bad) {  // (else every difference would be NaN)
    if (a.conf) {
#pragma unroll
      for (int i = 0; i < kLoads<T>; ++i)
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) out.soft += fast_exp2((z[i][e] - top) * kLog2e);
      out.soft = wave_reduce(out.soft, Add{});
    }
    // rows of few ids by count, and greedy ones, take no sum over all
    if (!st.greedy() && (st.top_k == 0 || st.top_k > kFewIds)) {
      const Weights w{pow16, static_cast<double>(top), weight_rate(st.temperature)};
#pragma unroll
      for (int i = 0; i < kLoads<T>; ++i)
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) out.sum += w(z[i][e]);
      out.sum = wave_reduce(out.sum, Add{});
    }
  }
  if (lane == 0) ws.stats[at] = out;
}

// ---------------------------------------------------------------------------------------
// Second launch: a workgroup per row.
// ---------------------------------------------------------------------------------------
struct Shared {
  uint64_t segment[kMaxSegments];  // a sum per segment, then the sum before it
  float segment_top[kMaxSegments];
  union {
    struct {
      uint64_t list[kList], mass[kList];
    };
    uint64_t bin_mass[kBins];
  };
  uint32_t bins[kBins];
  double pow16[16];
  uint64_t slots64[kWaves];
  double slots_d[kWaves];
  float slots_f[kWaves];
  uint32_t slots32[kWaves];
  uint32_t n_list, found, found_count, found_before;
  uint64_t found_mass, found_mass_before;
  int32_t found_id;
};

// x over all threads, on every thread; `slots` [kWaves] is free again behind the next barrier.
template <class V, class Op>
__device__ __forceinline__ V block_reduce(V x, V* slots, Op op) {
  x = wave_reduce(x, op);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = x;
  __syncthreads();
  V y = slots[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) y = op(y, slots[w]);
  return y;
}

// Sum of x over the threads before this one; `total` over all.
template <class V>
__device__ __forceinline__ V block_scan(V x, V* slots, V& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  V sum = x;
  for (int n = 1; n < 64; n <<= 1) {
    const V o = __shfl_up(sum, n);
    if (lane >= n) sum += o;
  }
  __syncthreads();
  if (lane == 63) slots[wave] = sum;
  __syncthreads();
  V before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) before = total;
    total += slots[w];
  }
  return before + sum - x;
}

// Sorts list[0 .. n) falling, in place: a value per thread, exchanged between lanes for distances
// below 64 and through LDS beyond.
__device__ __forceinline__ void sort_falling(uint64_t* list, int n) {
  const int t = threadIdx.x;
  int size = 64;
  while (size < n) size <<= 1;
  uint64_t x = t < n ? list[t] : 0;
  for (int k = 2; k <= size; k <<= 1) {
    for (int j = k >> 1; j > 0; j >>= 1) {
      uint64_t o;
      if (j >= 64) {
        __syncthreads();
        list[t] = x;
        __syncthreads();
        o = list[t ^ j];
      } else {
        o = __shfl_xor(x, j);
      }
      const bool larger = ((t & k) == 0) == ((t & j) == 0);  // this place takes the larger one
      x = (x > o) == larger ? x : o;
    }
  }
  __syncthreads();
  if (t < size) list[t] = x;
  __syncthreads();
}

// floor(sum * x) for x in [0, 1) (bits of x below 2^-64 are left out).
__device__ __forceinline__ uint64_t part_of(uint64_t sum, float x) {
  return __umul64hi(sum, static_cast<uint64_t>(static_cast<double>(x) * 0x1p64));
}
// The least whole number >= max(sum * p, 1), for p < 1.
__device__ __forceinline__ uint64_t share_of(uint64_t sum, float p) {
  const uint64_t q = static_cast<uint64_t>(static_cast<double>(fmaxf(p, 0.f)) * 0x1p64);
  return max(__umul64hi(sum, q) + (sum * q != 0), uint64_t{1});
}

template <class T>
struct Picker {
  const SampleArgs& a;
  const Workspace& ws;
  Shared& s;
  const T* row;
  int r;
  Settings st;
  Weights w;
  double scale;
  int segments;

  // ---- the row's segments, wave by wave -----------------------------------------------
  // f(z, id) for every id of segment g that this lane holds (ids behind the end as -inf).
  template <class F>
  __device__ __forceinline__ void visit(int g, F f) const {
#pragma unroll
    for (int i = 0; i < kLoads<T>; ++i) {
      const int at = g * kSegment + id_in_segment<T>(i, threadIdx.x & 63);
      float z[kVec<T>];
      load_logits(row, at, a.vocab, z);
#pragma unroll
      for (int e = 0; e < kVec<T>; ++e) f(z[e], at + e);
    }
  }
  // s.segment[g] <- sum of f(z, id) over the segments whose largest logit has a key of at least
  // key_low, 0 for the others.
  template <class F>
  __device__ __forceinline__ void segment_sums(uint32_t key_low, F f) const {
    __syncthreads();
    for (int g = threadIdx.x >> 6; g < segments; g += kWaves) {
      uint64_t sum = 0;
      if (order_key(s.segment_top[g]) >= key_low)
        visit(g, [&](float z, int id) { sum += f(z, id); });
      sum = wave_reduce(sum, Add{});
      if ((threadIdx.x & 63) == 0) s.segment[g] = sum;
    }
    __syncthreads();
  }
  // s.segment[g] <- the sum before segment g; returns the sum of all.
  __device__ __forceinline__ uint64_t segments_before() const {
    __syncthreads();
    const int t = threadIdx.x;
    uint64_t total;
    const uint64_t before = block_scan(t < segments ? s.segment[t] : 0, s.slots64, total);
    __syncthreads();
    s.segment[t] = before;
    __syncthreads();
    return total;
  }
  // The id whose running sum of f, over all ids in order, first exceeds x, from s.segment as
  // segments_before leaves it (x < the sum of all).  Where the segment's sum of f comes out a little
  // less than s.segment says (a sum of the first launch), its last id with f > 0.
  template <class F>
  __device__ __forceinline__ int find(uint64_t x, F f) const {
    const int t = threadIdx.x;
    if (t == 0) s.found_id = -1;
    if (t < segments && s.segment[t] <= x && (t + 1 == segments || s.segment[t + 1] > x))
      s.found = static_cast<uint32_t>(t);
    __syncthreads();
    const int g = min(static_cast<int>(s.found), segments - 1);
    // two ids a thread
    const int at = g * kSegment + 2 * t;
    uint64_t v[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) v[e] = at + e < a.vocab ? f(load_logit(row, at + e), at + e) : 0;
    uint64_t total;
    const uint64_t before = s.segment[g] + block_scan(v[0] + v[1], s.slots64, total);
    if (before <= x && before + v[0] > x)
      s.found_id = at;
    else if (before + v[0] <= x && before + v[0] + v[1] > x)
      s.found_id = at + 1;
    __syncthreads();
    if (s.found_id < 0) {  // uniform
      const uint32_t mine = v[1] ? at + 2 : v[0] ? at + 1 : 0;  // id + 1
      const uint32_t last = block_reduce(mine, s.slots32, Max{});
      return last ? static_cast<int>(last) - 1 : g * kSegment;
    }
    return s.found_id;
  }

  // ---- few ids, in LDS ------------------------------------------------------------------
  // Puts every id whose logit is at least `least` into s.list as (key, ~id), by way of the groups
  // whose largest logit is; returns their number, or -1 where they are more than kList.
  __device__ __forceinline__ int gather(float least) const {
    const int t = threadIdx.x, n_groups = segments * 64;
    const float* const tops = ws.group_top + static_cast<size_t>(r) * n_groups;
    uint32_t* const groups = s.bins;  // kBins of them at most
    __syncthreads();
    if (t == 0) s.n_list = s.found = 0;
    __syncthreads();
    for (int i = t; i < n_groups; i += kThreads)
      if (tops[i] >= least) {
        const uint32_t at = atomicAdd(&s.found, 1u);
        if (at < kList) groups[at] = static_cast<uint32_t>(i);
      }
    __syncthreads();
    const int found = static_cast<int>(s.found);
    if (found > kList) return -1;  // (each holds one such id at least)
    for (int i = t; i < found * kLoads<T>; i += kThreads) {
      const int group = static_cast<int>(groups[i / kLoads<T>]);
      const int at = (group >> 6) * kSegment + id_in_segment<T>(i % kLoads<T>, group & 63);
      float z[kVec<T>];
      load_logits(row, at, a.vocab, z);
#pragma unroll
      for (int e = 0; e < kVec<T>; ++e)
        if (z[e] >= least) {
          const uint32_t j = atomicAdd(&s.n_list, 1u);
          if (j < kList)
            s.list[j] = static_cast<uint64_t>(order_key(z[e])) << 32 | ~static_cast<uint32_t>(at + e);
        }
    }
    __syncthreads();
    return s.n_list <= kList ? static_cast<int>(s.n_list) : -1;
  }
  static __device__ __forceinline__ uint32_t entry_key(uint64_t x) {
    return static_cast<uint32_t>(x >> 32);
  }
  static __device__ __forceinline__ int entry_id(uint64_t x) {
    return static_cast<int>(~static_cast<uint32_t>(x));
  }
  __device__ __forceinline__ double entry_weight(uint64_t x) const {
    return w(key_logit(entry_key(x)));
  }

  // A logit such that at least `want` groups have a larger one or it, and not many more: the lowest in
  // the first so many bins of the groups' largest.  The lowest finite value when all groups above
  // -inf together hold at most kList ids.
  __device__ __forceinline__ float few_limit(uint32_t want, float top) const {
    const int t = threadIdx.x, n_groups = segments * 64;
    const float* const tops = ws.group_top + static_cast<size_t>(r) * n_groups;
    float low = INFINITY;
    uint32_t finite = 0;
    for (int i = t; i < n_groups; i += kThreads) {
      const float z = tops[i];
      if (z > -INFINITY) {
        low = fminf(low, z);
        ++finite;
      }
    }
    low = block_reduce(low, s.slots_f, Min{});
    finite = block_reduce(finite, s.slots32, Add{});
    if (finite * kGroup <= kList) return -FLT_MAX;
    // (what weighs less than e^-48 of the largest needs no bin of its own; halves: no overflow)
    const float from = fmaxf(low, top - 48.f * st.temperature);
    const float per = (kThreads - 1) / (0.5f * top - 0.5f * from);
    if (!(per < FLT_MAX)) return low;
    auto bin = [&](float z) {
      return static_cast<int>(fminf((0.5f * top - 0.5f * z) * per, kThreads - 1.f));
    };
    s.bins[t] = 0;
    if (t == 0) s.found = kThreads - 1;
    __syncthreads();
    for (int i = t; i < n_groups; i += kThreads)
      if (tops[i] > -INFINITY) atomicAdd(&s.bins[bin(tops[i])], 1u);
    __syncthreads();
    uint32_t total;
    const uint32_t mine = s.bins[t];
    const uint32_t before = block_scan(mine, s.slots32, total);
    if (before < want && before + mine >= want) s.found = static_cast<uint32_t>(t);
    __syncthreads();
    const int b = static_cast<int>(s.found);
    float edge = INFINITY;
    for (int i = t; i < n_groups; i += kThreads)
      if (tops[i] > -INFINITY && bin(tops[i]) <= b) edge = fminf(edge, tops[i]);
    return block_reduce(edge, s.slots_f, Min{});
  }

  // Cuts and draws from the n ids of s.list, which are the first n of the order; false where what is
  // kept may go on behind them.  whole_sum: the sum of all weights where no top-k limits it.
  __device__ __forceinline__ bool pick_from_list(int n, bool complete, uint64_t whole_sum, float u,
                                                 int& token, double& sum) const {
    const int t = threadIdx.x;
    sort_falling(s.list, n);
    const uint64_t entry = t < n ? s.list[t] : 0;
    const double x = t < n ? entry_weight(entry) : 0.0;
    const uint64_t mass = whole(x, scale);
    uint64_t total;
    const uint64_t before = block_scan(mass, s.slots64, total);
    int keep = n;
    bool closed = complete;  // nothing behind the list can be kept
    if (st.top_k > 0) {
      if (st.top_k > n && !complete) return false;
      keep = min(st.top_k, n);
      closed = true;
    }
    if (st.top_p < 1.f) {
      if (st.top_k > 0) {
        if (t == keep - 1) s.mass[0] = before + mass;
        __syncthreads();
        whole_sum = s.mass[0];
      } else if (complete) {
        whole_sum = total;
      }
      const uint64_t target = share_of(whole_sum, st.top_p);
      if (t == 0) s.found = n;
      __syncthreads();
      if (t < n && before < target && before + mass >= target) s.found = static_cast<uint32_t>(t);
      __syncthreads();
      if (static_cast<int>(s.found) < n) {
        keep = min(keep, static_cast<int>(s.found) + 1);
        closed = true;
      }
    }
    if (st.min_p > 0.f) {
      const uint32_t above =
          block_reduce(static_cast<uint32_t>(t < n && x >= st.min_p), s.slots32, Add{});
      if (static_cast<int>(above) < n) closed = true;
      keep = min(keep, static_cast<int>(above));
    }
    if (!closed) return false;
    // the kept ones in the order of their ids
    __syncthreads();
    if (t < n) s.mass[t] = mass;
    if (t < keep)
      s.list[t] = static_cast<uint64_t>(static_cast<uint32_t>(entry)) << 32 | static_cast<uint32_t>(t);
    __syncthreads();
    sort_falling(s.list, keep);  // (~id falls)
    const uint64_t by_id = t < keep ? s.list[t] : 0;
    const uint64_t m = t < keep ? s.mass[static_cast<uint32_t>(by_id)] : 0;
    const uint64_t up_to = block_scan(m, s.slots64, total);
    const uint64_t at = part_of(total, u);
    if (up_to <= at && at < up_to + m) s.found_id = static_cast<int>(~static_cast<uint32_t>(by_id >> 32));
    __syncthreads();
    token = s.found_id;
    sum = static_cast<double>(total) / scale;
    return true;
  }

  // ---- a cut anywhere in the row -----------------------------------------------------------
  // Puts the kept ids' sums into s.segment.
  __device__ __forceinline__ void sum_kept(const Cut& cut, uint32_t key_low) const {
    segment_sums(max(cut.key, key_low), [&](float z, int id) -> uint64_t {
      if (!cut.keeps(order_key(z), id)) return 0;
      const double x = w(z);
      return x >= st.min_p ? whole(x, scale) : 0;
    });
  }

  // The cut behind the first `target` ids of the order (kMass false), or behind the fewest whose
  // weights come to `target` (true).  `summed`: s.segment holds the sums of what it keeps.
  //
  // A histogram over [low, top] by value, of counts, or of weights in 32 bits, which is only to find
  // the bin; then the exact sums above the bin, segment by segment, with the bin's ids into the
  // list.  Where the histogram's rounding has led to the bin next to the right one, the exact sums say
  // so.
  template <bool kMass>
  __device__ __forceinline__ Cut search(uint64_t target, float low, float top, bool& summed) const {
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    summed = false;
    const float per = (kBins - 1) / (0.5f * top - 0.5f * low);  // (halves: no overflow)
    if (!(per < FLT_MAX)) return search_bits<kMass>(target);
    auto bin = [&](float z) {
      return static_cast<int>(fminf((0.5f * top - 0.5f * z) * per, kBins - 1.f));
    };
    __syncthreads();
    for (int i = t; i < kBins; i += kThreads) s.bins[i] = 0;
    if (t == 0) s.found = kBins - 1;
    __syncthreads();
    float* const fbins = reinterpret_cast<float*>(s.bins);
    const float rate = static_cast<float>(w.rate / 16.0);
    for (int g = wave; g < segments; g += kWaves)
      if (s.segment_top[g] > -INFINITY)
        visit(g, [&](float z, int) {
          if (!(z > -INFINITY)) return;
          if (kMass)
            atomicAdd(&fbins[bin(z)], fast_exp2((z - top) * rate));
          else
            atomicAdd(&s.bins[bin(z)], 1u);
        });
    __syncthreads();
    auto take = [&](auto before, auto x0, auto x1, auto want) {
      if (before < want && before + x0 >= want)
        s.found = 2 * t;
      else if (before + x0 < want && before + x0 + x1 >= want)
        s.found = 2 * t + 1;
    };
    if (kMass) {
      const double x0 = fbins[2 * t], x1 = fbins[2 * t + 1];
      double all;
      const double before = block_scan(x0 + x1, s.slots_d, all);
      take(before, x0, x1, static_cast<double>(target) / scale);
    } else {
      const uint64_t x0 = s.bins[2 * t], x1 = s.bins[2 * t + 1];
      uint64_t all;
      const uint64_t before = block_scan(x0 + x1, s.slots64, all);
      take(before, x0, x1, target);
    }
    __syncthreads();
    int at_bin = static_cast<int>(s.found);

    uint64_t above;
    for (int last_step = 0;;) {
      __syncthreads();
      if (t == 0) s.n_list = 0;
      __syncthreads();
      uint64_t n_above = 0, m_inside = 0;
      for (int g = wave; g < segments; g += kWaves) {
        uint64_t sum = 0;
        if (s.segment_top[g] > -INFINITY && bin(s.segment_top[g]) <= at_bin)
          visit(g, [&](float z, int id) {
            if (!(z > -INFINITY)) return;
            const int b = bin(z);
            if (b > at_bin) return;
            const uint64_t m = whole(w(z), scale);
            if (b < at_bin) {
              sum += m;
              ++n_above;
              return;
            }
            m_inside += m;
            const uint32_t j = atomicAdd(&s.n_list, 1u);
            if (j < kList)
              s.list[j] = static_cast<uint64_t>(order_key(z)) << 32 | ~static_cast<uint32_t>(id);
          });
        sum = wave_reduce(sum, Add{});
        if (lane == 0) s.segment[g] = sum;
      }
      uint64_t inside = block_reduce(kMass ? m_inside : uint64_t{0}, s.slots64, Add{});
      above = kMass ? (t < segments ? s.segment[t] : 0) : n_above;
      above = block_reduce(above, s.slots64, Add{});
      if (!kMass) inside = s.n_list;
      int step = 0;
      if (above >= target)
        step = -1;
      else if (above + inside < target)
        step = 1;
      // (a step back after one in the other direction, or off the end: by bits)
      if (step == 0) break;
      if (step == -last_step || at_bin + step < 0 || at_bin + step >= kBins)
        return search_bits<kMass>(target);
      last_step = step;
      at_bin += step;
    }
    const int n = static_cast<int>(s.n_list);
    if (n > kList) return search_bits<kMass>(target);
    sort_falling(s.list, n);
    const uint64_t entry = t < n ? s.list[t] : 0;
    const uint64_t mass = t < n ? whole(entry_weight(entry), scale) : 0;
    uint64_t total;
    const uint64_t unit = kMass ? mass : t < n ? 1 : 0;
    const uint64_t before = above + block_scan(unit, s.slots64, total);
    if (t < n && before < target) {  // kept
      atomicAdd(reinterpret_cast<unsigned long long*>(&s.segment[entry_id(entry) / kSegment]),
                static_cast<unsigned long long>(mass));
      if (before + unit >= target) s.found = static_cast<uint32_t>(t);
    }
    __syncthreads();
    const uint64_t last = s.list[s.found];
    summed = true;
    return Cut{entry_key(last), entry_id(last)};
  }

  // The same by three rounds over the row, which fix 11, 11 and 10 bits of the key, with exact sums;
  // then, where not all ids of that key are kept, their last one.
  template <bool kMass>
  __device__ __forceinline__ Cut search_bits(uint64_t target) const {
    const int t = threadIdx.x;
    uint32_t prefix = 0;
    uint64_t n_before = 0, m_before = 0;
    for (int level = 0; level < 3; ++level) {
      const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, above = level == 1 ? 21 : 10;
      const uint32_t mask = level == 2 ? 1023u : 2047u;
      __syncthreads();
      for (int i = t; i < kBins; i += kThreads) {
        s.bins[i] = 0;
        s.bin_mass[i] = 0;
      }
      if (t == 0) s.found_count = 0;
      __syncthreads();
      for (int g = t >> 6; g < segments; g += kWaves)
        if (s.segment_top[g] > -INFINITY)
          visit(g, [&](float z, int) {
            const uint32_t key = order_key(z);
            if (!(z > -INFINITY) || (level > 0 && (key >> above) != prefix)) return;
            const uint32_t bin = (key >> shift) & mask;
            atomicAdd(&s.bins[bin], 1u);
            atomicAdd(reinterpret_cast<unsigned long long*>(&s.bin_mass[bin]),
                      static_cast<unsigned long long>(whole(w(z), scale)));
          });
      __syncthreads();
      // bins from the highest down, two a thread
      const int hi = kBins - 1 - 2 * t;
      const uint64_t c0 = s.bins[hi], c1 = s.bins[hi - 1], m0 = s.bin_mass[hi],
                     m1 = s.bin_mass[hi - 1];
      uint64_t all;
      const uint64_t n0 = n_before + block_scan(c0 + c1, s.slots64, all);
      const uint64_t p0 = m_before + block_scan(m0 + m1, s.slots64, all);
      auto take = [&](int bin, uint64_t c, uint64_t m, uint64_t n, uint64_t p) {
        const uint64_t from = kMass ? p : n, to = kMass ? p + m : n + c;
        if (from < target && target <= to) {
          s.found = static_cast<uint32_t>(bin);
          s.found_count = static_cast<uint32_t>(c);
          s.found_before = static_cast<uint32_t>(n);
          s.found_mass = m;
          s.found_mass_before = p;
        }
      };
      take(hi, c0, m0, n0, p0);
      take(hi - 1, c1, m1, n0 + c0, p0 + m0);
      __syncthreads();
      if (s.found_count == 0) return kKeepAll;  // fewer ids, or less weight, than the target
      prefix = level == 0 ? s.found : (prefix << (level == 1 ? 11 : 10)) | s.found;
      n_before = s.found_before;
      m_before = s.found_mass_before;
    }
    // every id of the last bin has the same key and weight
    const uint64_t equal = s.found_count, each = s.found_mass / equal;
    const uint64_t keep = kMass ? (target - m_before + each - 1) / each : target - n_before;
    Cut cut{prefix, INT32_MAX};
    if (keep < equal) {
      auto ties = [&](float z, int id) -> uint64_t {
        return id < a.vocab && order_key(z) == cut.key ? 1 : 0;
      };
      segment_sums(cut.key, ties);
      segments_before();
      cut.last = find(keep - 1, ties);
    }
    return cut;
  }
};

template <class T>
__global__ __launch_bounds__(kThreads) void sample_pick_kernel(SampleArgs a, Workspace ws) {
  __shared__ Shared s;
  const int t = threadIdx.x, r = blockIdx.x;
  const Settings st = settings(a, find_sequence(a.cu_block, a.batch, r, t & 63));
  const float u = fminf(fmaxf(a.uniform[r], 0.f), 0x1.fffffep-1f);
  SegmentStats mine{-INFINITY, INFINITY, 0.f, 0.f, 0.0};
  if (t < ws.segments) mine = ws.stats[static_cast<size_t>(r) * ws.segments + t];
  s.segment_top[t] = mine.top;
  if (t < 16) s.pow16[t] = kPow16[t];
  const bool bad = __syncthreads_or(mine.top != mine.top);
  const float top = block_reduce(mine.top, s.slots_f, Max{});
  if (bad || top == -INFINITY) {  // a NaN or +inf; or nothing to draw from
    if (t == 0) {
      a.token[r] = -1;
      const float none = bad ? NAN : 0.f;
      if (a.prob) a.prob[r] = none;
      if (a.conf) a.conf[r] = none;
    }
    return;
  }
  Picker<T> p{a, ws, s, static_cast<const T*>(a.logits) + static_cast<size_t>(r) * a.pitch, r, st,
              Weights{s.pow16, static_cast<double>(top), weight_rate(st.temperature)}, 0.0,
              ws.segments};
  int token;
  double sum = 1.0;  // of the kept weights
  if (st.greedy()) {
    const uint32_t key = order_key(top);
    s.segment[t] = mine.top == top;
    p.segments_before();
    token = p.find(0, [&](float z, int) -> uint64_t { return order_key(z) == key; });
  } else {
    const bool few = st.top_k > 0 && st.top_k <= kFewIds;
    uint64_t whole_sum = 0;
    // s.segment <- the segments' sums as whole numbers of 1 / scale, from sums relative to their own top
    auto scale_sums = [&](double x) {
      const double all = block_reduce(x, s.slots_d, Add{});
      p.scale = ldexp(1.0, 61 - ilogb(all));
      const uint64_t part = whole(x, p.scale);
      s.segment[t] = part;
      whole_sum = block_reduce(part, s.slots64, Add{});
    };
    if (few)
      p.scale = 0x1p51;  // (at most kList weights of at most 1 are summed)
    else
      scale_sums(mine.top > -INFINITY ? mine.sum * p.w(mine.top) : 0.0);
    const bool limited = st.top_k > 0 || st.top_p < 1.f || st.min_p > 0.f;
    bool done = false;
    if (limited && (few || st.top_k == 0)) {
      const float least = p.few_limit(few ? st.top_k : kFewIds / 2, top);
      const int n = p.gather(least);
      done = n >= 0 && p.pick_from_list(n, least == -FLT_MAX, whole_sum, u, token, sum);
    }
    if (!done) {
      if (few) {  // the list has not done, and the sums have not been formed
        double x = 0.0;
        for (int g = t >> 6; g < ws.segments; g += kWaves)
          p.visit(g, [&](float z, int) { x += p.w(z); });
        scale_sums(x);
      }
      Cut cut = kKeepAll;
      bool summed = !limited;
      if (limited) {
        const float low = block_reduce(mine.low, s.slots_f, Min{});
        if (st.top_k > 0) {
          cut = p.template search<false>(static_cast<uint64_t>(st.top_k), low, top, summed);
          if (st.top_p < 1.f) {
            if (!summed) {
              p.segment_sums(cut.key, [&](float z, int id) -> uint64_t {
                return cut.keeps(order_key(z), id) ? whole(p.w(z), p.scale) : 0;
              });
              summed = true;
            }
            whole_sum = block_reduce(t < ws.segments ? s.segment[t] : uint64_t{0}, s.slots64, Add{});
          }
        }
        if (st.top_p < 1.f) {
          bool sums_of_it;
          const Cut c = p.template search<true>(share_of(whole_sum, st.top_p),
                                                fmaxf(low, top - 64.f * st.temperature), top,
                                                sums_of_it);
          summed = c.tighter(cut) && sums_of_it;
          if (c.tighter(cut)) cut = c;
        }
        uint32_t key_low = 0;
        if (st.min_p > 0.f) {
          // the cut may keep ids below min_p: none below this key is kept
          if (cut.key == 0 || p.w(key_logit(cut.key)) < st.min_p) summed = false;
          const double least = top + static_cast<double>(st.temperature) * log(static_cast<double>(st.min_p));
          key_low = order_key(static_cast<float>(least - 1e-6 * (1.0 + fabs(least))));
        }
        if (!summed) p.sum_kept(cut, key_low);
      }
      const uint64_t total = p.segments_before();
      token = p.find(part_of(total, u), [&](float z, int id) -> uint64_t {
        if (!cut.keeps(order_key(z), id)) return 0;
        const double x = p.w(z);
        return x >= st.min_p ? whole(x, p.scale) : 0;
      });
      sum = static_cast<double>(total) / p.scale;
    }
  }
  float soft = 0.f;
  if (a.conf)
    soft = block_reduce(mine.soft * fast_exp2((mine.top - top) * kLog2e), s.slots_f, Add{});
  if (t == 0) {
    const float z = load_logit(p.row, token);
    a.token[r] = token;
    if (a.prob) a.prob[r] = st.greedy() ? 1.f : static_cast<float>(p.w(z) / sum);
    if (a.conf) a.conf[r] = static_cast<float>(exp(static_cast<double>(z) - top) / soft);
  }
}

int segments_of(int vocab) { return (vocab + kSegment - 1) / kSegment; }
size_t stats_bytes(int n_rows, int vocab) {
  const size_t n = static_cast<size_t>(n_rows) * segments_of(vocab) * sizeof(SegmentStats);
  return (n + 255) / 256 * 256;
}

template <class T>
hipError_t launch(const SampleArgs& a, void* ws, hipStream_t s) {
  const int segments = segments_of(a.vocab);
  const Workspace w{static_cast<SegmentStats*>(ws),
                    reinterpret_cast<float*>(static_cast<char*>(ws) + stats_bytes(a.n_rows, a.vocab)),
                    segments};
  const int parts = (segments + kScanWaves - 1) / kScanWaves;
  hipLaunchKernelGGL(sample_scan_kernel<T>, dim3(a.n_rows * parts), dim3(kScanThreads), 0, s, a, w);
  hipLaunchKernelGGL(sample_pick_kernel<T>, dim3(a.n_rows), dim3(kThreads), 0, s, a, w);
  return hipGetLastError();
}

}  // namespace

size_t sample_ws_bytes(int n_rows, int vocab) {
  return stats_bytes(n_rows, vocab) +
         static_cast<size_t>(n_rows) * segments_of(vocab) * 64 * sizeof(float);
}

long sample_threads(int n_rows, int vocab) {
  const long parts = (segments_of(vocab) + kScanWaves - 1) / kScanWaves;
  return max(parts * kScanThreads, static_cast<long>(kThreads)) * n_rows;
}

hipError_t sample(bool bf16, const SampleArgs& a, void* ws, hipStream_t s) {
  if (a.n_rows == 0) return hipSuccess;
  return bf16 ? launch<uint16_t>(a, ws, s) : launch<float>(a, ws, s);
}

}  // namespace eb

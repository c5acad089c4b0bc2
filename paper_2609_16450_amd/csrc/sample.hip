// A token per row from its logits and a given random number: temperature, top-k, top-p, min-p.
//
// With w_v = exp((z_v - m) / t) and the vocabulary in the order (z falling, id rising), every
// filter keeps a prefix of that order, so what is kept is one cut: all ids whose logit lies above a
// value, and of those that equal it the lowest ids up to one.  The token is the lowest kept id
// whose running sum, over the kept ids in rising order, exceeds u times the sum of all of them.
//
// The drawn id depends on sums over up to the whole vocabulary next to a border, and has to be the
// same whatever cuts the sums into pieces.  So a weight is formed in 64 bits (to 2^-37 of itself,
// see Weights).  Within a segment of 2048 ids weights are summed as 64-bit floats, always the same
// ones in the same order.  Beyond that, and id by id next to a border, sums are of whole numbers of
// 2^-62 of (at least) the sum of all weights (in rows of a small top-k, of 2^-52 of the largest
// one): they are exact in any order, also by atomics, whichever segments a workgroup has.  A whole
// number is off by at most half a unit, a segment's sum by less than 2^-47 of itself, far below
// what the weights are off by.
//
// sample_scan_kernel reads every logit once and leaves, per segment of 2048 ids, its largest and
// lowest logit and its sums of weights, and the largest of each of its 64 groups of 32 ids.
// sample_pick_kernel, a workgroup per row, cuts and draws from these alone where that can be done:
// with a temperature only it reads the one segment that the draw falls into; with a small top-k, or
// where the nucleus is small, the groups that can hold what is kept (their largest logits say
// which), at most kPickList ids in LDS.  The rows left over (none of a vocabulary that the list
// holds whole) are read again: sample_bins_kernel makes a histogram which finds the few bins that
// the cut lies in, and sample_sums_kernel the exact sums above them and a list of the ids within,
// many workgroups to a row; sample_search_kernel, one workgroup to a row, orders the list, cuts and
// draws.  Rows whose bins hold more ids than the list it cuts by itself, the key found bit by bit:
// logits that tie; a few that lie far off the others, so that these share few bins; more than some
// 300000 ids, of which one bin holds too many.
//
// Bounds: many rows are bound by reading the logits, once in the scan (944 fp32 rows of 126464,
// mixed settings: 110 us, 4.3 TB/s), and once or twice more where they are left over; few rows by
// one dependent step after another (a single row with a small top-k: 20 us; two launches, and three
// that find nothing to do).
#include <float.h>
#include <stddef.h>

#include <type_traits>

#include "attn_common.hpp"
#include "eb_common.hpp"
#include "eb_internal.hpp"
#include "paged.hpp"
#include "wave_ops.hpp"

namespace eb {
namespace {

constexpr int kSegment = 2048;         // ids that a wave takes at a time
constexpr int kGroup = kSegment / 64;  // of them a lane's
constexpr int kScanThreads = 256;
constexpr int kScanWaves = kScanThreads / 64;
constexpr int kPickThreads = 256;
constexpr int kPickWaves = kPickThreads / 64;
constexpr int kPickList = kPickThreads;  // ids that the second launch settles a row among
constexpr int kThreads = 1024;           // of a workgroup that searches
constexpr int kWaves = kThreads / 64;
constexpr int kMaxSegments = kThreads;
constexpr int kList = kThreads;  // ids that it sorts in LDS
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

// Logits at .. at + kVec - 1 of a row, as they came; -inf behind its end.  (Loads without the test
// for segments that lie before the row's end: 108 -> 123 us for 944 rows of 126464.)
template <class T>
struct Chunk;
template <>
struct Chunk<float> {
  f32x4 x;
  __device__ __forceinline__ void load(const float* row, int at, int vocab) {
    if (at + 4 <= vocab) {
      x = *reinterpret_cast<const f32x4u*>(row + at);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = at + e < vocab ? row[at + e] : -INFINITY;
    }
  }
  __device__ __forceinline__ float operator[](int e) const { return x[e]; }
};
template <>
struct Chunk<uint16_t> {
  u32x4 x;
  __device__ __forceinline__ void load(const uint16_t* row, int at, int vocab) {
    if (at + 8 <= vocab) {
      x = *reinterpret_cast<const u32x4h*>(row + at);
    } else {
      auto bits = [&](int e) -> uint32_t { return at + e < vocab ? row[at + e] : 0xff80u; };
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = bits(2 * i) | bits(2 * i + 1) << 16;
    }
  }
  __device__ __forceinline__ float operator[](int e) const {
    const uint32_t w = x[e / 2];
    return __uint_as_float(e % 2 ? w & 0xffff0000u : w << 16);
  }
};
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

// 2^(i / 64)
__constant__ const double kPow64[64] = {
    0x1.0000000000000p+0, 0x1.02c9a3e778061p+0, 0x1.059b0d3158574p+0, 0x1.0874518759bc8p+0,
    0x1.0b5586cf9890fp+0, 0x1.0e3ec32d3d1a2p+0, 0x1.11301d0125b51p+0, 0x1.1429aaea92de0p+0,
    0x1.172b83c7d517bp+0, 0x1.1a35beb6fcb75p+0, 0x1.1d4873168b9aap+0, 0x1.2063b88628cd6p+0,
    0x1.2387a6e756238p+0, 0x1.26b4565e27cddp+0, 0x1.29e9df51fdee1p+0, 0x1.2d285a6e4030bp+0,
    0x1.306fe0a31b715p+0, 0x1.33c08b26416ffp+0, 0x1.371a7373aa9cbp+0, 0x1.3a7db34e59ff7p+0,
    0x1.3dea64c123422p+0, 0x1.4160a21f72e2ap+0, 0x1.44e086061892dp+0, 0x1.486a2b5c13cd0p+0,
    0x1.4bfdad5362a27p+0, 0x1.4f9b2769d2ca7p+0, 0x1.5342b569d4f82p+0, 0x1.56f4736b527dap+0,
    0x1.5ab07dd485429p+0, 0x1.5e76f15ad2148p+0, 0x1.6247eb03a5585p+0, 0x1.6623882552225p+0,
    0x1.6a09e667f3bcdp+0, 0x1.6dfb23c651a2fp+0, 0x1.71f75e8ec5f74p+0, 0x1.75feb564267c9p+0,
    0x1.7a11473eb0187p+0, 0x1.7e2f336cf4e62p+0, 0x1.82589994cce13p+0, 0x1.868d99b4492edp+0,
    0x1.8ace5422aa0dbp+0, 0x1.8f1ae99157736p+0, 0x1.93737b0cdc5e5p+0, 0x1.97d829fde4e50p+0,
    0x1.9c49182a3f090p+0, 0x1.a0c667b5de565p+0, 0x1.a5503b23e255dp+0, 0x1.a9e6b5579fdbfp+0,
    0x1.ae89f995ad3adp+0, 0x1.b33a2b84f15fbp+0, 0x1.b7f76f2fb5e47p+0, 0x1.bcc1e904bc1d2p+0,
    0x1.c199bdd85529cp+0, 0x1.c67f12e57d14bp+0, 0x1.cb720dcef9069p+0, 0x1.d072d4a07897cp+0,
    0x1.d5818dcfba487p+0, 0x1.da9e603db3285p+0, 0x1.dfc97337b9b5fp+0, 0x1.e502ee78b3ff6p+0,
    0x1.ea4afa2a490dap+0, 0x1.efa1bee615a27p+0, 0x1.f50765b6e4540p+0, 0x1.fa7c1819e90d8p+0};

// exp((z - top) / temperature) in 64 bits.  With y = (z - top) 64 log2(e) / temperature and n the
// whole number nearest to y, it is 2^(n / 64) 2^((y - n) / 64): a table in LDS and a polynomial in
// y - n (|y - n| <= 1/2) of the third degree, 1 at 0 and otherwise as near as one comes, which
// leaves 2^-37 of the value at most.  (A weight's error of that size moves a border of the draw by
// as much of the weight: one in 10^8 draws from 100000 ids of like weight across it.)  n comes from
// the low bits of y + 1.5 2^52, and 2^(n / 64 rounded down) goes into the result's exponent.  What
// a pass over a row costs is its weights: with 16 table values and a fifth degree 41 us for 131072
// on one compute unit, 20 us of them the weights.
struct Weights {
  const double* pow64;  // LDS
  double top, rate;     // largest logit; 64 log2(e) / temperature
  // Not 0 but 2^-1000 or so where that is the value or less, -inf among it.
  __device__ __forceinline__ double normal(float z) const {
    // the power series of exp(x ln 2 / 64) with the fourth term's best parabola in place of it
    constexpr double c1 = 0x1.62e42fefa39efp-7, c2 = 0x1.ebfc213e1c4f7p-15,
                     c3 = 0x1.c6b08d704a0c0p-23;
    constexpr double kRound = 0x1.8p52;
    const double y = fmax((static_cast<double>(z) - top) * rate, kLeast);
    const double shifted = y + kRound, r = y - (shifted - kRound);
    const int k = static_cast<int>(__double_as_longlong(shifted));  // low word
    const double p = fma(r, fma(r, fma(r, c3, c2), c1), 1.0);
    const uint64_t x = __double_as_longlong(pow64[k & 63] * p);
    return __longlong_as_double(x + (static_cast<uint64_t>(static_cast<uint32_t>(k >> 6)) << 52));
  }
  __device__ __forceinline__ double operator()(float z) const {
    const double x = normal(z);
    return x > kNothing ? x : 0.0;
  }
  static constexpr double kLeast = -64000.0;  // in y
  // Weights up to this one are 0; what normal() gives for those below 2^-1000, a segment of them
  // summed up too.
  static constexpr double kNothing = 0x1p-980;
};
__device__ __forceinline__ double weight_rate(float temperature) {
  return 0x1.71547652b82fep+6 / static_cast<double>(temperature);  // 64 log2(e) / t
}
// Weights as whole numbers of 1 / scale, a power of two; one that is not 0 counts at least 1.
__device__ __forceinline__ uint64_t whole(double w, double scale) {
  return w > Weights::kNothing ? max(static_cast<uint64_t>(rint(w * scale)), uint64_t{1}) : 0;
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

// Top-k small enough to be settled by the second launch: half the list, so that the ids which the
// groups' largest logits let through besides fit as well.
constexpr int kFewIds = kPickList / 2;
// Ids among which a top-p or min-p is tried otherwise: a sure model's nucleus.
constexpr int kNucleus = 64;

// A row's settings.
struct Settings {
  float temperature, top_p, min_p;
  int32_t top_k;  // 0: no limit
  __device__ __forceinline__ bool greedy() const { return !(temperature > 0.f); }
  // (the top_k largest of n groups let at most about -n ln(1 - top_k / n) ids through, 214 of 128
  // groups)
  __device__ __forceinline__ bool few(int vocab) const {
    const int groups = (vocab + kSegment - 1) / kSegment * 64;
    return top_k > 0 && top_k <= kFewIds && (vocab <= kPickList || 16 * top_k <= 13 * groups);
  }
  __device__ __forceinline__ bool limited() const {
    return top_k > 0 || top_p < 1.f || min_p > 0.f;
  }
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
// What the second launch knows of a row that it leaves to the next ones.
struct RowHeader {
  double scale;
  uint64_t whole_sum;
  float top, low;
  Settings st;
  uint32_t pending;  // 0: the row is settled, and the rest is not written
  uint32_t pad;
};
static_assert(sizeof(RowHeader) == 48, "packed");

// What the launches that search a row leave one another; zeroed by the second launch.
struct Border {
  uint64_t between;  // weight between `last` and bin_k
  uint32_t n_list[2];
  int32_t first, last;              // bins of the cut
  int32_t bin_k, bin_m;             // top-k's and min-p's (kBins: no limit)
  uint32_t before_first, before_k;  // ids in the bins before `first` and before bin_k, with a top-k
};
struct SearchState {
  uint32_t count[kBins], mass[kBins];  // ids and weights (of 2^-31 of their sum) per bin
  Border border;
  uint64_t pad;
  uint64_t list[2][kList];  // ids of bins first .. last, of bin_k where that lies behind them
};
static_assert(sizeof(SearchState) % 16 == 0, "whole 16-byte words");

struct Workspace {
  SegmentStats* stats;  // [n_rows, segments]
  float* group_top;     // [n_rows, segments, 64]: largest logit of a lane's ids
  RowHeader* headers;   // [n_rows]
  uint64_t* kept;       // [n_rows, segments]: sums above a cut's bin
  SearchState* states;  // [n_rows]
  int segments;
  int parts;  // workgroups per row of the launches that search
};

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
struct MaxOfBoth {  // of the two halves, each by itself
  __device__ __forceinline__ uint64_t operator()(uint64_t a, uint64_t b) const {
    const uint32_t hi = max(static_cast<uint32_t>(a >> 32), static_cast<uint32_t>(b >> 32));
    const uint32_t lo = max(static_cast<uint32_t>(a), static_cast<uint32_t>(b));
    return static_cast<uint64_t>(hi) << 32 | lo;
  }
};
struct Min {
  __device__ __forceinline__ uint64_t operator()(uint64_t a, uint64_t b) const { return min(a, b); }
  __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); }
};

// ---------------------------------------------------------------------------------------
// First launch: a wave per segment.
// ---------------------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(kScanThreads) void sample_scan_kernel(SampleArgs a, Workspace ws) {
  __shared__ double pow64[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int parts = (ws.segments + kScanWaves - 1) / kScanWaves;
  const int r = blockIdx.x / parts;
  const int g = (blockIdx.x - r * parts) * kScanWaves + wave;
  const T* const row = static_cast<const T*>(a.logits) + static_cast<size_t>(r) * a.pitch;
  Chunk<T> z[kLoads<T>];
#pragma unroll
  for (int i = 0; i < kLoads<T>; ++i)
    z[i].load(row, g * kSegment + id_in_segment<T>(i, lane), a.vocab);
  if (threadIdx.x < 64) pow64[threadIdx.x] = kPow64[threadIdx.x];
  const Settings st = settings(a, find_sequence(a.cu_block, a.batch, r, lane));
  __syncthreads();
  if (g >= ws.segments || r >= a.cu_block[a.batch]) return;

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
    // rows of few ids by count, and greedy ones, take no sum over all
    const bool sum = !st.greedy() && !st.few(a.vocab);
    if (sum) {
      const Weights w{pow64, static_cast<double>(top), weight_rate(st.temperature)};
#pragma unroll
      for (int i = 0; i < kLoads<T>; ++i)
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) out.sum += w.normal(z[i][e]);
      out.sum = wave_reduce(out.sum, Add{});
      out.soft = static_cast<float>(out.sum);  // (at temperature 1)
    }
    if (a.conf && !(sum && st.temperature == 1.f)) {
      out.soft = 0.f;
#pragma unroll
      for (int i = 0; i < kLoads<T>; ++i)
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) out.soft += fast_exp2((z[i][e] - top) * kLog2e);
      out.soft = wave_reduce(out.soft, Add{});
    }
  }
  if (lane == 0) ws.stats[at] = out;
}

// ---------------------------------------------------------------------------------------
// What the later launches share.
// ---------------------------------------------------------------------------------------
__device__ __forceinline__ int wave_index() {
  return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x >> 6));
}

// x over the kN waves of the workgroup, on every thread; `slots` [kN] is free again behind the next
// barrier.
template <int kN, class V, class Op>
__device__ __forceinline__ V block_reduce(V x, V* slots, Op op) {
  x = wave_reduce(x, op);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = x;
  __syncthreads();
  V y = slots[0];
#pragma unroll
  for (int w = 1; w < kN; ++w) y = op(y, slots[w]);
  return uniform(y);
}

// Sum of x over the threads before this one; `total` over all.
template <int kN, class V>
__device__ __forceinline__ V block_scan(V x, V* slots, V& total) {
  const int lane = threadIdx.x & 63, wave = wave_index();
  const V sum = wave_scan(x);
  __syncthreads();
  if (lane == 63) slots[wave] = sum;
  __syncthreads();
  V before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kN; ++w) {
    if (w == wave) before = all;
    all += slots[w];
  }
  total = uniform(all);
  return before + sum - x;
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

// A list's entry: (key, ~id), so that the order is that of falling entries.
__device__ __forceinline__ uint64_t entry_of(float z, int id) {
  return static_cast<uint64_t>(order_key(z)) << 32 | ~static_cast<uint32_t>(id);
}
__device__ __forceinline__ uint32_t entry_key(uint64_t x) { return static_cast<uint32_t>(x >> 32); }
__device__ __forceinline__ int entry_id(uint64_t x) {
  return static_cast<int>(~static_cast<uint32_t>(x));
}

// A row, as a workgroup of any size sees it.  Every wave reduces the segments' statistics by
// itself, without barriers, and all come to the same bits.
template <class T>
struct Row {
  const T* logits;
  const SegmentStats* stats;
  const float* group_top;
  int r, vocab, segments;
  Settings st;
  float top, low;
  Weights w;
  double scale;
  uint64_t whole_sum;  // of all weights, as whole numbers

  __device__ __forceinline__ void locate(const SampleArgs& a, const Workspace& ws, int row) {
    r = row;
    logits = static_cast<const T*>(a.logits) + static_cast<size_t>(r) * a.pitch;
    stats = ws.stats + static_cast<size_t>(r) * ws.segments;
    group_top = ws.group_top + static_cast<size_t>(r) * ws.segments * 64;
    vocab = a.vocab;
    segments = ws.segments;
  }
  // A row that the second launch has left: false where it has not.
  __device__ __forceinline__ bool reopen(const SampleArgs& a, const Workspace& ws, int row,
                                         const double* pow64) {
    const RowHeader& h = ws.headers[row];
    if (!uniform(h.pending)) return false;
    locate(a, ws, row);
    top = uniform(h.top);
    low = uniform(h.low);
    st = Settings{uniform(h.st.temperature), uniform(h.st.top_p), uniform(h.st.min_p),
                  uniform(h.st.top_k)};
    scale = uniform(h.scale);
    whole_sum = uniform(h.whole_sum);
    w = Weights{pow64, static_cast<double>(top), weight_rate(st.temperature)};
    return true;
  }
  __device__ __forceinline__ void set_scale(double sum) { scale = ldexp(1.0, 61 - ilogb(sum)); }
  // Where the running sum of parts(g) first exceeds x: the segment, with the sum before it.
  template <class F>
  __device__ __forceinline__ int find_segment(uint64_t x, F parts, uint64_t& before) const {
    const int lane = threadIdx.x & 63;
    uint64_t base = 0;
    for (int g0 = 0; g0 < segments; g0 += 64) {
      const uint64_t part = parts(g0 + lane), upto = base + wave_scan(part);
      const uint64_t hit = __ballot(upto > x);
      if (hit) {
        const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
        before = of_lane(upto - part, l);
        return g0 + l;
      }
      base = of_lane(upto, 63);
    }
    before = base;
    return segments - 1;
  }
  // The id whose running sum of f, over the ids of segment g in order and what lies before it,
  // first exceeds x.  Where the segment's sum of f comes out a little less than the sum that has
  // led to it (one of the first launch's), its last id with f > 0.
  template <int kN, class S, class F>
  __device__ __forceinline__ int find_id(S& s, int g, uint64_t before, uint64_t x, F f) const {
    constexpr int kIds = kSegment / (64 * kN);  // of a thread
    const int at = g * kSegment + static_cast<int>(threadIdx.x) * kIds;
    uint64_t v[kIds], mine = 0;
#pragma unroll
    for (int e = 0; e < kIds; ++e) {
      v[e] = at + e < vocab ? f(load_logit(logits, at + e), at + e) : 0;
      mine += v[e];
    }
    if (threadIdx.x == 0) s.found_id = -1;
    uint64_t total;
    uint64_t run = before + block_scan<kN>(mine, s.slots64, total);
    if (run <= x && run + mine > x) {
      int id = at;
#pragma unroll
      for (int e = 0; e < kIds - 1; ++e) {
        run += v[e];
        if (run <= x) id = at + e + 1;
      }
      s.found_id = id;
    }
    __syncthreads();
    const int id = uniform(s.found_id);
    if (id >= 0) return id;
    uint32_t last = 0;  // id + 1
#pragma unroll
    for (int e = 0; e < kIds; ++e)
      if (v[e]) last = at + e + 1;
    last = block_reduce<kN>(last, s.slots32, Max{});
    return last ? static_cast<int>(last) - 1 : g * kSegment;
  }
  // Row r's outputs, by the calling thread; soft: sum of the model's weights, for conf; sum: of the
  // kept weights.
  __device__ __forceinline__ float model_sum(const SampleArgs& a) const {
    float soft = 0.f;
    if (a.conf)
      for (int g = threadIdx.x & 63; g < segments; g += 64)
        soft += stats[g].soft * fast_exp2((stats[g].top - top) * kLog2e);
    return wave_reduce(soft, Add{});
  }
  __device__ __forceinline__ void write(const SampleArgs& a, int token, double sum,
                                        float soft) const {
    const float z = load_logit(logits, token);
    a.token[r] = token;
    if (a.prob) a.prob[r] = st.greedy() ? 1.f : static_cast<float>(w(z) / sum);
    if (a.conf) a.conf[r] = static_cast<float>(Weights{w.pow64, w.top, weight_rate(1.f)}(z)) / soft;
  }
};

__device__ __forceinline__ float random_number(const SampleArgs& a, int r) {
  return fminf(fmaxf(a.uniform[r], 0.f), 0x1.fffffep-1f);
}

// ---------------------------------------------------------------------------------------
// Second launch: a workgroup of four waves per row settles it where that takes one segment, or at
// most kPickList ids.
// ---------------------------------------------------------------------------------------
struct PickShared {
  double pow64[64];
  uint64_t list[kPickList][2];  // entry, weight
  alignas(16) uint32_t bins[kPickThreads];
  uint32_t groups[kPickList];
  uint64_t slots64[kPickWaves];
  uint32_t slots32[kPickWaves];
  float slots_f[kPickWaves];
  uint64_t sum_of_k;
  uint32_t n_list, n_groups, past_min_p, unsure;
  int32_t found_id;
};

// A row's segments, a few of them in this lane's registers (segments lane and lane + 64: rows of up
// to 2^18 ids), the others in memory.  Every wave goes through all of them by itself, without
// barriers, and all come to the same bits.
struct SegmentsOfRow {
  static constexpr int kHeld = 2;
  const SegmentStats* stats;
  int n;
  SegmentStats held[kHeld];
  __device__ __forceinline__ SegmentsOfRow(const SegmentStats* stats_, int n_)
      : stats(stats_), n(n_) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      held[j] = lane + 64 * j < n ? stats[lane + 64 * j]
                                  : SegmentStats{-INFINITY, INFINITY, 0.f, 0.f, 0.0};
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) f(held[j]);
    for (int g = (threadIdx.x & 63) + 64 * kHeld; g < n; g += 64) f(stats[g]);
  }
  // f(segment g), 0 behind the last one; g - lane is a multiple of 64
  template <class F>
  __device__ __forceinline__ uint64_t at(int g, F f) const {
    if (g < 64) return f(held[0]);
    if (g < 128) return f(held[1]);
    return g < n ? f(stats[g]) : 0;
  }
};

// Largest logits of a row's groups: thread t has groups 4 t .. 4 t + 3 of every 4 kPickThreads, the
// first ones (rows of up to 163840 ids) in registers.
struct GroupTops {
  static constexpr int kHeld = 5, kPass = 4 * kPickThreads;
  const float* tops;
  int n;  // a multiple of 64
  f32x4 held[kHeld];
  __device__ __forceinline__ GroupTops(const float* tops_, int n_) : tops(tops_), n(n_) {
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int i = j * kPass + 4 * static_cast<int>(threadIdx.x);
      held[j] = i < n ? *reinterpret_cast<const f32x4*>(tops + i)
                      : f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    }
  }
  // Number of this thread's first group of a pass.
  static __device__ __forceinline__ int first(int pass) {
    return pass * kPass + 4 * static_cast<int>(threadIdx.x);
  }
  template <class F>
  __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) f(held[j][e]);
    for (int i = first(kHeld); i < n; i += kPass)
      for (int e = 0; e < 4; ++e) f(tops[i + e]);
  }
};

// The first of `mine` places in a list for this lane; reserved once a wave.  (With a branch and an
// atomic to each item most of the kernel's time went here.)
__device__ __forceinline__ uint32_t reserve(uint32_t& length, uint32_t mine) {
  const uint32_t upto = wave_scan(mine), total = of_lane(upto, 63);
  uint32_t at = 0;
  if (total && (threadIdx.x & 63) == 0) at = atomicAdd(&length, total);
  return uniform(at) + upto - mine;
}

// The first ids of the order into s.list, by way of the groups whose largest logits are the first
// of these; all ids above -inf (then `complete`) where there are at most kPickList.  By count: at
// least `want` of them.  Otherwise about as many, less where the rest weighs less than e^-48 of the
// largest.  Returns their number, or -1 where they are more than kPickList.
//
// (Much of what a row costs here is the fetching of its code: with a bin and a branch to each item,
// 41 KB in the kernel, 16.0 us for 32 rows; with one comparison, with the lowest logit that is
// taken, 31 KB and 12.4 us.)
template <class T>
__device__ __forceinline__ int gather(const Row<T>& row, const GroupTops& tops, PickShared& s,
                                      uint32_t want, bool by_count, bool& complete) {
  constexpr int kLevels = 3;
  const int t = threadIdx.x, lane = t & 63;
  float hi = row.top, lo = fmaxf(row.low, row.top - 48.f * row.st.temperature);
  float least = row.low;  // that has a bin
  float cut;              // least logit that is taken
  // The bin of [lo, hi] that the want-th group lies in, the last one for what lies lower as well.
  // Where the groups up to it are more than the list, the bins are laid over that bin's: a sure
  // row's one logit far above all others, then perhaps a mask's far below them.
  uint32_t ahead = 0;  // groups above hi
  for (int level = 0;; ++level) {
    // (halves: no overflow)
    const float per = fminf((kPickThreads - 1) / (0.5f * hi - 0.5f * lo), FLT_MAX);
    auto bin = [&](float z) {
      return static_cast<int>(fminf((0.5f * hi - 0.5f * z) * per, kPickThreads - 1.f));
    };
    tops.each([&](float z) {
      if (z >= least && z <= hi) atomicAdd(&s.bins[bin(z)], 1u);
    });
    __syncthreads();
    // every wave for itself, four bins a lane
    const u32x4 c = *reinterpret_cast<const u32x4*>(&s.bins[4 * lane]);
    const uint32_t sum = c[0] + c[1] + c[2] + c[3], upto = ahead + wave_scan(sum);
    uint32_t through = of_lane(upto, 63), before = through;
    if (level == 0) complete = row.vocab <= kPickList || through * kGroup <= kPickList;
    int last = kPickThreads - 1;
    const uint64_t hit = __ballot(upto >= want);
    if (hit && !complete) {
      const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
      before = of_lane(upto - sum, l);
      last = 4 * l;
      through = before + of_lane(c[0], l);
      if (through < want) ++last, before = through, through += of_lane(c[1], l);
      if (through < want) ++last, before = through, through += of_lane(c[2], l);
      if (through < want) ++last, before = through, through += of_lane(c[3], l);
    }
    if (!by_count && !complete && lo > row.low) last = min(last, kPickThreads - 2);
    // (a bin lower than the one found, for the roundings of both)
    cut = last == kPickThreads - 1 ? least : fmaxf(2.f * (0.5f * hi - (last + 2) / per), least);
    if (!by_count || complete || through <= kPickList || level == kLevels - 1) break;
    float a = -INFINITY, b = INFINITY;
    tops.each([&](float z) {
      const bool in = z >= least && z <= hi && bin(z) == last;
      a = fmaxf(a, in ? z : -INFINITY);
      b = fminf(b, in ? z : INFINITY);
    });
    a = block_reduce<kPickWaves>(a, s.slots_f, Max{});
    s.bins[t] = 0;  // (every wave has read them)
    b = block_reduce<kPickWaves>(b, s.slots_f, Min{});
    hi = a;
    least = lo = b;
    ahead = before;
  }
  uint32_t taken = 0;  // bit 4 j + e: held[j][e]
#pragma unroll
  for (int j = 0; j < GroupTops::kHeld; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      taken |= static_cast<uint32_t>(tops.held[j][e] >= cut) << (4 * j + e);
  auto put_groups = [&](int pass) {
    uint32_t place = reserve(s.n_groups, __popc(taken));
    for (; taken; taken &= taken - 1) {
      const int bit = __ffs(taken) - 1;
      if (place < kPickList)
        s.groups[place++] = static_cast<uint32_t>(GroupTops::first(pass + bit / 4) + bit % 4);
    }
  };
  put_groups(0);
  for (int pass = GroupTops::kHeld; pass * GroupTops::kPass < tops.n; ++pass) {
    const int i = GroupTops::first(pass);
    for (int e = 0; e < 4; ++e)
      if (i < tops.n && tops.tops[i + e] >= cut) taken |= 1u << e;
    put_groups(pass);
  }
  __syncthreads();
  const int found = static_cast<int>(uniform(s.n_groups));
  if (found > kPickList) return -1;  // (each holds one such id at least)
  // the groups' ids, one a lane, 16 loads of a thread under way at once
  constexpr int kAtOnce = 16;
  for (int i0 = 0; i0 < found * kGroup; i0 += kAtOnce * kPickThreads) {
    float z[kAtOnce];
    int ids[kAtOnce];
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int item = i0 + j * kPickThreads + t, k = item % kGroup;
      const int group = static_cast<int>(s.groups[min(item / kGroup, found - 1)]);
      ids[j] = (group >> 6) * kSegment + id_in_segment<T>(k / kVec<T>, group & 63) + k % kVec<T>;
      z[j] = load_logit(row.logits, min(ids[j], row.vocab - 1));
      if (item >= found * kGroup || ids[j] >= row.vocab) z[j] = -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) mine += z[j] >= cut;
    uint32_t place = reserve(s.n_list, mine);
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (z[j] >= cut && place < kPickList) s.list[place++][0] = entry_of(z[j], ids[j]);
  }
  __syncthreads();
  const uint32_t n = uniform(s.n_list);
  return n <= kPickList ? static_cast<int>(n) : -1;
}

// Cuts and draws from the n ids of s.list, the first n of the order, an id a thread; false where
// what is kept may go on behind them.  An id's place in the order, the weight before it, and then
// the weight up to it in the order of ids come from one walk each over the list, which all lanes
// read at once: no sorting, and no sums across waves.
template <class T>
__device__ __forceinline__ bool pick_from_list(const SampleArgs& a, const Row<T>& row,
                                               PickShared& s, int n, bool complete, float soft) {
  const int t = threadIdx.x;
  const Settings& st = row.st;
  const bool open = !complete && !(st.top_k > 0 && st.top_k <= n);  // what limits it may lie behind
  if (open && st.few(row.vocab)) return false;
  const bool active = t < n;
  const uint64_t entry = active ? s.list[t][0] : 0;
  const double x = active ? row.w(key_logit(entry_key(entry))) : 0.0;
  const uint64_t mass = whole(x, row.scale);
  if (active)
    s.list[t][1] = mass;
  else
    s.list[t][0] = s.list[t][1] = 0;
  if (active && x < st.min_p) s.past_min_p = 1;
  const uint64_t of_list = block_reduce<kPickWaves>(mass, s.slots64, Add{});
  uint64_t all = complete ? of_list : row.whole_sum;
  // unless nothing behind the list can be kept
  if (open && !(st.top_p < 1.f && of_list >= share_of(all, st.top_p)) && !uniform(s.past_min_p))
    return false;
  uint64_t before = 0;
  int place = 0;
  // f(entry, weight) of the list's ids, eight at a time; behind its end 0, 0
  auto walk = [&](auto f) {
    if (wave_index() * 64 >= n) return;
    for (int j = 0; j < n; j += 8) {
      uint64_t e[8], m[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = s.list[j + i][0];
        m[i] = s.list[j + i][1];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) f(e[i], m[i]);
    }
  };
  walk([&](uint64_t e, uint64_t m) {
    const bool ahead = e > entry;
    place += ahead;
    before += ahead ? m : 0;
  });
  const int keep = st.top_k > 0 ? min(st.top_k, n) : n;
  bool kept = active && place < keep && x >= st.min_p;
  if (st.top_p < 1.f) {
    if (st.top_k > 0 && !open) {
      if (active && place == keep - 1) s.sum_of_k = before + mass;
      __syncthreads();
      all = uniform(s.sum_of_k);
    }
    // (of a top-k behind the list: its ids weigh no less than the list and no more than all)
    if (st.top_k > 0 && open && kept && before < share_of(all, st.top_p) &&
        before >= share_of(of_list, st.top_p))
      s.unsure = 1;
    kept &= before < share_of(all, st.top_p);
  }
  __syncthreads();  // the walks are over
  if (uniform(s.unsure)) return false;
  if (active && !kept) s.list[t][1] = 0;
  __syncthreads();
  if (wave_index() * 64 >= n) return true;
  uint64_t upto = 0, total = 0;
  walk([&](uint64_t e, uint64_t m) {
    total += m;
    // (~id falls as the id rises)
    upto += static_cast<uint32_t>(e) >= static_cast<uint32_t>(entry) ? m : 0;
  });
  const uint64_t at = part_of(total, random_number(a, row.r));
  if (kept && upto > at && upto - mass <= at)
    row.write(a, entry_id(entry), static_cast<double>(total) / row.scale, soft);
  return true;
}

// kLimits: the call has a top-k, top-p or min-p (of which a row may still have none).
template <class T, bool kLimits>
__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(SampleArgs a, Workspace ws) {
  __shared__ PickShared s;
  const int t = threadIdx.x, lane = t & 63;
  Row<T> row;
  row.locate(a, ws, blockIdx.x);
  const SegmentsOfRow segments(row.stats, row.segments);
  const GroupTops tops(row.group_top, kLimits ? row.segments * 64 : 0);
  row.st = settings(a, find_sequence(a.cu_block, a.batch, row.r, lane));
  if (t < 64) s.pow64[t] = kPow64[t];
  s.bins[t] = 0;
  if (t == 0) s.n_list = s.n_groups = s.past_min_p = s.unsure = 0;
  float hi = -INFINITY, lo = INFINITY;
  bool bad = false;
  segments.each([&](const SegmentStats& x) {
    bad |= x.top != x.top;
    hi = fmaxf(hi, x.top);
    lo = fminf(lo, x.low);
  });
  row.top = uniform(wave_reduce(hi, Max{}));
  row.low = uniform(wave_reduce(lo, Min{}));
  bad = __any(bad);
  RowHeader& header = ws.headers[row.r];
  if (row.r >= a.cu_block[a.batch]) {  // behind the last sequence
    if (t == 0) header.pending = 0;
    return;
  }
  if (bad || row.top == -INFINITY) {  // a NaN or +inf; or nothing to draw from
    if (t == 0) {
      a.token[row.r] = -1;
      const float none = bad ? NAN : 0.f;
      if (a.prob) a.prob[row.r] = none;
      if (a.conf) a.conf[row.r] = none;
      header.pending = 0;
    }
    return;
  }
  row.w = Weights{s.pow64, static_cast<double>(row.top), weight_rate(row.st.temperature)};
  __syncthreads();

  float soft = 0.f;  // sum of the model's weights, for conf
  if (a.conf) {
    segments.each([&](const SegmentStats& x) {
      soft += x.soft * fast_exp2((x.top - row.top) * kLog2e);
    });
    soft = wave_reduce(soft, Add{});
  }
  auto weight = [&](const SegmentStats& x) {
    return x.top > -INFINITY ? x.sum * row.w(x.top) : 0.0;
  };
  auto whole_part = [&](const SegmentStats& x) { return whole(weight(x), row.scale); };
  auto sum_segments = [&]() {  // sets scale and whole_sum
    double x = 0.0;
    segments.each([&](const SegmentStats& g) { x += weight(g); });
    x = uniform(wave_reduce(x, Add{}));
    row.set_scale(x);
    row.whole_sum = whole(x, row.scale);
  };
  if (row.st.greedy() || !row.st.limited()) {
    int token;
    double sum = 1.0;
    uint64_t before;
    if (row.st.greedy()) {
      const float top = row.top;
      const uint32_t key = order_key(top);
      const int g = row.find_segment(
          0, [&](int i) {
            return segments.at(i, [&](const SegmentStats& x) -> uint64_t { return x.top == top; });
          }, before);
      token = row.template find_id<kPickWaves>(
          s, g, 0, 0, [&](float z, int) -> uint64_t { return order_key(z) == key; });
    } else {
      sum_segments();
      uint64_t n = 0;  // as the segments' parts add up
      segments.each([&](const SegmentStats& g) { n += whole_part(g); });
      row.whole_sum = uniform(wave_reduce(n, Add{}));
      const uint64_t at = part_of(row.whole_sum, random_number(a, row.r));
      const int g =
          row.find_segment(at, [&](int i) { return segments.at(i, whole_part); }, before);
      token = row.template find_id<kPickWaves>(
          s, g, before, at, [&](float z, int) { return whole(row.w(z), row.scale); });
      sum = static_cast<double>(row.whole_sum) / row.scale;
    }
    if (t == 0) {
      row.write(a, token, sum, soft);
      header.pending = 0;
    }
    return;
  }
  if constexpr (kLimits) {
    const bool few = row.st.few(row.vocab);
    if (few) {
      row.scale = 0x1p52;  // (at most kPickList weights of at most 1 are summed)
      row.whole_sum = 0;
    } else {
      sum_segments();
    }
    bool done = false;
    // A list that holds the whole row settles it whatever limits it, and has to: such a call makes
    // no later launches, and its workspace has no states for them.
    const bool held = row.vocab <= kPickList;
    // (a list of weights of at most 1 does not come to top_p of more than its length)
    const bool hopeless =
        row.st.min_p <= 0.f &&
        static_cast<double>(share_of(row.whole_sum, fminf(row.st.top_p, 0x1.fffffep-1f))) >
            kPickList * row.scale;
    if (few || held || ((row.st.top_p < 1.f || row.st.min_p > 0.f) && !hopeless)) {
      bool complete;
      const int n = gather(row, tops, s, few ? row.st.top_k : kNucleus, few, complete);
      done = n > 0 && pick_from_list(a, row, s, n, complete, soft);
    }
    if (t == 0) {
      if (done)
        header.pending = 0;
      else
        header = RowHeader{row.scale, row.whole_sum, row.top, row.low, row.st, 1, 0};
    }
    if (!done && !held) {  // (all but the lists)
      u32x4* const state = reinterpret_cast<u32x4*>(&ws.states[row.r]);
      for (int i = t; i < static_cast<int>(offsetof(SearchState, list) / 16); i += kPickThreads)
        state[i] = u32x4{};
    }
  }
}

// ---------------------------------------------------------------------------------------
// The rows that the second launch has left: cuts anywhere.  Three launches: a histogram of a row by
// its parts' workgroups, which tells the bin that the cut lies in; the exact sums above the bin,
// segment by segment, with the bin's ids put into a list, by workgroups again; and a workgroup that
// orders the list, cuts and draws.  The last one alone also does the rows that the others have not
// found the cut of.  (That workgroup alone for rows of up to 32768 ids: 40 -> 48 us for a row of
// 9000, 588 -> 970 us for 4096 rows of 32000, wide nuclei.)
// ---------------------------------------------------------------------------------------
constexpr int kPartThreads = 256;
constexpr int kPartWaves = kPartThreads / 64;
// The histogram's workgroups do two parts each: what few rows wait for is its atomics on the row's
// state (4 waves: 14.6 us for 32 rows, 8: 11.0, 16: 10.2; but of 944 rows in all 199, 196 and 197
// us).
constexpr int kBinThreads = 2 * kPartThreads;
__host__ __device__ constexpr int bin_parts(int parts) { return (parts + 1) / 2; }

// f(z, id) for every id that this lane holds of segments first + wave, first + wave + kN, .. below
// `end` for which wanted(g); then each_segment(g) (by the whole wave) for these and the others.
// Two loads at a time, the next two under way meanwhile (four: 232 -> 237 us for 944 rows of
// 126464, mixed settings), worked on by two ids (with more the kernels of 16 waves, which have 128
// registers a lane, spill; the others take the same time with eight).
template <int kN, class T, class Wanted, class F, class End>
__device__ __forceinline__ void visit(const Row<T>& row, int first, int end, Wanted wanted, F f,
                                      End each_segment) {
  constexpr int kAtOnce = 2, kIds = 2;
  const int lane = threadIdx.x & 63;
  for (int g = first + wave_index(); g < end; g += kN) {
    if (wanted(g)) {
      Chunk<T> x[kAtOnce], next[kAtOnce];
      auto load = [&](int i0, Chunk<T> (&c)[kAtOnce]) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          c[i].load(row.logits, g * kSegment + id_in_segment<T>(i0 + i, lane), row.vocab);
      };
      load(0, x);
#pragma unroll 1
      for (int i0 = 0; i0 < kLoads<T>; i0 += kAtOnce) {
        if (i0 + kAtOnce < kLoads<T>) load(i0 + kAtOnce, next);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
          for (int e = 0; e < kVec<T>; ++e) {
            if ((i * kVec<T> + e) % kIds == 0) __builtin_amdgcn_sched_barrier(0);
            f(x[i][e], g * kSegment + id_in_segment<T>(i0 + i, lane) + e);
          }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) x[i] = next[i];
      }
    }
    each_segment(g);
  }
}

// Bins from a row's largest logit down; a higher logit never has a higher bin.  They are of equal
// width down to what weighs e^-64 of the largest, and the last one holds all that lies lower; but
// with a top-k, which counts that too, half of them are laid over it.
struct Bins {
  static constexpr int kLower = kBins / 2 - 1;
  float half_top, per, half_from, per_lower, upper;
  template <class T>
  __device__ __forceinline__ explicit Bins(const Row<T>& row) {
    // (halves: no overflow)
    const float from = fmaxf(row.low, row.top - 64.f * row.st.temperature);
    const bool split = row.st.top_k > 0 && from > row.low;
    upper = split ? kBins - 1 - kLower : kBins - 1;
    half_top = 0.5f * row.top;
    half_from = 0.5f * from;
    per = upper / (half_top - half_from);
    per_lower = split ? kLower / (half_from - 0.5f * row.low) : 0.f;
  }
  __device__ __forceinline__ bool usable() const { return per < FLT_MAX; }
  __device__ __forceinline__ int operator()(float z) const {
    const float x = fminf((half_top - 0.5f * z) * per, upper);
    // (a NaN, of 0 times infinity, becomes 0)
    const float y = fminf(fmaxf((half_from - 0.5f * z) * per_lower, 0.f), kLower);
    return static_cast<int>(x + y);
  }
};

// The least logit whose weight is at least min_p: from its formula, then, as the weights themselves
// round, by steps to the next float.
template <class T>
__device__ __forceinline__ float min_p_logit(const Row<T>& row) {
  const double z = row.top + static_cast<double>(row.st.temperature) *
                                 log(static_cast<double>(row.st.min_p));
  uint32_t key = order_key(fminf(fmaxf(static_cast<float>(z), -FLT_MAX), row.top));
  auto reaches = [&](uint32_t k) { return row.w(key_logit(k)) >= row.st.min_p; };
  for (int i = 0; i < 8 && !reaches(key); ++i) ++key;
  for (int i = 0; i < 8 && reaches(key - 1); ++i) --key;
  return key_logit(key);
}

// Whether the launches over parts have to do with a row (of those left).
template <class T>
__device__ __forceinline__ bool in_parts(const Row<T>& row) {
  return !row.st.few(row.vocab) && Bins(row).usable();
}

__device__ __forceinline__ int part_begin(int part, int parts, int segments) {
  return static_cast<int>(static_cast<long>(segments) * part / parts);
}

template <class T>
__global__ __launch_bounds__(kBinThreads) void sample_bins_kernel(SampleArgs a, Workspace ws) {
  __shared__ uint32_t count[kBins], mass[kBins + 64];
  const int parts = bin_parts(ws.parts);
  const int t = threadIdx.x, r = blockIdx.x / parts, part = blockIdx.x - r * parts;
  Row<T> row;
  if (!row.reopen(a, ws, r, nullptr) || !in_parts(row)) return;
  for (int i = t; i < kBins; i += kBinThreads) count[i] = mass[i] = 0;
  const bool by_count = row.st.top_k > 0, by_mass = row.st.top_p < 1.f;
  if (!by_count && !by_mass) return;
  __syncthreads();
  // weights as whole numbers of 2^-31 of (at most) their sum (a float's atomic sum takes 8 times as
  // long in LDS)
  const float rate = static_cast<float>(row.w.rate / 64.0);
  const float unit = static_cast<float>(ilogb(row.scale) - 31);
  const float top = row.top;
  const Bins bin(row);
  visit<kBinThreads / 64>(
      row, part_begin(part, parts, ws.segments), part_begin(part + 1, parts, ws.segments),
      [&](int g) { return uniform(row.stats[g].top) > -INFINITY; },
      [&](float z, int) {
        if (!(z > -INFINITY)) return;
        const int b = bin(z);
        if (by_count) atomicAdd(&count[b], 1u);
        if (by_mass) {
          // (most of a sure row's are 0, and in one bin: these go to a place of the lane's own)
          const uint32_t m = static_cast<uint32_t>(fast_exp2((z - top) * rate + unit) + 0.5f);
          atomicAdd(&mass[m ? b : kBins + (t & 63)], m);
        }
      },
      [](int) {});
  __syncthreads();
  SearchState& state = ws.states[r];
  for (int i = t; i < kBins; i += kBinThreads) {
    if (by_count && count[i]) atomicAdd(&state.count[i], count[i]);
    if (by_mass && mass[i]) atomicAdd(&state.mass[i], mass[i]);
  }
}

// The bins in which the running sum of x (kBins / kPartThreads bins a thread) reaches a first and a
// second target, kBins where none does, with the sum before the first of them.
struct FoundBins {
  int first, second;
  uint64_t before;
};
__device__ __forceinline__ FoundBins find_bins(const uint32_t* x, uint64_t first, uint64_t second,
                                               uint64_t* slots, FoundBins* found) {
  constexpr int kEach = kBins / kPartThreads;
  const int t = threadIdx.x;
  uint32_t v[kEach];
  uint64_t mine = 0, total;
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    v[e] = x[t * kEach + e];
    mine += v[e];
  }
  __syncthreads();  // (what an earlier call has found has been read)
  if (t == 0) *found = FoundBins{kBins, kBins, 0};
  uint64_t run = block_scan<kPartWaves>(mine, slots, total);
  if ((run < first && run + mine >= first) || (run < second && run + mine >= second)) {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const uint64_t upto = run + v[e];
      if (run < first && upto >= first) found->first = t * kEach + e, found->before = run;
      if (run < second && upto >= second) found->second = t * kEach + e;
      run = upto;
    }
  }
  __syncthreads();
  return FoundBins{uniform(found->first), uniform(found->second), uniform(found->before)};
}

template <class T>
__global__ __launch_bounds__(kPartThreads) void sample_sums_kernel(SampleArgs a, Workspace ws) {
  __shared__ double pow64[64];
  __shared__ uint64_t slots64[kPartWaves];
  __shared__ FoundBins found;
  __shared__ uint64_t list[2][kList];
  __shared__ uint32_t n_list[2], list_at[2];
  const int t = threadIdx.x, r = blockIdx.x / ws.parts, part = blockIdx.x - r * ws.parts;
  Row<T> row;
  if (!row.reopen(a, ws, r, pow64) || !in_parts(row)) return;
  if (t < 64) pow64[t] = kPow64[t];
  if (t < 2) n_list[t] = 0;
  __syncthreads();
  const Settings& st = row.st;
  const Bins bin(row);
  SearchState& state = ws.states[r];
  // The bins of each limit, kBins where it limits nothing; the cut lies in the first of them.
  // top-p's are those that its sum reaches within 2^-18 of the whole (hardly ever two) and, where
  // it is a part of the first top_k ids' weight, for all that this may be.  The histogram is mostly
  // nearer than 2^-18, but not always: each id's weight is off by up to half of 2^-31 of the sum,
  // all of a long tail to the same side perhaps (2^-15 of the sum for 126464 ids).  What has led to
  // a bin beside the cut's is found by the exact sums (cut_from_lists), and such a row is searched
  // by one workgroup.
  int bin_k = kBins, bin_m = kBins, p_first = kBins, p_last = kBins;
  uint64_t before_k = 0;
#pragma unroll 1
  for (int by_mass = 0; by_mass < 2; ++by_mass) {
    if (by_mass ? st.top_p >= 1.f : st.top_k == 0) continue;
    uint64_t low = static_cast<uint64_t>(st.top_k), high = low;
    if (by_mass) {
      uint64_t least = row.whole_sum >> 31, most = least;  // weight that top_p takes its part of
      if (bin_k < kBins) {  // the bins up to bin_k, without it and with it
        uint64_t x = 0;
        for (int i = t; i < bin_k; i += kPartThreads) x += state.mass[i];
        least = block_reduce<kPartWaves>(x, slots64, Add{});
        most = least + state.mass[bin_k];
      }
      const uint64_t slack = (most >> 18) + 1;
      low = share_of(least, st.top_p);
      low = low > slack ? low - slack : 1;
      high = share_of(most, st.top_p) + slack;
    }
    const FoundBins f = find_bins(by_mass ? state.mass : state.count, low, high, slots64, &found);
    if (by_mass) {
      p_first = f.first;
      p_last = f.second;
    } else {
      bin_k = f.first;
      before_k = f.before;
    }
  }
  if (st.min_p > 0.f) bin_m = bin(min_p_logit(row));
  const int first = min(min(bin_k, p_first), bin_m), last = min(min(bin_k, p_last), bin_m);
  const bool between = st.top_p < 1.f && bin_k < kBins && bin_k > last;
  const int end = between ? bin_k : last;
  if (part == 0) {
    uint64_t x = 0;
    if (st.top_k > 0)
      for (int i = t; i < min(first, kBins); i += kPartThreads) x += state.count[i];
    x = block_reduce<kPartWaves>(x, slots64, Add{});
    if (t == 0) {
      state.border.first = first;
      state.border.last = last;
      state.border.bin_k = bin_k;
      state.border.bin_m = bin_m;
      state.border.before_first = static_cast<uint32_t>(x);
      state.border.before_k = static_cast<uint32_t>(before_k);
    }
  }
  // (whole numbers from each segment's sums: which segments are a wave's depends on the call's
  // rows)
  double sum = 0.0, sum_between = 0.0;
  uint64_t weight_between = 0;
  visit<kPartWaves>(
      row, part_begin(part, ws.parts, ws.segments), part_begin(part + 1, ws.parts, ws.segments),
      [&](int g) {
        const float top = uniform(row.stats[g].top);
        return top > -INFINITY && uniform(bin(top)) <= end;
      },
      [&](float z, int id) {
        const int b = bin(z);
        if (b > end || !(z > -INFINITY)) return;
        if (b < first) {
          sum += row.w.normal(z);
        } else if (b > last && b < bin_k) {
          sum_between += row.w.normal(z);
        } else {
          const int which = b <= last ? 0 : 1;
          const uint32_t j = atomicAdd(&n_list[which], 1u);
          if (j < kList) list[which][j] = entry_of(z, id);
        }
      },
      [&](int g) {
        sum = wave_reduce(sum, Add{});
        if ((t & 63) == 0)
          ws.kept[static_cast<size_t>(r) * ws.segments + g] = whole(sum, row.scale);
        sum = 0.0;
        if (between) {
          weight_between += whole(wave_reduce(sum_between, Add{}), row.scale);
          sum_between = 0.0;
        }
      });
  // The listed ids by one reservation a workgroup.  (With an atomic on the
  // state for each 14.5 us for 32 wide nuclei, so 11.9.)
  __syncthreads();
  if (t < 2 && n_list[t]) list_at[t] = atomicAdd(&state.border.n_list[t], n_list[t]);
  __syncthreads();
#pragma unroll
  for (int which = 0; which < 2; ++which)
    for (uint32_t j = t; j < min(n_list[which], uint32_t{kList}); j += kPartThreads)
      if (list_at[which] + j < kList) state.list[which][list_at[which] + j] = list[which][j];
  if (between && (t & 63) == 0)
    atomicAdd(reinterpret_cast<unsigned long long*>(&state.border.between),
              static_cast<unsigned long long>(weight_between));
}

struct Shared {
  uint64_t segment[kMaxSegments];
  uint64_t list[kList];
  uint64_t bin_mass[kBins];
  uint32_t bins[kBins];
  double pow64[64];
  uint64_t slots64[kWaves];
  double slots_d[kWaves];
  uint32_t slots32[kWaves];
  uint32_t found, found_count, found_before;
  uint64_t found_mass, found_mass_before;
  int32_t found_id;
};

template <class T>
struct Searcher {
  Row<T>& row;
  Shared& s;

  // s.segment[g] <- sum of f(z, id) over the segments whose largest logit has a key of at least
  // key_low, 0 for the others.
  template <class F>
  __device__ __forceinline__ void segment_sums(uint32_t key_low, F f) const {
    __syncthreads();
    uint64_t sum = 0;
    visit<kWaves>(
        row, 0, row.segments,
        [&](int g) { return order_key(uniform(row.stats[g].top)) >= key_low; },
        [&](float z, int id) { sum += f(z, id); },
        [&](int g) {
          sum = wave_reduce(sum, Add{});
          if ((threadIdx.x & 63) == 0) s.segment[g] = sum;
          sum = 0;
        });
    __syncthreads();
  }
  // Sum of s.segment, as every wave finds it.
  __device__ __forceinline__ uint64_t sum_of_segments() const {
    uint64_t n = 0;
    for (int g = threadIdx.x & 63; g < row.segments; g += 64) n += s.segment[g];
    return uniform(wave_reduce(n, Add{}));
  }
  // The id whose running sum of f, over all ids in order, first exceeds x, from f's sums in
  // s.segment.
  template <class F>
  __device__ __forceinline__ int find(uint64_t x, F f) const {
    uint64_t before;
    const int g = row.find_segment(
        x, [&](int i) { return i < row.segments ? s.segment[i] : uint64_t{0}; }, before);
    return row.template find_id<kWaves>(s, g, before, x, f);
  }
  // s.segment <- sums of the kept ids' weights, none of which has a key below key_low.
  __device__ __forceinline__ void sum_kept(const Cut& cut, uint32_t key_low, float min_p) const {
    const uint32_t least = max(cut.key, key_low);
    double sum = 0.0;
    __syncthreads();
    visit<kWaves>(
        row, 0, row.segments,
        [&](int g) { return order_key(uniform(row.stats[g].top)) >= least; },
        [&](float z, int id) {
          const double x = row.w(z);
          if (cut.keeps(order_key(z), id) && x >= min_p) sum += x;
        },
        [&](int g) {
          sum = wave_reduce(sum, Add{});
          if ((threadIdx.x & 63) == 0) s.segment[g] = whole(sum, row.scale);
          sum = 0.0;
        });
    __syncthreads();
  }

  // One of a state's lists, an entry a thread.
  struct Listed {
    int n;
    uint64_t entry, mass;  // this thread's (0: none) and its weight
    double x;
    uint64_t before;  // in the order of entries: their weights before this one, their number
    uint32_t place;
    uint64_t total;  // weight of all
  };
  // The entries are first put into bins, whose numbers and sums of weights come by
  // atomics; within a bin, mostly of one to three, each walks over the others.  (Sorting up to 1024
  // entries across 16 waves took 4 us more.)
  __device__ __forceinline__ Listed listed(uint32_t n, uint64_t entry) const {
    constexpr int kListBins = kThreads;
    const int t = threadIdx.x;
    Listed l;
    l.n = static_cast<int>(uniform(n));
    const bool active = t < l.n;
    l.entry = active ? entry : 0;
    l.x = active ? row.w(key_logit(entry_key(l.entry))) : 0.0;
    l.mass = whole(l.x, row.scale);
    // entries as consecutive numbers as far as they go: keys from the list's lowest on (of bf16
    // logits their upper halves, so that equal ones are told apart by their ids), then the ids
    constexpr int kKeyShift = sizeof(T) == 2 ? 16 : 0;
    const uint32_t key = entry_key(l.entry) >> kKeyShift;
    const uint64_t ends = block_reduce<kWaves>(
        active ? static_cast<uint64_t>(key) << 32 | ~key : uint64_t{0}, s.slots64, MaxOfBoth{});
    const uint32_t high = static_cast<uint32_t>(ends >> 32), low = ~static_cast<uint32_t>(ends);
    const int id_bits = 32 - __clz(row.vocab);
    const uint64_t range = (static_cast<uint64_t>(high - low) + 1) << id_bits;
    const int shift = max(0, 64 - __clzll(static_cast<long long>(range)) - 10);
    static_assert(kListBins == 1 << 10, "range >> shift is a bin");
    uint64_t* const sums = s.bin_mass;
    uint32_t* const counts = s.bins;
    sums[t] = 0;
    counts[t] = 0;
    __syncthreads();
    const uint64_t number = static_cast<uint64_t>(high - key) << id_bits |
                            static_cast<uint32_t>(entry_id(l.entry));
    const uint32_t bin = active ? static_cast<uint32_t>(number >> shift) : 0;
    uint32_t at_in_bin = 0;
    if (active) {
      at_in_bin = atomicAdd(&counts[bin], 1u);
      atomicAdd(reinterpret_cast<unsigned long long*>(&sums[bin]),
                static_cast<unsigned long long>(l.mass));
    }
    __syncthreads();
    const uint32_t count = counts[t];
    uint32_t all;
    const uint32_t place = block_scan<kWaves>(count, s.slots32, all);
    const uint64_t before = block_scan<kWaves>(sums[t], s.slots64, l.total);
    __syncthreads();
    sums[t] = before;
    counts[t] = place;
    __syncthreads();
    // the entries bin by bin, in no order within one
    l.before = sums[bin];
    l.place = counts[bin];
    const uint32_t end = bin + 1 < kListBins ? counts[bin + 1] : static_cast<uint32_t>(l.n);
    const uint32_t begin = l.place;
    if (active) s.list[begin + at_in_bin] = l.entry;
    __syncthreads();
    for (uint32_t j = begin; active && j < end; ++j) {
      const uint64_t other = s.list[j];
      if (other > l.entry) {
        ++l.place;
        l.before += whole(row.w(key_logit(entry_key(other))), row.scale);
      }
    }
    return l;
  }

  // The cut from what the launches over parts have found, with the kept ids' sums in s.segment;
  // false where a list has run over, or a rounding of the histogram has led to a bin without the
  // cut. first_list, kept_sum: this thread's entry of the state's first list and segment's sum
  // above the bins.
  __device__ __forceinline__ bool cut_from_lists(const Border& border, uint64_t first_list,
                                                 const uint64_t* second_list, uint64_t kept_sum,
                                                 Cut& cut) const {
    const int t = threadIdx.x;
    const Settings& st = row.st;
    const int last = uniform(border.last), bin_k = uniform(border.bin_k);
    if (last >= kBins || uniform(border.n_list[0]) > kList || uniform(border.n_list[1]) > kList)
      return false;
    if (t < row.segments) s.segment[t] = kept_sum;
    const bool by_min_p = uniform(border.bin_m) == last;
    // the weight of a list's entries up to the top_k-th id
    auto up_to = [&](const Listed& l, uint32_t ids_before) {
      const uint32_t n = static_cast<uint32_t>(st.top_k) - uniform(ids_before);
      if (l.entry && l.place == n - 1) s.found_mass = l.before + l.mass;
      __syncthreads();
      return uniform(s.found_mass);
    };
    uint64_t of_k = 0;
    if (st.top_p < 1.f && bin_k < kBins && bin_k > last) {
      const Listed l = listed(border.n_list[1], second_list[t]);
      of_k = up_to(l, border.before_k) + uniform(border.between);
      __syncthreads();
    }
    const Listed l = listed(border.n_list[0], first_list);
    const uint64_t above = sum_of_segments();
    bool kept = l.entry != 0, closed = false;
    if (bin_k == last) {
      kept &= l.place < static_cast<uint32_t>(st.top_k) - uniform(border.before_first);
      closed = true;
    }
    if (st.top_p < 1.f) {
      uint64_t all = row.whole_sum;
      if (bin_k == last)
        all = above + up_to(l, border.before_first);
      else if (bin_k < kBins)
        all = above + l.total + of_k;
      const uint64_t target = share_of(all, st.top_p);
      if (above >= target) return false;
      kept &= above + l.before < target;
      closed |= above + l.total >= target;
    }
    if (st.min_p > 0.f) {
      kept &= l.x >= st.min_p;
      closed |= by_min_p;
    }
    if (!closed) return false;
    if (l.n == 0) {  // nothing between the bins above and min_p
      cut = kKeepAll;
      return by_min_p;
    }
    // (the kept ones of the list are its first; with none kept, the cut lies before all of them)
    const uint64_t none = ~uint64_t{0};
    const uint64_t end = block_reduce<kWaves>(kept ? l.entry : none, s.slots64, Min{});
    if (kept)  // (every wave has summed up the segments)
      atomicAdd(reinterpret_cast<unsigned long long*>(&s.segment[entry_id(l.entry) / kSegment]),
                static_cast<unsigned long long>(l.mass));
    if (end == none)
      cut = Cut{block_reduce<kWaves>(entry_key(l.entry), s.slots32, Max{}), -1};
    else
      cut = Cut{entry_key(end), entry_id(end)};
    return true;
  }

  // The cut behind the first `target` ids of the order (by_mass false), or behind the fewest whose
  // weights come to `target` (true), by three rounds over the row, which fix 11, 11 and 10 bits of
  // the key; then, where not all ids of that key are kept, their last one.
  __device__ __forceinline__ Cut search_bits(bool by_mass, uint64_t target) const {
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
      visit<kWaves>(
          row, 0, row.segments, [&](int g) { return uniform(row.stats[g].top) > -INFINITY; },
          [&](float z, int) {
            const uint32_t key = order_key(z);
            if (!(z > -INFINITY) || (level > 0 && (key >> above) != prefix)) return;
            const uint32_t bin = (key >> shift) & mask;
            atomicAdd(&s.bins[bin], 1u);
            if (by_mass)
              atomicAdd(reinterpret_cast<unsigned long long*>(&s.bin_mass[bin]),
                        static_cast<unsigned long long>(whole(row.w(z), row.scale)));
          },
          [](int) {});
      __syncthreads();
      // bins from the highest down, two a thread
      const int hi = kBins - 1 - 2 * t;
      const uint64_t c0 = s.bins[hi], c1 = s.bins[hi - 1], m0 = s.bin_mass[hi],
                     m1 = s.bin_mass[hi - 1];
      uint64_t all;
      const uint64_t n0 = n_before + block_scan<kWaves>(c0 + c1, s.slots64, all);
      const uint64_t p0 = m_before + block_scan<kWaves>(m0 + m1, s.slots64, all);
      auto take = [&](int bin, uint64_t c, uint64_t m, uint64_t n, uint64_t p) {
        const uint64_t from = by_mass ? p : n, to = by_mass ? p + m : n + c;
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
      // (fewer ids, or less weight, than the target)
      if (uniform(s.found_count) == 0) return kKeepAll;
      const uint32_t bin = uniform(s.found);
      prefix = level == 0 ? bin : (prefix << (level == 1 ? 11 : 10)) | bin;
      n_before = uniform(s.found_before);
      m_before = uniform(s.found_mass_before);
    }
    // every id of the last bin has the same key and weight
    const uint64_t equal = uniform(s.found_count);
    const uint64_t each = uniform(s.found_mass) / equal;  // (if by_mass)
    const uint64_t keep = by_mass ? (target - m_before + each - 1) / each : target - n_before;
    Cut cut{prefix, INT32_MAX};
    if (keep < equal) {
      auto ties = [&](float z, int id) -> uint64_t {
        return id < row.vocab && order_key(z) == cut.key ? 1 : 0;
      };
      segment_sums(cut.key, ties);
      cut.last = find(keep - 1, ties);
    }
    return cut;
  }
};

template <class T>
__global__ __launch_bounds__(kThreads) void sample_search_kernel(SampleArgs a, Workspace ws) {
  __shared__ Shared s;
  const int t = threadIdx.x, r = blockIdx.x;
  Row<T> row;
  // (read before it is known whether the row is left over: no waiting for one load after another)
  const SearchState& state = ws.states[r];
  const Border border = state.border;
  const uint64_t first_list = state.list[0][t];
  const uint64_t kept_sum =
      t < ws.segments ? ws.kept[static_cast<size_t>(r) * ws.segments + t] : uint64_t{0};
  if (!row.reopen(a, ws, r, s.pow64)) return;
  if (t < 64) s.pow64[t] = kPow64[t];
  __syncthreads();
  const Settings& st = row.st;
  const Searcher<T> p{row, s};
  Cut cut = kKeepAll;
  if (!in_parts(row) ||
      !p.cut_from_lists(border, first_list, state.list[1], kept_sum, cut)) {
    if (st.few(row.vocab)) {  // (for which the first launch forms no sums)
      double x = 0.0;
      visit<kWaves>(
          row, 0, row.segments, [&](int g) { return uniform(row.stats[g].top) > -INFINITY; },
          [&](float z, int) { x += row.w.normal(z); }, [](int) {});
      row.set_scale(block_reduce<kWaves>(x, s.slots_d, Add{}));
    }
    uint64_t sum = row.whole_sum;
    cut = kKeepAll;
    for (int kind = 0; kind < 2; ++kind) {  // top-k, then top-p of what it keeps
      if (kind == 0 ? st.top_k == 0 : st.top_p >= 1.f) continue;
      if (kind == 1 && st.top_k > 0) {
        p.sum_kept(cut, 0, 0.f);
        sum = p.sum_of_segments();
      }
      const Cut c = p.search_bits(kind == 1, kind == 1 ? share_of(sum, st.top_p) : st.top_k);
      if (c.tighter(cut)) cut = c;
    }
    p.sum_kept(cut, st.min_p > 0.f ? order_key(min_p_logit(row)) : 0, st.min_p);
  }
  __syncthreads();
  const uint64_t total = p.sum_of_segments();
  const int token = p.find(part_of(total, random_number(a, r)), [&](float z, int id) -> uint64_t {
    if (!cut.keeps(order_key(z), id)) return 0;
    const double x = row.w(z);
    return x >= st.min_p ? whole(x, row.scale) : 0;
  });
  const float soft = row.model_sum(a);
  if (t == 0) row.write(a, token, static_cast<double>(total) / row.scale, soft);
}

int segments_of(int vocab) { return (vocab + kSegment - 1) / kSegment; }

// Where a call's intermediate results lie in its workspace.
struct Layout {
  size_t tops, headers, kept, states, bytes;
  Layout(int n_rows, int vocab) {
    const size_t n = n_rows, segments = segments_of(vocab);
    auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    tops = up(n * segments * sizeof(SegmentStats));
    headers = tops + up(n * segments * 64 * sizeof(float));
    kept = headers + up(n * sizeof(RowHeader));
    states = bytes = kept;
    if (vocab > kPickList) {
      states = kept + up(n * segments * sizeof(uint64_t));
      bytes = states + n * sizeof(SearchState);
    }
  }
};

// Workgroups per row of the launches over parts: up to 8192 in all, as the rows left over are of
// unlike cost (2048: 300 -> 244 us for 944 rows, mixed settings), at most 32 of a row (a wave has a
// segment of its own then, up to 2^18 ids).
int parts_of(int n_rows, int vocab) {
  return max(1, min(min(8192 / n_rows, 32), (segments_of(vocab) + kPartWaves - 1) / kPartWaves));
}

template <class T>
hipError_t launch(const SampleArgs& a, void* ws, hipStream_t s) {
  const int segments = segments_of(a.vocab);
  const Layout at(a.n_rows, a.vocab);
  char* const base = static_cast<char*>(ws);
  const Workspace w{reinterpret_cast<SegmentStats*>(base),
                    reinterpret_cast<float*>(base + at.tops),
                    reinterpret_cast<RowHeader*>(base + at.headers),
                    reinterpret_cast<uint64_t*>(base + at.kept),
                    reinterpret_cast<SearchState*>(base + at.states),
                    segments,
                    parts_of(a.n_rows, a.vocab)};
  const int groups = (segments + kScanWaves - 1) / kScanWaves;
  hipLaunchKernelGGL(sample_scan_kernel<T>, dim3(a.n_rows * groups), dim3(kScanThreads), 0, s, a,
                     w);
  const bool limits = a.top_k || a.top_p || a.min_p;
  const auto pick = limits ? sample_pick_kernel<T, true> : sample_pick_kernel<T, false>;
  hipLaunchKernelGGL(pick, dim3(a.n_rows), dim3(kPickThreads), 0, s, a, w);
  // rows are left only where something limits them and the list does not hold them whole
  if (limits && a.vocab > kPickList) {
    if (a.top_k || a.top_p)
      hipLaunchKernelGGL(sample_bins_kernel<T>, dim3(a.n_rows * bin_parts(w.parts)),
                         dim3(kBinThreads), 0, s, a, w);
    hipLaunchKernelGGL(sample_sums_kernel<T>, dim3(a.n_rows * w.parts), dim3(kPartThreads), 0, s, a,
                       w);
    hipLaunchKernelGGL(sample_search_kernel<T>, dim3(a.n_rows), dim3(kThreads), 0, s, a, w);
  }
  return hipGetLastError();
}

}  // namespace

size_t sample_ws_bytes(int n_rows, int vocab) { return Layout(n_rows, vocab).bytes; }

long sample_threads(int n_rows, int vocab) {
  const long groups = (segments_of(vocab) + kScanWaves - 1) / kScanWaves;
  return max(groups * kScanThreads, static_cast<long>(kThreads)) * n_rows;
}

hipError_t sample(bool bf16, const SampleArgs& a, void* ws, hipStream_t s) {
  if (a.n_rows == 0) return hipSuccess;
  return bf16 ? launch<uint16_t>(a, ws, s) : launch<float>(a, ws, s);
}

}  // namespace eb

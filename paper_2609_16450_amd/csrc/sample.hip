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
#include <type_traits>

#include "attn_common.hpp"
#include "eb_common.hpp"
#include "eb_internal.hpp"
#include "paged.hpp"

namespace eb {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kSegment = 2048;  // ids that a wave takes at a time
constexpr int kMaxSegments = kThreads;
static_assert(kMaxSegments * kSegment >= kSampleMaxVocab, "a thread per segment");

typedef uint32_t u32x4h __attribute__((ext_vector_type(4), aligned(2)));  // at any 2 bytes

template <class T>
constexpr int kVec = 16 / sizeof(T);  // ids of a lane and load
template <class T>
constexpr int kLoads = kSegment / (64 * kVec<T>);  // loads of a lane per segment

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

// A whole number that orders as the float does (-0 as +0).
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}

// Weights of a row: in 64 bits, and as whole numbers.  A weight that is not 0 counts at least 1.
struct Weights {
  double top, inv_t;  // largest logit; 1 / temperature
  double scale;       // a power of two: scale times the sum of all weights lies in [2^61, 2^62]
  __device__ __forceinline__ double weight(float z) const {
    return z == -INFINITY ? 0.0 : exp((static_cast<double>(z) - top) * inv_t);
  }
  __device__ __forceinline__ uint64_t whole(double w) const {
    return w > 0.0 ? max(static_cast<uint64_t>(rint(w * scale)), uint64_t{1}) : 0;
  }
};

// Kept: above key, or equal to it with an id of at most last.
struct Cut {
  uint32_t key;
  int32_t last;
  __device__ __forceinline__ bool keeps(uint32_t k, int id) const {
    return k > key || (k == key && id <= last);
  }
};

template <class V, class Op>
__device__ __forceinline__ V wave_reduce(V x, Op op) {
  for (int mask = 32; mask >= 1; mask >>= 1) x = op(x, __shfl_xor(x, mask));
  return x;
}

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

constexpr int kBins = 2048;  // of one round of the search for a cut

struct Shared {
  uint32_t count[kBins];
  uint64_t mass[kBins];
  uint64_t segment[kMaxSegments];
  uint64_t slots64[kWaves];
  double slots_d[kWaves];
  float slots_f[kWaves];
  uint32_t slots32[kWaves];
  uint32_t found_bin, found_count, found_before;
  uint64_t found_mass, found_mass_before;
  int32_t found_id;
};

// The row of one workgroup: wave w takes segments w, w + kWaves, ...
template <class T>
struct Row {
  const T* logits;
  int vocab;
  // f(z, id) for every id of segment g that lane `lane` holds (ids behind the end as -inf)
  template <class F>
  __device__ __forceinline__ void segment(int g, int lane, F f) const {
#pragma unroll
    for (int i = 0; i < kLoads<T>; ++i) {
      const int at = g * kSegment + (i * 64 + lane) * kVec<T>;
      float z[kVec<T>];
      load_logits(logits, at, vocab, z);
#pragma unroll
      for (int e = 0; e < kVec<T>; ++e) f(z[e], at + e);
    }
  }
  template <class F>
  __device__ __forceinline__ void all(F f) const {
    const int n = (vocab + kSegment - 1) / kSegment;
    for (int g = threadIdx.x >> 6; g < n; g += kWaves) segment(g, threadIdx.x & 63, f);
  }
  // f() summed over each segment's ids, into s.segment; then the segment and what lies before it
  // whose running sum first exceeds x, on every thread.
  template <class F>
  __device__ __forceinline__ uint64_t segment_sums(Shared& s, F f) const {
    const int n = (vocab + kSegment - 1) / kSegment;
    for (int g = threadIdx.x >> 6; g < n; g += kWaves) {
      uint64_t sum = 0;
      segment(g, threadIdx.x & 63, [&](float z, int id) { sum += f(z, id); });
      sum = wave_reduce(sum, [](uint64_t a, uint64_t b) { return a + b; });
      if ((threadIdx.x & 63) == 0) s.segment[g] = sum;
    }
    __syncthreads();
    uint64_t total;
    const uint64_t own = static_cast<int>(threadIdx.x) < n ? s.segment[threadIdx.x] : 0;
    const uint64_t before = block_scan(own, s.slots64, total);
    __syncthreads();
    s.segment[threadIdx.x] = before;
    __syncthreads();
    return total;
  }
  // Lowest id whose running sum of f() exceeds x < total, after segment_sums of the same f.
  template <class F>
  __device__ __forceinline__ int find(Shared& s, uint64_t x, F f) const {
    const int n = (vocab + kSegment - 1) / kSegment, t = threadIdx.x;
    if (t < n && s.segment[t] <= x && (t + 1 == n || s.segment[t + 1] > x))
      s.found_bin = static_cast<uint32_t>(t);
    __syncthreads();
    const int g = min(static_cast<int>(s.found_bin), n - 1);
    if (t < 64) {
      if (t == 0) s.found_id = g * kSegment;
      uint64_t before = s.segment[g];
      bool found = false;
      for (int i = 0; i < kLoads<T> && !found; ++i) {
        const int at = g * kSegment + (i * 64 + t) * kVec<T>;
        float z[kVec<T>];
        load_logits(logits, at, vocab, z);
        uint64_t sum = 0;
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) sum += f(z[e], at + e);
        uint64_t upto = sum;
        for (int k = 1; k < 64; k <<= 1) {
          const uint64_t o = __shfl_up(upto, k);
          if (t >= k) upto += o;
        }
        const uint64_t hit = __ballot(before + upto > x);
        if (hit) {
          if (t == __ffsll(static_cast<unsigned long long>(hit)) - 1) {
            uint64_t run = before + upto - sum;
            int id = at;
#pragma unroll
            for (int e = 0; e < kVec<T>; ++e) {
              run += f(z[e], at + e);
              if (run <= x) id = at + e + 1;
            }
            s.found_id = id;
          }
          found = true;
        }
        before += __shfl(upto, 63);
      }
    }
    __syncthreads();
    return s.found_id;
  }
};

// The cut behind the first `target` ids of the order (kMass false) or behind the fewest whose
// weights come to at least `target` (kMass true; 1 <= target <= their sum).  `mass`: the weight of
// all that it keeps.  Three rounds over the row fix 11, 11 and 10 bits of the key.
template <bool kMass, class T>
__device__ __forceinline__ Cut find_cut(const Row<T>& row, const Weights& w, Shared& s,
                                        uint64_t target, uint64_t& mass) {
  const int t = threadIdx.x;
  uint32_t prefix = 0;
  uint64_t n_before = 0, m_before = 0;
  constexpr int kShift[3] = {21, 10, 0};
  for (int level = 0; level < 3; ++level) {
    const int shift = kShift[level];
    const uint32_t mask = level == 2 ? 1023u : 2047u;
    for (int i = t; i < kBins; i += kThreads) {
      s.count[i] = 0;
      s.mass[i] = 0;
    }
    __syncthreads();
    row.all([&](float z, int id) {
      const uint32_t key = order_key(z);
      if (id >= row.vocab) return;
      if (level > 0 && (key >> (level == 1 ? 21 : 10)) != prefix) return;
      const uint32_t bin = (key >> shift) & mask;
      atomicAdd(&s.count[bin], 1u);
      atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[bin]),
                static_cast<unsigned long long>(w.whole(w.weight(z))));
    });
    __syncthreads();
    // bins from the highest down, two a thread
    const int hi = kBins - 1 - 2 * t;
    const uint32_t c0 = s.count[hi], c1 = s.count[hi - 1];
    const uint64_t m0 = s.mass[hi], m1 = s.mass[hi - 1];
    uint64_t all;
    const uint64_t n0 = n_before + block_scan(static_cast<uint64_t>(c0) + c1, s.slots64, all);
    const uint64_t p0 = m_before + block_scan(m0 + m1, s.slots64, all);
    auto take = [&](int bin, uint32_t c, uint64_t m, uint64_t n, uint64_t p) {
      const uint64_t from = kMass ? p : n, to = kMass ? p + m : n + c;
      if (from < target && target <= to) {
        s.found_bin = static_cast<uint32_t>(bin);
        s.found_count = c;
        s.found_before = static_cast<uint32_t>(n);
        s.found_mass = m;
        s.found_mass_before = p;
      }
    };
    take(hi, c0, m0, n0, p0);
    take(hi - 1, c1, m1, n0 + c0, p0 + m0);
    __syncthreads();
    prefix = level == 0 ? s.found_bin : (prefix << (level == 1 ? 11 : 10)) | s.found_bin;
    n_before = s.found_before;
    m_before = s.found_mass_before;
    __syncthreads();
  }
  // every id of the last bin has the same key and weight
  const uint64_t equal = s.found_count, each = s.found_mass / equal;
  const uint64_t keep = kMass ? (target - m_before + each - 1) / each : target - n_before;
  mass = m_before + keep * each;
  Cut cut{prefix, INT32_MAX};
  if (keep < equal) {
    auto ties = [&](float z, int id) -> uint64_t {
      return id < row.vocab && order_key(z) == cut.key ? 1 : 0;
    };
    row.segment_sums(s, ties);
    cut.last = row.find(s, keep - 1, ties);
  }
  return cut;
}

// floor(sum * x) for x in [0, 1) (bits of x below 2^-64 are left out).
__device__ __forceinline__ uint64_t part_of(uint64_t sum, float x) {
  return __umul64hi(sum, static_cast<uint64_t>(static_cast<double>(x) * 0x1p64));
}

template <class T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared s;
  const int t = threadIdx.x, r = blockIdx.x;
  const int b = find_sequence(a.cu_block, a.batch, r, t & 63);
  const Row<T> row{static_cast<const T*>(a.logits) + static_cast<size_t>(r) * a.pitch, a.vocab};
  const float temperature = a.temperature ? a.temperature[b] : 1.f;
  const int32_t top_k = a.top_k ? a.top_k[b] : 0;
  const float top_p = a.top_p ? a.top_p[b] : 1.f;
  const double min_p = a.min_p ? fmin(static_cast<double>(a.min_p[b]), 1.0) : 0.0;
  const bool greedy = !(temperature > 0.f);
  auto add = [](auto x, auto y) { return x + y; };

  float m = -INFINITY;
  bool bad = false;
  row.all([&](float z, int) {
    m = fmaxf(m, z);
    bad |= !(z < INFINITY);
  });
  m = block_reduce(m, s.slots_f, [](float x, float y) { return fmaxf(x, y); });
  bad = block_reduce(static_cast<uint32_t>(bad), s.slots32, add) != 0;
  if (bad || m == -INFINITY) {  // a NaN or +inf; or nothing to draw from
    if (t == 0) {
      a.token[r] = -1;
      const float none = bad ? NAN : 0.f;
      if (a.prob) a.prob[r] = none;
      if (a.conf) a.conf[r] = none;
    }
    return;
  }

  Weights w{static_cast<double>(m), greedy ? 1.0 : 1.0 / static_cast<double>(temperature), 1.0};
  double sum = 0.0;
  float soft = 0.f;
  row.all([&](float z, int) {
    if (!greedy) sum += w.weight(z);
    if (a.conf) soft += fast_exp2((z - m) * kLog2e);
  });
  soft = block_reduce(soft, s.slots_f, add);
  int token;
  double total = 1.0;  // sum of the kept weights
  if (greedy) {
    const uint32_t key = order_key(m);
    auto equal = [&](float z, int id) -> uint64_t {
      return id < a.vocab && order_key(z) == key ? 1 : 0;
    };
    row.segment_sums(s, equal);
    token = row.find(s, 0, equal);
  } else {
    sum = block_reduce(sum, s.slots_d, add);
    w.scale = ldexp(1.0, 61 - ilogb(sum));
    Cut cut{0, INT32_MAX};
    uint64_t mass = 0;
    if (top_k > 0 && top_k < a.vocab)
      cut = find_cut<false>(row, w, s, static_cast<uint64_t>(top_k), mass);
    if (top_p < 1.f) {
      if (mass == 0) {
        uint64_t x = 0;
        row.all([&](float z, int) { x += w.whole(w.weight(z)); });
        mass = block_reduce(x, s.slots64, add);
      }
      const double p = fmax(static_cast<double>(top_p), 0.0) * 0x1p64;
      const uint64_t q = static_cast<uint64_t>(p);
      const uint64_t target = __umul64hi(mass, q) + (mass * q != 0);  // rounded up
      const Cut c = find_cut<true>(row, w, s, max(target, uint64_t{1}), mass);
      if (c.key > cut.key || (c.key == cut.key && c.last < cut.last)) cut = c;
    }
    auto kept = [&](float z, int id) -> uint64_t {
      const double x = w.weight(z);
      return cut.keeps(order_key(z), id) && x >= min_p ? w.whole(x) : 0;
    };
    mass = row.segment_sums(s, kept);
    const float u = fminf(fmaxf(a.uniform[r], 0.f), 0x1.fffffep-1f);
    token = row.find(s, part_of(mass, u), kept);
    total = static_cast<double>(mass) / w.scale;
  }
  if (t == 0) {
    float z;
    if constexpr (sizeof(T) == 4)
      z = row.logits[token];
    else
      z = bf16_bits_to_f32(row.logits[token]);
    a.token[r] = token;
    if (a.prob) a.prob[r] = greedy ? 1.f : static_cast<float>(w.weight(z) / total);
    if (a.conf) a.conf[r] = static_cast<float>(exp(static_cast<double>(z) - m) / soft);
  }
}

}  // namespace

size_t sample_ws_bytes(bool, int, int) { return 0; }

hipError_t sample(bool bf16, const SampleArgs& a, void*, hipStream_t s) {
  if (a.n_rows == 0) return hipSuccess;
  if (bf16)
    hipLaunchKernelGGL(sample_kernel<uint16_t>, dim3(a.n_rows), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(sample_kernel<float>, dim3(a.n_rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace eb

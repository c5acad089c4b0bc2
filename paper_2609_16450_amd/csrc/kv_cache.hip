// Rows into and out of the paged key/value cache.
//
// Both directions move every byte once and compute next to nothing, so they are bound by memory for
// many rows and by latency for few.  A row (token, K/V head) of D values is moved by D / 8 lanes of
// 8 values each; a wavefront takes consecutive tokens of one head, which lie one behind the other
// in a page (a line of an 8-bit cache with 64-wide heads holds two of them), while the packed side
// sees whole rows of 128 bytes or more.  Workgroups run over the heads first: the packed rows of a
// few tokens are then taken as one piece of memory (heads last: 5-13% slower).
// Quantising is a maximum over bf16 pairs and lane exchanges, and one instruction per two values,
// exact because the scale is a power of two; rows with a NaN or an infinity take the long way.
// Measured, bytes read and written together: prompts of 501 to 2048 rows x 32 heads x 128 into 8
// bits and back 95 us (5.0 TB/s, as a large copy; 99 us with the values unpacked one by one), the
// same into bf16 pages 53 us (5.0 TB/s), 64 prefixes of 1001 to 4096 rows x 4 heads out of 8 bits
// 105 us (4.6 TB/s).  Without gain: two, four or eight rows per lane, an eighth of the rows to each
// XCD.
#include <type_traits>

#include "eb_internal.hpp"
#include "paged.hpp"

namespace eb {
namespace {

constexpr int kThreads = 256;  // 4 waves
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(4)));  // at any word

// Eight values of a row, as they came.
template <class T>
struct Row8;
template <>
struct Row8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const f32x4u*>(p);
    b = *reinterpret_cast<const f32x4u*>(p + 4);
  }
  __device__ __forceinline__ void store(float* p) const {
    *reinterpret_cast<f32x4*>(p) = a;
    *reinterpret_cast<f32x4*>(p + 4) = b;
  }
  __device__ __forceinline__ float value(int i) const { return i < 4 ? a[i] : b[i - 4]; }
  // largest magnitude, as bits
  __device__ __forceinline__ uint32_t magnitude() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(value(i)) & 0x7fffffffu);
    return m;
  }
  // E4M3 bytes of the values over `scale` = 2^e, all finite and at most 448 2^e
  __device__ __forceinline__ u32x2 e4m3(float scale) const {
    return u32x2{f32x4_to_e4m3(a, scale), f32x4_to_e4m3(b, scale)};
  }
};
template <>
struct Row8<uint16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const u32x4*>(p); }
  __device__ __forceinline__ void store(uint16_t* p) const { *reinterpret_cast<u32x4*>(p) = w; }
  __device__ __forceinline__ float value(int i) const {
    return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  __device__ __forceinline__ uint32_t magnitude() const {  // of bf16 pairs, two at a time
    u16x2 m = pair(0);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, pair(i));
    return static_cast<uint32_t>(max(m[0], m[1])) << 16;
  }
  __device__ __forceinline__ u32x2 e4m3(float scale) const {
    return u32x2{bf16x4_to_e4m3(w[0], w[1], scale), bf16x4_to_e4m3(w[2], w[3], scale)};
  }

 private:
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  __device__ __forceinline__ u16x2 pair(int i) const {
    const uint32_t x = w[i] & 0x7fff7fffu;
    return __builtin_bit_cast(u16x2, x);
  }
};

// Largest x of each group of kLanes lanes (8 or 16), on every lane of the group.
template <int kLanes>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  auto with = [&](auto ctrl) {
    constexpr int kCtrl = decltype(ctrl)::value;
    x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(
                   0, static_cast<int>(x), kCtrl, 0xf, 0xf, true)));
  };
  with(std::integral_constant<int, 0xb1>{});   // lane ^ 1
  with(std::integral_constant<int, 0x4e>{});   // lane ^ 2
  with(std::integral_constant<int, 0x141>{});  // lane ^ 7
  if (kLanes == 16) with(std::integral_constant<int, 0x140>{});  // lane ^ 15
  return x;
}

// Where a packed row goes to or comes from: the row's number in the pool, (page hkv + head)
// page_size + slot, or -1 for a row that is left out.
__device__ __forceinline__ long pool_row(const PagedKv& kv, int b, int pos, int head) {
  const int page_at = pos >> kv.page_shift;
  if (pos < 0 || page_at >= kv.max_pages) return -1;
  const int page = kv.table[static_cast<size_t>(b) * kv.max_pages + page_at];
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(kv.n_pages)) return -1;
  const long row = static_cast<long>(page) * kv.hkv + head;
  return (row << kv.page_shift) + (pos & ((1 << kv.page_shift) - 1));
}

// Sequence of each lane's token, given the wave's first one: lanes step forward from its sequence.
__device__ __forceinline__ int lane_sequence(const int32_t* cu, int batch, int b, int token) {
  while (b + 1 < batch && cu[b + 1] <= token) ++b;
  return b;
}

// One (token, head) row per D / 8 lanes.  T: the rows' type; kE4m3: the cache holds 8 bits.
template <int D, class T, bool kE4m3>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(PagedKv kv, const int32_t* cu_block,
                                                            const int32_t* cu_prefix,
                                                            const int32_t* pos, int batch,
                                                            int total, const T* __restrict__ k,
                                                            const T* __restrict__ v) {
  constexpr int kLanes = D / 8;         // lanes per row
  constexpr int kTokens = 64 / kLanes;  // tokens per wave
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int head = blockIdx.x % kv.hkv, col = (lane % kLanes) * 8;
  const int first = (blockIdx.x / kv.hkv * (kThreads / 64) + wave) * kTokens;
  if (first >= total) return;  // uniform per wavefront
  const int token = min(first + lane / kLanes, total - 1);
  const size_t src = (static_cast<size_t>(token) * kv.hkv + head) * D + col;
  Row8<T> x[2];
  x[0].load(k + src);
  x[1].load(v + src);
  int at = pos ? pos[token] : 0;
  const int b = lane_sequence(cu_block, batch, find_sequence(cu_block, batch, first, lane), token);
  if (!pos) at = cu_prefix[b + 1] - cu_prefix[b] + token - cu_block[b];
  const long row = first + lane / kLanes < total ? pool_row(kv, b, at, head) : -1;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint8_t* const pool = i ? kv.v : kv.k;
    if constexpr (kE4m3) {
      uint32_t amax = group_max<kLanes>(x[i].magnitude());
      int e = e4m3_exponent(amax);
      u32x2 w = x[i].e4m3(e8m0(e + 127));
      if (__any(amax >= 0x7f800000u)) {  // a NaN or an infinity somewhere: its row's others count
        amax = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) amax = max(amax, finite_mag(x[i].value(j)));
        e = e4m3_exponent(group_max<kLanes>(amax));
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[i].value(j);
        w = u32x2{pack4_e4m3(y, e8m0(127 - e)), pack4_e4m3(y + 4, e8m0(127 - e))};
      }
      if (row >= 0) {
        *reinterpret_cast<u32x2*>(pool + row * D + col) = w;
        if (col == 0) (i ? kv.v_scale : kv.k_scale)[row] = static_cast<uint8_t>(e + 127);
      }
    } else if (row >= 0) {
      x[i].store(reinterpret_cast<T*>(pool) + row * D + col);
    }
  }
}

// The same rows the other way.  T: the type of the packed rows; kE4m3: the cache holds 8 bits.
template <int D, class T, bool kE4m3>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(PagedKv kv, const int32_t* cu_prefix,
                                                           int batch, int total,
                                                           T* __restrict__ k, T* __restrict__ v) {
  constexpr int kLanes = D / 8;
  constexpr int kTokens = 64 / kLanes;
  constexpr int kWords = kE4m3 ? 1 : sizeof(T) / 2;  // loads per 8 values, 16 bytes (8 bits: 8)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int head = blockIdx.x % kv.hkv, col = (lane % kLanes) * 8;
  const int first = (blockIdx.x / kv.hkv * (kThreads / 64) + wave) * kTokens;
  if (first >= total) return;  // uniform per wavefront
  const int token = min(first + lane / kLanes, total - 1);
  const int b =
      lane_sequence(cu_prefix, batch, find_sequence(cu_prefix, batch, first, lane), token);
  const long row = pool_row(kv, b, token - cu_prefix[b], head);
  const size_t from = row < 0 ? 0 : row;  // rows without a page: loaded from the first, then zeros
  u32x4 w[2][kWords];
  uint32_t scale[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint8_t* const pool = i ? kv.v : kv.k;
    if constexpr (kE4m3) {
      const u32x2 y = *reinterpret_cast<const u32x2*>(pool + from * D + col);
      w[i][0] = u32x4{y[0], y[1], 0, 0};
      scale[i] = (i ? kv.v_scale : kv.k_scale)[from];
    } else {
#pragma unroll
      for (int e = 0; e < kWords; ++e)
        w[i][e] = *reinterpret_cast<const u32x4*>(pool + (from * D + col) * sizeof(T) + 16 * e);
    }
  }
  if (first + lane / kLanes >= total) return;
  const size_t dst = (static_cast<size_t>(token) * kv.hkv + head) * D + col;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    T* const out = (i ? v : k) + dst;
    if (row < 0) {
      scale[i] = 127;  // (what was loaded may stand for infinity, and zero times that is NaN)
#pragma unroll
      for (int e = 0; e < kWords; ++e) w[i][e] = u32x4{};
    }
    if constexpr (!kE4m3) {
#pragma unroll
      for (int e = 0; e < kWords; ++e)  // (fp32 rows may start at any float)
        *reinterpret_cast<u32x4u*>(reinterpret_cast<uint8_t*>(out) + 16 * e) = w[i][e];
    } else if constexpr (sizeof(T) == 2) {
      u32x4 lo, hi;
      e4m3_widen(w[i][0], e8m0(scale[i]), lo, hi);
      *reinterpret_cast<u32x4*>(out) = lo;
    } else {
      const float f = e8m0(scale[i]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const f32x2 a = e4m3_pair_f32<false>(w[i][0][e], f), c = e4m3_pair_f32<true>(w[i][0][e], f);
        *reinterpret_cast<f32x4u*>(out + 4 * e) = f32x4u{a[0], a[1], c[0], c[1]};
      }
    }
  }
}

// Calls go.run<head dimension, row type, 8-bit cache>().
template <class Go>
hipError_t by_type(const PagedKv& kv, bool bf16, const Go& go) {
  const bool e4m3 = kv.type == CacheType::kE4m3;
  if (kv.head_dim == 128) {
    if (bf16)
      e4m3 ? go.template run<128, uint16_t, true>() : go.template run<128, uint16_t, false>();
    else
      e4m3 ? go.template run<128, float, true>() : go.template run<128, float, false>();
  } else {
    if (bf16)
      e4m3 ? go.template run<64, uint16_t, true>() : go.template run<64, uint16_t, false>();
    else
      e4m3 ? go.template run<64, float, true>() : go.template run<64, float, false>();
  }
  return hipGetLastError();
}

dim3 grid_of(const PagedKv& kv, int rows) {
  const long per = kThreads / (kv.head_dim / 8);
  return dim3(static_cast<unsigned>((rows + per - 1) / per * kv.hkv));
}

struct WriteLaunch {
  const PagedKv& kv;
  const int32_t *cu_block, *cu_prefix, *pos;
  int batch, total;
  const void *k, *v;
  hipStream_t s;
  template <int D, class T, bool kE4m3>
  void run() const {
    hipLaunchKernelGGL((kv_write_kernel<D, T, kE4m3>), grid_of(kv, total), dim3(kThreads), 0, s, kv,
                       cu_block, cu_prefix, pos, batch, total, static_cast<const T*>(k),
                       static_cast<const T*>(v));
  }
};

struct ReadLaunch {
  const PagedKv& kv;
  const int32_t* cu_prefix;
  int batch, total;
  void *k, *v;
  hipStream_t s;
  template <int D, class T, bool kE4m3>
  void run() const {
    hipLaunchKernelGGL((kv_read_kernel<D, T, kE4m3>), grid_of(kv, total), dim3(kThreads), 0, s, kv,
                       cu_prefix, batch, total, static_cast<T*>(k), static_cast<T*>(v));
  }
};

}  // namespace

hipError_t kv_write(bool bf16, const PagedKv& kv, int batch, int total, const int32_t* cu_block,
                    const int32_t* cu_prefix, const int32_t* pos, const void* k, const void* v,
                    hipStream_t s) {
  if (total == 0) return hipSuccess;
  return by_type(kv, bf16, WriteLaunch{kv, cu_block, cu_prefix, pos, batch, total, k, v, s});
}

hipError_t kv_read(bool bf16, const PagedKv& kv, int batch, int total, const int32_t* cu_prefix,
                   void* k, void* v, hipStream_t s) {
  if (total == 0) return hipSuccess;
  return by_type(kv, bf16, ReadLaunch{kv, cu_prefix, batch, total, k, v, s});
}

}  // namespace eb

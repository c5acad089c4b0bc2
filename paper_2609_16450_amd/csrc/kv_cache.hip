// Rows into and out of the paged key/value cache.
//
// Both directions move every byte once and compute next to nothing, so they are bound by memory for
// many rows and by latency for few.  A row (token, K/V head) of D values is moved by D / 8 lanes of
// 8 values each; a wavefront takes consecutive tokens of one head, which lie one behind the other
// in a page (a line of an 8-bit cache with 64-wide heads holds two of them, and a line of scales
// 128), while the packed side sees whole rows of 128 bytes or more.
#include "eb_internal.hpp"
#include "paged.hpp"

namespace eb {
namespace {

constexpr int kThreads = 256;  // 4 waves

// Eight values of a row, in fp32.
template <class T>
__device__ __forceinline__ void load8(const T* p, float* x);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* x) {
  const f32x4u a = *reinterpret_cast<const f32x4u*>(p), b = *reinterpret_cast<const f32x4u*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
template <>
__device__ __forceinline__ void load8<uint16_t>(const uint16_t* p, float* x) {
  const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(a[i] << 16);
    x[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
  }
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
  constexpr int kLanes = D / 8;           // lanes per row
  constexpr int kTokens = 64 / kLanes;    // tokens per wave
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long first = (static_cast<long>(blockIdx.x) * (kThreads / 64) + wave) * kTokens;
  if (first >= total) return;  // uniform per wavefront
  const int head = blockIdx.y;
  const int token = static_cast<int>(min(first + lane / kLanes, static_cast<long>(total) - 1));
  const bool live = first + lane / kLanes < total;
  const int col = (lane % kLanes) * 8;
  const size_t src = (static_cast<size_t>(token) * kv.hkv + head) * D + col;
  float x[2][8];
  load8(k + src, x[0]);
  load8(v + src, x[1]);
  const int b0 = find_sequence(cu_block, batch, static_cast<int>(first), lane);
  const int b = lane_sequence(cu_block, batch, b0, token);
  const int at = pos ? pos[token] : cu_prefix[b + 1] - cu_prefix[b] + token - cu_block[b];
  const long row = live ? pool_row(kv, b, at, head) : -1;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint8_t* const pool = i ? kv.v : kv.k;
    if constexpr (kE4m3) {
      uint32_t amax = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = max(amax, finite_mag(x[i][e]));
#pragma unroll
      for (int m = 1; m < kLanes; m <<= 1)
        amax = max(amax, static_cast<uint32_t>(__shfl_xor(static_cast<int>(amax), m)));
      const int e = e4m3_exponent(amax);
      const float inv = e8m0(127 - e);
      const u32x2 w{pack4_e4m3(x[i], inv), pack4_e4m3(x[i] + 4, inv)};
      if (row >= 0) {
        *reinterpret_cast<u32x2*>(pool + row * D + col) = w;
        if (col == 0) (i ? kv.v_scale : kv.k_scale)[row] = static_cast<uint8_t>(e + 127);
      }
    } else if (row >= 0) {
      T* dst = reinterpret_cast<T*>(pool) + row * D + col;
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4*>(dst) = f32x4{x[i][0], x[i][1], x[i][2], x[i][3]};
        *reinterpret_cast<f32x4*>(dst + 4) = f32x4{x[i][4], x[i][5], x[i][6], x[i][7]};
      } else {
        // the bf16 bits as they came
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = (__float_as_uint(x[i][2 * e]) >> 16) | __float_as_uint(x[i][2 * e + 1]);
        *reinterpret_cast<u32x4*>(dst) = w;
      }
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
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long first = (static_cast<long>(blockIdx.x) * (kThreads / 64) + wave) * kTokens;
  if (first >= total) return;  // uniform per wavefront
  const int head = blockIdx.y;
  if (first + lane / kLanes >= total) return;
  const int token = static_cast<int>(first) + lane / kLanes;
  const int col = (lane % kLanes) * 8;
  const size_t dst = (static_cast<size_t>(token) * kv.hkv + head) * D + col;
  const int b0 = find_sequence(cu_prefix, batch, static_cast<int>(first), lane);
  const int b = lane_sequence(cu_prefix, batch, b0, token);
  const long row = pool_row(kv, b, token - cu_prefix[b], head);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint8_t* const pool = i ? kv.v : kv.k;
    T* const out = (i ? v : k) + dst;
    if constexpr (kE4m3) {
      u32x2 w{};
      float scale = 0.f;
      if (row >= 0) {
        w = *reinterpret_cast<const u32x2*>(pool + row * D + col);
        scale = e8m0((i ? kv.v_scale : kv.k_scale)[row]);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if constexpr (sizeof(T) == 4) {
          const f32x2 lo = e4m3_pair_f32<false>(w[j], scale), hi = e4m3_pair_f32<true>(w[j], scale);
          *reinterpret_cast<f32x4u*>(out + 4 * j) = f32x4u{lo[0], lo[1], hi[0], hi[1]};
        } else {
          *reinterpret_cast<u32x2*>(out + 4 * j) =
              u32x2{e4m3_pair_bf16<false>(w[j], scale), e4m3_pair_bf16<true>(w[j], scale)};
        }
      }
    } else {
      constexpr int kWords = sizeof(T) / 2;  // 16-byte words of 8 values
#pragma unroll
      for (int j = 0; j < kWords; ++j) {
        u32x4 w{};
        if (row >= 0)
          w = *reinterpret_cast<const u32x4*>(pool + (row * D + col) * sizeof(T) + 16 * j);
        typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(4)));
        *reinterpret_cast<u32x4u*>(reinterpret_cast<uint8_t*>(out) + 16 * j) = w;
      }
    }
  }
}

template <class Go>
hipError_t by_type(const PagedKv& kv, bool bf16, Go go) {
  const bool e4m3 = kv.type == CacheType::kE4m3;
  if (kv.head_dim == 128) {
    if (bf16) e4m3 ? go.template run<128, uint16_t, true>() : go.template run<128, uint16_t, false>();
    else e4m3 ? go.template run<128, float, true>() : go.template run<128, float, false>();
  } else {
    if (bf16) e4m3 ? go.template run<64, uint16_t, true>() : go.template run<64, uint16_t, false>();
    else e4m3 ? go.template run<64, float, true>() : go.template run<64, float, false>();
  }
  return hipGetLastError();
}

dim3 grid_of(const PagedKv& kv, int rows) {
  const int per = kThreads / (kv.head_dim / 8);
  return dim3(static_cast<unsigned>((rows + static_cast<long>(per) - 1) / per),
              static_cast<unsigned>(kv.hkv));
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

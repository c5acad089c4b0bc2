// Reductions and running sums over a wavefront, for values of one word or more.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace eb {

// x, which is the same on every lane, as a scalar: what depends on it alone takes no vector
// registers, and branches on it no lane masks.
template <class V>
__device__ __forceinline__ V uniform(V x) {
  static_assert(sizeof(V) == 4 || sizeof(V) == 8, "one or two words");
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(
        V, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int32_t, x)));
  } else {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b));
    const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b >> 32));
    return __builtin_bit_cast(V, static_cast<uint64_t>(hi) << 32 | lo);
  }
}

// x of lane l, which is the same on every lane, as a scalar.
template <class V>
__device__ __forceinline__ V of_lane(V x, int l) {
  static_assert(sizeof(V) == 4 || sizeof(V) == 8, "one or two words");
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int32_t, x), l));
  } else {
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(b), l);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(b >> 32), l);
    return __builtin_bit_cast(V, static_cast<uint64_t>(hi) << 32 | lo);
  }
}

// x of another lane by DPP, word by word; `old` where no lane is there or the row is masked out.
template <int kCtrl, int kRows = 0xf, class V>
__device__ __forceinline__ V dpp(V old, V x) {
  constexpr int kWords = sizeof(V) / 4;
  struct Words {
    int32_t w[kWords];
  };
  const Words o = __builtin_bit_cast(Words, old), a = __builtin_bit_cast(Words, x);
  Words r;
#pragma unroll
  for (int i = 0; i < kWords; ++i)
    r.w[i] = __builtin_amdgcn_update_dpp(o.w[i], a.w[i], kCtrl, kRows, 0xf, false);
  return __builtin_bit_cast(V, r);
}

// x over the wave, on every lane.  Within rows of 16 lanes by DPP (a third of the time that
// exchanges through LDS take), then by the swaps of rows and halves; both lanes of a pair combine
// the same two values, so all lanes end with the same bits.
template <class V, class Op>
__device__ __forceinline__ V wave_reduce(V x, Op op) {
  x = op(x, dpp<0xb1>(x, x));   // lane ^ 1
  x = op(x, dpp<0x4e>(x, x));   // lane ^ 2
  x = op(x, dpp<0x141>(x, x));  // lane ^ 7: the other four of eight
  x = op(x, dpp<0x140>(x, x));  // lane ^ 15: the other eight of a row
  constexpr int kWords = sizeof(V) / 4;
  struct Words {
    uint32_t w[kWords];
  };
  auto swapped = [&](auto swap) {
    const Words a = __builtin_bit_cast(Words, x);
    Words lo, hi;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const auto r = swap(a.w[i]);
      lo.w[i] = r[0];
      hi.w[i] = r[1];
    }
    x = op(__builtin_bit_cast(V, lo), __builtin_bit_cast(V, hi));
  };
  swapped([](uint32_t v) { return __builtin_amdgcn_permlane16_swap(v, v, false, false); });
  swapped([](uint32_t v) { return __builtin_amdgcn_permlane32_swap(v, v, false, false); });
  return x;
}
// Sum of x over this lane and the lanes before it: within rows of 16, then with the last lanes of
// the rows before.
template <class V>
__device__ __forceinline__ V wave_scan(V x) {
  x += dpp<0x111>(V{}, x);       // row_shr:1
  x += dpp<0x112>(V{}, x);       // row_shr:2
  x += dpp<0x114>(V{}, x);       // row_shr:4
  x += dpp<0x118>(V{}, x);       // row_shr:8
  x += dpp<0x142, 0xa>(V{}, x);  // row_bcast:15 into rows 1 and 3
  x += dpp<0x143, 0xc>(V{}, x);  // row_bcast:31 into rows 2 and 3
  return x;
}

}  // namespace eb

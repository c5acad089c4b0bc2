// The 8-bit values of a paged key/value cache, and the search for a packed row's sequence.
#pragma once

#include "eb_common.hpp"

namespace eb {

// 2^(s - 127) of a scale byte, 1 <= s <= 254.
__device__ __forceinline__ float e8m0(uint32_t s) { return __uint_as_float(s << 23); }

// Exponent of a row's scale from the bits of its largest finite magnitude a: the smallest e with
// a <= 448 * 2^e (448 = 1.75 * 2^8 is the largest E4M3 value), kept in [-100, 120].  Within that
// range 2^-e and every value of the row are ordinary fp32 and bf16 numbers.
__device__ __forceinline__ int e4m3_exponent(uint32_t amax_bits) {
  const int e = static_cast<int>(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7fffffu) > 0x600000u);
  return min(max(e, -100), 120);
}

// |x| as bits where x is finite, else 0.
__device__ __forceinline__ uint32_t finite_mag(float x) {
  const uint32_t m = __float_as_uint(x) & 0x7fffffffu;
  return m < 0x7f800000u ? m : 0u;
}

// Four values times `inv` (a power of two, so the product is exact) as E4M3 bytes, rounded to
// nearest even; infinities and NaN become NaN.
__device__ __forceinline__ uint32_t pack4_e4m3(const float* x, float inv) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = __float_as_uint(x[i]);
    y[i] = (b & 0x7fffffffu) < 0x7f800000u ? x[i] * inv : __uint_as_float(0x7fc00000u);
  }
  int w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  return static_cast<uint32_t>(w);
}

// Four values over `scale` (a power of two) as E4M3 bytes, rounded once to nearest even; for finite
// values of at most 448 scale.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t f32x4_to_e4m3(f32x4 x, float scale) {
  s16x2 w{};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[0], x[1], scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[2], x[3], scale, true);
  return __builtin_bit_cast(uint32_t, w);
}
__device__ __forceinline__ uint32_t bf16x4_to_e4m3(uint32_t lo, uint32_t hi, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  s16x2 w{};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, lo), scale, false);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, hi), scale, true);
  return __builtin_bit_cast(uint32_t, w);
}

// Two of four E4M3 bytes (the low two, or with kHigh the high two) times `scale` (a power of two)
// as bf16, exactly; and as fp32.
typedef float f32x2 __attribute__((ext_vector_type(2)));
template <bool kHigh>
__device__ __forceinline__ uint32_t e4m3_pair_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, kHigh));
}
template <bool kHigh>
__device__ __forceinline__ f32x2 e4m3_pair_f32(uint32_t w, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, kHigh);
}

// Sixteen bytes per lane, two, or one, at byte `off` of a buffer; zeros past its end.  In functions
// of their own, like every builtin that the host pass does not know.
__device__ __forceinline__ u32x4 buffer_load16(__amdgpu_buffer_rsrc_t rs, uint32_t off) {
  return __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0);
}
__device__ __forceinline__ uint32_t buffer_load1(__amdgpu_buffer_rsrc_t rs, uint32_t off) {
  return __builtin_amdgcn_raw_buffer_load_b8(rs, off, 0, 0);
}
__device__ __forceinline__ uint32_t buffer_load2(__amdgpu_buffer_rsrc_t rs, uint32_t off) {
  return __builtin_amdgcn_raw_buffer_load_b16(rs, off, 0, 0);
}

// Sixteen E4M3 values times `scale` as sixteen bf16.
__device__ __forceinline__ void e4m3_widen(u32x4 w, float scale, u32x4& lo, u32x4& hi) {
  lo = u32x4{e4m3_pair_bf16<false>(w[0], scale), e4m3_pair_bf16<true>(w[0], scale),
             e4m3_pair_bf16<false>(w[1], scale), e4m3_pair_bf16<true>(w[1], scale)};
  hi = u32x4{e4m3_pair_bf16<false>(w[2], scale), e4m3_pair_bf16<true>(w[2], scale),
             e4m3_pair_bf16<false>(w[3], scale), e4m3_pair_bf16<true>(w[3], scale)};
}

// Reductions over the wavefront by lane shifts within rows of 16 and broadcasts between them, which
// cost an instruction each (a shuffle goes through LDS).  `op` combines a lane's value with that of
// lanes before it; `none` is its neutral value.  lanes_up_to: over the lanes up to this one;
// lanes_all: over all, uniform.
template <class Op>
__device__ __forceinline__ int lanes_up_to(int x, int none, Op op) {
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x111, 0xf, 0xf, false));  // from lane - 1
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x112, 0xf, 0xf, false));  // - 2
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x114, 0xf, 0xf, false));  // - 4
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x118, 0xf, 0xf, false));  // - 8
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x142, 0xa, 0xf, false));  // lanes 15 and 47
  x = op(x, __builtin_amdgcn_update_dpp(none, x, 0x143, 0xc, 0xf, false));  // lane 31
  return x;
}
template <class Op>
__device__ __forceinline__ int lanes_all(int x, int none, Op op) {
  return __builtin_amdgcn_readlane(lanes_up_to(x, none, op), 63);
}
struct AddOp {
  __device__ __forceinline__ int operator()(int a, int b) const { return a + b; }
};
struct MaxOp {
  __device__ __forceinline__ int operator()(int a, int b) const { return max(a, b); }
};
struct MinOp {
  __device__ __forceinline__ int operator()(int a, int b) const { return min(a, b); }
};

// The sequence that owns packed row `row` of a batch with offsets cu: the number of sequences that
// end at or before it, found by the whole wavefront with one load per 64 sequences (`row` is
// uniform).  At most batch - 1.
__device__ __forceinline__ int find_sequence(const int32_t* cu, int batch, int row, int lane) {
  int b = 0;
  for (int b0 = 0; b0 < batch; b0 += 64) {
    const bool before = b0 + lane < batch && cu[b0 + lane + 1] <= row;
    const int n = __popcll(__ballot(before));
    b += n;
    if (n < 64) break;
  }
  return min(b, batch - 1);
}

}  // namespace eb

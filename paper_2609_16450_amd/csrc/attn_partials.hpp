// One output row from the partials (O, running maximum in log2 units, sum of weights) of the parts
// of its keys, by one wavefront.
#pragma once

#include "eb_common.hpp"

namespace eb {
namespace {

// A row of D values held by the first D / 4 lanes, four each, before its division by l.
template <int D>
struct PartialRow {
  f32x4 x;
  float l;
  __device__ __forceinline__ void store(uint16_t* out, int lane) const {
    if (lane >= D / 4) return;
    const float inv = 1.0f / l;
    *reinterpret_cast<u32x2*>(out + 4 * lane) =
        u32x2{pack2_bf16(x[0] * inv, x[1] * inv), pack2_bf16(x[2] * inv, x[3] * inv)};
  }
};

// Rescaling by 2^d with d <= 0.  An infinity or NaN stays one even where 2^d is zero, as it does in
// the kernels' own accumulators, so that no cut of the keys makes its column finite.
__device__ __forceinline__ void rescale(f32x4& x, float& l, float d) {
  const float f = fast_exp2(d);
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= f;
  l *= f;
}

// Partial k of n lies at row at(k) of o [., D], m and l.  64 / (D / 4) of them are taken side by
// side, kBatch per lane in flight, each lane in the order of k with a running maximum; then the
// lanes of a column are merged.  The order is fixed by n alone.
template <int D, int kBatch, class At>
__device__ __forceinline__ PartialRow<D> merge_partials_by(At at, int n, const float* o,
                                                           const float* m, const float* l,
                                                           int lane) {
  constexpr int kCols = D / 4, kSide = 64 / kCols;
  const int c = 4 * (lane % kCols), sub = lane / kCols;
  f32x4 x{};
  float sum = 0.f, M = kNegBig;
  for (int k0 = 0; k0 < n; k0 += kBatch * kSide) {
    f32x4 y[kBatch];
    float mk[kBatch], lk[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const size_t i = at(min(k0 + j * kSide + sub, n - 1));
      y[j] = *reinterpret_cast<const f32x4*>(o + i * D + c);
      mk[j] = m[i];
      lk[j] = l[i];
    }
    float M_new = M;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      // no such partial (what was loaded is another's, and may be infinite)
      if (k0 + j * kSide + sub >= n) mk[j] = -INFINITY, y[j] = f32x4{};
      M_new = fmaxf(M_new, mk[j]);
    }
    rescale(x, sum, M - M_new);
    M = M_new;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const float f = fast_exp2(mk[j] - M);
      sum = fmaf(f, lk[j], sum);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = fmaf(f, y[j][e], x[e]);
    }
  }
  for (int d = kCols; d < 64; d <<= 1) {
    const float M_new = fmaxf(M, __shfl_xor(M, d));
    rescale(x, sum, M - M_new);
    M = M_new;
    sum += __shfl_xor(sum, d);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], d);
  }
  return PartialRow<D>{x, sum};
}

// A batch loads as many rows however few there are: two or four partials in a batch for eight took
// 27 against 11 us (1000 rows x 32 heads x 128 in two ranges).
template <int D, class At>
__device__ __forceinline__ PartialRow<D> merge_partials(At at, int n, const float* o,
                                                        const float* m, const float* l, int lane) {
  constexpr int kSide = 64 / (D / 4);
  if (n <= kSide) return merge_partials_by<D, 1>(at, n, o, m, l, lane);
  if (n <= 4 * kSide) return merge_partials_by<D, 4>(at, n, o, m, l, lane);
  return merge_partials_by<D, 8>(at, n, o, m, l, lane);
}

}  // namespace
}  // namespace eb

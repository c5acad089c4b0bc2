// Block attention over a paged cache for few query rows per K/V head (single tokens, small blocks),
// bf16.  Such calls read every cached key and value for a handful of multiply-adds: they are bound
// by memory, and the kernel is built around its loads.
//
// A workgroup of four waves per (sequence, K/V head, key range, 16 kTiles query rows).  The waves
// split the keys, not the rows: each takes every fourth piece of the range, holds all query rows
// and keeps an online softmax of its own, so that no wave waits for another until the range ends
// and their results are merged through LDS.
//
// A piece is kKeys keys.  K goes from memory straight into the registers of the MFMA's A operand
// (S^T = K Q^T by 16x16x32: lane l holds row l % 16).  V has to be transposed for O^T = V^T P^T: it
// goes through the wave's own part of LDS, row-major, and comes back by transposing reads
// (attn_small.hpp).  As soon as a piece's K is in S and its V in LDS, the loads of the wave's next
// piece go out into the same registers, and stay in flight over the softmax and the second product.
// An 8-bit cache is converted to bf16 on the way, exactly: K rows by the lane that holds them, V
// rows before they go to LDS.
//
// Every 16 keys of a piece lie in one page; a buffer resource per group of 16 ends with the last
// cached row, so rows past it arrive as zeros, and one of no length stands for a missing page.
#pragma once

#include "attn_common.hpp"
#include "attn_small.hpp"
#include "paged.hpp"

namespace eb {
namespace {

constexpr int kFewWaves = 4;
constexpr int kFewBlockKeys = 32;  // keys of a piece of the block's own rows

struct FewParams {
  AttnParams a;  // without the prefix segment
  PagedKv kv;
  int row_tiles;  // groups of query rows per (sequence, K/V head)
  int units;      // batch * nsplit * hkv
};

template <int D, bool kE4m3, int kKeys, int kTiles>
__global__ __launch_bounds__(kFewWaves * 64, 2) void attn_paged_few_kernel(FewParams fp) {
  const AttnParams& p = fp.a;
  constexpr int kDSteps = D / 32;         // MFMA k-steps of S^T
  constexpr int kDTiles = D / 16;         // 16-row tiles of O^T
  constexpr int kGroups = kKeys / 16;     // groups of 16 keys of a piece
  constexpr int kRow = kE4m3 ? D : 2 * D; // bytes of a cached row
  constexpr int kVPitch = D + 16;         // V row pitch in LDS (see attn_small.hpp)
  constexpr int kOPitch = D + 4;          // row pitch of a wave's O in LDS (fp32)
  constexpr int kVBytes = kKeys * kVPitch * 2;
  constexpr int kOBytes = kSmallTile * kOPitch * 4;
  constexpr int kWaveBytes = kVBytes > kOBytes ? kVBytes : kOBytes;
  constexpr int kStage = kFewWaves * kKeys;
  static_assert(kKeys >= kFewBlockKeys, "a block piece fits the wave's part of LDS");
  __shared__ __attribute__((aligned(16))) uint8_t smem[kFewWaves * kWaveBytes];
  __shared__ float s_m[kFewWaves][kTiles * kSmallTile], s_l[kFewWaves][kTiles * kSmallTile];

  // the row tiles of a unit run on one XCD, one after another (see attn_bf16_kernel)
  const int xcd = blockIdx.x % 8, jx = blockIdx.x / 8;
  const int unit = 8 * (jx / fp.row_tiles) + xcd;
  if (unit >= fp.units) return;  // whole workgroup: padding of the last round
  const int tile = jx % fp.row_tiles;
  const int z = unit / p.hkv, g = unit % p.hkv;
  const int b = z / p.nsplit, sp = z % p.nsplit;
  const int G = p.group;
  const int bbeg = p.cu_block[b];
  const int len = p.cu_block[b + 1] - bbeg;
  const int plen = p.cu_prefix[b + 1] - p.cu_prefix[b];
  const int n_rows = len * G;
  const int row0 = tile * kTiles * kSmallTile;
  const int cached = (plen + kStage - 1) / kStage * kStage;  // the block's first key
  const int n_keys = cached + len;
  const int kbeg = sp * p.kps;
  if (row0 >= n_rows || kbeg >= n_keys) return;  // whole workgroup
  const int kend = min(n_keys, kbeg + p.kps);

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = lane >> 4, l16 = lane & 15;
  uint16_t* const Vs = reinterpret_cast<uint16_t*>(smem + wave * kWaveBytes);

  // Columns of lane group grp in k-step s: the contraction index is permuted so that 16 bytes of an
  // 8-bit row hold the lane's columns of two steps.
  auto col_of = [&](int s) { return kE4m3 ? 64 * (s / 2) + 16 * grp + 8 * (s % 2) : 32 * s + 8 * grp; };
  bf16x8 qf[kTiles][kDSteps];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int r = min(row0 + t * kSmallTile + l16, n_rows - 1);
    const uint16_t* q = p.q + (static_cast<size_t>(bbeg + r / G) * p.hq + g * G + r % G) * D;
#pragma unroll
    for (int s = 0; s < kDSteps; ++s) qf[t][s] = *reinterpret_cast<const bf16x8*>(q + col_of(s));
  }
  f32x4 o[kTiles][kDTiles];
  float m_run[kTiles], l_run[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    m_run[t] = kNegBig;  // the lowest finite value: scores of -inf have weights of zero
    l_run[t] = 0.f;
#pragma unroll
    for (int d = 0; d < kDTiles; ++d) o[t][d] = f32x4{};
  }

  // V^T fragment of keys kbase + 4 grp + 0..3 at d = d0 + l16, as in attn_small_role
  auto vt_read = [&](int kbase, int d0) -> v4i16 {
    const uint16_t* a = Vs + (kbase + 4 * grp + (l16 >> 2)) * kVPitch + d0 + 4 * (l16 & 3);
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(const_cast<uint16_t*>(a)));
  };
  // Softmax and O^T += V^T P^T of one piece with scores sc[t][j] (16 keys each) whose first `valid`
  // keys exist; V lies in LDS.
  auto finish = [&](auto& sc, int valid) {
    constexpr int kG = sizeof(sc[0]) / sizeof(f32x4);
    u32x2 pk[kTiles][kG];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      if (valid < 16 * kG) {
#pragma unroll
        for (int j = 0; j < kG; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * j + 4 * grp + r >= valid) sc[t][j][r] = -INFINITY;
      }
      float mloc = -INFINITY;
#pragma unroll
      for (int j = 0; j < kG; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) mloc = fmaxf(mloc, sc[t][j][r]);
      mloc = fmaxf(mloc, __shfl_xor(mloc, 16));
      mloc = fmaxf(mloc, __shfl_xor(mloc, 32));
      // scale > 0, so max(scale * s) = scale * max(s); e = 2^(scale s - m) with one FMA
      const float m_new = fmaxf(m_run[t], mloc * p.scale_log2);
      const float alpha = fast_exp2(m_run[t] - m_new);
      m_run[t] = m_new;
      float lsum = 0.f;
#pragma unroll
      for (int j = 0; j < kG; ++j) {
        float e[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          e[r] = fast_exp2(fmaf(sc[t][j][r], p.scale_log2, -m_new));
          lsum += e[r];
        }
        pk[t][j] = u32x2{pack2_bf16(e[0], e[1]), pack2_bf16(e[2], e[3])};
      }
      l_run[t] = l_run[t] * alpha + lsum;
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int d = 0; d < kDTiles; ++d) o[t][d] *= alpha;
      }
    }
#pragma unroll
    for (int u = 0; u < kG / 2; ++u)
#pragma unroll
      for (int d = 0; d < kDTiles; ++d) {
        const v4i16 lo = vt_read(32 * u, 16 * d), hi = vt_read(32 * u + 16, 16 * d);
        const bf16x8 vf = __builtin_bit_cast(
            bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          const u32x4 w{pk[t][2 * u][0], pk[t][2 * u][1], pk[t][2 * u + 1][0], pk[t][2 * u + 1][1]};
          o[t][d] = mfma16(vf, __builtin_bit_cast(bf16x8, w), o[t][d]);
        }
      }
  };

  // ---- cached rows ----------------------------------------------------------------------
  constexpr int kKPer = kRow / 64;             // 16-byte loads per lane of 16 rows of K
  constexpr int kVRows = 1024 / kRow;          // rows of V per load instruction
  constexpr int kVPer = 16 / kVRows;           // the same of V
  constexpr int kVLanes = kRow / 16;           // lanes per row of V
  u32x4 kraw[kGroups][kKPer], vraw[kGroups][kVPer];
  uint32_t kscale[kGroups], vscale[kGroups][kVPer];
  const uint32_t koff = l16 * kRow + 16 * grp;
  const int vrow = lane / kVLanes;
  const uint32_t voff = lane * 16;
  const int32_t* const table = fp.kv.table + static_cast<size_t>(b) * fp.kv.max_pages;
  const int pmask = (1 << fp.kv.page_shift) - 1;
  // Pages of the piece at key k0 (uniform); groups past the cached rows take the last page, and no
  // rows of it.
  auto pages = [&](int k0, int (&page)[kGroups]) {
#pragma unroll
    for (int j = 0; j < kGroups; ++j)
      page[j] = table[min(k0 + 16 * j, plen - 1) >> fp.kv.page_shift];
  };
  auto load = [&](int k0, const int (&page_)[kGroups]) {
#pragma unroll
    for (int j = 0; j < kGroups; ++j) {
      const int page = __builtin_amdgcn_readfirstlane(page_[j]);
      const bool ok = static_cast<unsigned>(page) < static_cast<unsigned>(fp.kv.n_pages);
      const size_t row =
          ((static_cast<size_t>(ok ? page : 0) * p.hkv + g) << fp.kv.page_shift) +
          ((k0 + 16 * j) & pmask);
      const int rows = ok ? min(max(plen - (k0 + 16 * j), 0), 16) : 0;
      const __amdgpu_buffer_rsrc_t rk = make_rsrc(fp.kv.k + row * kRow, rows * kRow);
      const __amdgpu_buffer_rsrc_t rv = make_rsrc(fp.kv.v + row * kRow, rows * kRow);
#pragma unroll
      for (int i = 0; i < kKPer; ++i) kraw[j][i] = buffer_load16(rk, koff + 64 * i);
      if constexpr (kE4m3) kscale[j] = buffer_load1(make_rsrc(fp.kv.k_scale + row, rows), l16);
#pragma unroll
      for (int i = 0; i < kVPer; ++i) {
        vraw[j][i] = buffer_load16(rv, voff + 1024 * i);
        if constexpr (kE4m3)
          vscale[j][i] = buffer_load1(make_rsrc(fp.kv.v_scale + row, rows), vrow + kVRows * i);
      }
    }
  };
  const int kcached = min(kend, cached);
  int k0 = kbeg + wave * kKeys;
  if (k0 < min(kcached, plen)) {
    int page[kGroups];
    pages(k0, page);
    load(k0, page);
    for (; k0 < min(kcached, plen); k0 += kStage) {
      const int next = k0 + kStage;
      const bool more = next < min(kcached, plen);
      if (more) pages(next, page);
      // V into LDS (the reads of the piece before are done: they fed the MFMAs above)
#pragma unroll
      for (int j = 0; j < kGroups; ++j)
#pragma unroll
        for (int i = 0; i < kVPer; ++i) {
          uint16_t* dst = Vs + (16 * j + kVRows * i + vrow) * kVPitch;
          if constexpr (kE4m3) {
            u32x4 lo, hi;
            e4m3_widen(vraw[j][i], e8m0(vscale[j][i]), lo, hi);
            dst += 16 * (lane % kVLanes);
            *reinterpret_cast<u32x4*>(dst) = lo;
            *reinterpret_cast<u32x4*>(dst + 8) = hi;
          } else {
            *reinterpret_cast<u32x4*>(dst + 8 * (lane % kVLanes)) = vraw[j][i];
          }
        }
      f32x4 sc[kTiles][kGroups];
#pragma unroll
      for (int j = 0; j < kGroups; ++j) {
        bf16x8 kf[kDSteps];
        if constexpr (kE4m3) {
#pragma unroll
          for (int i = 0; i < kKPer; ++i) {
            u32x4 lo, hi;
            e4m3_widen(kraw[j][i], e8m0(kscale[j]), lo, hi);
            kf[2 * i] = __builtin_bit_cast(bf16x8, lo);
            kf[2 * i + 1] = __builtin_bit_cast(bf16x8, hi);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kKPer; ++i) kf[i] = __builtin_bit_cast(bf16x8, kraw[j][i]);
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          sc[t][j] = f32x4{};
#pragma unroll
          for (int s = 0; s < kDSteps; ++s) sc[t][j] = mfma16(kf[s], qf[t][s], sc[t][j]);
        }
      }
      if (more) load(next, page);
      // the wave's own LDS stores before its transposing reads, and those before the next stores
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      finish(sc, plen - k0);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  }
  // ---- the block's own rows (bf16), pieces of 32 keys dealt to the waves ------------------
  if (kend > cached) {
    const int jend = kend - cached;
    const uint32_t key_bytes = static_cast<uint32_t>(p.hkv) * 2 * D;
    for (int j0 = max(kbeg - cached, 0) + wave * kFewBlockKeys; j0 < jend;
         j0 += kFewWaves * kFewBlockKeys) {
      const size_t at = (static_cast<size_t>(bbeg + j0) * p.hkv + g) * D;
      const int rows = min(len - j0, kFewBlockKeys);
      const uint32_t bytes = (rows - 1) * key_bytes + 2 * D;
      const __amdgpu_buffer_rsrc_t rk = make_rsrc(p.k_blk + at, bytes);
      const __amdgpu_buffer_rsrc_t rv = make_rsrc(p.v_blk + at, bytes);
      constexpr int kLanes = D / 8, kPer = kFewBlockKeys * kLanes / 64;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int r = i * (64 / kLanes) + lane / kLanes, c = 8 * (lane % kLanes);
        *reinterpret_cast<u32x4*>(Vs + r * kVPitch + c) = buffer_load16(rv, r * key_bytes + 2 * c);
      }
      f32x4 sc[kTiles][kFewBlockKeys / 16];
#pragma unroll
      for (int j = 0; j < kFewBlockKeys / 16; ++j) {
        bf16x8 kf[kDSteps];
#pragma unroll
        for (int s = 0; s < kDSteps; ++s)
          kf[s] = __builtin_bit_cast(
              bf16x8, buffer_load16(rk, (16 * j + l16) * key_bytes + 2 * col_of(s)));
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
          sc[t][j] = f32x4{};
#pragma unroll
          for (int s = 0; s < kDSteps; ++s) sc[t][j] = mfma16(kf[s], qf[t][s], sc[t][j]);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      finish(sc, rows);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  }

  // ---- the waves' results, in wave order --------------------------------------------------
  float* const so = reinterpret_cast<float*>(smem);
  constexpr int kWaveFloats = kWaveBytes / 4;
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    float l = l_run[t] + __shfl_xor(l_run[t], 16);
    l += __shfl_xor(l, 32);
    if (grp == 0) s_m[wave][t * kSmallTile + l16] = m_run[t], s_l[wave][t * kSmallTile + l16] = l;
  }
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    if (t > 0) __syncthreads();  // the tile before has been read
    // register r of o[t][d]: column 16 d + 4 grp + r of query l16
#pragma unroll
    for (int d = 0; d < kDTiles; ++d)
      *reinterpret_cast<f32x4*>(so + wave * kWaveFloats + l16 * kOPitch + 16 * d + 4 * grp) = o[t][d];
    __syncthreads();
    for (int i = tid; i < kSmallTile * (D / 4); i += kFewWaves * 64) {
      const int r = i / (D / 4), c = 4 * (i % (D / 4)), rt = t * kSmallTile + r;
      const int row = row0 + rt;
      if (row >= n_rows) break;
      float m = s_m[0][rt];
#pragma unroll
      for (int w = 1; w < kFewWaves; ++w) m = fmaxf(m, s_m[w][rt]);
      f32x4 x{};
      float l = 0.f;
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        const float f = fast_exp2(s_m[w][rt] - m);
        l = fmaf(f, s_l[w][rt], l);
        const f32x4 y = *reinterpret_cast<const f32x4*>(so + w * kWaveFloats + r * kOPitch + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(f, y[e], x[e]);
      }
      const size_t at = static_cast<size_t>(bbeg + row / G) * p.hq + g * G + row % G;
      if (p.nsplit > 1) {
        const size_t idx = at * p.nsplit + sp;
        *reinterpret_cast<f32x4*>(p.o_part + idx * D + c) = x;
        if (c == 0) p.m_part[idx] = m, p.l_part[idx] = l;
      } else {
        const float inv = 1.0f / l;
        *reinterpret_cast<u32x2*>(p.out + at * D + c) =
            u32x2{pack2_bf16(x[0] * inv, x[1] * inv), pack2_bf16(x[2] * inv, x[3] * inv)};
      }
    }
  }
}

}  // namespace
}  // namespace eb

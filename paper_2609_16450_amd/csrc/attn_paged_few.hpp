// Block attention over a paged cache for few query rows per K/V head (single tokens, small blocks),
// bf16.  Such calls read every cached key and value for a handful of multiply-adds: they are bound
// by memory, and the kernel is built around its loads.
//
// A workgroup is four waves.  The waves split the keys, not the rows: each takes every fourth
// piece, holds all 16 kTiles query rows and keeps an online softmax of its own, so that no wave
// waits for another until its keys end; their results are then merged through LDS.
//
// Contexts of a served batch are of very different lengths, and one launch should keep every
// compute unit busy to its end.  So the keys of all sequences form one line, for each (K/V head,
// tile of query rows): n_b stages for sequence b (its cached rows in stages of four pieces, and one
// stage for the block's own rows), and workgroup w takes stages w chunk .. (w + 1) chunk - 1 of it,
// wherever sequences begin and end in them.  A sequence that lies within one workgroup is written
// out at once.  Otherwise each of its workgroups leaves a partial: the first in its slot 1 (the
// sequence goes on), the others in their slot 0 (it came from before), merged by a second launch.
// Measured against ranges of equal length for every sequence: see few_plan.  64 tokens behind 501
// to 8192 rows, 28/4 heads x 128, 8 bits: 56 us (4.9 TB/s), bf16 pages 108 us with the merge (5.1);
// 16 blocks of 32 rows behind 1001 to 4096, 32/32 heads, 8 bits: 80 us (4.0 TB/s); with 33 to 64
// query rows two workgroups read and widen the same keys (32 blocks of 8, 28/4 heads, behind 1001
// to 8192, 8 bits: 65 us with the merge, 2.4 TB/s).
//
// A piece is kFewKeys keys.  K goes from memory straight into the registers of the MFMA's A operand
// (S^T = K Q^T by 16x16x32: lane l holds row l % 16).  V has to be transposed for O^T = V^T P^T: it
// goes through the wave's own part of LDS, row-major, and comes back by transposing reads
// (attn_small.hpp).  As soon as a piece's K is in S and its V in LDS, the loads of the wave's next
// piece go out into the same registers, and stay in flight over the softmax and the second product
// (a second piece in flight: 0-8% slower).
// An 8-bit cache is converted to bf16 on the way, exactly: K rows by the lane that holds them, V
// rows before they go to LDS.
//
// The MFMA takes the probabilities in bf16.  Two of them hold a probability to 2^-16 and cost as
// many MFMAs of the second product again, which wait for memory anyway: the result is then as far
// from 64 bits (2-norm) as its own rounding makes it, 0.00166, with one bf16 0.0019 to 0.0020, and
// no call is slower (64 tokens as above 60.6 and 60.3 us with one, with the merge; bf16 pages, 16
// blocks of 32 rows, 145 and 146).  Only two tiles over 8 bits, whose widening leaves no issue
// slots, keep one bf16, as the tile kernels do: 3 to 14% slower with two (16 blocks of 32 rows 92
// against 89 us, 32 of 8 rows x 7 heads 70 against 65, 100 of 10 rows x 4 heads of 64 59 against
// 51).  l sums them in fp32.
//
// Every 16 keys of a piece lie in one page; a buffer resource per group of 16 ends with the last
// cached row, so rows past it arrive as zeros, and one of no length stands for a missing page.
#pragma once

#include "attn_common.hpp"
#include "attn_partials.hpp"
#include "attn_small.hpp"
#include "paged.hpp"

namespace eb {
namespace {

constexpr int kFewWaves = 4;
constexpr int kFewKeys = 32;  // keys of a piece
constexpr int kFewStage = kFewWaves * kFewKeys;

struct FewParams {
  AttnParams a;  // without the prefix segment and the key split
  PagedKv kv;
  int batch;
  int row_tiles;  // tiles of query rows per (sequence, K/V head)
  int groups;     // workgroups along the line of a (K/V head, tile)
  int chunk;      // stages per workgroup; 0: workgroup w takes sequence w whole
  int most;       // sequences of more query rows per K/V head are another launch's
  // partials of (line, workgroup, slot), line = K/V head * row_tiles + tile
  float* o_part;  // [rows of a tile, D]
  float* m_part;  // [rows of a tile], log2 units
  float* l_part;
};

// Stages of sequence b in the line of the tile at query row row0 (none if the tile lies past its
// rows, or it has too many): its cached rows, then the block's.
__device__ __forceinline__ int few_stages(const FewParams& fp, int b, int row0) {
  const AttnParams& p = fp.a;
  const int rows = (p.cu_block[b + 1] - p.cu_block[b]) * p.group;
  const int plen = p.cu_prefix[b + 1] - p.cu_prefix[b];
  return row0 < rows && rows <= fp.most ? (plen + kFewStage - 1) / kFewStage + 1 : 0;
}

// The sequence that holds stage s of the line, and its first stage, found by the whole wavefront;
// batch if the line ends before s.
__device__ __forceinline__ int few_find(const FewParams& fp, int row0, int s, int lane,
                                        int& first) {
  first = 0;
  for (int b0 = 0; b0 < fp.batch; b0 += 64) {
    const int n = b0 + lane < fp.batch ? few_stages(fp, b0 + lane, row0) : 0;
    const int upto = lanes_up_to(n, 0, AddOp{});
    const uint64_t past = __ballot(first + upto > s);
    if (past) {
      const int l = __builtin_ctzll(past);
      first += __builtin_amdgcn_readlane(upto - n, l);
      return b0 + l;
    }
    first += __builtin_amdgcn_readlane(upto, 63);
  }
  return fp.batch;
}

// Two values >= 0, each as a bf16 below it and a bf16 of the rest, to 2^-16 of itself.  The rest is
// made 2^-20 of the value too large, so that it is zero only where the value is: infinity times the
// pair stays infinity.
__device__ __forceinline__ void split2(float a, float b, uint32_t& most, uint32_t& rest) {
  const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
  most = __builtin_amdgcn_perm(y, x, 0x07060302u);  // high halves
  rest = pack2_bf16(fmaf(a, 0x1p-20f, a - __uint_as_float(x & 0xffff0000u)),
                    fmaf(b, 0x1p-20f, b - __uint_as_float(y & 0xffff0000u)));
}

template <int D, bool kE4m3, int kTiles>
__global__ __launch_bounds__(kFewWaves * 64, 2) void attn_paged_few_kernel(FewParams fp) {
  const AttnParams& p = fp.a;
  constexpr int kDSteps = D / 32;         // MFMA k-steps of S^T
  constexpr int kDTiles = D / 16;         // 16-row tiles of O^T
  constexpr int kGroups = kFewKeys / 16;     // groups of 16 keys of a piece
  constexpr int kRow = kE4m3 ? D : 2 * D; // bytes of a cached row
  constexpr bool kTwoBf16 = !kE4m3 || kTiles == 1;  // a probability in two bf16
  constexpr int kVPitch = D + 16;         // V row pitch in LDS (see attn_small.hpp)
  constexpr int kOPitch = D + 4;          // row pitch of a wave's O in LDS (fp32)
  constexpr int kVBytes = kFewKeys * kVPitch * 2;
  constexpr int kOBytes = kSmallTile * kOPitch * 4;
  constexpr int kWaveBytes = kVBytes > kOBytes ? kVBytes : kOBytes;
  __shared__ __attribute__((aligned(16))) uint8_t smem[kFewWaves * kWaveBytes];
  __shared__ float s_m[kFewWaves][kTiles * kSmallTile], s_l[kFewWaves][kTiles * kSmallTile];

  // the row tiles of a unit (K/V head, workgroup of the line) run on one XCD, one after another,
  // and read its keys from that XCD's L2
  const int xcd = blockIdx.x % 8, jx = blockIdx.x / 8;
  const int unit = 8 * (jx / fp.row_tiles) + xcd;
  const int tile = jx % fp.row_tiles;
  const int w = unit / p.hkv, g = unit % p.hkv;
  if (w >= fp.groups) return;  // whole workgroup: padding of the last round
  const int G = p.group;
  const int row0 = tile * kTiles * kSmallTile;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = lane >> 4, l16 = lane & 15;
  uint16_t* const Vs = reinterpret_cast<uint16_t*>(smem + wave * kWaveBytes);

  int b, first, from, to;  // sequence, its first stage in the line, stages of this workgroup
  if (fp.chunk) {
    from = w * fp.chunk;
    to = from + fp.chunk;
    b = few_find(fp, row0, from, lane, first);
  } else {
    b = w, first = 0, from = 0, to = 1 << 30;
  }
  for (; b < fp.batch && from < to; ++b) {
    const int n_stages = few_stages(fp, b, row0);
    if (n_stages == 0) {
      if (!fp.chunk) return;  // uniform, as the rest of the loop's conditions
      continue;
    }
    const int bbeg = p.cu_block[b];
    const int len = p.cu_block[b + 1] - bbeg;
    const int plen = p.cu_prefix[b + 1] - p.cu_prefix[b];
    const int n_rows = len * G;
    const int sbeg = from - first, send = min(to - first, n_stages);  // stages of the sequence
    // its cached rows among them
    const int kbeg = sbeg * kFewStage, kend = min(send * kFewStage, plen);

    // Columns of lane group grp in k-step s: the contraction index is permuted so that 16 bytes of
    // an 8-bit row hold the lane's columns of two steps.
    auto col_of = [&](int s, int grp_) {
      return kE4m3 ? 64 * (s / 2) + 16 * grp_ + 8 * (s % 2) : 32 * s + 8 * grp_;
    };
    bf16x8 qf[kTiles][kDSteps];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int r = min(row0 + t * kSmallTile + l16, n_rows - 1);
      const uint16_t* q = p.q + (static_cast<size_t>(bbeg + r / G) * p.hq + g * G + r % G) * D;
#pragma unroll
      for (int s = 0; s < kDSteps; ++s)
        qf[t][s] = *reinterpret_cast<const bf16x8*>(q + col_of(s, grp));
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
    // Softmax and O^T += V^T P^T of one piece with scores sc[t][j] (16 keys each) whose first
    // `valid` keys exist; V lies in LDS.
    auto finish = [&](auto& sc, int valid) {
      constexpr int kG = sizeof(sc[0]) / sizeof(f32x4);
      u32x2 pk[kTiles][kG], rest[kTiles][kG];  // P in one bf16, or in two (split2)
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
          if constexpr (kTwoBf16) {
            uint32_t most[2], less[2];
            split2(e[0], e[1], most[0], less[0]);
            split2(e[2], e[3], most[1], less[1]);
            pk[t][j] = u32x2{most[0], most[1]};
            rest[t][j] = u32x2{less[0], less[1]};
          } else {
            pk[t][j] = u32x2{pack2_bf16(e[0], e[1]), pack2_bf16(e[2], e[3])};
          }
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
            auto weights = [&](const u32x2& lo2, const u32x2& hi2) {
              return __builtin_bit_cast(bf16x8, u32x4{lo2[0], lo2[1], hi2[0], hi2[1]});
            };
            o[t][d] = mfma16(vf, weights(pk[t][2 * u], pk[t][2 * u + 1]), o[t][d]);
            if constexpr (kTwoBf16)
              o[t][d] = mfma16(vf, weights(rest[t][2 * u], rest[t][2 * u + 1]), o[t][d]);
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
    // Pages of the piece at key k0 (uniform); groups past the cached rows take the last page, and
    // no rows of it.
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
    int k0 = kbeg + wave * kFewKeys;
    if (k0 < kend) {
      int page[kGroups];
      pages(k0, page);
      load(k0, page);
      for (; k0 < kend; k0 += kFewStage) {
        const int next = k0 + kFewStage;
        const bool more = next < kend;
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
    if (send == n_stages) {
      const uint32_t key_bytes = static_cast<uint32_t>(p.hkv) * 2 * D;
      int lane_ = lane;  // addresses formed here: kept over the cached rows they would spill
      asm volatile("" : "+v"(lane_));
      for (int j0 = wave * kFewKeys; j0 < len; j0 += kFewWaves * kFewKeys) {
        const size_t at = (static_cast<size_t>(bbeg + j0) * p.hkv + g) * D;
        const int rows = min(len - j0, kFewKeys);
        const uint32_t bytes = (rows - 1) * key_bytes + 2 * D;
        const __amdgpu_buffer_rsrc_t rk = make_rsrc(p.k_blk + at, bytes);
        const __amdgpu_buffer_rsrc_t rv = make_rsrc(p.v_blk + at, bytes);
        constexpr int kLanes = D / 8, kPer = kFewKeys * kLanes / 64;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int r = i * (64 / kLanes) + lane_ / kLanes, c = 8 * (lane_ % kLanes);
          *reinterpret_cast<u32x4*>(Vs + r * kVPitch + c) =
              buffer_load16(rv, r * key_bytes + 2 * c);
        }
        f32x4 sc[kTiles][kFewKeys / 16];
#pragma unroll
        for (int j = 0; j < kFewKeys / 16; ++j) {
          bf16x8 kf[kDSteps];
#pragma unroll
          for (int s = 0; s < kDSteps; ++s)
            kf[s] = __builtin_bit_cast(
                bf16x8, buffer_load16(
                            rk, (16 * j + (lane_ & 15)) * key_bytes + 2 * col_of(s, lane_ >> 4)));
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
    const bool whole = sbeg == 0 && send == n_stages;
    const size_t slot =
        ((static_cast<size_t>(g) * fp.row_tiles + tile) * fp.groups + w) * 2 + (sbeg == 0 ? 1 : 0);
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
        *reinterpret_cast<f32x4*>(so + wave * kWaveFloats + l16 * kOPitch + 16 * d + 4 * grp) =
            o[t][d];
      __syncthreads();
      int tid_ = tid;  // (as lane_ above)
      asm volatile("" : "+v"(tid_));
      for (int i = tid_; i < kSmallTile * (D / 4); i += kFewWaves * 64) {
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
        if (whole) {
          const size_t at = static_cast<size_t>(bbeg + row / G) * p.hq + g * G + row % G;
          const float inv = 1.0f / l;
          *reinterpret_cast<u32x2*>(p.out + at * D + c) =
              u32x2{pack2_bf16(x[0] * inv, x[1] * inv), pack2_bf16(x[2] * inv, x[3] * inv)};
        } else {
          const size_t at = slot * kTiles * kSmallTile + rt;
          *reinterpret_cast<f32x4*>(fp.o_part + at * D + c) = x;
          if (c == 0) fp.m_part[at] = m, fp.l_part[at] = l;
        }
      }
    }
    __syncthreads();  // before the next sequence's values take the waves' places in LDS
    first += n_stages;
    from = first;
    if (!fp.chunk) return;
  }
}

// The partials of one (sequence, K/V head, tile of query rows) per workgroup, in the order of the
// line; a wave per query row, its lanes over kParts partials side by side.
template <int D>
__global__ __launch_bounds__(512) void attn_paged_few_merge_kernel(FewParams fp,
                                                                   int tile_rows) {
  const AttnParams& p = fp.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = blockIdx.x % fp.row_tiles, z = blockIdx.x / fp.row_tiles;
  const int g = z % p.hkv, b = z / p.hkv;
  const int row0 = tile * tile_rows;
  // first stage of the sequence in the line
  int before = 0;
  for (int b0 = 0; b0 < b; b0 += 64)
    before += b0 + lane < b ? few_stages(fp, b0 + lane, row0) : 0;
  before = lanes_all(before, 0, AddOp{});
  const int n = few_stages(fp, b, row0);
  const int w0 = before / fp.chunk, w1 = (before + n - 1) / fp.chunk;
  if (n == 0 || w0 == w1) return;  // nothing here, or written out by its only workgroup
  const int bbeg = p.cu_block[b], G = p.group;
  const int n_rows = min((p.cu_block[b + 1] - bbeg) * G - row0, tile_rows);
  const size_t line = static_cast<size_t>(g * fp.row_tiles + tile) * fp.groups;
  const int parts = w1 - w0 + 1;
  for (int r = wave; r < n_rows; r += 8) {
    // row of partial k: slot 1 of the first workgroup, slot 0 of the others
    auto at = [&](int k) {
      return ((line + w0 + k) * 2 + (k == 0 ? 1 : 0)) * tile_rows + r;
    };
    const int row = row0 + r;
    const size_t dst = static_cast<size_t>(bbeg + row / G) * p.hq + g * G + row % G;
    merge_partials<D>(at, parts, fp.o_part, fp.m_part, fp.l_part, lane)
        .store(p.out + dst * D, lane);
  }
}

}  // namespace
}  // namespace eb

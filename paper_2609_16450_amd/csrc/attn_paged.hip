// Block attention over a paged key/value cache.
//
// Keys of a sequence are its cached rows, read through the page table, and the block's own rows.
// The cached rows are padded to whole stages, so that a stage lies either in the cache or in the
// block and a piece of 16 keys in one page (page sizes are multiples of 16); keys of the padding
// get scores of -inf and values of zero, whatever the page holds there.
#include <algorithm>

#include "attn_common.hpp"
#include "attn_paged_few.hpp"
#include "attn_tiles.hpp"
#include "eb_common.hpp"
#include "eb_internal.hpp"
#include "paged.hpp"

namespace eb {
namespace {

// ---------------------------------------------------------------------------------------
// fp32 arithmetic throughout, on 16x16x4 fp32 MFMAs.
//
// A workgroup of kPf32Waves wavefronts per (16 query rows, K/V head, sequence, key range).  Wave w
// takes the 16-key chunks w, w + kPf32Waves, ... of the range with an online softmax of its own;
// the waves' results are merged through LDS and, with a key split, the ranges' by a second kernel.
// Scores are formed transposed, S^T = K Q^T: lane l owns query l % 16 and holds keys 4 (l / 16) + r
// of the chunk, which are the k-slots of the B operand of O^T = V^T P^T, one register per MFMA.
// ---------------------------------------------------------------------------------------
constexpr int kPf32Waves = 8;
constexpr int kPf32Rows = 16;
constexpr int kPf32Keys = 16;
constexpr int kPf32Stage = kPf32Waves * kPf32Keys;  // keys that the waves take in one go

struct PagedF32Params {
  PagedKv kv;
  const int32_t* cu_block;
  const int32_t* cu_prefix;
  int hq, group, tiles;
  float scale;
  const void* q;
  const void* k_blk;
  const void* v_blk;
  void* out;
  // key split, in ranges of kps keys of the padded key space; partials as in AttnParams, the
  // maxima in natural units
  int nsplit, kps;
  float* o_part;
  float* m_part;
  float* l_part;
};

template <class T>
__device__ __forceinline__ f32x4 widen4(const T* p);
template <>
__device__ __forceinline__ f32x4 widen4<float>(const float* p) {
  return *reinterpret_cast<const f32x4u*>(p);
}
template <>
__device__ __forceinline__ f32x4 widen4<uint8_t>(const uint8_t* p) {
  const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
  const f32x2 a = e4m3_pair_f32<false>(w, 1.f), b = e4m3_pair_f32<true>(w, 1.f);
  return f32x4{a[0], a[1], b[0], b[1]};
}
template <int D, class C>
__global__ __launch_bounds__(kPf32Waves * 64) void attn_paged_f32_kernel(PagedF32Params p) {
  constexpr int kChunks = D / 16;
  constexpr int kPitch = D + 4;
  __shared__ __attribute__((aligned(16))) float s_o[kPf32Waves][kPf32Rows * kPitch];
  __shared__ float s_m[kPf32Waves][kPf32Rows], s_l[kPf32Waves][kPf32Rows];
  const int tile = blockIdx.x % p.tiles, sp = blockIdx.x / p.tiles, g = blockIdx.y, b = blockIdx.z;
  const int row0 = tile * kPf32Rows;
  const int bbeg = p.cu_block[b], len = p.cu_block[b + 1] - bbeg;
  const int G = p.group, n_rows = len * G;
  if (row0 >= n_rows) return;  // whole workgroup
  const int plen = p.cu_prefix[b + 1] - p.cu_prefix[b];
  const int cached = (plen + kPf32Keys - 1) / kPf32Keys * kPf32Keys;  // the block's first key
  const int n_keys = cached + len;
  const int kbeg = sp * p.kps;
  if (kbeg >= n_keys) return;  // whole workgroup
  const int kend = min(n_keys, kbeg + p.kps);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int grp = lane >> 4, l16 = lane & 15;
  auto row_at = [&](int i) {  // element offset of a query row (rows past the end repeat the last)
    const int r = min(row0 + i, n_rows - 1);
    return (static_cast<size_t>(bbeg + r / G) * p.hq + g * G + r % G);
  };

  f32x4 qf[kChunks], o[kChunks];
  const float* q = static_cast<const float*>(p.q) + row_at(l16) * D + 4 * grp;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) qf[c] = widen4(q + 16 * c), o[c] = f32x4{};
  // from the lowest finite value on: keys with scores of -inf have weights of zero
  float m_run = -3.402823466e38f, l_run = 0.f;
  for (int k0 = kbeg + wave * kPf32Keys; k0 < kend; k0 += kPf32Stage) {
    f32x4 kf[kChunks];
    f32x4 vf[4][kChunks / 4];  // V of key k0 + 4 grp + r at d = kChunks l16 + 4 i + e
    int valid;             // keys of this chunk
    if (k0 < cached) {
      valid = min(kPf32Keys, plen - k0);
      int page = p.kv.table[static_cast<size_t>(b) * p.kv.max_pages + (k0 >> p.kv.page_shift)];
      const bool ok = static_cast<unsigned>(page) < static_cast<unsigned>(p.kv.n_pages);
      page = ok ? page : 0;
      const size_t slab = ((static_cast<size_t>(page) * p.kv.hkv + g) << p.kv.page_shift) +
                          (k0 & ((1 << p.kv.page_shift) - 1));
      const size_t kr = slab + min(l16, valid - 1);
      float ks = ok ? 1.f : 0.f;
      if (sizeof(C) == 1 && ok) ks = e8m0(p.kv.k_scale[kr]);
      const C* kp = reinterpret_cast<const C*>(p.kv.k) + kr * D + 4 * grp;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        kf[c] = widen4(kp + 16 * c) * ks;
        if (!ok) kf[c] = f32x4{};
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const size_t vr = slab + min(4 * grp + r, valid - 1);
        float vs = 1.f;
        if (sizeof(C) == 1) vs = e8m0(p.kv.v_scale[vr]);
        const C* vp = reinterpret_cast<const C*>(p.kv.v) + vr * D + kChunks * l16;
        const bool live = ok && 4 * grp + r < valid;  // a weight of zero times infinity is NaN
#pragma unroll
        for (int i = 0; i < kChunks / 4; ++i) {
          vf[r][i] = widen4(vp + 4 * i) * vs;
          if (!live) vf[r][i] = f32x4{};
        }
      }
    } else {
      const int j0 = k0 - cached;
      valid = min(kPf32Keys, len - j0);
      const size_t kr = static_cast<size_t>(bbeg + j0 + min(l16, valid - 1)) * p.kv.hkv + g;
      const float* kp = static_cast<const float*>(p.k_blk) + kr * D + 4 * grp;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) kf[c] = widen4(kp + 16 * c);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const size_t vr =
            static_cast<size_t>(bbeg + j0 + min(4 * grp + r, valid - 1)) * p.kv.hkv + g;
        const float* vp = static_cast<const float*>(p.v_blk) + vr * D + kChunks * l16;
#pragma unroll
        for (int i = 0; i < kChunks / 4; ++i) {
          vf[r][i] = widen4(vp + 4 * i);
          if (4 * grp + r >= valid) vf[r][i] = f32x4{};
        }
      }
    }
    f32x4 acc[2] = {f32x4{}, f32x4{}};
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e & 1] = mfma16_f32(kf[c][e], qf[c][e], acc[e & 1]);
    float sc[4], mloc = -INFINITY;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sc[r] = 4 * grp + r < valid ? (acc[0][r] + acc[1][r]) * p.scale : -INFINITY;
      mloc = fmaxf(mloc, sc[r]);
    }
    mloc = fmaxf(mloc, __shfl_xor(mloc, 16));
    mloc = fmaxf(mloc, __shfl_xor(mloc, 32));
    const float m_new = fmaxf(m_run, mloc);
    const float alpha = expf(m_run - m_new);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) o[c] *= alpha;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float e = expf(sc[r] - m_new);
      l_run += e;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) o[c] = mfma16_f32(vf[r][c / 4][c % 4], e, o[c]);
    }
  }
  float l_tot = l_run + __shfl_xor(l_run, 16);
  l_tot += __shfl_xor(l_tot, 32);
  if (grp == 0) {
    s_m[wave][l16] = m_run;
    s_l[wave][l16] = l_tot;
  }
  // register r of o[c]: d = kChunks (4 (l / 16) + r) + c of query l % 16
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int i = 0; i < kChunks / 4; ++i)
      *reinterpret_cast<f32x4*>(&s_o[wave][l16 * kPitch + kChunks * (4 * grp + r) + 4 * i]) =
          f32x4{o[4 * i][r], o[4 * i + 1][r], o[4 * i + 2][r], o[4 * i + 3][r]};
  __syncthreads();
  // merge in wave order; a wave without keys has l = 0 and o = 0
  for (int i = tid; i < kPf32Rows * D; i += kPf32Waves * 64) {
    const int r = i / D, d = i % D;
    if (row0 + r >= n_rows) break;
    float m = s_m[0][r];
#pragma unroll
    for (int w = 1; w < kPf32Waves; ++w) m = fmaxf(m, s_m[w][r]);
    float l = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < kPf32Waves; ++w) {
      const float f = expf(s_m[w][r] - m);
      l = fmaf(f, s_l[w][r], l);
      x = fmaf(f, s_o[w][r * kPitch + d], x);
    }
    const size_t at = row_at(r);
    if (p.nsplit > 1) {
      p.o_part[(at * p.nsplit + sp) * D + d] = x;
      if (d == 0) p.m_part[at * p.nsplit + sp] = m, p.l_part[at * p.nsplit + sp] = l;
    } else {
      static_cast<float*>(p.out)[at * D + d] = x / l;
    }
  }
}

// The ranges of one (block row, query head) per wavefront, in order.
template <int D>
__global__ __launch_bounds__(256) void attn_paged_f32_merge_kernel(PagedF32Params p, int batch,
                                                                   int total) {
  constexpr int kPer = D / 64;
  const long rh = static_cast<long>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (rh >= static_cast<long>(total) * p.hq) return;  // uniform per wavefront
  const int b = find_sequence(p.cu_block, batch, static_cast<int>(rh / p.hq), lane);
  const int plen = p.cu_prefix[b + 1] - p.cu_prefix[b];
  const int cached = (plen + kPf32Keys - 1) / kPf32Keys * kPf32Keys;
  const int n_keys = cached + p.cu_block[b + 1] - p.cu_block[b];
  const int n = min(p.nsplit, (n_keys + p.kps - 1) / p.kps);
  const size_t base = static_cast<size_t>(rh) * p.nsplit;
  float m = -INFINITY, l = 0.f, x[kPer] = {};
  for (int k = lane; k < n; k += 64) m = fmaxf(m, p.m_part[base + k]);
  for (int mask = 32; mask >= 1; mask >>= 1) m = fmaxf(m, __shfl_xor(m, mask));
  for (int k = 0; k < n; ++k) {
    const float f = expf(p.m_part[base + k] - m);
    l = fmaf(f, p.l_part[base + k], l);
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      x[e] = fmaf(f, p.o_part[(base + k) * D + lane * kPer + e], x[e]);
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e)
    static_cast<float*>(p.out)[rh * D + lane * kPer + e] = x[e] / l;
}

// Ranges of whole stages, enough for a workgroup per compute unit (two per compute unit: 29 against
// 24 us for 4 sequences of 64 rows behind 1024, 16/4 heads x 64); up to four stages stay whole (the
// merge takes as long).
SplitPlan f32_plan(const PagedAttnArgs& a) {
  const long tiles =
      (static_cast<long>(a.max_block) * (a.hq / a.kv.hkv) + kPf32Rows - 1) / kPf32Rows;
  const long base = tiles * a.kv.hkv * a.batch;
  const int keys = (a.max_prefix + kPf32Keys - 1) / kPf32Keys * kPf32Keys + a.max_block;
  const long stages = (keys + kPf32Stage - 1) / kPf32Stage;
  const long want = stages <= 4 ? 1 : std::max(1L, std::min((256 + base - 1) / base, stages));
  const long per = (stages + want - 1) / want;
  return SplitPlan{static_cast<int>((stages + per - 1) / per), static_cast<int>(per * kPf32Stage)};
}

template <int D, class C>
hipError_t launch_f32(const PagedAttnArgs& a, void* ws, hipStream_t s) {
  const SplitPlan sp = f32_plan(a);
  const size_t n = static_cast<size_t>(a.total_block) * a.hq * sp.nsplit;
  float* o = static_cast<float*>(ws);
  const int group = a.hq / a.kv.hkv;
  const int tiles = static_cast<int>((static_cast<long>(a.max_block) * group + kPf32Rows - 1) /
                                     kPf32Rows);
  const PagedF32Params p{a.kv, a.cu_block, a.cu_prefix, a.hq, group, tiles, a.scale, a.q, a.k_blk,
                      a.v_blk, a.out, sp.nsplit, sp.kps, o, o + n * D, o + n * D + n};
  const dim3 grid(static_cast<unsigned>(tiles * sp.nsplit), static_cast<unsigned>(a.kv.hkv),
                  static_cast<unsigned>(a.batch));
  hipLaunchKernelGGL((attn_paged_f32_kernel<D, C>), grid, dim3(kPf32Waves * 64), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || sp.nsplit == 1) return e;
  const long pairs = static_cast<long>(a.total_block) * a.hq;
  hipLaunchKernelGGL((attn_paged_f32_merge_kernel<D>), dim3(static_cast<unsigned>((pairs + 3) / 4)),
                     dim3(256), 0, s, p, a.batch, a.total_block);
  return hipGetLastError();
}

// ---- few query rows per K/V head, bf16 ----------------------------------------------------
// Up to this many query rows per K/V head.  Over bf16 pages the tile kernel is the faster from 33
// rows on (32 heads x 128, 16 blocks of 64 rows: 137 against 165 us); widening 8 bits costs it more
// (28/4 heads, 64 blocks of 8: 112 against 106 us; 16/4 heads x 64, 32 blocks of 16: 67 against
// 48).
constexpr int kFewRowsBf16 = 32, kFewRowsE4m3 = 64;
constexpr int kFewMaxBatch = 2048;
// A sequence this many stages longer than a part still takes one workgroup: the merge's launch
// costs as much (one token behind 100 rows, 28/4 heads: 6.8 against 9.3 us; behind 1000 rows, 9
// stages, 14.5 whole against 9.2 us).
constexpr int kFewWhole = 5;

// Query rows per K/V head up to which sequences of this call go to the kernel for few rows; the
// others go to the tile kernel, in a launch of their own.  Over 8 bits that is worth two launches
// where a long block comes with many short ones: 63 tokens and a chunk of 1024 behind 1000 to 4000
// rows, 28/4 heads x 128, 141 us in one launch, 112 in two, 255 and a chunk of 2048 362 and 288
// (32/32 heads 1741 and 1150, 16/4 heads x 64 244 and 167).  Over bf16 pages the tile kernel reads
// the keys of a few rows about as fast.  The sizes of single blocks are on the device; the host
// goes by the mean of all but the longest, and by the cached rows, whether the launch can gain more
// than it takes (16 tokens and a chunk of 256, 28/4 heads: 42 us in one, 50 in two).
constexpr long kFewWorth = 4096;  // cached stages of 64 rows, over the K/V heads
long few_rows(const PagedAttnArgs& a) {
  const bool e4m3 = a.kv.type == CacheType::kE4m3;
  const long group = a.hq / a.kv.hkv, rows = a.max_block * group;
  if (rows <= (e4m3 ? kFewRowsE4m3 : kFewRowsBf16)) return rows;
  const long others = (a.total_block - a.max_block) * group;  // of batch - 1 sequences
  const long stages = static_cast<long>(a.total_prefix) / kKeys * a.kv.hkv;
  if (!e4m3 || a.batch == 1 || stages < kFewWorth) return 0;
  for (long most = kSmallTile; most <= 2 * kSmallTile; most *= 2)
    if (2 * others <= most * (a.batch - 1)) return most;
  return 0;
}

// The line of stages (attn_paged_few.hpp) in as many equal parts as workgroups that run at a time,
// two per compute unit: one round, and all of it ends together.  Ranges of equal length for every
// sequence, 1024 workgroups of them, took as long as their last round: 64 tokens behind 501 to 8192
// rows 143 against 110 us (bf16), 256 behind 100 to 4000 rows 278 against 222 us, 32 blocks of 8
// behind 1001 to 8192 rows (8 bits) 92 against 76 us (28/4 heads x 128).  768 or 1024 parts: 0-15%
// slower.  Every workgroup looks at all sequences to find its part, so more than kFewMaxBatch
// sequences take one workgroup each.
struct FewPlan {
  int most;       // query rows per K/V head
  int row_tiles, groups, chunk;
  size_t slots;  // partial rows of the workspace
};
FewPlan few_plan(const PagedAttnArgs& a, long rows) {
  FewPlan f;
  f.most = static_cast<int>(rows);
  const int per = (rows <= kSmallTile ? 1 : 2) * kSmallTile;
  f.row_tiles = (f.most + per - 1) / per;
  const long lines = static_cast<long>(f.row_tiles) * a.kv.hkv;
  if (a.batch > kFewMaxBatch) {
    f.groups = a.batch, f.chunk = 0, f.slots = 0;
    return f;
  }
  // stages of a line, at most
  const long most = std::min(a.total_prefix / kFewStage + 2L * a.batch,
                        a.batch * ((a.max_prefix + kFewStage - 1L) / kFewStage + 1));
  const long chunk = (most * lines + kAttnTargetWgs - 1) / kAttnTargetWgs;
  const long longest = (a.max_prefix + kFewStage - 1L) / kFewStage + 1;
  if (longest <= chunk + kFewWhole) {
    f.groups = a.batch, f.chunk = 0, f.slots = 0;
    return f;
  }
  f.chunk = static_cast<int>(chunk);
  f.groups = static_cast<int>((most + chunk - 1) / chunk);
  f.slots = f.groups > 1 ? static_cast<size_t>(lines) * f.groups * 2 * per : 0;
  return f;
}

// The call as one on packed rows whose prefix is empty, for what the kernels share.
AttnArgs packed_args(const PagedAttnArgs& a) {
  return AttnArgs{a.batch, a.total_block, a.max_block, a.total_prefix, a.max_prefix, a.cu_block,
                  a.cu_prefix, a.hq, a.kv.hkv, a.kv.head_dim, a.scale, a.q, a.k_blk, a.v_blk,
                  nullptr, nullptr, a.out};
}

template <int D, bool kE4m3, int kTiles>
hipError_t launch_few(const PagedAttnArgs& a, const FewPlan& f, void* ws, hipStream_t s) {
  float* const o = static_cast<float*>(ws);
  float* const m = o + f.slots * D;
  const FewParams p{attn_params(packed_args(a), SplitPlan{1, 0}, nullptr), a.kv, a.batch,
                    f.row_tiles, f.groups, f.chunk, f.most, o, m, m + f.slots};
  const long units = static_cast<long>(f.groups) * a.kv.hkv;
  const dim3 grid(static_cast<unsigned>(8 * ((units + 7) / 8) * f.row_tiles));
  hipLaunchKernelGGL((attn_paged_few_kernel<D, kE4m3, kTiles>), grid,
                     dim3(kFewWaves * 64), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || f.slots == 0) return e;
  hipLaunchKernelGGL(attn_paged_few_merge_kernel<D>,
                     dim3(static_cast<unsigned>(a.batch * a.kv.hkv * f.row_tiles)), dim3(512), 0, s,
                     p, kTiles * kSmallTile);
  return hipGetLastError();
}

template <int D>
hipError_t launch_few_any(const PagedAttnArgs& a, long rows, void* ws, hipStream_t s) {
  const bool e4m3 = a.kv.type == CacheType::kE4m3;
  const FewPlan f = few_plan(a, rows);
  if (rows <= kSmallTile)
    return e4m3 ? launch_few<D, true, 1>(a, f, ws, s) : launch_few<D, false, 1>(a, f, ws, s);
  return e4m3 ? launch_few<D, true, 2>(a, f, ws, s) : launch_few<D, false, 2>(a, f, ws, s);
}

// ---- many query rows, bf16: the tile kernels of the packed prefix ---------------------------
// Items of whole sequences (a K/V head and a tile of query rows each) up to which a launch may cut
// sequences into ranges, for one, two or four rounds of workgroups: the fewer items, the fewer
// rounds are needed to make them even.  With more than kSplitItems sequences stay whole (32 heads,
// 32 blocks of 8 to 128 rows behind 2048, 1024 items, two full rounds: 212 us whole, 227 us with the
// plan); a third round that is not full then costs as much as a full one (33, 36, 40 and 48 such
// blocks: 254, 272, 288 and 329 us).  The borders lie between the shapes measured.
constexpr long kSplitItems1 = 160, kSplitItems2 = 420, kSplitItems = 900;
// Up to this many stages sequences stay whole: one block of 100 rows behind 300, 28/4 heads, 7
// stages, 16 against 19 us; behind 600, 12 stages, 18 us either way.
constexpr long kWholeStages = 8;

// With blocks of unlike lengths, counting every sequence as the longest leaves workgroups without
// an item, and while these come and go the others wait: 255 tokens and a chunk of 2048 behind 1000
// to 4000, 28/4 heads x 128, 115000 workgroups for at most 1500 items, 1009 us, counted off 362 us
// (32/32 heads 5125 and 1986; 64 blocks of 16 to 256 rows, 3584 for 2160, 621 and 573).  Counting
// costs a workgroup a look at the lengths of 64 sequences at a time, about a quarter of such a
// visit.
constexpr long kCountBatch = 256;
constexpr long kCountTurns = 8;  // runs per XCD, at least
// Items counted off that may leave partials: twice what the plan aims at.  Only where more blocks
// than are likely have items of their own (few_rows) would there be more of them; the sequences
// behind these stay whole.  (The host can only bound the blocks that have items, by a good ten
// times what there usually are: a chunk of 512 among 255 tokens took 239 MB for 336 items.)
constexpr long kMostPartials = 2 * kAttnTargetWgs;

struct TilesLaunch {
  TilePlan plan;
  long grid;
  size_t parts;  // items that may leave partials
};
// (of the sequences with more than `skip` query rows per K/V head)
TilesLaunch tiles_plan(const PagedAttnArgs& a, long skip) {
  const long group = a.hq / a.kv.hkv, hkv = a.kv.hkv;
  const long row_tiles = (a.max_block * group + kRowsPerWg - 1) / kRowsPerWg;
  const long stages = (a.max_prefix + kKeys - 1L) / kKeys + (a.max_block + kKeys - 1) / kKeys;
  // items of whole sequences, at most
  const long rows = a.total_block * group;
  const long sequences = std::min(static_cast<long>(a.batch), rows / (skip + 1));
  const long whole = hkv * std::min(sequences * row_tiles, rows / kRowsPerWg + sequences);
  TilesLaunch t{};
  t.plan.batch = a.batch;
  t.plan.row_tiles = static_cast<int>(row_tiles);
  t.plan.skip = static_cast<int>(skip);
  if (a.batch <= kPlanMaxBatch && whole <= kSplitItems && stages > kWholeStages) {
    const int rounds = whole <= kSplitItems1 ? 1 : whole <= kSplitItems2 ? 2 : 4;
    // no more than there are (range, K/V head, tile)s; a power of two, for find_item
    int cap = kXcdCount;
    while (cap < rounds * kAttnTargetWgs && cap < whole * stages) cap *= 2;
    t.plan.cap = cap;
    t.grid = t.plan.cap;
    t.parts = t.plan.cap;
    return t;
  }
  const long all = row_tiles * hkv * a.batch;
  const bool counted = all * kCountBatch > whole * (kCountBatch + a.batch);
  // items of whole sequences as they are likely to be (few_rows skips short ones, not knowing them)
  const long likely = skip ? std::min(whole, hkv * (rows / kRowsPerWg + 1)) : whole;
  const long base = counted ? likely : all;
  // (to the nearest: 400 sequences whole 89 us, halved 97; 280 of them 82 and 68, 16/4 heads x 64)
  const long most = std::max(1L, std::min((kAttnTargetWgs + base / 2) / base, stages));
  const long want = stages <= kWholeStages ? 1 : most;
  const long chunk = (stages + want - 1) / want;
  t.plan.chunk = static_cast<int>(chunk);
  t.plan.nsplit = static_cast<int>((stages + chunk - 1) / chunk);
  if (counted) {
    const long items = std::min(whole * t.plan.nsplit, whole + kMostPartials);
    const long run =
        std::max(1L, std::min(row_tiles, likely * t.plan.nsplit / (kXcdCount * kCountTurns)));
    t.plan.run = static_cast<int>(run);
    t.plan.most = static_cast<int>(kMostPartials);
    t.grid = kXcdCount * run * ((items + kXcdCount * run - 1) / (kXcdCount * run));
  } else {
    t.grid = kXcdCount * ((a.batch * hkv * t.plan.nsplit + kXcdCount - 1) / kXcdCount) * row_tiles;
  }
  t.parts = t.plan.nsplit == 1 ? 0 : counted ? std::min(t.grid, kMostPartials) : t.grid;
  return t;
}

// Waves of the merge that run at a time; with more rows x heads than these a wave takes several
// heads of a row, as most find little or nothing to merge (32 heads, 1000 rows behind 3000, 92 ->
// 88 us, 8 blocks of 64 to 512 behind 300 to 2400 134 -> 127 us; with 16384 95 and 124).
constexpr long kMergeWaves = 8192;

template <int D, bool kE4m3>
hipError_t launch_tiles(const PagedAttnArgs& a, long skip, void* ws, hipStream_t s) {
  const TilesLaunch t = tiles_plan(a, skip);
  const AttnParams p = attn_params(packed_args(a), SplitPlan{1, 0}, nullptr);
  using Keys = PagedKeys<kE4m3>;
  Keys keys{a.kv, t.plan};
  const size_t rows = t.parts * kRowsPerWg;
  keys.plan.o_part = static_cast<float*>(ws);
  keys.plan.m_part = keys.plan.o_part + rows * D;
  keys.plan.l_part = keys.plan.m_part + rows;
  keys.plan.found = reinterpret_cast<int32_t*>(keys.plan.l_part + rows);
  if constexpr (D == 128)
    hipLaunchKernelGGL(attn_bf16_d128_kernel<Keys>, dim3(static_cast<unsigned>(t.grid)),
                       dim3(kThreads), 0, s, p, keys, 0, 0);
  else
    hipLaunchKernelGGL((attn_bf16_kernel<D, Keys>), dim3(static_cast<unsigned>(t.grid)),
                       dim3(kThreads), 0, s, p, keys, 0, 0);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || t.parts == 0) return e;
  const long pairs = static_cast<long>(a.total_block) * a.hq;
  const long heads = std::max(1L, std::min(pairs / kMergeWaves, 8L));  // per wave
  const int per_row = static_cast<int>((a.hq + heads - 1) / heads);
  const long waves = static_cast<long>(a.total_block) * per_row;
  hipLaunchKernelGGL(attn_tiles_merge_kernel<D>,
                     dim3(static_cast<unsigned>((waves + kThreads / 64 - 1) / (kThreads / 64))),
                     dim3(kThreads), 0, s, p, keys.plan, a.total_block, per_row);
  return hipGetLastError();
}

}  // namespace

long attn_paged_threads(bool bf16, const PagedAttnArgs& a) {
  if (a.total_block == 0 || a.max_block == 0) return 0;
  const long group = a.hq / a.kv.hkv, rows = a.max_block * group;
  const long merge = static_cast<long>(a.total_block) * a.hq * 64;  // a wave per query row
  if (!bf16) {
    const SplitPlan sp = f32_plan(a);
    const long tiles = (rows + kPf32Rows - 1) / kPf32Rows;
    return std::max(tiles * sp.nsplit * kPf32Waves * 64, sp.nsplit > 1 ? merge : 0);
  }
  long most = 0;
  const long few = few_rows(a);
  if (few > 0) {
    const FewPlan f = few_plan(a, few);
    most = std::max((static_cast<long>(f.groups) * a.kv.hkv + 7) * f.row_tiles * kFewWaves * 64,
               f.slots ? static_cast<long>(a.batch) * a.kv.hkv * f.row_tiles * 512 : 0);
    if (few == rows) return most;
  }
  const TilesLaunch t = tiles_plan(a, few);
  return std::max(most, std::max(t.grid * kThreads, t.parts ? merge : 0));
}

size_t attn_paged_ws_bytes(bool bf16, const PagedAttnArgs& a) {
  if (a.total_block == 0 || a.max_block == 0) return 0;
  if (bf16) {  // one launch after the other, in the same memory
    const long few = few_rows(a);
    const size_t row = (a.kv.head_dim + 2) * sizeof(float);
    const size_t bytes = few ? few_plan(a, few).slots * row : 0;
    if (few == static_cast<long>(a.max_block) * (a.hq / a.kv.hkv)) return bytes;
    const TilesLaunch t = tiles_plan(a, few);
    const size_t found = t.plan.cap ? kFoundPlan : t.plan.run ? a.batch : 0;
    return std::max(bytes, t.parts * kRowsPerWg * row + found * sizeof(int32_t));
  }
  const SplitPlan sp = f32_plan(a);
  if (sp.nsplit == 1) return 0;
  return static_cast<size_t>(a.total_block) * a.hq * sp.nsplit * (a.kv.head_dim + 2) *
         sizeof(float);
}

hipError_t attn_paged(bool bf16, const PagedAttnArgs& a, void* ws, hipStream_t s) {
  if (a.total_block == 0 || a.max_block == 0) return hipSuccess;
  const bool e4m3 = a.kv.type == CacheType::kE4m3, d128 = a.kv.head_dim == 128;
  if (!bf16) {
    if (d128) return e4m3 ? launch_f32<128, uint8_t>(a, ws, s) : launch_f32<128, float>(a, ws, s);
    return e4m3 ? launch_f32<64, uint8_t>(a, ws, s) : launch_f32<64, float>(a, ws, s);
  }
  const long few = few_rows(a);
  if (few > 0) {
    const hipError_t e =
        d128 ? launch_few_any<128>(a, few, ws, s) : launch_few_any<64>(a, few, ws, s);
    if (e != hipSuccess || few == static_cast<long>(a.max_block) * (a.hq / a.kv.hkv)) return e;
  }
  if (d128)
    return e4m3 ? launch_tiles<128, true>(a, few, ws, s) : launch_tiles<128, false>(a, few, ws, s);
  return e4m3 ? launch_tiles<64, true>(a, few, ws, s) : launch_tiles<64, false>(a, few, ws, s);
}

}  // namespace eb

// The bf16 block-attention kernels of 128 query rows per workgroup, over a packed prefix or a paged
// cache.
#pragma once

#include "attn_common.hpp"
#include "attn_partials.hpp"
#include "attn_small.hpp"
#include "eb_common.hpp"
#include "paged.hpp"

namespace eb {
namespace {

constexpr int kThreads = 256;   // 4 waves
constexpr int kRowsPerWg = kAttnRowsPerWg;
constexpr int kKeys = kAttnKeys;
constexpr int kXcdCount = 8;  // XCDs of the chip (workgroups are dealt to them round-robin)

// Where the cached keys and values lie: packed rows (the prefix and suffix segments of AttnParams),
// or pages.  With pages the cached rows are padded to whole stages, so that a stage lies either in
// the cache or in the block: the block's first key is `cached` below, a stage of the cache may have
// fewer than 64 keys, and nothing is read for the others.
struct PackedKeys {
  static constexpr bool kPaged = false, kE4m3 = false;
};
// Page numbers of one sequence: the wave holds 64 entries of its row of the table, a lane each, and
// the 64 behind them on their way, so that taking one costs no memory access.  Entries are asked
// for in rising order, and none is left out by a whole window.
struct PageWindow {
  const int32_t* row;
  int last, first, now, next;  // last entry of the row; entries first .. first + 63 and the next 64
  __device__ __forceinline__ void start(const PagedKv& kv, int b, int entry, int lane) {
    row = kv.table + static_cast<size_t>(b) * kv.max_pages;
    last = kv.max_pages - 1;
    first = entry;
    now = row[min(first + lane, last)];
    next = row[min(first + 64 + lane, last)];
  }
  // makes entries up to `entry` (uniform) available
  __device__ __forceinline__ void advance(int entry, int lane) {
    if (entry - first < 64) return;
    first += 64;
    now = next;
    next = row[min(first + 64 + lane, last)];
  }
  __device__ __forceinline__ int uniform(int entry) const {
    return __builtin_amdgcn_readlane(now, entry - first);
  }
};

// Key ranges of a launch over pages.  A sequence's stages (its cached rows, then the block's) are
// cut into n_b nearly equal ranges of at most `chunk` stages, and an item is one (range, K/V head,
// tile of query rows); the row tiles of a range are neighbours, so that they run on one XCD at a
// time and share its keys. With cap > 0 every workgroup finds chunk itself, from the lengths, which
// the host does not know: of kPlanCandidates cuts of the longest sequence the cheapest with at most
// cap items, by the rounds of kAttnTargetWgs workgroups and the partials.  (The lanes hold a
// sequence each, so this is for at most 64 of them, and takes a microsecond.)  Against as many
// ranges for every sequence as fill the chip when all are as long as the longest: 28/4 heads x 128,
// 16 blocks of 32 to 256 rows behind 2000 to 16000, 576 -> 453 us; 8 of 20 to 100 behind 1000 to
// 8000, 71 -> 60 us; 16/4 heads x 64, the same, 49 -> 32 us.  Equal lengths gain nothing (32 heads,
// 1000 rows behind 3000: 89 and 91 us).  Where whole sequences make more than one round of
// workgroups, the alternative is to leave those of the full rounds whole, and to cut the few of the
// last round into as many ranges as make it full: few partials, and no round half empty.  A chunk
// of 2500 rows behind 8000, 28/4 heads, 440 -> 369 us; 2 of 1000 to 2048 behind 7001 to 12000
// 507 -> 458 us; 18 blocks of 100 to 128 behind 1500, 32 heads, 8 bits, 142 -> 115 us; taken
// always, unlike lengths suffer (5 of 300 to 500 behind 500 to 9000, 32 heads: 211 against 282 us),
// so the costs decide here too.
// With cap = 0 chunk is the host's; then either every sequence counts as the longest, with as many
// row tiles, and many a workgroup may find nothing to do, or (run > 0) the items are counted off,
// and a workgroup finds its own by a scan over the lengths.
struct TilePlan {
  int batch, row_tiles;
  int skip;  // sequences of at most this many query rows per K/V head have no items
  int cap;
  int chunk, nsplit;  // cap = 0: stages per range, ranges per sequence
  int run;            // > 0: items counted off, dealt to the XCDs in runs of so many
  int most;           // run > 0: items that may leave partials
  float* o_part;      // [items, kRowsPerWg, D], then m and l [items, kRowsPerWg]
  float* m_part;
  float* l_part;
  // cap > 0: of each of kPlanMaxBatch sequences its first item, then its ranges, then a LastRound;
  // run > 0: of each sequence of more than `chunk` stages its first item, or -1 if it stayed whole
  int32_t* found;
};
template <bool kBits8>
struct PagedKeys {
  static constexpr bool kPaged = true, kE4m3 = kBits8;
  PagedKv kv;
  TilePlan plan;
};
constexpr int kPlanMaxBatch = 64;
constexpr int kPlanCandidates = 32;
// Costs in stages of one of two workgroups of a compute unit: of a last round that leaves each
// compute unit one (which is the faster for it), of a workgroup's start and end, of the merge's
// launch, and of one row's partial, written and read.
constexpr float kPlanHalf = 0.65f, kPlanRange = 3.f, kPlanMerge = 2.f, kPlanRow = 1.f / 8192;

// Stages and row tiles of a sequence.
__device__ __forceinline__ int tile_stages(int plen, int len) {
  return len > 0 ? (plen + kKeys - 1) / kKeys + (len + kKeys - 1) / kKeys : 0;
}
__device__ __forceinline__ int tile_rows(int len, int group) {
  return (len * group + kRowsPerWg - 1) / kRowsPerWg;
}
// Parts of the longest sequence that candidate j stands for: 1 .. 16, 20 .. 48, 64 .. 176.
__device__ __forceinline__ int plan_parts(int j) {
  return j < 16 ? j + 1 : j < 24 ? 16 + 4 * (j - 15) : 48 + 16 * (j - 23);
}

// Block rows of a sequence, as far as they have items here.
__device__ __forceinline__ int tile_len(const AttnParams& p, const TilePlan& tp, int b) {
  const int len = p.cu_block[b + 1] - p.cu_block[b];
  return len * p.group > tp.skip ? len : 0;
}

// More items than one round has workgroups: the first `full` stay whole, each of the `rest` behind
// them is cut into (at most) `ranges`.
struct LastRound {
  int full, rest, ranges;
};
constexpr int kFoundPlan = 2 * kPlanMaxBatch + sizeof(LastRound) / sizeof(int);
// The lengths of a wave's sequences (lane = sequence) and the cut they get.
struct LanePlan {
  int ranges, items, upto;  // of the lane's sequence; upto: items of all up to it
  int total;
  int stages;
  LastRound last;  // full > 0: in place of the sequences' ranges
};
__device__ __forceinline__ LanePlan lane_plan(const AttnParams& p, const TilePlan& tp, int lane) {
  const int own = min(lane, tp.batch - 1);
  const int len = lane < tp.batch ? tile_len(p, tp, own) : 0;
  const int stages = tile_stages(p.cu_prefix[own + 1] - p.cu_prefix[own], len);
  const int per_range = tile_rows(len, p.group) * p.hkv;
  const int longest = max(lanes_all(stages, 0, MaxOp{}), 1);
  const int whole = lanes_all(per_range, 0, AddOp{});
  const int rows = lanes_all(len * p.group, 0, AddOp{});
  // A lane per candidate, twice: lanes 0-31 add up the even sequences' items, 32-63 the odd ones'.
  const int parts = plan_parts(lane % kPlanCandidates);
  int chunk = (longest + parts - 1) / parts;
  const float inv = 1.0f / chunk;
  int items = 0;
  for (int b = 0; b < tp.batch; b += 2) {
    const int st0 = __builtin_amdgcn_readlane(stages, b);
    const int st1 = __builtin_amdgcn_readlane(stages, b + 1);
    const int per0 = __builtin_amdgcn_readlane(per_range, b);
    const int per1 = __builtin_amdgcn_readlane(per_range, b + 1);
    // ceil(st / chunk) = floor((st - 1) / chunk) + 1
    const float st = static_cast<float>(lane < kPlanCandidates ? st0 : st1) - 0.5f;
    items += (static_cast<int>(st * inv) + 1) * (lane < kPlanCandidates ? per0 : per1);
  }
  items += __shfl_xor(items, kPlanCandidates);
  const int rest = items % kAttnTargetWgs;
  float cost = items / kAttnTargetWgs +
               (rest == 0 ? 0.f : rest <= kAttnTargetWgs / 2 ? kPlanHalf : 1.f);
  cost *= chunk + kPlanRange;
  if (parts > 1)
    cost += kPlanMerge + static_cast<float>(items) * rows * p.hkv / max(whole, 1) * kPlanRow;
  if (items > tp.cap) cost = 1e30f;
  // the cheapest, of equals the one with fewer parts (costs are positive: their bits order them)
  const int least = lanes_all(__float_as_int(cost), 0x7fffffff, MinOp{});
  const uint64_t win = __ballot(__float_as_int(cost) == least);
  chunk = __builtin_amdgcn_readlane(chunk, __builtin_ctzll(win));
  LanePlan l;
  auto cut = [&](int by) {
    l.ranges = (stages + by - 1) / by;
    l.items = l.ranges * per_range;
    l.upto = lanes_up_to(l.items, 0, AddOp{});
    l.total = __builtin_amdgcn_readlane(l.upto, 63);
  };
  cut(chunk);
  l.stages = stages;
  l.last = LastRound{};
  if (whole > kAttnTargetWgs) {
    const int full = whole / kAttnTargetWgs, rest = whole - full * kAttnTargetWgs;
    const int ranges = max(kAttnTargetWgs / max(rest, 1), 1);
    const float last = static_cast<float>(longest) / ranges + kPlanRange + kPlanMerge +
                       kAttnTargetWgs * kRowsPerWg * kPlanRow;
    if (full * (longest + kPlanRange) + (rest ? last : 0.f) < __int_as_float(least)) {
      cut(longest);
      l.last = LastRound{full * kAttnTargetWgs, rest, ranges};
    }
  }
  if (l.total > tp.cap) cut(longest);  // (a count in floats was off: whole sequences always fit)
  return l;
}

// First stage of a range.
__device__ __forceinline__ int range_start(int stages, int range, int ranges) {
  const int each = stages / ranges, more = stages % ranges;
  return range * each + min(range, more);
}

// One workgroup's item.
struct TileItem {
  int b, g, tile, item, range, ranges;
};
// Item number `local` of a sequence.
__device__ __forceinline__ void place_item(TileItem& it, int local, int row_tiles, int hkv) {
  it.tile = local % row_tiles;
  it.g = local / row_tiles % hkv;
  it.range = local / row_tiles / hkv;
}
// An item counted off (run > 0), by the whole wavefront.
__device__ __forceinline__ bool count_off(const AttnParams& p, const TilePlan& tp, int xcd, int j,
                                          int lane, int wave, TileItem& it) {
  it.item = (j / tp.run * kXcdCount + xcd) * tp.run + j % tp.run;
  int first = 0, b = tp.batch, row_tiles = 1;
  int cut = 0;  // items so far if every sequence is cut
  bool whole = false;
  for (int b0 = 0; b0 < tp.batch; b0 += 64) {
    const int own = min(b0 + lane, tp.batch - 1);
    const int len = b0 + lane < tp.batch ? tile_len(p, tp, own) : 0;
    const int stages = tile_stages(p.cu_prefix[own + 1] - p.cu_prefix[own], len);
    const int tiles = tile_rows(len, p.group);
    int ranges = (stages + tp.chunk - 1) / tp.chunk;
    if (tp.nsplit > 1) {  // (uniform) sequences are cut while the partials' places last
      const int upto = cut + lanes_up_to(ranges * tiles * p.hkv, 0, AddOp{});
      cut = __builtin_amdgcn_readlane(upto, 63);
      if (upto > tp.most) ranges = min(ranges, 1);
    }
    const int n = ranges * tiles * p.hkv;
    const int upto = lanes_up_to(n, 0, AddOp{});
    const uint64_t past = __ballot(first + upto > it.item);
    if (past) {
      const int l = __builtin_ctzll(past);
      first += __builtin_amdgcn_readlane(upto - n, l);
      b = b0 + l;
      it.ranges = __builtin_amdgcn_readlane(ranges, l);
      whole = it.ranges == 1 && __builtin_amdgcn_readlane(stages, l) > tp.chunk;
      row_tiles = __builtin_amdgcn_readlane(tiles, l);
      break;
    }
    first += __builtin_amdgcn_readlane(upto, 63);
  }
  if (b >= tp.batch) return false;
  it.b = __builtin_amdgcn_readfirstlane(b);
  place_item(it, it.item - first, row_tiles, p.hkv);
  if (it.item == first && (it.ranges > 1 || whole) && wave == 0 && lane == 0)  // for the merge
    tp.found[b] = whole ? -1 : first;
  return true;
}
// The item of this workgroup; false if there is none.
__device__ __forceinline__ bool find_item(const AttnParams& p, const TilePlan& tp, int lane,
                                          int wave, TileItem& it) {
  const int xcd = blockIdx.x % kXcdCount, j = blockIdx.x / kXcdCount;
  if (tp.run > 0) return count_off(p, tp, xcd, j, lane, wave, it);
  if (tp.cap == 0) {
    const int unit = kXcdCount * (j / tp.row_tiles) + xcd;
    it.tile = j % tp.row_tiles;
    it.g = unit % p.hkv;
    it.range = unit / p.hkv % tp.nsplit;
    it.b = unit / p.hkv / tp.nsplit;
    it.item = unit * tp.row_tiles + it.tile;
    if (it.b >= tp.batch) return false;
    const int stages =
        tile_stages(p.cu_prefix[it.b + 1] - p.cu_prefix[it.b], tile_len(p, tp, it.b));
    it.ranges = (stages + tp.chunk - 1) / tp.chunk;
    return it.range < it.ranges;
  }
  // The items in 8 turns equal runs, dealt to the XCDs in turn: runs of at least as many items as
  // the longest block has row tiles, for the sharing.  turns divides 64, so that an XCD gets no
  // more items than its share of the cap.
  const LanePlan l = lane_plan(p, tp, lane);
  const LastRound last = l.last;
  if (blockIdx.x == 0 && wave == 0) {  // for the merge
    tp.found[lane] = l.upto - l.items;
    tp.found[kPlanMaxBatch + lane] = l.ranges;
    if (lane == 0) *reinterpret_cast<LastRound*>(tp.found + 2 * kPlanMaxBatch) = last;
  }
  // (the full rounds by themselves, in runs of a power of two of items, 64 at most, as an XCD has
  // 64 workgroups at a time)
  const int in_full = last.full / kXcdCount, at = j - in_full;
  const int total = last.full ? last.rest * last.ranges : l.total;
  if (at < 0) {
    int run = 64;
    while (run >= 2 * tp.row_tiles) run /= 2;
    it.item = (j / run * kXcdCount + xcd) * run + j % run;
  } else {
    int turns = 1;
    while (turns < 64 && 2 * turns * kXcdCount * tp.row_tiles <= total) turns *= 2;
    const int runs = turns * kXcdCount, most = max((total + runs - 1) / runs, 1);
    const int run = at / most * kXcdCount + xcd;
    const int n = run * total / runs + at % most;
    if (run >= runs || n >= (run + 1) * total / runs) return false;
    it.item = last.full + n;
  }
  const int whole = at < 0 || !last.full ? it.item : last.full + (it.item - last.full) % last.rest;
  const int b = __builtin_ctzll(__ballot(l.upto > whole));
  const int local = whole - __builtin_amdgcn_readlane(l.upto - l.items, b);
  const int row_tiles = tile_rows(p.cu_block[b + 1] - p.cu_block[b], p.group);
  it.b = b;
  place_item(it, local, row_tiles, p.hkv);
  it.ranges = __builtin_amdgcn_readlane(l.ranges, b);
  if (at >= 0 && last.full) {
    it.range = (it.item - last.full) / last.rest;
    it.ranges = min(last.ranges, __builtin_amdgcn_readlane(l.stages, b));
  }
  return it.range < it.ranges;
}

// Two workgroups per compute unit (<= 256 VGPRs per lane, no spills at D = 128), so one
// wave's softmax arithmetic overlaps another wave's MFMAs on the same SIMD (batch 64 at
// D = 128: 1.85 ms with one workgroup per compute unit, 1.07 ms with two).
//
// The probabilities are rounded to bf16 for the product with V, the MFMA's type; l sums them
// unrounded, in fp32.  Over pages at D = 64 the result's distance from 64 bits (2-norm) is then
// 0.0020 of it, 0.00166 with the output's rounding alone.  A second bf16 for the rest of each
// probability, as in the kernel for few rows, takes that away and costs 10 to 27% here, over pages
// (16/4 heads, 32 blocks of 16 to 128 behind 2048 71 -> 86 us, 2 chunks behind 7001 and 12000 301
// -> 382): not kept.
template <int D, class Keys>
__global__ __launch_bounds__(kThreads, 2) void attn_bf16_kernel(AttnParams p, Keys keys,
                                                                int row_tiles, int units) {
  constexpr int kKRow = D + 8;       // K tile pitch (bf16)
  constexpr int kVRow = kKeys + 8;   // V^T tile pitch (bf16): 144-byte rows, 16-byte aligned
  constexpr int kDSteps = D / 16;    // MFMA k-steps over the head dimension
  constexpr int kDBlocks = D / 32;   // 32-row blocks of O^T
  __shared__ __attribute__((aligned(16))) uint16_t Ks[kKeys * kKRow];
  __shared__ __attribute__((aligned(16))) uint16_t Vt[D * kVRow];

  // Workgroup id -> (unit, row tile) so that the row tiles of one unit (sequence, K/V head, key
  // range) all run on one XCD, one after another: workgroups are dealt to the 8 XCDs round-robin
  // by id, and the tiles of unit u take ids 8 (row_tiles (u / 8) + tile) + u % 8.  They then read
  // the unit's K/V stages from that XCD's L2 instead of each XCD fetching them.
  [[maybe_unused]] TileItem it;
  int b, g, sp, tile;
  if constexpr (Keys::kPaged) {
    if (!find_item(p, keys.plan, threadIdx.x & 63,
                   __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), it))
      return;  // whole workgroup
    b = it.b, g = it.g, sp = it.range, tile = it.tile;
  } else {
    const int xcd = blockIdx.x % kXcdCount, j = blockIdx.x / kXcdCount;
    const int unit = kXcdCount * (j / row_tiles) + xcd;
    if (unit >= units) return;  // whole workgroup: padding of the last round
    tile = j % row_tiles;
    const int z = unit / p.hkv;
    b = z / p.nsplit;
    sp = z % p.nsplit;
    g = unit % p.hkv;
  }
  const int G = p.group;
  const int bbeg = p.cu_block[b];
  const int len = p.cu_block[b + 1] - bbeg;
  const int pbeg = p.cu_prefix[b];
  const int plen = p.cu_prefix[b + 1] - pbeg;
  const int n_rows = len * G;
  const int row0 = tile * kRowsPerWg;
  if (row0 >= n_rows) return;  // whole workgroup: this tile lies past the block
  const int sbeg = p.cu_suffix ? p.cu_suffix[b] : 0;
  const int slen = p.cu_suffix ? p.cu_suffix[b + 1] - sbeg : 0;
  const int cached = Keys::kPaged ? (plen + kKeys - 1) / kKeys * kKeys : plen;
  const int n_keys = cached + len + slen;
  int kbeg = sp * p.kps, kend = kbeg + p.kps;
  if constexpr (Keys::kPaged) {
    const int stages = tile_stages(plen, len);
    kbeg = range_start(stages, it.range, it.ranges) * kKeys;
    kend = range_start(stages, it.range + 1, it.ranges) * kKeys;
  }
  if (kbeg >= n_keys) return;  // whole workgroup: this key range lies past the sequence
  kend = min(n_keys, kend);

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int half = lane >> 5, l32 = lane & 31;

  // This lane's query row.
  const int myrow = row0 + wave * 32 + l32;
  const bool row_ok = myrow < n_rows;
  const int rr = row_ok ? myrow : 0;
  const int pos = rr / G, hh = rr % G;
  const size_t q_off = (static_cast<size_t>(bbeg + pos) * p.hq + g * G + hh) * D;

  // Q^T fragments (B operand): step s, half hf holds d = 16 s + 8 hf .. +7.
  bf16x8 qf[kDSteps];
#pragma unroll
  for (int s = 0; s < kDSteps; ++s)
    qf[s] = *reinterpret_cast<const bf16x8*>(p.q + q_off + 16 * s + 8 * half);

  f32x16 o[kDBlocks];
#pragma unroll
  for (int db = 0; db < kDBlocks; ++db) o[db] = f32x16{};
  // with pages from the lowest finite value on: scores of -inf then have weights of zero
  float m_run = Keys::kPaged ? kNegBig : -INFINITY, l_run = 0.f;
  // where the keys that the stage at kv0 may hold end
  auto end_of = [&](int kv0) { return Keys::kPaged && kv0 < cached ? plen : kend; };

  // Loader assignments.  K: 16-byte chunks, chunk c = key c / (D/8), columns 8 (c % (D/8)).
  constexpr int kKChunks = kKeys * (D / 8);
  constexpr int kKPer = kKChunks / kThreads;
  // V: thread handles keys 2 kp, 2 kp + 1 (kp = tid % 32) and d range [dg * D/8, +D/8).
  const int kp = tid & 31, dg = tid >> 5;
  constexpr int kVd = D / 8;

  // key j of the sequence: prefix rows, then block rows, then suffix rows (an unordered set)
  auto key_src = [&](int j, const uint16_t* pre, const uint16_t* blk,
                     const uint16_t* suf) -> const uint16_t* {
    if (j < plen) return pre + (static_cast<size_t>(pbeg + j) * p.hkv + g) * D;
    if (j < plen + len) return blk + (static_cast<size_t>(bbeg + j - plen) * p.hkv + g) * D;
    return suf + (static_cast<size_t>(sbeg + j - plen - len) * p.hkv + g) * D;
  };

  // Loads are unconditional with clamped key indices (a conditional load would be waited for
  // on the spot); keys past the end are replaced by zeros when stored to LDS.
  u32x4 kreg[kKPer];
  u32x4 vreg[2][kVd / 8];
  const int key_stride = p.hkv * D;  // elements between consecutive keys of one K/V head
  [[maybe_unused]] PageWindow window;
  [[maybe_unused]] uint32_t kscale[kKPer], vscale[2];  // of the rows of an 8-bit cache
  [[maybe_unused]] uint32_t gone;  // bit i: row i of kreg, then of vreg, does not exist
  [[maybe_unused]] bool bits8;     // the stage in kreg and vreg holds 8-bit values
  if constexpr (Keys::kPaged) window.start(keys.kv, b, kbeg >> keys.kv.page_shift, lane);
  auto gload = [&](int kv0) {
    if constexpr (Keys::kPaged) {
      gone = 0;
      bits8 = Keys::kE4m3 && kv0 < cached;
      if (kv0 >= cached) {
        const int j0 = kv0 - cached;
        auto load = [&](int i, int key, const uint16_t* base, int col) {
          if (j0 + key >= len) gone |= 1u << i;
          const int j = min(j0 + key, len - 1);
          return *reinterpret_cast<const u32x4*>(
              base + (static_cast<size_t>(bbeg + j) * p.hkv + g) * D + col);
        };
#pragma unroll
        for (int i = 0; i < kKPer; ++i) {
          const int c = tid + i * kThreads;
          kreg[i] = load(i, c / (D / 8), p.k_blk, (c % (D / 8)) * 8);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int c = 0; c < kVd / 8; ++c)
            vreg[e][c] = load(kKPer + e, 2 * kp + e, p.v_blk, dg * kVd + 8 * c);
        return;
      }
      const PagedKv& kv = keys.kv;
      // (a range starts at a whole stage, so a window holds all pages of a stage or none)
      window.advance(kv0 >> kv.page_shift, lane);
      // pool row of position kv0 + key; a row that is none of the cache's comes from page 0
      auto row_of = [&](int i, int key) {
        const int at = kv0 + key;
        const int page = __shfl(window.now, (at >> kv.page_shift) - window.first);
        const bool ok =
            at < plen && static_cast<unsigned>(page) < static_cast<unsigned>(kv.n_pages);
        if (!ok) gone |= 1u << i;
        return ((static_cast<size_t>(ok ? page : 0) * p.hkv + g) << kv.page_shift) +
               (at & ((1 << kv.page_shift) - 1));
      };
      auto load = [&](const uint8_t* pool, size_t row, int col) -> u32x4 {
        if constexpr (Keys::kE4m3) {
          const u32x2 w = *reinterpret_cast<const u32x2*>(pool + row * D + col);
          return u32x4{w[0], w[1], 0, 0};
        } else {
          return *reinterpret_cast<const u32x4*>(pool + (row * D + col) * 2);
        }
      };
#pragma unroll
      for (int i = 0; i < kKPer; ++i) {
        const int c = tid + i * kThreads;
        const size_t row = row_of(i, c / (D / 8));
        kreg[i] = load(kv.k, row, (c % (D / 8)) * 8);
        if constexpr (Keys::kE4m3) kscale[i] = kv.k_scale[row];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const size_t row = row_of(kKPer + e, 2 * kp + e);
#pragma unroll
        for (int c = 0; c < kVd / 8; ++c) vreg[e][c] = load(kv.v, row, dg * kVd + 8 * c);
        if constexpr (Keys::kE4m3) vscale[e] = kv.v_scale[row];
      }
      return;
    }
    if (kv0 + kKeys <= plen) {
      // the whole stage lies in the prefix: one base pointer per tensor, no per-key segment choice
      const size_t base = (static_cast<size_t>(pbeg + kv0) * p.hkv + g) * D;
      const uint16_t* kb = p.k_pre + base;
      const uint16_t* vb = p.v_pre + base;
#pragma unroll
      for (int i = 0; i < kKPer; ++i) {
        const int c = tid + i * kThreads;
        const int key = c / (D / 8), col = (c % (D / 8)) * 8;
        kreg[i] = *reinterpret_cast<const u32x4*>(kb + key * key_stride + col);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int c = 0; c < kVd / 8; ++c)
          vreg[e][c] = *reinterpret_cast<const u32x4*>(vb + (2 * kp + e) * key_stride +
                                                       dg * kVd + 8 * c);
      return;
    }
#pragma unroll
    for (int i = 0; i < kKPer; ++i) {
      const int c = tid + i * kThreads;
      const int key = c / (D / 8), col = (c % (D / 8)) * 8;
      const int j = min(kv0 + key, kend - 1);
      kreg[i] = *reinterpret_cast<const u32x4*>(key_src(j, p.k_pre, p.k_blk, p.k_suf) + col);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int j = min(kv0 + 2 * kp + e, kend - 1);
#pragma unroll
      for (int c = 0; c < kVd / 8; ++c)
        vreg[e][c] = *reinterpret_cast<const u32x4*>(key_src(j, p.v_pre, p.v_blk, p.v_suf) +
                                                     dg * kVd + 8 * c);
    }
  };
  // Keys past the end were loaded from a clamped (valid) row: finite values whose scores are
  // masked to -inf below, so their probabilities are exactly 0 and they add nothing to O.
  auto sstore = [&]() {
    if constexpr (Keys::kPaged) {
      // 8 bits to bf16; rows that do not exist to zeros (whatever a page holds there)
      auto widen = [](u32x4& w, float scale) {
        w = u32x4{e4m3_pair_bf16<false>(w[0], scale), e4m3_pair_bf16<true>(w[0], scale),
                  e4m3_pair_bf16<false>(w[1], scale), e4m3_pair_bf16<true>(w[1], scale)};
      };
      if (Keys::kE4m3 && bits8) {
#pragma unroll
        for (int i = 0; i < kKPer; ++i) widen(kreg[i], e8m0(kscale[i]));
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int c = 0; c < kVd / 8; ++c) widen(vreg[e][c], e8m0(vscale[e]));
      }
      if (__any(gone != 0)) {
#pragma unroll
        for (int i = 0; i < kKPer; ++i)
          if (gone >> i & 1) kreg[i] = u32x4{};
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int c = 0; c < kVd / 8; ++c)
            if (gone >> (kKPer + e) & 1) vreg[e][c] = u32x4{};
      }
    }
#pragma unroll
    for (int i = 0; i < kKPer; ++i) {
      const int c = tid + i * kThreads;
      const int key = c / (D / 8), col = (c % (D / 8)) * 8;
      *reinterpret_cast<u32x4*>(Ks + key * kKRow + col) = kreg[i];
    }
    // V^T: the 16-bit values of keys 2 kp and 2 kp + 1 at one d form one 32-bit word.  Within
    // each 16-key group, key w sits at column 8 ((w / 4) % 2) + 4 (w / 8) + w % 4, so the eight
    // keys one lane contracts over in an MFMA (4 half + 0..3 and 8 + 4 half + 0..3) are
    // contiguous; keys 2 kp and 2 kp + 1 stay adjacent.
    const int w16 = (2 * kp) & 15;
    const int vcol = (2 * kp - w16) + 8 * ((w16 >> 2) & 1) + 4 * (w16 >> 3) + (w16 & 3);
#pragma unroll
    for (int c = 0; c < kVd / 8; ++c)
#pragma unroll
      for (int w4 = 0; w4 < 4; ++w4) {
        const int d = dg * kVd + 8 * c + 2 * w4;
        const uint32_t k0 = vreg[0][c][w4], k1 = vreg[1][c][w4];
        *reinterpret_cast<uint32_t*>(Vt + d * kVRow + vcol) =
            __builtin_amdgcn_perm(k1, k0, 0x05040100u);  // low halves: value at d
        *reinterpret_cast<uint32_t*>(Vt + (d + 1) * kVRow + vcol) =
            __builtin_amdgcn_perm(k1, k0, 0x07060302u);  // high halves: value at d + 1
      }
  };

  const int n_stages = (kend - kbeg + kKeys - 1) / kKeys;
  gload(kbeg);
  for (int st = 0; st < n_stages; ++st) {
    const int kv0 = kbeg + st * kKeys;
    __syncthreads();  // previous stage's LDS reads are done
    sstore();
    __syncthreads();
    if (st + 1 < n_stages) gload(kv0 + kKeys);

    // S^T for two 32-key blocks: acc[kb][r] = S[query l32][key kb*32 + 8(r/4) + 4 half + r%4]
    f32x16 sacc[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      sacc[kb] = f32x16{};
#pragma unroll
      for (int s = 0; s < kDSteps; ++s) {
        const bf16x8 kf =
            *reinterpret_cast<const bf16x8*>(Ks + (kb * 32 + l32) * kKRow + 16 * s + 8 * half);
        sacc[kb] = mfma32(kf, qf[s], sacc[kb]);
      }
    }
    // raw scores; keys past the end (last stage only) masked to -inf
    const int end = end_of(kv0);
    if (kv0 + kKeys > end) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = kv0 + kb * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
          if (key >= end) sacc[kb][r] = -INFINITY;
        }
    }
    float mloc = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mloc = fmaxf(mloc, sacc[kb][r]);
    mloc = fmaxf(mloc, __shfl_xor(mloc, 32));
    // scale > 0, so max(scale * s) = scale * max(s); e = 2^(scale s - m) with one FMA
    const float m_new = fmaxf(m_run, mloc * p.scale_log2);
    const float alpha = fast_exp2(m_run - m_new);
    m_run = m_new;
    float lsum = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = fast_exp2(fmaf(sacc[kb][r], p.scale_log2, -m_new));
        sacc[kb][r] = e;
        lsum += e;
      }
    l_run = l_run * alpha + lsum;
    if (__any(alpha != 1.0f)) {  // some row's running max moved (alpha = 1 leaves O as it is)
#pragma unroll
      for (int db = 0; db < kDBlocks; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
    }

    // O^T += V^T P^T.  MFMA u of key block kb covers keys kb*32 + 16u + {4 half + 0..3,
    // 8 + 4 half + 0..3}, which are exactly accumulator registers 8u .. 8u+7 of sacc[kb].
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 pb;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          pb[e] = pack2_bf16(sacc[kb][8 * u + 2 * e], sacc[kb][8 * u + 2 * e + 1]);
        const bf16x8 pf = __builtin_bit_cast(bf16x8, pb);
        const int kbase = kb * 32 + 16 * u + 8 * half;  // the lane's 8 keys, contiguous
#pragma unroll
        for (int db = 0; db < kDBlocks; ++db) {
          const bf16x8 va =
              *reinterpret_cast<const bf16x8*>(Vt + (db * 32 + l32) * kVRow + kbase);
          o[db] = mfma32(va, pf, o[db]);
        }
      }
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32);
  if (!row_ok) return;
  if (Keys::kPaged ? it.ranges > 1 : p.nsplit > 1) {
    float *o_part = p.o_part, *m_part = p.m_part, *l_part = p.l_part;
    size_t idx = (static_cast<size_t>(bbeg + pos) * p.hq + g * G + hh) * p.nsplit + sp;
    if constexpr (Keys::kPaged) {
      idx = static_cast<size_t>(it.item) * kRowsPerWg + wave * 32 + l32;
      o_part = keys.plan.o_part, m_part = keys.plan.m_part, l_part = keys.plan.l_part;
    }
    float* dst = o_part + idx * D;
#pragma unroll
    for (int db = 0; db < kDBlocks; ++db)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int d = db * 32 + 8 * q4 + 4 * half;
        *reinterpret_cast<f32x4*>(dst + d) =
            f32x4{o[db][4 * q4 + 0], o[db][4 * q4 + 1], o[db][4 * q4 + 2], o[db][4 * q4 + 3]};
      }
    if (half == 0) {
      m_part[idx] = m_run;
      l_part[idx] = l_tot;
    }
    return;
  }
  const float inv = 1.0f / l_tot;
  uint16_t* dst = p.out + q_off;
#pragma unroll
  for (int db = 0; db < kDBlocks; ++db)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const int d = db * 32 + 8 * q4 + 4 * half;
      const u32x2 v{pack2_bf16(o[db][4 * q4 + 0] * inv, o[db][4 * q4 + 1] * inv),
                    pack2_bf16(o[db][4 * q4 + 2] * inv, o[db][4 * q4 + 3] * inv)};
      *reinterpret_cast<u32x2*>(dst + d) = v;
    }
}

// Head dimension 128: the main path of the bf16 block attention.
//
// Staging.  K and V tiles of 64 keys reach LDS by buffer loads straight into LDS (no staging
// registers, no LDS store instructions): waves 0-1 load K tiles, waves 2-3 V tiles, two slots
// each.  K runs one stage ahead of V, so iteration st needs K(st + 1) and V(st) and one barrier
// per iteration suffices: after it, K(st + 2) goes into the slot K(st) left and V(st + 1) into
// the slot V(st - 1) left.  Rows are 256 bytes of 16 sixteen-byte chunks; chunk c of key row r
// sits in slot c ^ (r % 16) for K (the 32-row fragment reads of S^T then touch 16 distinct slots
// per 16 lanes) and in slot c ^ 4 (r % 4) for V (the 4 rows x 4 chunks of a transposing read by
// 16 lanes then touch distinct slots).  A load instruction writes 1 KB, 4 key rows, lane L
// filling slot L % 16 of row L / 16, so each lane fetches the global chunk that lands there.
//
// Schedule.  Iteration st issues the 16 MFMAs of S(st + 1) = K(st + 1) Q^T, each followed by the
// VALU work of one bf16 word (two probabilities) of P(st) from the scores of the previous
// iteration, then the 16 MFMAs of O^T += V(st)^T P(st)^T, each followed by one step of the
// maximum of S(st + 1).  Scheduling barriers keep that interleave, so one wave's exponentials
// run while its matrix pipe works.  V^T fragments come from transposing LDS reads of the
// row-major V tile.  The loop runs two iterations per trip, the score arrays of S(st) and
// S(st + 1) trading places between them, so no scores are copied.
//
// Softmax.  The running maximum m (log2 units) moves only when some row's stage maximum
// exceeds it by more than kAttnSlack, so probabilities 2^(s - m) stay below 2^kAttnSlack and
// O, l are rescaled rarely.  l sums the bf16-rounded probabilities that P V multiplies, two per
// dot instruction.  The final O / l and the split partials (m, l, O) mean the same as in
// attn_bf16_kernel.  With the slack even a row's largest probability is rounded: 0.0023 from 64
// bits (2-norm, packed or paged), 0.00166 with the output's rounding alone.
//
// Registers: 234 vector registers over bf16 pages, 251 over 8 bits, none of them in memory; 24 and
// 30 scalar values do not fit and are kept in lanes of vector registers, some of those of the 8-bit
// form read back in every iteration.
constexpr float kAttnSlack = 8.0f;
constexpr int kDmaKeys = 64;  // keys per tile (the schedule pairs 16 S MFMAs with 16 P words)
static_assert(kDmaKeys == kKeys, "stages of the key-split plan");

template <class Keys>
__global__ __launch_bounds__(kThreads, 2) void attn_bf16_d128_kernel(AttnParams p, Keys keys,
                                                                     int row_tiles, int units) {
  constexpr int D = 128;
  constexpr int kRowBytes = D * 2;
  constexpr int kTileBytes = kDmaKeys * kRowBytes;  // 16 KB
  constexpr int kDSteps = D / 16;                   // MFMA k-steps of S^T over the head dim
  constexpr int kDBlocks = D / 32;                  // 32-row blocks of O^T
  constexpr int kKB = kDmaKeys / 32;                // 32-key blocks per tile
  constexpr int kMfmas = kKB * kDSteps;             // S MFMAs per tile = P V MFMAs per tile
  static_assert(kMfmas == 16 && kKB * 2 * kDBlocks == kMfmas, "schedule");
  constexpr int kInstPerTile = kTileBytes / 1024;            // 1 KB per load instruction
  constexpr int kInstPerWave = 2 * kInstPerTile / (kThreads / 64);
  static_assert(kInstPerTile % kInstPerWave == 0, "a wave loads K or V, not both");
  // K and V fragment reads are issued this many MFMAs ahead (one less where a tile waits in
  // registers: a third would spill)
  constexpr int kPreK = Keys::kE4m3 ? 2 : 3;
  constexpr int kPreV = Keys::kE4m3 ? 2 : 3;
  // K tiles in slots 0, 1; V tiles in slots 2, 3
  __shared__ __attribute__((aligned(16))) uint8_t smem[4 * kTileBytes];

  // Workgroup id -> (unit, row tile) as in attn_bf16_kernel: the row tiles of one unit run on
  // one XCD, one after another, and share that XCD's L2.
  [[maybe_unused]] TileItem it;
  int b, g, sp, tile;
  if constexpr (Keys::kPaged) {
    if (!find_item(p, keys.plan, threadIdx.x & 63,
                   __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), it))
      return;  // whole workgroup
    b = it.b, g = it.g, sp = it.range, tile = it.tile;
  } else {
    const int xcd = blockIdx.x % kXcdCount, jx = blockIdx.x / kXcdCount;
    const int unit = kXcdCount * (jx / row_tiles) + xcd;
    if (unit >= units) return;  // whole workgroup: padding of the last round
    tile = jx % row_tiles;
    const int z = unit / p.hkv;
    b = z / p.nsplit;
    sp = z % p.nsplit;
    g = unit % p.hkv;
  }
  const int G = p.group;
  const int bbeg = p.cu_block[b];
  const int len = p.cu_block[b + 1] - bbeg;
  const int pbeg = p.cu_prefix[b];
  const int plen = p.cu_prefix[b + 1] - pbeg;
  const int n_rows = len * G;
  const int row0 = tile * kRowsPerWg;
  if (row0 >= n_rows) return;  // whole workgroup: this tile lies past the block
  const int sbeg = p.cu_suffix ? p.cu_suffix[b] : 0;
  const int slen = p.cu_suffix ? p.cu_suffix[b + 1] - sbeg : 0;
  const int cached = Keys::kPaged ? (plen + kKeys - 1) / kKeys * kKeys : plen;
  const int n_keys = cached + len + slen;
  int kbeg = sp * p.kps, kend = kbeg + p.kps;
  if constexpr (Keys::kPaged) {
    const int stages = tile_stages(plen, len);
    kbeg = range_start(stages, it.range, it.ranges) * kKeys;
    kend = range_start(stages, it.range + 1, it.ranges) * kKeys;
  }
  if (kbeg >= n_keys) return;  // whole workgroup: this key range lies past the sequence
  kend = min(n_keys, kend);

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // uniform: scalar buffer resources
  const int half = lane >> 5, l32 = lane & 31;

  // This lane's query row.
  const int myrow = row0 + wave * 32 + l32;
  const bool row_ok = myrow < n_rows;
  const int rr = row_ok ? myrow : 0;
  const int pos = rr / G, hh = rr % G;
  const size_t q_off = (static_cast<size_t>(bbeg + pos) * p.hq + g * G + hh) * D;

  // Q^T fragments (B operand): step s, half hf holds d = 16 s + 8 hf .. +7.
  bf16x8 qf[kDSteps];
#pragma unroll
  for (int s = 0; s < kDSteps; ++s)
    qf[s] = *reinterpret_cast<const bf16x8*>(p.q + q_off + 16 * s + 8 * half);

  f32x16 o[kDBlocks];
#pragma unroll
  for (int db = 0; db < kDBlocks; ++db) o[db] = f32x16{};
  // with pages from the lowest finite value on: scores of -inf then have weights of zero
  float m_run = Keys::kPaged ? kNegBig : -INFINITY, l_run = 0.f;
  // where the keys that the stage at kv0 may hold end
  auto end_of = [&](int kv0) { return Keys::kPaged && kv0 < cached ? plen : kend; };

  // Loads: per segment (prefix, block, suffix) a buffer resource at the segment's first key of
  // head g; key j of a segment lies j * key_bytes further.  Instruction i of a wave covers tile
  // rows 4 n .. 4 n + 3, n = (wave * kInstPerWave + i) % kInstPerTile.
  const bool k_wave = wave * kInstPerWave < kInstPerTile;  // wave-uniform
  const uint32_t key_bytes = static_cast<uint32_t>(p.hkv) * kRowBytes;
  // (an empty prefix or suffix segment, never read, takes the block's resource)
  const uint16_t* blk0 = (k_wave ? p.k_blk : p.v_blk) + (static_cast<size_t>(bbeg) * p.hkv + g) * D;
  const __amdgpu_buffer_rsrc_t rs_blk = make_rsrc(blk0);
  const __amdgpu_buffer_rsrc_t rs_pre = make_rsrc(
      plen > 0 ? (k_wave ? p.k_pre : p.v_pre) + (static_cast<size_t>(pbeg) * p.hkv + g) * D : blk0);
  const __amdgpu_buffer_rsrc_t rs_suf = make_rsrc(
      slen > 0 ? (k_wave ? p.k_suf : p.v_suf) + (static_cast<size_t>(sbeg) * p.hkv + g) * D : blk0);
  // slot of a chunk in tile row 4 n + lane / 16 (n mod 4 = i): XORed with this
  auto swz = [&](int lane_, int i) {
    const int r = 4 * (i & 3) + (lane_ >> 4);
    return k_wave ? r : 4 * (r & 3);
  };
  int lrow[kInstPerWave];       // tile row this lane fills in instruction i
  uint32_t coff[kInstPerWave];  // byte offset of the global chunk it fetches within the row
#pragma unroll
  for (int i = 0; i < kInstPerWave; ++i) {
    const int n = (wave * kInstPerWave + i) % kInstPerTile;
    const int r = 4 * n + (lane >> 4);
    lrow[i] = r;
    coff[i] = 16u * static_cast<uint32_t>((lane & 15) ^ swz(lane, n));
  }
  // This wave's half (K or V) of the tile of keys kv0 .. kv0 + 63 into dst.  Keys past kend come
  // from a clamped, valid row; their scores are set to -inf.
  [[maybe_unused]] PageWindow window;
  [[maybe_unused]] int page_shift, page_mask;
  [[maybe_unused]] unsigned n_pages;
  [[maybe_unused]] size_t page_bytes;      // a page of every head
  [[maybe_unused]] const uint8_t* pool_g;  // this head's rows of page 0
  [[maybe_unused]] const uint8_t* scale_g;
  [[maybe_unused]] const uint8_t* blk_g = reinterpret_cast<const uint8_t*>(blk0);
  if constexpr (Keys::kPaged) {
    constexpr int kHeld = Keys::kE4m3 ? D : kRowBytes;  // bytes of a cached row
    window.start(keys.kv, b, kbeg >> keys.kv.page_shift, lane);
    page_shift = keys.kv.page_shift;
    page_mask = (1 << page_shift) - 1;
    n_pages = keys.kv.n_pages;
    page_bytes = (static_cast<size_t>(p.hkv) << page_shift) * kHeld;
    pool_g = (k_wave ? keys.kv.k : keys.kv.v) + (static_cast<size_t>(g) << page_shift) * kHeld;
    if constexpr (Keys::kE4m3)
      scale_g =
          (k_wave ? keys.kv.k_scale : keys.kv.v_scale) + (static_cast<size_t>(g) << page_shift);
  }
  auto issue = [&](int kv0, uint8_t* dst) {
    if constexpr (Keys::kPaged) {
      // A wave loads 32 keys in two groups of 16, each within one page (or within the block): a
      // buffer resource per load, at its first row, ends with the group's last existing row, so
      // rows past it arrive as zeros.
      const bool paged = !Keys::kE4m3 && kv0 < cached;  // 8-bit tiles: fetch and place
      const uint32_t stride = paged ? kRowBytes : key_bytes;
      int lane_ = lane;
      if constexpr (Keys::kE4m3) asm volatile("" : "+v"(lane_));  // (as in place)
      const uint32_t row_off = static_cast<uint32_t>(lane_ >> 4) * stride;
      if (paged) window.advance(kv0 >> page_shift, lane);
      // where the wave's rows go (formed here, not kept per load over the loop)
      uint32_t to = static_cast<uint32_t>(dst - smem) + (wave & 1) * (kTileBytes / 2);
      asm volatile("" : "+s"(to));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = kv0 + 32 * (wave & 1) + 16 * h;
        const uint8_t* base;
        int rows;
        if (paged) {
          const int page = window.uniform(at >> page_shift);
          const bool ok = static_cast<unsigned>(page) < n_pages;
          base = pool_g + (ok ? page : 0) * page_bytes + (at & page_mask) * kRowBytes;
          rows = ok ? plen - at : 0;
        } else {
          const int j = at - cached;
          base = blk_g + min(j, len) * static_cast<size_t>(key_bytes);
          rows = len - j;
        }
        const int bytes =
            rows > 0 ? (min(rows, 16) - 1) * static_cast<int>(stride) + kRowBytes : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          buffer_load_to_lds(make_rsrc(base + 4 * i * static_cast<size_t>(stride),
                                       max(bytes - 4 * i * static_cast<int>(stride), 0)),
                             smem + to + (4 * h + i) * 1024,
                             row_off + 16u * ((lane_ & 15) ^ swz(lane_, i)), 0);
        }
      }
      return;
    }
    if (kv0 + kDmaKeys <= plen) {  // the whole tile lies in the prefix
#pragma unroll
      for (int i = 0; i < kInstPerWave; ++i) {
        const int n = (wave * kInstPerWave + i) % kInstPerTile;
        buffer_load_to_lds(rs_pre, dst + n * 1024,
                           static_cast<uint32_t>(lrow[i]) * key_bytes + coff[i],
                           static_cast<uint32_t>(kv0) * key_bytes);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < kInstPerWave; ++i) {
      const int n = (wave * kInstPerWave + i) % kInstPerTile;
      const int j = min(kv0 + lrow[i], kend - 1);
      if (j < plen)
        buffer_load_to_lds(rs_pre, dst + n * 1024, static_cast<uint32_t>(j) * key_bytes + coff[i],
                           0);
      else if (j < plen + len)
        buffer_load_to_lds(rs_blk, dst + n * 1024,
                           static_cast<uint32_t>(j - plen) * key_bytes + coff[i], 0);
      else
        buffer_load_to_lds(rs_suf, dst + n * 1024,
                           static_cast<uint32_t>(j - plen - len) * key_bytes + coff[i], 0);
    }
  };
  // Tiles of an 8-bit cache go through registers: fetch() loads this wave's half of a tile (four
  // loads of 16 bytes per lane, 8 rows each, and the scales of the lane's two rows per group of
  // 16), an iteration later place() widens it to bf16, exactly, and stores it where the loads into
  // LDS would have put it.  2 chunks of 1000 to 2048 rows behind 7001 to 12000, 28/4 heads: 506 us
  // (0.87 PFLOP/s), over bf16 pages 444.  Widening in the slots of the S loop instead, with the
  // next tile's loads behind it: 2% slower, the loads then have half the time; a swap of halves
  // between lanes that takes away the stores' bank conflicts: no change.
  constexpr int kRawLoads = 4;
  [[maybe_unused]] u32x4 raw[kRawLoads];
  [[maybe_unused]] uint32_t raw_scale[2];
  // where the lane's first row and chunk of a group go: row r = 2 (lane / 8), chunk 2 (lane % 8);
  // its second chunk lies in the slot ^ 1, row r + 1 in the slot ^ 1 (K: r % 16 is XORed) or ^ 4
  // (V)
  [[maybe_unused]] uint32_t raw_at =
      2 * (lane >> 3) * kRowBytes +
      16 * ((2 * (lane & 7)) ^ (k_wave ? 2 * (lane >> 3) : 8 * ((lane >> 3) & 1)));
  auto fetch = [&](int kv0) {
    if constexpr (Keys::kE4m3) {
      if (kv0 >= cached) return;
      window.advance(kv0 >> page_shift, lane);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = kv0 + 32 * (wave & 1) + 16 * h;
        const int page = window.uniform(at >> page_shift);
        const bool ok = static_cast<unsigned>(page) < n_pages;
        const size_t from = (ok ? page : 0) * page_bytes;
        const int row = at & page_mask, rows = ok ? min(max(plen - at, 0), 16) : 0;
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(pool_g + from + row * D, rows * D);
        // load i of the group: rows 2 (lane / 8) + i
#pragma unroll
        for (int i = 0; i < 2; ++i)
          raw[2 * h + i] = buffer_load16(rs, (2 * (lane >> 3) + i) * D + 16 * (lane & 7));
        raw_scale[h] = buffer_load2(make_rsrc(scale_g + from / D + row, (rows + 1) & ~1),
                                    2 * (lane >> 3));
      }
    }
  };
  auto place = [&](int kv0, uint8_t* dst) {
    if (kv0 >= cached) {
      issue(kv0, dst);
      return;
    }
    // the tile's rows of this wave begin at a multiple of 8 KB, so slots can be XORed into
    // addresses
    uint32_t base = static_cast<uint32_t>(dst - smem) + (wave & 1) * (kTileBytes / 2);
    asm volatile("" : "+s"(base));  // (formed here, not kept per slot over the loop)
    const uint32_t row0 = raw_at + base, row1 = (row0 ^ (k_wave ? 16 : 64)) + kRowBytes;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // (a scale byte of 255 can only come with the zeros of a row that does not exist: 254 then)
        const uint32_t scale = min(raw_scale[h] << (i ? 15 : 23) & 0x7f800000u, 0x7f000000u);
        u32x4 lo, hi;
        e4m3_widen(raw[2 * h + i], __uint_as_float(scale), lo, hi);
        uint8_t* const to = smem + h * 16 * kRowBytes;
        *reinterpret_cast<u32x4*>(to + (i ? row1 : row0)) = lo;
        *reinterpret_cast<u32x4*>(to + ((i ? row1 : row0) ^ 16)) = hi;
      }
  };
  auto ktile = [&](int i) { return smem + (i & 1) * kTileBytes; };
  auto vtile = [&](int i) { return smem + (2 + (i & 1)) * kTileBytes; };

  // S^T of tile st into acc (unmasked):
  // acc[kb][r] = S[query l32][key kb*32 + 8(r/4) + 4 half + r%4]
  auto scores = [&](int st, f32x16 (&acc)[kKB]) {
    const uint8_t* Kt = ktile(st);
#pragma unroll
    for (int kb = 0; kb < kKB; ++kb) acc[kb] = f32x16{};
#pragma unroll
    for (int s = 0; s < kDSteps; ++s)
#pragma unroll
      for (int kb = 0; kb < kKB; ++kb) {
        const int r = kb * 32 + l32;
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(
            Kt + r * kRowBytes + 16 * ((2 * s + half) ^ (r & 15)));
        acc[kb] = mfma32(kf, qf[s], acc[kb]);
      }
  };
  // Scores of keys past the tile's last to -inf; returns this lane's maximum over the tile.
  auto mask_max = [&](int st, f32x16 (&acc)[kKB]) {
    const int kv0 = kbeg + st * kDmaKeys, end = end_of(kv0);
    float mloc = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < kKB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = kv0 + kb * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
        if (key >= end) acc[kb][r] = -INFINITY;
        mloc = fmaxf(mloc, acc[kb][r]);
      }
    return mloc;
  };
  // Running maximum from this lane's tile maximum (both halves of a row agree).
  auto update_max = [&](float mloc) {
    mloc = fmaxf(mloc, __shfl_xor(mloc, 32));
    const float mcand = mloc * p.scale_log2;  // scale > 0: max(scale s) = scale max(s)
    if (__any(mcand > m_run + kAttnSlack)) {
      const float m_new = fmaxf(m_run, mcand);
      const float alpha = fast_exp2(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < kDBlocks; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
    }
  };

  const int n_stages = (kend - kbeg + kDmaKeys - 1) / kDmaKeys;
  // prologue: K(0), K(1), V(0); then S(0) and its maximum
  auto tile_at = [&](int st) { return kbeg + st * kDmaKeys; };
  if constexpr (Keys::kE4m3) {
    fetch(tile_at(0));
    place(tile_at(0), k_wave ? ktile(0) : vtile(0));
    if (n_stages > 1) fetch(tile_at(1));
    if (k_wave && n_stages > 1) {
      place(tile_at(1), ktile(1));
      if (n_stages > 2) fetch(tile_at(2));
    }
  } else if (k_wave) {
    issue(kbeg, ktile(0));
    if (n_stages > 1) issue(kbeg + kDmaKeys, ktile(1));
  } else {
    issue(kbeg, vtile(0));
  }
  wait_vm_lds_and_barrier<0>();
  f32x16 scur[kKB];
  scores(0, scur);
  update_max(mask_max(0, scur));

  const int q4 = lane & 3, j4 = (lane >> 2) & 3;
  const int d0 = 16 * ((lane >> 4) & 1);
  // Iteration st: S(st + 1) into snxt_ while P(st) comes from scur_.  Two iterations per trip
  // with the two score arrays swapping roles, so the next tile's scores are never copied.
  auto step = [&](int st, f32x16 (&scur_)[kKB], f32x16 (&snxt_)[kKB]) {
    // this wave's loads of K(st + 1) and V(st) have landed; after the barrier every wave's
    // have, and every wave is done with K(st) and V(st - 1)
    wait_vm_lds_and_barrier<0>();
    if constexpr (Keys::kE4m3) {
      const int to = st + (k_wave ? 2 : 1);  // the tile in the registers
      if (to < n_stages) place(tile_at(to), k_wave ? ktile(st) : vtile(st + 1));
      if (to + 1 < n_stages) fetch(tile_at(to + 1));
    } else if constexpr (Keys::kPaged) {
      const int to = st + (k_wave ? 2 : 1);
      if (to < n_stages) issue(tile_at(to), k_wave ? ktile(st) : vtile(st + 1));
    } else if (k_wave) {
      if (st + 2 < n_stages) issue(kbeg + (st + 2) * kDmaKeys, ktile(st));
    } else {
      if (st + 1 < n_stages) issue(kbeg + (st + 1) * kDmaKeys, vtile(st + 1));
    }
    const bool more = st + 1 < n_stages;
    // on the last iteration S of a stale K tile is computed and discarded (no branch)
    const uint8_t* Kt = ktile(more ? st + 1 : st);
    const uint8_t* Vt = vtile(st);
    auto kread = [&](int m) {  // K fragment of S MFMA m = 2 s + kb
      const int s = m / kKB, kb = m % kKB, r = kb * 32 + l32;
      return *reinterpret_cast<const bf16x8*>(Kt + r * kRowBytes +
                                              16 * ((2 * s + half) ^ (r & 15)));
    };
    // V^T fragment of P V MFMA n = (2 kb + u) kDBlocks + db: keys kb*32 + 16u + {4 half + 0..3,
    // 8 + 4 half + 0..3} at d = 32 db + l32.  Lane 4 j + q of a 16-lane group addresses key row
    // kbase + j at d = d0 + 4 q .. +3; the transposing read hands lane i of the group
    // d = d0 + i of rows kbase .. kbase + 3.
    auto vread = [&](int n) {
      const int db = n % kDBlocks, u = (n / kDBlocks) % 2, kb = n / (2 * kDBlocks);
      const int c = (32 * db + d0) / 8 + (q4 >> 1);  // 16-byte chunk of columns d0 + 4 q
      v4i16 part[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = kb * 32 + 16 * u + 8 * x + 4 * half + j4;
        const uint8_t* a = Vt + r * kRowBytes + 16 * (c ^ (4 * (r & 3))) + 8 * (q4 & 1);
        part[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(const_cast<uint8_t*>(a)));
      }
      return __builtin_bit_cast(bf16x8,
                                __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int kb = 0; kb < kKB; ++kb) snxt_[kb] = f32x16{};
    bf16x8 kf[kMfmas], vf[kMfmas];
    u32x4 pw[2 * kKB];  // P(st) as bf16 pairs: word e of MFMA group 2 kb + u
    float lsum = 0.f;
#pragma unroll
    for (int m = 0; m < kPreK; ++m) kf[m] = kread(m);
    __builtin_amdgcn_sched_barrier(0);
    // S(st + 1), each MFMA followed by the P(st) work of one slot: registers 8u + 2e, 8u + 2e + 1
    // of scur_[kb] are keys kb*32 + 16u + 4 half + ... -- exactly the B operand layout of P V.
    // The P words are software-pipelined over the slots: slot m forms the exponents of word
    // m + 1, the exponentials of word m and the bf16 pair and running sum of word m - 1, so an
    // instruction does not wait on the one just before it (a wave issues in order).
    auto expo = [&](int w, float (&y)[2]) {
      const int kb = w / 8, u = (w / 4) % 2, e = w % 4;
      y[0] = fmaf(scur_[kb][8 * u + 2 * e], p.scale_log2, -m_run);
      y[1] = fmaf(scur_[kb][8 * u + 2 * e + 1], p.scale_log2, -m_run);
    };
    float ya[2][2], ea[2][2];
    auto commit = [&](int w) {
      const uint32_t wd = pack2_bf16(ea[w & 1][0], ea[w & 1][1]);
      pw[w / 4][w % 4] = wd;
      lsum = sum2_bf16(wd, lsum);
    };
    expo(0, ya[0]);
#pragma unroll
    for (int m = 0; m < kMfmas; ++m) {
      if (m + kPreK < kMfmas) kf[m + kPreK] = kread(m + kPreK);
      if (m >= kMfmas - kPreV) vf[m - (kMfmas - kPreV)] = vread(m - (kMfmas - kPreV));
      snxt_[m % kKB] = mfma32(kf[m], qf[m / kKB], snxt_[m % kKB]);
      if (m + 1 < kMfmas) expo(m + 1, ya[(m + 1) & 1]);
      ea[m & 1][0] = fast_exp2(ya[m & 1][0]);
      ea[m & 1][1] = fast_exp2(ya[m & 1][1]);
      if (m >= 1) commit(m - 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    commit(kMfmas - 1);
    // O^T += V^T P^T, each MFMA followed by a step of the maximum of S(st + 1)
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < kMfmas; ++n) {
      if (n + kPreV < kMfmas) vf[n + kPreV] = vread(n + kPreV);
      o[n % kDBlocks] =
          mfma32(vf[n], __builtin_bit_cast(bf16x8, pw[n / kDBlocks]), o[n % kDBlocks]);
      mx[n & 1] = fmaxf(mx[n & 1], fmaxf(snxt_[n / 8][2 * (n % 8)], snxt_[n / 8][2 * (n % 8) + 1]));
      asm volatile("" : "+v"(mx[n & 1]));  // keep the step here, between the MFMAs
      __builtin_amdgcn_sched_barrier(0);
    }
    l_run += lsum;
    if (more) {
      float mloc = fmaxf(mx[0], mx[1]);
      // a partial tile: the last, and with pages the last of the cached rows
      if (kbeg + (st + 2) * kDmaKeys > end_of(kbeg + (st + 1) * kDmaKeys))
        mloc = mask_max(st + 1, snxt_);
      update_max(mloc);
    }
  };
  f32x16 salt[kKB];
  for (int st = 0; st < n_stages; st += 2) {
    step(st, scur, salt);
    if (st + 1 < n_stages) step(st + 1, salt, scur);
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32);
  if (!row_ok) return;
  if (Keys::kPaged ? it.ranges > 1 : p.nsplit > 1) {
    float *o_part = p.o_part, *m_part = p.m_part, *l_part = p.l_part;
    size_t idx = (static_cast<size_t>(bbeg + pos) * p.hq + g * G + hh) * p.nsplit + sp;
    if constexpr (Keys::kPaged) {
      idx = static_cast<size_t>(it.item) * kRowsPerWg + wave * 32 + l32;
      o_part = keys.plan.o_part, m_part = keys.plan.m_part, l_part = keys.plan.l_part;
    }
    float* dst = o_part + idx * D;
#pragma unroll
    for (int db = 0; db < kDBlocks; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int d = db * 32 + 8 * q + 4 * half;
        *reinterpret_cast<f32x4*>(dst + d) =
            f32x4{o[db][4 * q + 0], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
      }
    if (half == 0) {
      m_part[idx] = m_run;
      l_part[idx] = l_tot;
    }
    return;
  }
  const float inv = 1.0f / l_tot;
  uint16_t* dst = p.out + q_off;
#pragma unroll
  for (int db = 0; db < kDBlocks; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int d = db * 32 + 8 * q + 4 * half;
      const u32x2 v{pack2_bf16(o[db][4 * q + 0] * inv, o[db][4 * q + 1] * inv),
                    pack2_bf16(o[db][4 * q + 2] * inv, o[db][4 * q + 3] * inv)};
      *reinterpret_cast<u32x2*>(dst + d) = v;
    }
}

// The ranges of every (block row, query head) of a launch over pages, in key order: a wave per row
// and every `waves`-th head (neighbouring heads have one K/V head and are cut alike), its lanes
// over a head's partials side by side.
template <int D>
__global__ __launch_bounds__(kThreads) void attn_tiles_merge_kernel(AttnParams p, TilePlan tp,
                                                                    int total, int waves) {
  const int lane = threadIdx.x & 63;
  const long unit = static_cast<long>(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (unit >= static_cast<long>(total) * waves) return;  // uniform per wavefront
  const int row = static_cast<int>(unit / waves), h0 = static_cast<int>(unit % waves);
  const int b = find_sequence(p.cu_block, tp.batch, row, lane);
  const int len = tile_len(p, tp, b);
  if (len == 0) return;  // another launch's
  const int stages = tile_stages(p.cu_prefix[b + 1] - p.cu_prefix[b], len);
  LastRound last{};
  int first, row_tiles = tile_rows(len, p.group), ranges;
  if (tp.cap > 0) {
    first = tp.found[b];
    ranges = tp.found[kPlanMaxBatch + b];
    last = *reinterpret_cast<const LastRound*>(tp.found + 2 * kPlanMaxBatch);
  } else {
    ranges = (stages + tp.chunk - 1) / tp.chunk;
    if (tp.run == 0) row_tiles = tp.row_tiles;
    first = tp.run == 0 ? b * tp.nsplit * p.hkv * row_tiles : ranges > 1 ? tp.found[b] : 0;
    if (first < 0) ranges = 1;
  }
  for (int h = h0; h < p.hq; h += waves) {
    const int g = h / p.group, r = (row - p.cu_block[b]) * p.group + h % p.group;
    const long item = first + g * row_tiles + r / kRowsPerWg;
    const bool cut = last.full && item >= last.full;  // one of the last round
    const int n = cut ? min(last.ranges, stages) : ranges;
    const long step = cut ? last.rest : p.hkv * row_tiles;
    if (n <= 1) continue;  // written out by its only workgroup
    auto at = [&](int k) {
      return static_cast<size_t>(item + k * step) * kRowsPerWg + r % kRowsPerWg;
    };
    const PartialRow<D> x = merge_partials<D>(at, n, tp.o_part, tp.m_part, tp.l_part, lane);
    x.store(p.out + (static_cast<size_t>(row) * p.hq + h) * D, lane);
  }
}

}  // namespace
}  // namespace eb

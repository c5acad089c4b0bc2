// Pages for the rows that a step adds to the cache, from the sequences' lengths, on the device.
//
// Everything follows from exclusive sums over the sequences: of their new rows (where a sequence's
// rows begin), of the pages that they need (which of the free pages are theirs) and of the pages
// that finished ones give back (where in the ring those go).  One launch does all of it: every
// workgroup forms the sums of all sequences for itself, kThreads sequences at a time, which costs
// it less than a second launch would, and then writes its own rows' positions and slots; a new
// page's first row also writes the page's number into the table, and given-back pages are spread
// over all workgroups.  A few thousand integers: bound by the launch and the three or four
// dependent loads behind it (length, table or ring, then the stores), not by memory: 4.3 us for one
// sequence, 6.2 us for 64 with 16 to 256 rows each, 9.0 us for 1024 with 205000 rows (of a copy of
// their 2.5 MB: 0.5 us).  Running sums by DPP: 5.3 -> 4.3, 7.1 -> 6.2 and 10.0 -> 9.0 us against
// exchanges through LDS.
#include "eb_common.hpp"
#include "eb_internal.hpp"
#include "wave_ops.hpp"

namespace eb {
namespace {

constexpr int kThreads = 1024;  // sequences per pass, and rows per workgroup and turn
constexpr int kWaves = kThreads / 64;
constexpr int kMaxGroups = 2048;

// Per sequence: rows, prefix rows, pages needed, pages given back.
struct Sums {
  uint32_t rows, prefix, need, back;
  __device__ __forceinline__ Sums operator+(const Sums& o) const {
    return Sums{rows + o.rows, prefix + o.prefix, need + o.need, back + o.back};
  }
  __device__ __forceinline__ Sums& operator+=(const Sums& o) { return *this = *this + o; }
};

// Last index t in [0, n) with first[t] <= x, where first[0] <= x and first never decreases.
__device__ __forceinline__ int last_at_or_before(const uint32_t* first, int n, uint32_t x) {
  int lo = 0;
  for (int step = kThreads / 2; step >= 1; step >>= 1)
    if (lo + step < n && first[lo + step] <= x) lo += step;
  return lo;
}

// write_state false: the call's state_out is its state, which other workgroups may still be
// reading, and kv_assign_state_kernel writes it behind this launch.
template <bool kStateOnly>
__device__ __forceinline__ void assign(const KvAssign& a, bool write_state) {
  __shared__ uint32_t row_first[kThreads], need_first[kThreads], back_first[kThreads];
  __shared__ int32_t cached_rows[kThreads], held_pages[kThreads], shared_pages[kThreads];
  __shared__ uint8_t is_served[kThreads];
  __shared__ Sums wave_sum[kWaves];
  __shared__ uint32_t taken_pages;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool first_group = blockIdx.x == 0;
  const int page = 1 << a.page_shift;
  const uint32_t n_pages = static_cast<uint32_t>(a.n_pages);
  const uint32_t head = static_cast<uint32_t>(a.state[0]) % n_pages;
  const uint32_t free_pages = static_cast<uint32_t>(min(max(a.state[1], 0), a.n_pages));
  const uint32_t tail = (head + free_pages) % n_pages;
  if (tid == 0) taken_pages = 0;

  Sums before{0, 0, 0, 0};  // of the sequences of earlier passes
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + tid, in_pass = min(kThreads, a.batch - b0);
    Sums own{0, 0, 0, 0};
    int32_t cached = 0, held = 0, keep = 0;
    bool fits = true;
    if (b < a.batch) {
      cached = max(a.cached[b], 0);
      const int32_t rows = max(a.new_rows[b], 0);
      const bool done = a.done && a.done[b];
      held = static_cast<int32_t>((static_cast<int64_t>(cached) + page - 1) >> a.page_shift);
      if (done) {
        held = min(held, a.max_pages);
        keep = min(a.shared ? max(a.shared[b], 0) : 0, held);
        own.back = static_cast<uint32_t>(held - keep);
      } else {
        const int64_t end = static_cast<int64_t>(cached) + rows;
        const int64_t want = (end + page - 1) >> a.page_shift;
        fits = want <= a.max_pages && end <= INT32_MAX;
        own.rows = static_cast<uint32_t>(rows);
        own.prefix = static_cast<uint32_t>(cached);
        own.need = fits ? static_cast<uint32_t>(want - held) : 0;
      }
    }
    Sums sum = wave_scan(own);  // then over the waves before
    __syncthreads();  // the pass before is done with its arrays
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    Sums total = before;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w == wave) sum += total;
      total += wave_sum[w];
    }
    const bool served = fits && (own.need == 0 || sum.need <= free_pages);
    row_first[tid] = sum.rows - own.rows;
    need_first[tid] = sum.need - own.need;
    back_first[tid] = sum.back - own.back;
    cached_rows[tid] = cached;
    held_pages[tid] = held;
    shared_pages[tid] = keep;
    is_served[tid] = served;
    if (first_group && served && own.need) atomicMax(&taken_pages, sum.need);
    if (!kStateOnly && first_group && b < a.batch) {
      a.cu_block[b + 1] = static_cast<int32_t>(sum.rows);
      a.cu_prefix[b + 1] = static_cast<int32_t>(sum.prefix);
      if (b == 0) a.cu_block[0] = a.cu_prefix[0] = 0;
      if (a.shorted) a.shorted[b] = !served;
    }
    __syncthreads();
    if constexpr (!kStateOnly) {
      const uint32_t stride = gridDim.x * kThreads;
      // rows of this pass's sequences
      const uint32_t r_end = min(total.rows, static_cast<uint32_t>(a.n_rows));
      uint32_t r = blockIdx.x * kThreads + tid;
      if (r < before.rows) r += (before.rows - r + stride - 1) / stride * stride;
      for (; r < r_end; r += stride) {
        const int t = last_at_or_before(row_first, in_pass, r);
        const int64_t at = static_cast<int64_t>(cached_rows[t]) + (r - row_first[t]);
        const int64_t j = at >> a.page_shift;  // page of the sequence
        int32_t* const entry = a.page_table + static_cast<size_t>(b0 + t) * a.max_pages + j;
        const bool opens = j >= held_pages[t] && (at & (page - 1)) == 0;
        int32_t number = -1;
        if (is_served[t]) {  // (j < max_pages)
          if (j < held_pages[t]) {
            number = *entry;
          } else {
            const uint32_t i = need_first[t] + static_cast<uint32_t>(j - held_pages[t]);
            number = a.free_pages[(head + i % n_pages) % n_pages];
          }
        }
        if (opens && j < a.max_pages) *entry = number;
        a.pos[r] = is_served[t] ? static_cast<int32_t>(at) : -1;
        if (a.slot)
          a.slot[r] = static_cast<uint32_t>(number) < n_pages
                          ? (static_cast<int64_t>(number) << a.page_shift) + (at & (page - 1))
                          : -1;
      }
      // pages that this pass's finished sequences give back
      uint32_t p = blockIdx.x * kThreads + tid;
      if (p < before.back) p += (before.back - p + stride - 1) / stride * stride;
      for (; p < total.back; p += stride) {
        const int t = last_at_or_before(back_first, in_pass, p);
        const uint32_t j = p - back_first[t] + static_cast<uint32_t>(shared_pages[t]);
        a.free_pages[(tail + p % n_pages) % n_pages] =
            a.page_table[static_cast<size_t>(b0 + t) * a.max_pages + j];
      }
    }
    before = total;
  }
  if constexpr (!kStateOnly) {  // rows behind the last sequence's
    const uint32_t stride = gridDim.x * kThreads;
    uint32_t r = blockIdx.x * kThreads + tid;
    if (r < before.rows) r += (before.rows - r + stride - 1) / stride * stride;
    for (; r < static_cast<uint32_t>(a.n_rows); r += stride) {
      a.pos[r] = -1;
      if (a.slot) a.slot[r] = -1;
    }
  }
  if (first_group && tid == 0 && write_state) {
    a.state_out[0] = static_cast<int32_t>((head + taken_pages) % n_pages);
    a.state_out[1] = static_cast<int32_t>(free_pages - taken_pages + before.back);
  }
}

__global__ __launch_bounds__(kThreads) void kv_assign_kernel(KvAssign a, bool write_state) {
  assign<false>(a, write_state);
}

// The state alone, of the same call, when every workgroup of kv_assign_kernel has read the old one.
__global__ __launch_bounds__(kThreads) void kv_assign_state_kernel(KvAssign a) {
  assign<true>(a, true);
}

}  // namespace

hipError_t kv_assign(const KvAssign& a, hipStream_t s) {
  const int groups = max(1, min(kMaxGroups, a.n_rows / kThreads + (a.n_rows % kThreads != 0)));
  const bool apart = groups > 1 && a.state_out == a.state;
  hipLaunchKernelGGL(kv_assign_kernel, dim3(groups), dim3(kThreads), 0, s, a, !apart);
  if (apart) hipLaunchKernelGGL(kv_assign_state_kernel, dim3(1), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace eb

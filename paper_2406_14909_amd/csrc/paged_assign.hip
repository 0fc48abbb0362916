// Page tables from lengths: pages that no later query sees go back to the free list, new
// tokens get pages from it, and the row of each new token and head is written down.
//
// For each (sequence, KV head) pair, with p the position of its first new token and lo the first
// key behind the sinks that a query at p or later sees:
//   gone   present entries i with i * page >= sinks and (i + 1) * page <= lo; of a fresh sequence all
//   need   absent entries of the new tokens' positions
// Both are numbered in the order of the table: gone entry k goes to free[n + k], and need
// entry k takes free[n + gone in all - 1 - k].  No atomics: the numbers are prefix sums.
//
// Bound by latency.  The first kernel, one work-group, counts the pairs' entries, adds them up
// and gives pages back; the second takes pages and writes rows, a wave per pair.  Between the two
// lies the one dependence of the whole: pages taken may be pages given back.
#include "paged_device.h"

namespace moa {

namespace {

constexpr int kCountThreads = 1024;
constexpr int kCountWaves = kCountThreads / 64;
constexpr int kTakeThreads = 256;
constexpr int kTakeWaves = kTakeThreads / 64;
constexpr int kHead = 2;                 // plan: pages on the list before step 2, pages needed; then (gone, need) per pair

// What a pair's entries [lo, hi) and [first, last) are about.
struct Pair {
  int b, g;
  bool fresh;
  int gone_lo, gone_hi;      // entries that go back where present
  int need_lo, need_hi;      // entries that get pages where absent
  int64_t row, tokens;       // packed rows of the new tokens
  int64_t pos;
};

__device__ __forceinline__ Pair pair_of(const AssignArgs& a, int p) {
  Pair r;
  r.b = p / a.hkv;
  r.g = p - r.b * a.hkv;
  r.fresh = a.fresh != nullptr && a.fresh[r.b] != 0;
  r.pos = a.positions[r.b];
  r.row = r.b;
  r.tokens = 1;
  if (a.seq_start != nullptr) {
    r.row = a.seq_start[r.b];
    r.tokens = int64_t(a.seq_start[r.b + 1]) - r.row;
    if (r.row < 0 || r.row + r.tokens > a.n_tokens) r.tokens = 0;
  }
  if (r.pos < 0 || r.tokens < 0) r.tokens = 0;
  const int shift = a.page_shift;
  r.gone_lo = r.gone_hi = 0;
  if (r.fresh) {
    r.gone_hi = a.max_pages;
  } else if (r.pos >= 0) {
    const int64_t w = a.window[r.g];
    int64_t lo = r.pos - w + 1;
    if (a.block_band) lo = min(lo, ((r.pos >> 6) - ((w + 63) >> 6) + 1) * 64);
    static_assert(MOA_BAND_BLOCK == 64, "blocks of 64 positions");
    r.gone_lo = static_cast<int>((int64_t(a.num_sink) + (1 << shift) - 1) >> shift);
    r.gone_hi = static_cast<int>(min(max(lo, int64_t(0)) >> shift, int64_t(a.max_pages)));
  }
  r.gone_hi = max(r.gone_hi, r.gone_lo);
  r.need_lo = r.need_hi = 0;
  if (r.tokens > 0) {
    r.need_lo = static_cast<int>(min(r.pos >> shift, int64_t(a.max_pages)));
    r.need_hi = static_cast<int>(min(((r.pos + r.tokens - 1) >> shift) + 1, int64_t(a.max_pages)));
  }
  return r;
}

__device__ __forceinline__ bool present(const AssignArgs& a, int entry) {
  return static_cast<uint32_t>(entry) < static_cast<uint32_t>(a.num_pages);
}

__device__ __forceinline__ int64_t free_at_start(const AssignArgs& a) {
  return min(max(a.counts[0], 0), a.num_pages);
}

// Entries of table[lo, hi) that are present (or absent), by the whole wave.
__device__ __forceinline__ int64_t count_entries(const AssignArgs& a, const int32_t* table, int lo, int hi, bool want) {
  const int lane = threadIdx.x & 63;
  int64_t n = 0;
  for (int i = lo; i < hi; i += 64) {
    const bool in = i + lane < hi && present(a, table[i + lane]) == want;
    n += __builtin_popcountll(__ballot(in));
  }
  return n;
}

__global__ void __launch_bounds__(kCountThreads) paged_release_kernel(AssignArgs a) {
  __shared__ int64_t s_gone[kCountWaves], s_need[kCountWaves];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int pairs = a.batch * a.hkv;
  int64_t* const sums = a.plan + kHead;
  const int64_t n = free_at_start(a);
  for (int p = wave; p < pairs; p += kCountWaves) {
    const Pair r = pair_of(a, p);
    const int32_t* table = a.table + int64_t(p) * a.max_pages;
    const int64_t gone = count_entries(a, table, r.gone_lo, r.gone_hi, true);
    const int64_t need = r.fresh ? r.need_hi - r.need_lo : count_entries(a, table, r.need_lo, r.need_hi, false);
    if (lane == 0) {
      sums[2 * p] = gone;
      sums[2 * p + 1] = need;
    }
  }
  __syncthreads();
  // Exclusive prefix sums in place: every thread adds up a run of pairs.
  const int each = (pairs + kCountThreads - 1) / kCountThreads;
  const int p0 = min(pairs, static_cast<int>(threadIdx.x) * each), p1 = min(pairs, p0 + each);
  int64_t gone = 0, need = 0;
  for (int p = p0; p < p1; ++p) {
    gone += sums[2 * p];
    need += sums[2 * p + 1];
  }
  int64_t gone_to = gone, need_to = need;
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const int64_t x = __shfl_up(gone_to, off, 64), y = __shfl_up(need_to, off, 64);
    gone_to += lane >= off ? x : 0;
    need_to += lane >= off ? y : 0;
  }
  if (lane == 63) {
    s_gone[wave] = gone_to;
    s_need[wave] = need_to;
  }
  __syncthreads();
  int64_t gone_at = gone_to - gone, need_at = need_to - need, all_gone = 0, all_need = 0;
#pragma unroll
  for (int v = 0; v < kCountWaves; ++v) {
    gone_at += v < wave ? s_gone[v] : 0;
    need_at += v < wave ? s_need[v] : 0;
    all_gone += s_gone[v];
    all_need += s_need[v];
  }
  for (int p = p0; p < p1; ++p) {
    const int64_t x = sums[2 * p], y = sums[2 * p + 1];
    sums[2 * p] = gone_at;
    sums[2 * p + 1] = need_at;
    gone_at += x;
    need_at += y;
  }
  const int64_t listed = min(n + all_gone, int64_t(a.num_pages));
  if (threadIdx.x == 0) {
    a.plan[0] = listed;
    a.plan[1] = all_need;
  }
  __syncthreads();
  if (all_gone == 0) return;
  for (int p = wave; p < pairs; p += kCountWaves) {
    const Pair r = pair_of(a, p);
    int32_t* table = a.table + int64_t(p) * a.max_pages;
    int64_t at = n + sums[2 * p];
    for (int i = r.gone_lo; i < r.gone_hi; i += 64) {
      const int entry = i + lane < r.gone_hi ? table[i + lane] : -1;
      const uint64_t which = __ballot(present(a, entry));
      if (present(a, entry)) {
        const int64_t to = at + __builtin_popcountll(which & ((uint64_t(1) << lane) - 1));
        if (to < a.num_pages) a.free_pages[to] = entry;      // more only if a page stands in two entries
        table[i + lane] = -1;
      }
      at += __builtin_popcountll(which);
    }
  }
}

// A wave takes the pages of one pair and writes its tokens' rows.
__global__ void __launch_bounds__(kTakeThreads) paged_take_kernel(AssignArgs a) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int pairs = a.batch * a.hkv;
  const int p = static_cast<int>(blockIdx.x) * kTakeWaves + wave;
  const int64_t listed = a.plan[0];
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const int64_t all = a.plan[1];
    a.counts[0] = static_cast<int>(max(listed - all, int64_t(0)));
    a.counts[1] = static_cast<int>(min(max(all - listed, int64_t(0)), int64_t(0x7fffffff)));
  }
  if (p >= pairs) return;
  const Pair r = pair_of(a, p);
  int32_t* table = a.table + int64_t(p) * a.max_pages;
  int64_t at = listed - 1 - a.plan[kHead + 2 * p + 1];
  for (int i = r.need_lo; i < r.need_hi; i += 64) {
    const bool need = i + lane < r.need_hi && !present(a, table[i + lane]);
    const uint64_t which = __ballot(need);
    const int64_t from = at - __builtin_popcountll(which & ((uint64_t(1) << lane) - 1));
    if (need && from >= 0) table[i + lane] = a.free_pages[from];
    at -= __builtin_popcountll(which);
  }
  if (a.slots == nullptr || r.tokens == 0) return;
  __threadfence_block();                  // the wave reads what its lanes have written
  for (int64_t t = lane; t < r.tokens; t += 64) {
    const int64_t pos = r.pos + t, i = pos >> a.page_shift;
    const int entry = i < a.max_pages ? table[i] : -1;
    a.slots[(r.row + t) * a.hkv + r.g] =
        present(a, entry) ? static_cast<int>((int64_t(entry) << a.page_shift) + (pos & ((1 << a.page_shift) - 1))) : -1;
  }
}

}  // namespace

int launch_paged_assign(const AssignArgs& a, void* stream) {
  AssignArgs copy = a;
  void* args[] = {&copy};
  hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&paged_release_kernel), dim3(1), dim3(kCountThreads), args,
                                 0, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return static_cast<int>(e);
  const unsigned groups = static_cast<unsigned>((int64_t(a.batch) * a.hkv + kTakeWaves - 1) / kTakeWaves);
  e = hipLaunchKernel(reinterpret_cast<const void*>(&paged_take_kernel), dim3(groups), dim3(kTakeThreads), args, 0,
                      static_cast<hipStream_t>(stream));
  return static_cast<int>(e);
}

}  // namespace moa

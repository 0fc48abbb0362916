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
// Bound by latency: trips to memory, one after the other.  A wave per pair counts and takes
// back, a wave per pair gives out; between the two lies the one dependence of the whole, that pages
// given out may be pages taken back in the same call.  Few pairs (the usual case): the first kernel
// leaves what it takes back in the workspace, and every work-group of the second adds up all
// pairs' counts by itself and finds a page wherever it is.  Many pairs, or tables that the workspace has
// no room for: the counts are added up and the pages put on the list by kernels of their own.
// Rows of many tokens are written by a kernel of their own, in whole lines (16,000 tokens of 32 heads
// 16.1 us in all, without it 22.9).  48 sequences x 8 heads, 3 of them new with 1,600 tokens: 8.4 us; by one
// work-group for all counts 57.  With scales and notes of lacked pages, captured: 8.4 -> 8.9 us, and the
// many tokens 17.8 -> 18.5.
#include <type_traits>

#include "paged_device.h"

namespace moa {

namespace {

constexpr int kThreads = 256;            // a wave per pair
constexpr int kWaves = kThreads / 64;
constexpr int kScanThreads = 1024;
constexpr int kScanWaves = kScanThreads / 64;
constexpr int kFewPairs = 4096;          // counts of all pairs in LDS
constexpr int kSlotTokens = 16;          // tokens per work-group of the rows' kernel
constexpr int kManyTokens = 4096;        // from here on rows have a kernel of their own
constexpr int kQuantShift = 4;
static_assert(kQuantBlock == 1 << kQuantShift, "positions of one scale");

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Pages that pairs give back and need.
struct Counts {
  int32_t gone, need;
};

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

// The workspace: the length of the free list before the call, the length after step 1 and the pages
// needed in all (many pairs); then the counts of each pair, or their sums in front of it (many pairs), and
// behind those the pages that each pair gives back.
struct Space {
  int64_t* head;
  Counts* counts;
  int64_t* sums;
  int32_t* stash;
  __device__ __forceinline__ explicit Space(const AssignArgs& a) : head(a.plan) {
    const int64_t pairs = int64_t(a.batch) * a.hkv;
    counts = reinterpret_cast<Counts*>(head + 4);
    sums = head + 4 + pairs;
    stash = reinterpret_cast<int32_t*>(counts + pairs);
  }
};

__device__ __forceinline__ int below(uint64_t which) {          // set bits of the lanes in front
  return __builtin_popcountll(which & ((uint64_t(1) << (threadIdx.x & 63)) - 1));
}

// Counts a pair's entries.  kStash: takes those that go back out of the table and keeps them.  kState: of
// a sequence that lacked a page none are needed until it is fresh.
template <bool kStash, bool kState>
__global__ void __launch_bounds__(kThreads) paged_count_kernel(AssignArgs a) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const Space ws(a);
  if (blockIdx.x == 0 && threadIdx.x == 0) ws.head[0] = min(max(a.counts[0], 0), a.num_pages);
  const int p = static_cast<int>(blockIdx.x) * kWaves + wave;
  if (p >= a.batch * a.hkv) return;
  const Pair r = pair_of(a, p);
  int32_t* table = a.table + int64_t(p) * a.max_pages;
  int gone = 0, need = 0;
  for (int i = r.gone_lo; i < r.gone_hi; i += 64) {
    const int entry = i + lane < r.gone_hi ? table[i + lane] : -1;
    const uint64_t which = __ballot(present(a, entry));
    if (kStash && present(a, entry)) {
      ws.stash[int64_t(p) * a.max_pages + gone + below(which)] = entry;
      table[i + lane] = -1;
    }
    gone += __builtin_popcountll(which);
  }
  if (r.fresh) {
    need = r.need_hi - r.need_lo;
  } else {
    for (int i = r.need_lo; i < r.need_hi; i += 64)
      need += __builtin_popcountll(__ballot(i + lane < r.need_hi && !present(a, table[i + lane])));
  }
  if constexpr (kState) {
    if (a.lacked != nullptr) {
      if (!r.fresh) need = a.lacked[r.b] != 0 ? 0 : need;
      else if (r.g == 0 && lane == 0) a.lacked[r.b] = 0;       // which no wave of this sequence reads
    }
  }
  if (lane == 0) ws.counts[p] = {gone, need};
}

// Many pairs: the sums in front of each, by one work-group.
__global__ void __launch_bounds__(kScanThreads) paged_scan_kernel(AssignArgs a) {
  __shared__ int64_t s_gone[kScanWaves], s_need[kScanWaves];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int pairs = a.batch * a.hkv;
  const Space ws(a);
  const int each = (pairs + kScanThreads - 1) / kScanThreads;
  const int p0 = min(pairs, static_cast<int>(threadIdx.x) * each), p1 = min(pairs, p0 + each);
  int64_t gone = 0, need = 0;
  for (int p = p0; p < p1; ++p) {
    gone += ws.counts[p].gone;
    need += ws.counts[p].need;
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
  for (int v = 0; v < kScanWaves; ++v) {
    gone_at += v < wave ? s_gone[v] : 0;
    need_at += v < wave ? s_need[v] : 0;
    all_gone += s_gone[v];
    all_need += s_need[v];
  }
  for (int p = p0; p < p1; ++p) {
    ws.sums[2 * p] = gone_at;
    ws.sums[2 * p + 1] = need_at;
    gone_at += ws.counts[p].gone;
    need_at += ws.counts[p].need;
  }
  if (threadIdx.x == 0) {
    ws.head[1] = min(ws.head[0] + all_gone, int64_t(a.num_pages));
    ws.head[2] = all_need;
  }
}

// Many pairs: a wave puts the pages that its pair gives back on the list.
__global__ void __launch_bounds__(kThreads) paged_release_kernel(AssignArgs a) {
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const Space ws(a);
  const int p = static_cast<int>(blockIdx.x) * kWaves + wave;
  if (p >= a.batch * a.hkv || ws.counts[p].gone == 0) return;
  const Pair r = pair_of(a, p);
  int32_t* table = a.table + int64_t(p) * a.max_pages;
  int64_t at = ws.head[0] + ws.sums[2 * p];
  for (int i = r.gone_lo; i < r.gone_hi; i += 64) {
    const int entry = i + lane < r.gone_hi ? table[i + lane] : -1;
    const uint64_t which = __ballot(present(a, entry));
    if (present(a, entry)) {
      const int64_t to = at + below(which);
      if (to < a.num_pages) a.free_pages[to] = entry;      // more only if a page stands in two entries
      table[i + lane] = -1;
    }
    at += __builtin_popcountll(which);
  }
}

__device__ __forceinline__ int row_of_pool(const AssignArgs& a, int entry, int64_t pos) {
  return present(a, entry) ? static_cast<int>((int64_t(entry) << a.page_shift) + (pos & ((1 << a.page_shift) - 1))) : -1;
}

// A wave gives out the pages of one pair, and writes its tokens' rows where there are few.  kStash:
// it adds up all pairs' counts first and puts its pair's pages on the list.  kState: the scales of
// the pages that it gives out become 0, and it notes what sequence lacks one (a kernel of its own, as calls without
// either would take 8.7 us for 8.4 and 16.7 for 16.3).
template <bool kStash, bool kState>
__global__ void __launch_bounds__(kThreads) paged_take_kernel(AssignArgs a) {
  __shared__ int s_gone[kStash ? kFewPairs + 1 : 1], s_need[kStash ? kFewPairs : 1], s_wave[2][kWaves];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int pairs = a.batch * a.hkv;
  const Space ws(a);
  const int p = static_cast<int>(blockIdx.x) * kWaves + wave;
  const Pair r = pair_of(a, min(p, pairs - 1));           // asked for along with the counts
  const int64_t n = ws.head[0];
  const int needs = kState ? ws.counts[min(p, pairs - 1)].need : 0;
  int64_t listed, all_need;
  if constexpr (kStash) {
    const int each = (pairs + kThreads - 1) / kThreads;
    const int p0 = min(pairs, static_cast<int>(threadIdx.x) * each), p1 = min(pairs, p0 + each);
    int gone = 0, need = 0;
    for (int i = p0; i < p1; ++i) {
      const Counts c = ws.counts[i];
      s_gone[i] = gone;
      s_need[i] = need;
      gone += c.gone;
      need += c.need;
    }
    int gone_to = gone, need_to = need;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
      const int x = __shfl_up(gone_to, off, 64), y = __shfl_up(need_to, off, 64);
      gone_to += lane >= off ? x : 0;
      need_to += lane >= off ? y : 0;
    }
    if (lane == 63) {
      s_wave[0][wave] = gone_to;
      s_wave[1][wave] = need_to;
    }
    __syncthreads();
    int gone_at = gone_to - gone, need_at = need_to - need, all_gone = 0, need_sum = 0;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      gone_at += v < wave ? s_wave[0][v] : 0;
      need_at += v < wave ? s_wave[1][v] : 0;
      all_gone += s_wave[0][v];
      need_sum += s_wave[1][v];
    }
    for (int i = p0; i < p1; ++i) {
      s_gone[i] += gone_at;
      s_need[i] += need_at;
    }
    if (threadIdx.x == 0) s_gone[pairs] = all_gone;
    __syncthreads();
    listed = min(n + all_gone, int64_t(a.num_pages));
    all_need = need_sum;
  } else {
    listed = ws.head[1];
    all_need = ws.head[2];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.counts[0] = static_cast<int>(max(listed - all_need, int64_t(0)));
    a.counts[1] = static_cast<int>(min(max(all_need - listed, int64_t(0)), int64_t(0x7fffffff)));
  }
  if (p >= pairs) return;
  // Page i of the list as step 1 leaves it: what this call has put there may still be under way.
  auto page = [&](int64_t i) {
    if constexpr (!kStash) return a.free_pages[i];
    if (i < n) return a.free_pages[i];
    const int k = static_cast<int>(i - n);
    int lo = 0, hi = pairs;                               // s_gone[lo] <= k < s_gone[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_gone[mid] <= k) lo = mid;
      else hi = mid;
    }
    return ws.stash[int64_t(lo) * a.max_pages + k - s_gone[lo]];
  };
  int32_t* table = a.table + int64_t(p) * a.max_pages;
  int64_t at = listed - 1;
  if constexpr (kStash) at -= s_need[p];
  else at -= ws.sums[2 * p + 1];
  if constexpr (kState) {
    if (a.lacked != nullptr && needs > at + 1 && needs > 0 && lane == 0) a.lacked[r.b] = 1;   // nothing reads it here
  }
  const bool rows = a.slots != nullptr && a.n_tokens < kManyTokens;
  const int64_t end = r.pos + r.tokens;
  auto write_rows = [&](int64_t lo, int64_t hi, auto entry_of) {      // of the tokens at positions lo .. hi - 1
    for (int64_t x = lo; x < hi; x += 64) {
      const int64_t pos = x + lane;
      const int entry = entry_of(pos);
      if (pos < hi) a.slots[(r.row + pos - r.pos) * a.hkv + r.g] = row_of_pool(a, entry, pos);
    }
  };
  for (int i = r.need_lo; i < r.need_hi; i += 64) {
    const bool in = i + lane < r.need_hi;
    int entry = r.fresh || !in ? -1 : table[i + lane];
    const bool need = in && !present(a, entry) && (!kState || needs > 0);
    const uint64_t which = __ballot(need);
    const int64_t from = at - below(which);
    if (need && from >= 0) {
      entry = page(from);
      table[i + lane] = entry;
      if constexpr (kState) {
        if (a.scales != nullptr && present(a, entry)) {
          f32x2* const of = reinterpret_cast<f32x2*>(a.scales) + (int64_t(entry) << (a.page_shift - kQuantShift));
          for (int k = 0; k < 1 << (a.page_shift - kQuantShift); ++k) of[k] = f32x2{0.0f, 0.0f};
        }
      }
    }
    at -= __builtin_popcountll(which);
    if (rows)
      write_rows(max(r.pos, int64_t(i) << a.page_shift), min(end, int64_t(i + 64) << a.page_shift),
                 [&](int64_t pos) { return __shfl(entry, static_cast<int>(pos >> a.page_shift) - i, 64); });
  }
  if (rows) write_rows(max(r.pos, int64_t(a.max_pages) << a.page_shift), end, [](int64_t) { return -1; });
  if constexpr (kStash) {
    const int first = s_gone[p], mine = s_gone[p + 1] - first;
    for (int i = lane; i < mine; i += 64)
      if (n + first + i < a.num_pages) a.free_pages[n + first + i] = ws.stash[int64_t(p) * a.max_pages + i];
  }
}

// Rows of the pool of kSlotTokens tokens, for all heads.
__global__ void __launch_bounds__(kThreads) paged_slots_kernel(AssignArgs a) {
  const int t0 = static_cast<int>(blockIdx.x) * kSlotTokens, t1 = min(t0 + kSlotTokens, a.n_tokens);
  int b0 = 0, b1 = 0;                     // the sequences of these tokens lie within
  if (a.seq_start != nullptr) {
    b0 = max(sequence_at(a.seq_start, a.batch, t0), 0);
    b1 = max(sequence_at(a.seq_start, a.batch, t1 - 1), b0);
  }
  for (int x = threadIdx.x; x < (t1 - t0) * a.hkv; x += kThreads) {
    const int t = t0 + x / a.hkv, g = x % a.hkv;
    int b = t;
    int64_t first = t;
    if (a.seq_start != nullptr) {
      b = b0;                               // the last with seq_start[b] <= t
      for (int hi = b1; b < hi;) {
        const int mid = (b + hi + 1) >> 1;
        if (a.seq_start[mid] <= t) b = mid;
        else hi = mid - 1;
      }
      first = a.seq_start[b];
      const int end = a.seq_start[b + 1];
      if (first < 0 || t < first || t >= end || end > a.n_tokens) continue;
    }
    const int64_t p0 = a.positions[b], pos = p0 + t - first, i = pos >> a.page_shift;
    if (p0 < 0) continue;
    a.slots[int64_t(t) * a.hkv + g] =
        row_of_pool(a, i < a.max_pages ? a.table[(int64_t(b) * a.hkv + g) * a.max_pages + i] : -1, pos);
  }
}

}  // namespace

int launch_paged_assign(const AssignArgs& a, size_t ws_bytes, void* stream) {
  AssignArgs copy = a;
  void* args[] = {&copy};
  auto run = [&](auto kernel, int64_t groups, int threads) {
    return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(static_cast<unsigned>(groups)), dim3(threads), args, 0,
                           static_cast<hipStream_t>(stream));
  };
  const int64_t pairs = int64_t(a.batch) * a.hkv, groups = (pairs + kWaves - 1) / kWaves;
  const int64_t row_groups = a.slots == nullptr ? 0 : (int64_t(a.n_tokens) + kSlotTokens - 1) / kSlotTokens;
  if (row_groups * kThreads >= kMaxGridThreads) return kGridTooLarge;      // nothing is launched
  // Few pairs are added up in 32 bits.
  const bool few = pairs <= kFewPairs && pairs * a.max_pages <= INT32_MAX &&
                   32 + pairs * (8 + int64_t(4) * a.max_pages) <= static_cast<int64_t>(ws_bytes);
  const bool state = a.scales != nullptr || a.lacked != nullptr;
  auto count = [&](auto stash) {
    constexpr bool kStash = decltype(stash)::value;
    return state ? run(&paged_count_kernel<kStash, true>, groups, kThreads) : run(&paged_count_kernel<kStash, false>, groups, kThreads);
  };
  hipError_t e = few ? count(std::true_type{}) : count(std::false_type{});
  if (e == hipSuccess && !few) e = run(&paged_scan_kernel, 1, kScanThreads);
  if (e == hipSuccess && !few) e = run(&paged_release_kernel, groups, kThreads);
  auto take = [&](auto stash) {
    constexpr bool kStash = decltype(stash)::value;
    return state ? run(&paged_take_kernel<kStash, true>, groups, kThreads) : run(&paged_take_kernel<kStash, false>, groups, kThreads);
  };
  if (e == hipSuccess) e = few ? take(std::true_type{}) : take(std::false_type{});
  if (e == hipSuccess && a.slots != nullptr && a.n_tokens >= kManyTokens)
    e = run(&paged_slots_kernel, row_groups, kThreads);
  return static_cast<int>(e);
}

}  // namespace moa

// How the work of paged attention of many query rows is shared out: ragged chunks of tokens
// over their caches, or the tokens of a whole batch over a shared prefix.
//
// Rows are (token, query head) pairs of one KV head, token by token, in tiles of ROWS; the
// keys of a row tile are walked in tiles of 64 positions.  A row tile costs the keys that
// its last token may see, and kTileCost more for its start and end.  The cost of all row
// tiles of all (sequence, KV head) pairs, laid end to end, is cut into equal pieces, one
// per work-group ("worker"); a worker walks the row tiles that its piece touches.  A row
// tile inside one piece writes its output, one that is cut leaves partial results, in a slot
// of the worker, and a merge follows.  Where there are row tiles enough, every work-group
// takes a whole one instead: no partial results, and neighbours share keys in their die's L2.
//
// The lengths live on the device.  Each work-group forms the plan for itself: one trip to
// memory and a prefix sum over the pairs; a row tile's place within its pair has a closed form.
#pragma once

#include "paged_device.h"
#include "paged_split.h"

namespace moa {

constexpr float kRescaleSlack = 8.0f;   // log2 headroom before a running maximum is raised

// One row tile and a part [num0, num1) of den of its key tiles.
struct PagedItem {
  int g;
  int64_t table;     // first entry in the page table
  int token;         // packed token of the first row
  int rows;
  int pos;           // position of the first row (prefill)
  int64_t num0, num1, den;
  int slot;          // of the partial result, -1: none
};

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(x & 0xffffffff));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32));
  return static_cast<int64_t>((uint64_t(hi) << 32) | lo);
}

// The same in scalar registers.
__device__ __forceinline__ PagedItem uniform(const PagedItem& i) {
  PagedItem u;
  u.g = uniform(i.g);
  u.table = uniform64(i.table);
  u.token = uniform(i.token);
  u.rows = uniform(i.rows);
  u.pos = uniform(i.pos);
  u.num0 = uniform64(i.num0);
  u.num1 = uniform64(i.num1);
  u.den = uniform64(i.den);
  u.slot = uniform(i.slot);
  return u;
}

// A (sequence, KV head) pair: its sequence's packed rows and position, its head, its cost.
// Pairs of a sequence are in the order of their heads' windows, widest first.
struct RowPair {
  int b, order, start, pos;
  int64_t tokens;
  PairCost cost;
};
struct RowPlanLds {
  int64_t cost[8], longest[8];     // of each wave
  int64_t tiles[8];
  // where this work-group begins
  int index, tile;
  int64_t before;                // cost in front of the pair
  RowPair pair;
};
__device__ __forceinline__ RowPair uniform(const RowPair& p) {
  return {uniform(p.b), uniform(p.order), uniform(p.start), uniform(p.pos), uniform64(p.tokens),
          {uniform(p.cost.tiles), uniform(p.cost.first), uniform(p.cost.shift), uniform(p.cost.most)}};
}

template <int ROWS>
__device__ __forceinline__ RowPair row_pair(const PagedArgs& a, int pair) {
  RowPair p;
  p.b = pair / a.hkv;
  p.order = pair - p.b * a.hkv;
  p.start = a.seq_start[p.b];
  const int end = a.seq_start[p.b + 1];
  p.pos = a.positions[p.b];
  p.tokens = p.start < 0 || end > a.n_tokens ? 0 : int64_t(end) - p.start;
  p.cost = pair_cost(p.tokens, p.pos, a.window_in_order[p.order], a.band_shift, a.num_sink, a.group_shift, ROWS,
                     int64_t(a.max_pages) << a.page_shift);
  return p;
}

// Calls tile(item) for each row tile that work-group `block` of WAVES waves has a part in.
// Work-group uniform; `tile` ends with a barrier where LDS is used again.  kWhole: of a launch without pieces
// (a.plan null), whose code then has one copy of `tile`.
template <int ROWS, int WAVES, bool kWhole = false, class Tile>
__device__ __forceinline__ void for_each_row_tile(const PagedArgs& a, int block, RowPlanLds& s, Tile&& tile) {
  constexpr int kThreads = WAVES * 64;
  const int pairs = a.batch * a.hkv;
  const int each = (pairs + kThreads - 1) / kThreads;
  const int p0 = static_cast<int>(threadIdx.x) * each;
  const int p1 = min(pairs, p0 + each);
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  int64_t cost = 0, longest = 0, tiles = 0;
  RowPair mine = {};                                 // the thread's last pair, of one the only one
  for (int p = p0; p < p1; ++p) {
    mine = row_pair<ROWS>(a, p);
    const PairCost& c = mine.cost;
    cost += c.before(c.tiles);
    longest = max(longest, c.longest());
    tiles += c.tiles;
  }
  int64_t cost_to = cost, tiles_to = tiles;
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const int64_t c = __shfl_up(cost_to, off, 64);
    const int64_t t = __shfl_up(tiles_to, off, 64);
    cost_to += lane >= off ? c : 0;
    tiles_to += lane >= off ? t : 0;
    longest = max(longest, static_cast<int64_t>(__shfl_xor(longest, off, 64)));
  }
  if (lane == 63) {
    s.cost[wave] = cost_to;
    s.longest[wave] = longest;
    s.tiles[wave] = tiles_to;
  }
  __syncthreads();
  int64_t units = 0, before = cost_to - cost, all = 0, tiles_before = tiles_to - tiles;
  longest = 0;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    before += v < wave ? s.cost[v] : 0;
    tiles_before += v < wave ? s.tiles[v] : 0;
    units += s.cost[v];
    all += s.tiles[v];
    longest = max(longest, s.longest[v]);
  }
  units = uniform64(units);
  longest = uniform64(longest);
  all = uniform64(all);

  // A row tile of a pair, whole or in part.
  auto item_of = [&](const RowPair& p, int i, int64_t num0, int64_t num1, int64_t den, int slot) {
    const int first = i * (ROWS >> a.group_shift);           // token of the sequence's new ones
    PagedItem it;
    it.g = a.kv_order[p.order];
    it.table = (int64_t(p.b) * a.hkv + it.g) * a.max_pages;
    it.token = p.start + first;
    it.rows = static_cast<int>(min(int64_t(ROWS), (p.tokens << a.group_shift) - int64_t(i) * ROWS));
    it.pos = static_cast<int>(min(int64_t(p.pos) + first, int64_t(0x7fffffff) - ROWS));
    it.num0 = num0;
    it.num1 = num1;
    it.den = den;
    it.slot = slot;
    return it;
  };

  // More row tiles than n_tokens rows can have: seq_start is no packing of them, and nothing
  // is done (all sums below rest on there being no more).
  if (all > a.most_tiles) {
    if (a.plan != nullptr && block < a.slots && threadIdx.x == 0) reinterpret_cast<PagedSeg*>(a.plan)[block].rows = 0;
    return;
  }

  // Whole row tiles, where the longest takes little more than an equal share of the work.
  PagedSeg* const segs = reinterpret_cast<PagedSeg*>(a.plan);
  const int worth = 4 * all >= 3 * a.slots ? a.full_cost : a.whole_cost;
  if (kWhole || a.plan == nullptr || (longest - worth) * a.slots <= units) {
    if (a.plan != nullptr && block < a.slots && threadIdx.x == 0) segs[block].rows = 0;
    // Dealt to the dies in units of 16 neighbours, one unit to each die in turn and back
    // again; few singly.  Of a pair the last first: theirs are the most keys.
    const uint32_t unit = all >= 16 * kNumXcd * 4 ? 16 : 1;
    const uint32_t die = block % kNumXcd, local = block / kNumXcd;
    const uint32_t round = local / unit;
    const uint32_t n = (round * kNumXcd + (round & 1 ? kNumXcd - 1 - die : die)) * unit + local % unit;
    if (n >= all) return;
    if (n >= tiles_before && n < tiles_before + tiles) {     // one thread
      int64_t at = tiles_before;
      for (int p = p0; each > 1; ++p) {
        mine = row_pair<ROWS>(a, p);
        if (n < at + mine.cost.tiles) break;
        at += mine.cost.tiles;
      }
      s.tile = static_cast<int>(mine.cost.tiles - 1 - (n - at));
      s.pair = mine;
    }
    __syncthreads();
    const RowPair p = uniform(s.pair);
    const int i = uniform(s.tile);
    tile(item_of(p, i, 0, 1, 1, -1));
    return;
  }

  if constexpr (kWhole) return;

  // Pieces.  Workers of neighbouring pieces sit on one die.
  const RowSplit split = row_split(units, a.least_cost, a.log_slots);
  if (block >= a.slots) return;
  const int workers = split.workers(), per_die = max(1, workers / kNumXcd);
  int w = block;
  if (w < workers && workers >= kNumXcd) w = w % kNumXcd * per_die + w / kNumXcd;
  PagedSeg cut = {0, 0, 0, 0};
  if (w < workers) {
    int64_t x = uniform64(split.start(w));
    const int64_t x_end = uniform64(split.start(w + 1));
    if (x >= before && x < before + cost) {                  // one thread
      int64_t at = before;
      int p = p0;
      for (; each > 1; ++p) {
        mine = row_pair<ROWS>(a, p);
        const int64_t n = mine.cost.before(mine.cost.tiles);
        if (x < at + n) break;
        at += n;
      }
      s.index = p;
      s.before = at;
      s.pair = mine;
    }
    __syncthreads();
    int pair = uniform(s.index);
    int64_t at = uniform64(s.before);
    RowPair p = uniform(s.pair);
    int i = 0;                                               // the row tile that x lies in: 64 probes at once
    for (int n = p.cost.tiles; n > 1;) {
      const int stride = (n + 63) >> 6;
      const bool below = lane * stride < n && p.cost.before(i + lane * stride) <= x - at;
      const int k = __builtin_popcountll(__ballot(below)) - 1;
      i += k * stride;
      n = min(stride, n - k * stride);
    }
    i = uniform(i);
    while (true) {
      const int n = p.cost.tiles;
      for (; i < n && x < x_end; ++i) {
        const int64_t c0 = at + uniform64(p.cost.before(i)), c1 = at + uniform64(p.cost.before(i + 1));
        const int64_t end = min(x_end, c1);
        const bool whole = x == c0 && end == c1;
        const PagedItem it = item_of(p, i, x - c0, end - c0, c1 - c0, whole ? -1 : x == c0 ? 2 * w + 1 : 2 * w);
        if (x == c0 && !whole) cut = {it.token, it.g, it.rows, split.worker_of(c1 - 1) - w + 1};
        tile(it);
        x = end;
      }
      if (x >= x_end) break;
      at += uniform64(p.cost.before(n));
      i = 0;
      ++pair;
      p = uniform(row_pair<ROWS>(a, pair));
    }
  }
  if (threadIdx.x == 0) segs[w] = cut;
}

// The item of work-group w over a shared prefix: rows are (sequence, query head) pairs, all
// heads have the same number of row tiles, and head g's keys are cut into
// a.prefix_piece[g + 1] - a.prefix_piece[g] pieces.  The row tiles of a piece are neighbours,
// on one die at one time, so that its keys come from memory once.  All items leave partial
// results, in slot w.  rows = 0: no item.
template <int ROWS>
__device__ __forceinline__ PagedItem prefix_item(const PagedArgs& a, int w) {
  const int lane = threadIdx.x & 63;
  const int tiles = prefix_row_tiles<ROWS>(a.batch, a.group_shift);
  const int piece = w / tiles, i = w - piece * tiles;
  const int my_end = a.prefix_piece[min(lane, a.hkv - 1) + 1];
  const int g = __builtin_popcountll(__ballot(lane < a.hkv && my_end <= piece));
  PagedItem it = {};
  if (g >= a.hkv) return it;
  const int first = a.prefix_piece[g];
  it.g = g;
  it.table = int64_t(g) * a.max_pages;
  it.token = i * (ROWS >> a.group_shift);
  it.rows = static_cast<int>(min(int64_t(ROWS), (int64_t(a.batch) << a.group_shift) - int64_t(i) * ROWS));
  it.num0 = piece - first;
  it.num1 = piece - first + 1;
  it.den = a.prefix_piece[g + 1] - first;
  it.slot = w;
  return it;
}

// What work-group `block` of a launch over a shared prefix does: an item of the prefix, or a worker's
// piece of the keys behind it.  The two kinds alternate, in eights, or (kFirst) the prefix comes first:
// a die's work-groups go to its compute units in turn, so that each then has one of either kind (of those
// that alternate, an even number of units away, two of one).  Neighbours of the prefix's items share a die.
struct SharedWork {
  bool prefix;
  int index;
};
template <bool kFirst = false>
__device__ __forceinline__ SharedWork shared_work(const PagedArgs& a, int block) {
  const int prefix = (a.prefix_items + kNumXcd - 1) / kNumXcd, own = (a.slots + kNumXcd - 1) / kNumXcd;
  const int eight = block / kNumXcd, die = block % kNumXcd;
  if constexpr (kFirst)
    return eight < prefix ? SharedWork{true, die * prefix + eight} : SharedWork{false, (eight - prefix) * kNumXcd + die};
  const int both = 2 * min(prefix, own);
  const bool is_prefix = eight < both ? eight % 2 == 0 : prefix > own;
  const int nth = eight < both ? eight / 2 : eight - both / 2;     // of its kind on this die
  return {is_prefix, is_prefix ? die * prefix + nth : nth * kNumXcd + die};
}
inline unsigned shared_groups(const PagedArgs& a) {
  return ((a.prefix_items + kNumXcd - 1) / kNumXcd + (a.slots + kNumXcd - 1) / kNumXcd) * kNumXcd;
}

}  // namespace moa

// Work items of the paged attention of many query rows: ragged chunks of tokens over
// their caches, or the tokens of a whole batch over a shared prefix.
//
// Rows are (token, query head of the KV head) pairs, token by token, in tiles of ROWS; the
// keys of a tile are walked in tiles of 64 positions.  An item is one row tile and one of
// the pieces that its key tiles are cut into.  A row tile that is not cut writes its
// output, the others leave partial results and a merge follows.
//
// The lengths live on the device.  Each work-group forms the plan for itself: a (sequence,
// KV head) pair with T row tiles of at most E key tiles is work for T * E steps; pieces
// have at most L = max(least, all steps / groups) of them, so that there are no more pieces
// of cut tiles than 2 * groups, whatever the lengths, and long prompts are not cut at all.
#pragma once

#include "paged_device.h"

namespace moa {

// What the merge has to know of a row tile that was cut.
struct PagedSeg {
  int32_t token;     // first packed token
  int32_t head;      // KV head
  int32_t rows;
  int32_t slot;      // of its first piece
  int32_t pieces;
  int32_t pad[3];
};

struct PagedItem {
  int g;
  int pair;          // b * hkv + g (prefill)
  int token;         // packed token of the row tile's first row
  int rows;          // rows of the tile
  int pos;           // position of the first row (prefill)
  int piece, pieces;
  int slot;          // of the partial result, -1: none
};

// The same in scalar registers.
__device__ __forceinline__ PagedItem uniform(const PagedItem& i) {
  PagedItem u;
  u.g = uniform(i.g);
  u.pair = uniform(i.pair);
  u.token = uniform(i.token);
  u.rows = uniform(i.rows);
  u.pos = uniform(i.pos);
  u.piece = uniform(i.piece);
  u.pieces = uniform(i.pieces);
  u.slot = uniform(i.slot);
  return u;
}

struct PagedPlanLds {
  double steps[4];
  uint32_t sum[4][3];
  int pair;
  uint32_t before[3];
};

template <int ROWS>
__device__ __forceinline__ void pair_work(const PagedArgs& a, int pair, int& tiles, int& keys) {
  const int b = pair / a.hkv, g = a.kv_order[pair - b * a.hkv];
  const int p0 = a.positions[b];
  const int64_t n = int64_t(a.seq_start[b + 1]) - a.seq_start[b];
  tiles = keys = 0;
  if (p0 < 0 || n <= 0 || a.seq_start[b] < 0 || a.seq_start[b + 1] > a.n_tokens) return;
  constexpr int kShift = __builtin_ctz(ROWS);
  tiles = static_cast<int>(((n << a.group_shift) + ROWS - 1) >> kShift);
  const int64_t end = min(int64_t(p0) + n, int64_t(a.max_pages) << a.page_shift);
  const int64_t span = (int64_t(a.window[g]) << a.band_shift) + (ROWS >> a.group_shift) + a.num_sink;
  keys = static_cast<int>(min((end + 63) >> 6, (span >> 6) + 3));
}

// The item of this work-group, of kThreads = 256 threads; rows = 0: none.
template <int ROWS>
__device__ __forceinline__ PagedItem paged_item(const PagedArgs& a, PagedPlanLds& s) {
  constexpr int kThreads = 256;
  const int pairs = a.batch * a.hkv;
  const int each = (pairs + kThreads - 1) / kThreads;
  const int p0 = static_cast<int>(threadIdx.x) * each;
  const int p1 = min(pairs, p0 + each);
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  int tiles = 0, keys = 0;
  double steps = 0.0;
  for (int p = p0; p < p1; ++p) {
    pair_work<ROWS>(a, p, tiles, keys);
    steps += double(tiles) * keys;
  }
#pragma unroll
  for (int off = 1; off < 64; off *= 2) steps += __shfl_xor(steps, off, 64);
  if (lane == 0) s.steps[wave] = steps;
  __syncthreads();
  steps = s.steps[0] + s.steps[1] + s.steps[2] + s.steps[3];
  const int longest = max(a.least_tiles, static_cast<int>(min(ceil(steps / a.slots), 1.0e9)));   // L

  // items, pieces of cut tiles, cut tiles
  uint32_t own[3] = {0, 0, 0};
  auto add = [&](uint32_t (&c)[3]) {
    const uint32_t pieces = min((keys + longest - 1) / max(longest, 1), kPagedMaxPieces);
    c[0] += tiles * pieces;
    c[1] += pieces > 1 ? tiles * pieces : 0;
    c[2] += pieces > 1 ? tiles : 0;
    return pieces;
  };
  for (int p = p0; p < p1; ++p) {
    if (each > 1) pair_work<ROWS>(a, p, tiles, keys);
    add(own);
  }
  uint32_t incl[3] = {own[0], own[1], own[2]};
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
#pragma unroll
    for (int c = 0; c < 3; ++c) {
      const uint32_t other = __shfl_up(incl[c], off, 64);
      incl[c] += lane >= off ? other : 0;
    }
  }
  if (lane == 63) {
#pragma unroll
    for (int c = 0; c < 3; ++c) s.sum[wave][c] = incl[c];
  }
  __syncthreads();
  uint32_t total = 0, cut = 0, at[3];
#pragma unroll
  for (int c = 0; c < 3; ++c) at[c] = incl[c] - own[c];
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    total += s.sum[v][0];
    cut += s.sum[v][2];
#pragma unroll
    for (int c = 0; c < 3; ++c) at[c] += v < wave ? s.sum[v][c] : 0;
  }
  // (more items than work-groups: seq_start is no packing of n_tokens rows, and nothing is merged)
  if (blockIdx.x == 0 && threadIdx.x == 0)
    a.plan[0] = total <= gridDim.x ? static_cast<int32_t>(min(cut, static_cast<uint32_t>(a.slots))) : 0;

  // Items go to the dies in units of 16 neighbours, which share keys, one unit to each die
  // in turn and back again; few items singly.
  const uint32_t unit = total >= 16 * kNumXcd * 4 ? 16 : 1;
  const uint32_t die = blockIdx.x % kNumXcd, local = blockIdx.x / kNumXcd;
  const uint32_t round = local / unit;
  const uint32_t item = (round * kNumXcd + (round & 1 ? kNumXcd - 1 - die : die)) * unit + local % unit;
  PagedItem it = {};
  if (item >= total) return it;
  if (item >= at[0] && item < at[0] + own[0]) {      // one thread
    int p = p0;
    while (true) {
      if (each > 1) pair_work<ROWS>(a, p, tiles, keys);
      uint32_t c[3] = {0, 0, 0};
      add(c);
      if (item < at[0] + c[0]) break;
#pragma unroll
      for (int k = 0; k < 3; ++k) at[k] += c[k];
      ++p;
    }
    s.pair = p;
#pragma unroll
    for (int k = 0; k < 3; ++k) s.before[k] = at[k];
  }
  __syncthreads();
  const int pair = uniform(s.pair);
  const uint32_t k = item - uniform(s.before[0]);
  pair_work<ROWS>(a, pair, tiles, keys);
  tiles = uniform(tiles);
  it.pieces = uniform(min((keys + longest - 1) / max(longest, 1), kPagedMaxPieces));
  const int b = pair / a.hkv;
  it.g = uniform(a.kv_order[pair - b * a.hkv]);
  it.pair = b * a.hkv + it.g;
  const int start = uniform(a.seq_start[b]);
  const int64_t rows = (int64_t(uniform(a.seq_start[b + 1])) - start) << a.group_shift;
  const int from_end = k / it.pieces;                // the last row tiles first: theirs are the most keys
  it.piece = k - from_end * it.pieces;
  const int tile = tiles - 1 - from_end;
  const int tok = tile * (ROWS >> a.group_shift);
  it.token = start + tok;
  it.rows = static_cast<int>(min(int64_t(ROWS), rows - int64_t(tile) * ROWS));
  it.pos = static_cast<int>(min(int64_t(uniform(a.positions[b])) + tok, int64_t(0x7fffffff) - ROWS));
  it.slot = -1;
  if (it.pieces > 1) {
    it.slot = uniform(s.before[1]) + k;
    const uint32_t seg = uniform(s.before[2]) + from_end;
    if (it.slot >= 2 * a.slots || seg >= static_cast<uint32_t>(a.slots)) {   // not for a well-formed seq_start
      it.rows = 0;
    } else if (it.piece == 0 && threadIdx.x == 0) {
      reinterpret_cast<PagedSeg*>(a.plan + 8)[seg] = {it.token, it.g, it.rows, it.slot, it.pieces, {0, 0, 0}};
    }
  }
  return it;
}

// The item of a work-group over the shared prefix: rows are (sequence, query head) pairs.
// The pieces of the heads are counted on the host; all of them leave partial results.
template <int ROWS>
__device__ __forceinline__ PagedItem prefix_item(const PagedArgs& a) {
  const int item = static_cast<int>(blockIdx.x);
  const int lane = threadIdx.x & 63;
  const int end = a.prefix_slot[min(lane, a.hkv - 1) + 1];
  PagedItem it = {};
  it.g = __builtin_popcountll(__ballot(lane < a.hkv && end <= item));
  if (it.g >= a.hkv) return it;
  const int first = a.prefix_slot[it.g];
  const int tiles = static_cast<int>(((int64_t(a.batch) << a.group_shift) + ROWS - 1) / ROWS);
  it.pieces = (a.prefix_slot[it.g + 1] - first) / tiles;
  const int tile = (item - first) / it.pieces;
  it.piece = (item - first) - tile * it.pieces;
  it.token = tile * (ROWS >> a.group_shift);
  it.rows = min(ROWS, (a.batch << a.group_shift) - tile * ROWS);
  it.slot = item;
  return it;
}

}  // namespace moa

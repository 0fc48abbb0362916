// How the work of a paged call is cut into workers' pieces: of a decode call the keys of its
// caches, of many query rows (a prefill, or a batch over a shared prefix) the key tiles of
// its row tiles.  The lengths live on the device, so every work-group forms the split
// itself.  Plain C++, so that it also compiles without a GPU toolchain.
#pragma once

#include "paged.h"

namespace moa {

// All rounds of all caches ((sequence, KV head) pairs, in that order), laid end to end,
// cut into `workers` pieces of `per` rounds, the first `rem` of them one longer.  A round
// is what a work-group's waves read at once; every cache starts a new one.
struct PagedSplit {
  uint32_t workers, per, rem;
  MOA_PAGED_FN uint32_t start(uint32_t w) const { return w * per + (w < rem ? w : rem); }
  MOA_PAGED_FN uint32_t worker_of(uint32_t x) const {
    const uint32_t first = rem * (per + 1);
    return x < first ? x / (per + 1) : rem + (x - first) / per;
  }
};

constexpr uint32_t kPagedMaxParts = 256;   // pieces that a cache is cut into, about
constexpr uint32_t kPagedFewParts = 64;    // the same where all slots hold the call twice

// units: rounds of the call, longest: of one cache, slots: resident work-groups.
MOA_PAGED_FN PagedSplit paged_split(uint32_t units, uint32_t longest, uint32_t slots) {
  const uint32_t parts = units <= 2 * slots && longest <= 4 * kPagedFewParts ? kPagedFewParts : kPagedMaxParts;
  const uint32_t least = (longest + parts - 1) / parts;    // 0 only without any work
  PagedSplit s;
  s.workers = least ? (units + least - 1) / least : 0;
  if (s.workers > slots) s.workers = slots;
  s.per = s.workers ? units / s.workers : 0;
  s.rem = units - s.per * s.workers;
  return s;
}

// Rounds of one cache.  A token that sees no key still has its output written (zeros),
// by a worker, unless the merge writes all outputs anyway.
MOA_PAGED_FN uint32_t paged_rounds(int32_t pos, int32_t count, int round_shift, bool merge_writes) {
  if (pos < 0) return 0;
  const uint32_t n = (uint32_t(count) + (1u << round_shift) - 1) >> round_shift;
  return n == 0 && !merge_writes ? 1 : n;
}

// Rounds that each cache's start counts as, in front of its own: of at least as many caches as workers, of two
// rounds or more on average, one, as workers would else differ in starts.
MOA_PAGED_FN uint32_t paged_start_rounds(uint32_t units, uint32_t pairs, uint32_t slots) {
  return pairs >= slots && units >= 2 * pairs ? 1 : 0;
}

// Of a cache of n rounds, `start` of them its start: what a piece that has rounds [lo, hi) of them
// reads, rounds [first, last) of the keys (none where it has the start alone), and whether that is all.
struct PagedPart {
  uint32_t first, last;
  bool whole;
  MOA_PAGED_FN PagedPart(uint32_t lo, uint32_t hi, uint32_t n, uint32_t start)
      : first((lo > start ? lo : start) - start), last((hi > start ? hi : start) - start), whole(lo <= start && hi == n) {}
};

// A cache's pages in the order of its visible keys: those of the sinks, then those of
// the band (one of them may be in both).
struct VisiblePages {
  int32_t first_sink, sink_pages, first_band;
  MOA_PAGED_FN VisiblePages(const VisibleKeys& v, int shift)
      : first_sink(v.from >> shift),
        sink_pages(v.sinks > 0 ? ((v.from + v.sinks - 1) >> shift) - (v.from >> shift) + 1 : 0),
        first_band(v.band >> shift) {}
  MOA_PAGED_FN int32_t index(int32_t n) const {            // in the table, of page n
    return n < sink_pages ? first_sink + n : first_band + (n - sink_pages);
  }
  MOA_PAGED_FN int32_t number(bool sink, int32_t index) const {
    return sink ? index - first_sink : index - first_band + sink_pages;
  }
};

// ---------------------------------------------------------------------------
// Row tiles.
// ---------------------------------------------------------------------------
// Keys: what a row tile's start and end cost, about (8 heads x 4 query heads x 5,000 tokens: 239 us
// with 96, 234 with 192 and 288; fp32, 16 heads of 64, 1,501
// tokens of 2 sequences: 69.6, 69.1, 70.7).
constexpr int kTileCost = 192;

// A piece costs a start and partial results of 128 rows on their way out and back (67 KB
// each way), so it has kLeastRowCost at least (8 heads x 4 query heads, 64 tokens behind
// 8,000: 37, 35, 36 and 47 us in pieces of 128, 256, 512 and 1,024), and a call is cut only
// where the longest row tile costs kWholeRowCost more than an equal share of all (the same
// heads, whole and cut: 3,000 tokens 98 and 139 us, 2,048 68 and 87, 1,500 52 and 66; fp32,
// where a key takes longer, 16 heads of 64, 1,501 tokens of 2 sequences 91 and 69).  With row tiles for most
// work-groups, whose pieces would nearly all be parts, it takes kFullRowCost in bf16 (8 heads x 4
// query heads, 2,000 tokens behind 1,000 and 2,000, 1,426 and 1,647 more: whole 83 and 104 us, cut
// 102 and 124; 32 heads, 1,513 and 1,959 more: 108 and 140, cut 106 and 130).
constexpr int kLeastRowCost = 256;
constexpr int kWholeRowCost = 1200;
constexpr int kWholeRowCostF32 = 600;
constexpr int kFullRowCost = 1700;
// Where the table has no room for longer row tiles than these, nothing is cut, and the merge
// is left out (512 tokens 22.3 -> 18.9 us); and so few that each work-group can have a compute
// unit for itself are walked by two groups of waves (1,500 tokens, 376 tiles, 55 -> 47 us; 504
// tiles 51 -> 59).  Very few are worth cutting all the same, unless they are shorter still (30
// tokens behind 1,900, 8 tiles: whole 40 us, cut 29).
constexpr int kShortRowCost = 2200;
constexpr int kShortRowCostF32 = 600;
constexpr int kKeyGroupTiles = 400;
constexpr int kFewRowTiles = 128;

// Cost of the row tiles of one (sequence, KV head) pair: tile i ends at key
// min(first + step * (i + 1), most), step being its tokens.
struct PairCost {
  int tiles, first, shift, most;     // step = 1 << shift
  MOA_PAGED_FN int64_t before(int64_t i) const {                  // of tiles 0 .. i - 1
    int64_t ramp = most > first ? (most - first) >> shift : 0;    // tiles that end within `most`
    ramp = ramp < i ? ramp : i;
    return i * kTileCost + ramp * first + ((ramp * (ramp + 1)) << shift) / 2 + (i - ramp) * most;
  }
  MOA_PAGED_FN int64_t longest() const { return tiles > 0 ? before(tiles) - before(tiles - 1) : 0; }
};

MOA_PAGED_FN PairCost pair_cost(int64_t tokens, int pos, int window, int band_shift, int num_sink, int group_shift,
                                int tile_rows, int64_t capacity) {
  const int step = tile_rows >> group_shift;
  PairCost c = {0, 0, __builtin_ctz(static_cast<unsigned>(step)), 0};
  if (pos < 0 || tokens <= 0) return c;
  c.tiles = static_cast<int>(((tokens << group_shift) + tile_rows - 1) / tile_rows);
  int64_t most = (int64_t(window) << band_shift) + step + num_sink + 64;
  most = most < capacity ? most : capacity;
  const int64_t end = int64_t(pos) + tokens;
  c.most = static_cast<int>(most < end ? most : end);
  c.first = static_cast<int>(pos < capacity ? pos : capacity);
  return c;
}

// 2^log_workers pieces of equal cost, to one: a power of two, so that no piece's start takes
// a division (a chain of several hundred cycles, in 64 bits).
struct RowSplit {
  int64_t units;
  int32_t log_workers;
  MOA_PAGED_FN int32_t workers() const { return units > 0 ? 1 << log_workers : 0; }
  MOA_PAGED_FN int64_t start(int64_t w) const { return (units * w) >> log_workers; }
  MOA_PAGED_FN int32_t worker_of(int64_t x) const {
    // near enough in fp32, then set right
    int32_t w = static_cast<int32_t>(static_cast<float>(x) * (static_cast<float>(1 << log_workers) / static_cast<float>(units)));
    w = w < (1 << log_workers) ? w : (1 << log_workers) - 1;
    while (start(w) > x) --w;
    while (start(w + 1) <= x) ++w;
    return w;
  }
};
// As many pieces of at least `least` as there are, up to 2^log_most.
MOA_PAGED_FN RowSplit row_split(int64_t units, int32_t least, int32_t log_most) {
  RowSplit s = {units, log_most};
  while (s.log_workers > 0 && (units >> s.log_workers) < least) --s.log_workers;
  return s;
}
// Key tile of `n` at which the part [0, num) of den of a row tile ends: the same for the
// worker in front and the one behind, 0 at 0 and n at den, and rising with num.
MOA_PAGED_FN int32_t row_part(int32_t n, int64_t num, int64_t den) {
  if (num >= den) return n;
  const int32_t t = static_cast<int32_t>(static_cast<float>(n) * (static_cast<float>(num) / static_cast<float>(den)));
  return t < n ? t : n;
}

// What the merge has to know of a row tile that was cut: its pieces are those of `pieces`
// workers, the first of which wrote to slot 2 w + 1 and the others to 2 w.
struct PagedSeg {
  int32_t token;     // first packed token
  int32_t head;      // KV head
  int32_t rows;      // 0: nothing to merge
  int32_t pieces;
};

// Row tiles of a KV head's queries over a shared prefix.
template <int ROWS>
MOA_PAGED_FN int prefix_row_tiles(int batch, int group_shift) {
  return static_cast<int>(((int64_t(batch) << group_shift) + ROWS - 1) / ROWS);
}

}  // namespace moa

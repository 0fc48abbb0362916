// How the keys of a paged decode call are cut into workers' pieces.  The lengths live on
// the device, so every work-group forms the split itself, from the positions, and the
// first one leaves it to the merge.  Plain C++, so that it also compiles without a GPU
// toolchain.
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

}  // namespace moa

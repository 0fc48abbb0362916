// Arguments and key arithmetic of the paged entry points, shared by the host and the
// kernels.  Plain C++, so that it also compiles without a GPU toolchain.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "moa_internal.h"

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define MOA_PAGED_FN __host__ __device__ __forceinline__
#else
#define MOA_PAGED_FN inline
#endif

namespace moa {

constexpr int kMinPageShift = 4;         // 16 positions: the rows that a wave of a tile load covers
constexpr int kMaxPageShift = 8;
constexpr int64_t kMaxPosition = int64_t(1) << 30;
constexpr int64_t kMaxPageRows = int64_t(1) << 31;   // rows of a page pool

// New tokens into the pages, rotated on the way.
struct PagedAppendArgs {
  const void* q;             // null: only keys and values
  const void* kn;
  const void* vn;
  void* q_out;
  void* kp;
  void* vp;
  const int32_t* table;      // [batch, hkv, max_pages]
  const int32_t* positions;  // [batch]
  const int32_t* seq_start;  // [batch + 1], or null: one token per sequence
  const float* inv_freq;     // [rotary / 2]
  int64_t q_stride;          // bytes from token to token
  int64_t k_stride;
  int64_t v_stride;
  int32_t n_tokens;
  int32_t batch;
  int32_t hq;                // 0 without queries
  int32_t hkv;
  int32_t num_pages;
  int32_t page_shift;
  int32_t max_pages;
  int32_t rotary;            // 0: nothing is rotated
  int32_t interleaved;
};

// Attention over the pages.
struct PagedArgs {
  const void* q;
  void* o;
  const void* kp;
  const void* vp;
  const int32_t* table;
  const int32_t* prefix_table;   // [hkv, max_pages] of the keys in front of prefix_len, or null
  const int32_t* positions;
  const int32_t* seq_start;      // null: one token per sequence
  float* part;                   // workspace: partial results
  int32_t* plan;                 // workspace: the split, from the first kernel of a call to the merge
  float* rows_part;              // workspace: partial results of row tiles (decode: of the shared prefix, or null)
  int32_t slots;                 // work-groups that the keys are cut for
  int32_t most_tiles;            // rows: as many row tiles as there can be
  int32_t least_cost;            // rows: keys of a piece, at least
  int32_t whole_cost;            // rows: keys of a row tile that is not worth cutting,
  int32_t full_cost;             // and with row tiles for most of the work-groups
  int32_t log_slots;             // rows: log2(slots)
  int32_t prefix_items;          // work-groups over a shared prefix
  int32_t n_tokens;
  int32_t batch;
  int32_t hq;
  int32_t hkv;
  int32_t num_pages;
  int32_t page_shift;
  int32_t max_pages;
  int32_t num_sink;
  int32_t prefix_len;
  int32_t group_shift;           // log2(hq / hkv)
  int32_t band_shift;            // the band of position i starts at ((i >> shift) - window + 1) << shift
  float scale_log2;
  int32_t window[MOA_MAX_KV_HEADS];
  int32_t window_in_order[MOA_MAX_KV_HEADS];   // and the same, widest first,
  int16_t kv_order[MOA_MAX_KV_HEADS];          // of these KV heads
  int32_t prefix_piece[MOA_MAX_KV_HEADS + 1];  // first piece of each head's keys of a shared prefix
};

// Keys of one query position, as a run of sinks and a band behind them, both cut at
// `from` (keys in front of it are read elsewhere) and at the end of the table.  Key x
// of the `count` visible ones, counted from 0, is at position at(x).
struct VisibleKeys {
  int32_t from, sinks, band, count;
  MOA_PAGED_FN int32_t at(int32_t x) const { return x < sinks ? from + x : band + (x - sinks); }
};
MOA_PAGED_FN VisibleKeys visible_keys(int32_t pos, int32_t window, int32_t band_shift, int32_t num_sink, int32_t from,
                                      int32_t capacity) {
  const int32_t end = pos < capacity ? pos + 1 : capacity;
  VisibleKeys v;
  v.from = from;
  const int32_t s = num_sink < end ? num_sink : end;
  v.sinks = s > from ? s - from : 0;
  const int32_t first = ((pos >> band_shift) - window + 1) * (1 << band_shift);
  const int32_t low = num_sink > from ? num_sink : from;
  v.band = first > low ? first : low;
  v.count = v.sinks + (end > v.band ? end - v.band : 0);
  return v;
}

constexpr int kPagedPartPad = 4;         // a partial row: head_dim sums, m, l, 2 pad floats
constexpr int kPagedMaxWorkers = 4096;   // decode workers (work-groups) per launch, at most

int launch_paged_append(const PagedAppendArgs& a, int dtype, int head_dim, void* stream);
constexpr int kPagedLogRowGroups = 9;
// Work-groups that row tiles are cut for, at most, two per compute unit (twice as many: 6 chunks behind
// 16,000 keys 258 -> 263 us; fp32, 16 heads of 64, 1,501 tokens of 2 sequences, 69 -> 82).
constexpr int kPagedRowGroups = 1 << kPagedLogRowGroups;
// Work-groups over a shared prefix, about, and over the keys behind it: one of each per
// compute unit, whatever the two have to read.  Sequences x KV heads x query heads of each on a
// prefix, with up to so many keys of their own (us):
//                                     256 + 256   384 + 256   192 + 256   256 + 512
//   16 x 8 x 4 on 8,001, 500               22.7        27.2        24.2        24.7
//   48 x 8 x 8 on 32,700, 1,000            50.8        58.7        55.3        57.1
//   16 x 32 x 1 on 8,001, 500              39.5        47.2        44.9        45.3
//   48 x 32 x 1 on 8,001, 1,500             166         172         166         146
// Most keys of the last are the sequences' own: there more work-groups for them pay.
constexpr int kPagedPrefixItems = 256;
MOA_PAGED_FN int paged_tile_rows(int dtype) { return dtype == MOA_BF16 ? 128 : 64; }

// groups: no fewer than there are row tiles, nor than a.slots.
int launch_paged_rows(const PagedArgs& a, int dtype, int head_dim, int key_groups, int64_t groups, void* stream);
int launch_paged_merge(const PagedArgs& a, int dtype, int head_dim, void* stream);
int launch_paged_shared(const PagedArgs& a, int dtype, int head_dim, int group, void* stream);
int launch_paged_decode(const PagedArgs& a, int dtype, int head_dim, int group, void* stream);

}  // namespace moa

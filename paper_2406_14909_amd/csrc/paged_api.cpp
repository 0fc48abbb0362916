// Host side of the paged entry points: argument checks and dispatch to the launchers.
#include <string.h>

#include <algorithm>
#include <string>

#include "moa_internal.h"
#include "paged_split.h"

namespace moa {

namespace {

constexpr int kMaxBatch = 65535;

moa_status_t invalid(const char* who, const char* what) {
  return fail(MOA_ERR_INVALID_ARG, std::string(who) + ": " + what);
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

bool aligned8(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

// Pages of either kind: of the plan's type, or in 8 bits with scales.
struct Pool : moa_pages_t {
  bool quant;
  float* scales;
};
const Pool* pool_of(const moa_pages_t* pages, Pool* pool) {
  if (!pages) return nullptr;
  static_cast<moa_pages_t&>(*pool) = *pages;
  pool->quant = false;
  pool->scales = nullptr;
  return pool;
}
const Pool* pool_of(const moa_quant_pages_t* pages, Pool* pool) {
  if (!pages) return nullptr;
  static_cast<moa_pages_t&>(*pool) = {pages->k_pages, pages->v_pages, pages->table, pages->num_pages, pages->page_size,
                                      pages->max_pages};
  pool->quant = true;
  pool->scales = pages->scales;
  return pool;
}

size_t pool_bytes(const moa_plan_s& p, const Pool& pages) {
  return (pages.quant ? 1 : elem_size(p)) * static_cast<size_t>(pages.num_pages) * pages.page_size * p.desc.head_dim;
}

size_t scale_bytes(const Pool& pages) {
  return pages.quant ? sizeof(float) * 2 * static_cast<size_t>(pages.num_pages) * (pages.page_size / kQuantBlock) : 0;
}

size_t rows_bytes(const moa_plan_s& p, int64_t n, int heads) {
  return elem_size(p) * static_cast<size_t>(n) * heads * p.desc.head_dim;
}

moa_status_t check_sizes(const char* who, int32_t ps, int64_t num_pages, int32_t max_pages, int32_t batch,
                         int64_t n_tokens) {
  if (ps < (1 << kMinPageShift) || ps > (1 << kMaxPageShift) || (ps & (ps - 1)) != 0)
    return fail(MOA_ERR_UNSUPPORTED, std::string(who) + ": page_size must be 16, 32, 64, 128 or 256");
  if (num_pages < 1 || num_pages > kMaxPageRows / ps)
    return invalid(who, "need num_pages >= 1 and num_pages * page_size <= 2^31");
  if (max_pages < 1 || max_pages > kMaxPosition / ps)
    return invalid(who, "need max_pages >= 1 and max_pages * page_size <= 2^30");
  if (batch < 1 || batch > kMaxBatch) return invalid(who, "batch must be in [1, 65535]");
  if (n_tokens < 0 || n_tokens >= (int64_t(1) << 30)) return invalid(who, "n_tokens must be in [0, 2^30)");
  return MOA_OK;
}

moa_status_t check_pages(const char* who, const moa_plan_t* plan, const Pool* pages, const int32_t* positions,
                         int32_t batch, int64_t n_tokens) {
  if (!plan || !pages) return invalid(who, "null plan or pages");
  if (!pages->k_pages || !pages->v_pages || !pages->table || !positions) return invalid(who, "null pointer");
  if (!aligned16(pages->k_pages) || !aligned16(pages->v_pages) || !aligned4(pages->table) || !aligned4(positions))
    return invalid(who, "pages must be 16-byte aligned, table and positions 4-byte");
  if (pages->quant) {
    if (plan->desc.dtype != MOA_BF16) return fail(MOA_ERR_UNSUPPORTED, std::string(who) + ": an 8-bit cache takes bf16 plans");
    if (!pages->scales || !aligned8(pages->scales)) return invalid(who, "null or misaligned scales (8-byte aligned)");
  }
  const moa_status_t st = check_sizes(who, pages->page_size, pages->num_pages, pages->max_pages, batch, n_tokens);
  if (st != MOA_OK) return st;
  const size_t pool = pool_bytes(*plan, *pages);
  if (overlaps(pages->k_pages, pool, pages->v_pages, pool)) return invalid(who, "k_pages overlaps v_pages");
  if (const size_t sb = scale_bytes(*pages))
    if (overlaps(pages->scales, sb, pages->k_pages, pool) || overlaps(pages->scales, sb, pages->v_pages, pool))
      return invalid(who, "scales overlap the pages");
  return MOA_OK;
}

int page_shift(const moa_pages_t& pages) { return __builtin_ctz(static_cast<unsigned>(pages.page_size)); }

// Checks the arguments that the three attention calls have in common and fills in
// those of the kernels.
moa_status_t attention_args(const char* who, const moa_plan_t* plan, const Pool* pages, const void* q, void* o,
                            const int32_t* positions, int32_t batch, int64_t n_tokens, void* workspace, size_t ws_bytes,
                            PagedArgs* a) {
  const moa_status_t st = check_pages(who, plan, pages, positions, batch, n_tokens);
  if (st != MOA_OK) return st;
  if (!q || !o) return invalid(who, "null tensor pointer");
  if (!aligned16(q) || !aligned16(o)) return invalid(who, "tensors must be 16-byte aligned");
  const moa_plan_s& p = *plan;
  const moa_desc_t& d = p.desc;
  const size_t need = moa_paged_workspace_bytes(plan, batch, n_tokens);
  if (!workspace || ws_bytes < need)
    return fail(MOA_ERR_WORKSPACE, std::string(who) + ": workspace missing or smaller than moa_paged_workspace_bytes (" +
                                       std::to_string(need) + " bytes)");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u)
    return fail(MOA_ERR_WORKSPACE, std::string(who) + ": workspace must be 256-byte aligned");
  const size_t qb = rows_bytes(p, n_tokens, d.num_q_heads), pool = pool_bytes(p, *pages);
  const size_t tb = sizeof(int32_t) * static_cast<size_t>(batch) * d.num_kv_heads * pages->max_pages;
  const struct { const void* p; size_t n; } reads[] = {
      {q, qb}, {pages->k_pages, pool}, {pages->v_pages, pool}, {pages->table, tb}, {positions, sizeof(int32_t) * batch},
      {pages->scales, scale_bytes(*pages)}};
  for (const auto& r : reads)
    if (r.n && (overlaps(o, qb, r.p, r.n) || overlaps(workspace, need, r.p, r.n)))
      return invalid(who, "o or the workspace overlaps another argument");
  if (overlaps(o, qb, workspace, need)) return invalid(who, "o overlaps the workspace");
  memset(a, 0, sizeof(*a));
  a->q = q; a->o = o; a->kp = pages->k_pages; a->vp = pages->v_pages;
  a->scales = pages->scales;
  a->table = pages->table;
  a->positions = positions;
  a->part = static_cast<float*>(workspace);
  a->n_tokens = static_cast<int32_t>(n_tokens);
  a->batch = batch;
  a->hq = d.num_q_heads;
  a->hkv = d.num_kv_heads;
  a->num_pages = static_cast<int32_t>(std::min<int64_t>(pages->num_pages, INT32_MAX));
  a->page_shift = page_shift(*pages);
  a->max_pages = pages->max_pages;
  a->num_sink = d.num_sink;
  a->scale_log2 = p.scale * 1.4426950408889634f;
  a->group_shift = __builtin_ctz(static_cast<unsigned>(p.group));
  for (int h = 0; h < d.num_kv_heads; ++h) {
    a->window[h] = p.window[h];
    a->kv_order[h] = p.kv_order[h];
  }
  return MOA_OK;
}

size_t up256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }

size_t row_bytes(const moa_plan_s& p) { return sizeof(float) * (p.desc.head_dim + kPagedPartPad); }

// Row tiles of `tokens` tokens in `sequences` sequences, for one KV head, at most.
int64_t row_tiles(const moa_plan_s& p, int64_t tokens, int64_t sequences) {
  return tokens * p.group / paged_tile_rows(p.desc.dtype) + std::min(tokens, sequences);
}

// Workspaces.  Decode: partial results fp32 [workers + pairs][group][head_dim + 4], one
// slot per worker and per (sequence, KV head) pair, the split of the call, int32
// [4 + pairs + 1], and where a prefix is shared the partial results of its row tiles.
// Prefill: partial results of the row tiles that are cut, and what the merge needs of them.
struct DecodeSpace {
  size_t plan, rows, bytes;      // offsets of the split and the row tiles' results, and the end
};
DecodeSpace decode_space(const moa_plan_s& p, int32_t batch) {
  const size_t pairs = static_cast<size_t>(batch) * p.desc.num_kv_heads;
  const int rows = paged_tile_rows(p.desc.dtype);
  const size_t tiles = (static_cast<size_t>(batch) * p.group + rows - 1) / rows * p.desc.num_kv_heads;
  DecodeSpace s;
  s.plan = up256((kPagedMaxWorkers + pairs) * p.group * row_bytes(p));
  s.rows = s.plan + up256((pairs + 5) * sizeof(int32_t));
  s.bytes = s.rows + up256(std::max<size_t>(tiles, kPagedPrefixItems) * rows * row_bytes(p));
  return s;
}
struct PrefillSpace {
  size_t plan, bytes;
};
PrefillSpace prefill_space(const moa_plan_s& p) {
  PrefillSpace s;
  s.plan = up256(size_t(2) * kPagedRowGroups * paged_tile_rows(p.desc.dtype) * row_bytes(p));
  s.bytes = s.plan + up256(size_t(kPagedRowGroups) * 16);
  return s;
}

// Rounds of all caches of a decode call are counted in 31 bits.
bool countable(const moa_plan_s& p, const Pool& pages, int32_t batch) {
  int64_t keys = 0;
  for (int h = 0; h < p.desc.num_kv_heads; ++h)
    keys += std::min<int64_t>(p.capacity[h], int64_t(pages.max_pages) * pages.page_size) / 64 + 1;
  return keys * batch < (int64_t(1) << 31);
}

moa_status_t launched(const char* who, int err) {
  if (err == kGridTooLarge) return fail(MOA_ERR_UNSUPPORTED, std::string(who) + ": too much work for one launch");
  if (err) return fail(MOA_ERR_HIP, std::string(who) + ": kernel launch failed (hipError " + std::to_string(err) + ")");
  return ok();
}

moa_status_t paged_append(const char* who, const moa_plan_t* plan, const Pool* pages, const void* q, int64_t q_stride,
                              const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, void* q_out,
                              const moa_rope_t* rope, const int32_t* positions, const int32_t* seq_start,
                              int32_t batch, int64_t n_tokens, void* hip_stream) {
  const moa_status_t st = check_pages(who, plan, pages, positions, batch, n_tokens);
  if (st != MOA_OK) return st;
  if (!seq_start && n_tokens != batch) return invalid(who, "without seq_start there is one token per sequence");
  if (n_tokens == 0) return ok();
  if (!k_new || !v_new || !q != !q_out) return invalid(who, "null tensor pointer");
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(q_out) || !aligned4(seq_start))
    return invalid(who, "tensors must be 16-byte aligned (seq_start 4-byte)");
  const moa_desc_t& d = plan->desc;
  const int64_t es = static_cast<int64_t>(elem_size(*plan));
  const int64_t q_row = int64_t(d.num_q_heads) * d.head_dim, k_row = int64_t(d.num_kv_heads) * d.head_dim;
  // a token's heads are contiguous; tokens do not run into each other
  const struct { int64_t stride, row; } rows[] = {{q ? q_stride : q_row, q_row}, {k_stride, k_row}, {v_stride, k_row}};
  for (const auto& r : rows)
    if (r.stride < r.row || r.stride > (int64_t(1) << 40) || r.stride * es % 16 != 0)
      return invalid(who, "a token stride is smaller than a token or no multiple of 16 bytes");
  if (rope) {
    if (!rope->inv_freq || !aligned4(rope->inv_freq)) return invalid(who, "null or misaligned inv_freq");
    if (rope->rotary_dim < 16 || rope->rotary_dim > d.head_dim || rope->rotary_dim % 16 != 0)
      return fail(MOA_ERR_UNSUPPORTED, std::string(who) + ": rotary_dim must be a multiple of 16, at most head_dim");
    if (rope->interleaved != 0 && rope->interleaved != 1) return invalid(who, "interleaved must be 0 or 1");
  }
  const size_t pool = pool_bytes(*plan, *pages);
  const size_t qb = static_cast<size_t>(((n_tokens - 1) * (q ? q_stride : q_row) + q_row) * es);
  const size_t kb = static_cast<size_t>(((n_tokens - 1) * k_stride + k_row) * es);
  const size_t vb = static_cast<size_t>(((n_tokens - 1) * v_stride + k_row) * es);
  const size_t ob = rows_bytes(*plan, n_tokens, d.num_q_heads);
  const size_t tb = sizeof(int32_t) * static_cast<size_t>(batch) * d.num_kv_heads * pages->max_pages;
  const struct { const void* p; size_t n; } reads[] = {
      {k_new, kb}, {v_new, vb}, {pages->table, tb}, {positions, sizeof(int32_t) * batch},
      {seq_start, seq_start ? sizeof(int32_t) * (batch + 1) : 0},
      {rope ? rope->inv_freq : nullptr, rope ? sizeof(float) * (rope->rotary_dim / 2) : 0}};
  const struct { const void* p; size_t n; } written[] = {
      {pages->k_pages, pool}, {pages->v_pages, pool}, {pages->scales, scale_bytes(*pages)}};
  for (const auto& w : written) {
    if (!w.n) continue;
    for (const auto& r : reads)
      if (r.n && overlaps(w.p, w.n, r.p, r.n)) return invalid(who, "the pages overlap another argument");
    if (q && (overlaps(w.p, w.n, q, qb) || overlaps(w.p, w.n, q_out, ob)))
      return invalid(who, "the pages overlap another argument");
  }
  if (q) {
    for (const auto& r : reads)
      if (r.n && overlaps(q_out, ob, r.p, r.n)) return invalid(who, "q_out overlaps another argument");
    if (overlaps(q_out, ob, q, qb) && !(q_out == q && q_stride == q_row))
      return invalid(who, "q_out overlaps q without being q");
  }
  QuantAppendArgs args;
  memset(&args, 0, sizeof(args));
  args.scales = pages->scales;
  PagedAppendArgs& a = args.a;
  a.q = q; a.kn = k_new; a.vn = v_new; a.q_out = q_out;
  a.kp = pages->k_pages; a.vp = pages->v_pages; a.table = pages->table;
  a.positions = positions;
  a.seq_start = seq_start;
  a.q_stride = q_stride * es;
  a.k_stride = k_stride * es;
  a.v_stride = v_stride * es;
  a.n_tokens = static_cast<int32_t>(n_tokens);
  a.batch = batch;
  a.hq = q ? d.num_q_heads : 0;
  a.hkv = d.num_kv_heads;
  a.num_pages = static_cast<int32_t>(std::min<int64_t>(pages->num_pages, INT32_MAX));
  a.page_shift = page_shift(*pages);
  a.max_pages = pages->max_pages;
  if (rope) {
    a.inv_freq = rope->inv_freq;
    a.rotary = rope->rotary_dim;
    a.interleaved = rope->interleaved;
  }
  return launched(who, pages->quant ? launch_quant_append(args, d.head_dim, hip_stream)
                                    : launch_paged_append(a, d.dtype, d.head_dim, hip_stream));
}

moa_status_t paged_prefill(const char* who, const moa_plan_t* plan, const Pool* pages, const void* q, void* o,
                               const int32_t* positions, const int32_t* seq_start, int32_t batch, int64_t n_tokens,
                               void* workspace, size_t ws_bytes, void* hip_stream) {
  PagedArgs a;
  if (n_tokens == 0) {
    const moa_status_t none = check_pages(who, plan, pages, positions, batch, 0);
    return none != MOA_OK ? none : seq_start ? ok() : invalid(who, "null or misaligned seq_start");
  }
  const moa_status_t st = attention_args(who, plan, pages, q, o, positions, batch, n_tokens, workspace, ws_bytes, &a);
  if (st != MOA_OK) return st;
  if (!seq_start || !aligned4(seq_start)) return invalid(who, "null or misaligned seq_start");
  const moa_desc_t& d = plan->desc;
  const size_t sb = sizeof(int32_t) * (static_cast<size_t>(batch) + 1);
  if (overlaps(o, rows_bytes(*plan, n_tokens, d.num_q_heads), seq_start, sb) ||
      overlaps(workspace, moa_paged_workspace_bytes(plan, batch, n_tokens), seq_start, sb))
    return invalid(who, "o or the workspace overlaps seq_start");
  a.seq_start = seq_start;
  if (d.flags & MOA_BLOCK_BAND) {
    a.band_shift = 6;
    static_assert(MOA_BAND_BLOCK == 64, "band_shift is log2(MOA_BAND_BLOCK)");
    for (int h = 0; h < d.num_kv_heads; ++h) a.window[h] = (a.window[h] + MOA_BAND_BLOCK - 1) / MOA_BAND_BLOCK;
  }
  const int64_t tiles = row_tiles(*plan, n_tokens, batch) * d.num_kv_heads;
  char* ws = static_cast<char*>(workspace);
  a.rows_part = static_cast<float*>(workspace);
  a.plan = reinterpret_cast<int32_t*>(ws + prefill_space(*plan).plan);
  int64_t widest = 0;
  for (int h = 0; h < d.num_kv_heads; ++h) {
    a.window_in_order[h] = a.window[a.kv_order[h]];
    widest = std::max(widest, int64_t(a.window[h]) << a.band_shift);
  }
  const bool bf16 = d.dtype == MOA_BF16;
  const int rows = paged_tile_rows(d.dtype);
  const int64_t longest = pair_cost(n_tokens, pages->max_pages * pages->page_size - 1, static_cast<int>(widest >> a.band_shift),
                                    a.band_shift, d.num_sink, a.group_shift, rows,
                                    int64_t(pages->max_pages) * pages->page_size).longest();
  // The cost of a call is added up in 64 bits, whatever seq_start holds, and cut in 53.
  const double one = double(n_tokens) * plan->group / rows + 1;
  if (tiles >= kMaxGrid || double(tiles) * longest >= 9.0e15 || one * batch * d.num_kv_heads * longest >= 4.0e18)
    return launched(who, kGridTooLarge);
  const int64_t most = bf16 ? kShortRowCost : kShortRowCostF32;
  const bool whole = longest <= (tiles >= kFewRowTiles ? most : most / 3);   // nothing is cut: no merge
  const int key_groups = bf16 && whole && tiles <= kKeyGroupTiles ? 2 : 1;
  if (whole) a.plan = nullptr;
  // fp32 at head_dim 128 has one work-group per compute unit (32/8 heads, 100 tokens behind
  // 4,000: 80 us in twice as many pieces, 63 in these; 500 tokens 222 and 203)
  a.log_slots = kPagedLogRowGroups - (bf16 || d.head_dim == 64 ? 0 : 1);
  a.slots = 1 << a.log_slots;
  a.most_tiles = static_cast<int32_t>(tiles);
  a.least_cost = kLeastRowCost;
  a.whole_cost = bf16 ? kWholeRowCost : kWholeRowCostF32;
  a.full_cost = bf16 ? kFullRowCost : kWholeRowCostF32;
  // a work-group per row tile, dealt to the dies in whole rounds, or per piece
  const int64_t groups = std::max<int64_t>((tiles + 127) / 128 * 128, whole ? 0 : a.slots);
  int err = pages->quant ? launch_quant_rows(a, d.head_dim, key_groups, groups, hip_stream)
                         : launch_paged_rows(a, d.dtype, d.head_dim, key_groups, groups, hip_stream);
  if (!err && !whole) err = launch_paged_merge(a, d.dtype, d.head_dim, hip_stream);
  return launched(who, err);
}

int run_decode(const moa_plan_s& p, const Pool& pages, const PagedArgs& a, void* hip_stream) {
  return pages.quant ? launch_quant_decode(a, p.desc.head_dim, p.group, hip_stream)
                     : launch_paged_decode(a, p.desc.dtype, p.desc.head_dim, p.group, hip_stream);
}

moa_status_t paged_decode(const char* who, const moa_plan_t* plan, const Pool* pages, const void* q, void* o,
                              const int32_t* positions, int32_t batch, void* workspace, size_t ws_bytes,
                              void* hip_stream) {
  PagedArgs a;
  const moa_status_t st = attention_args(who, plan, pages, q, o, positions, batch, batch, workspace, ws_bytes, &a);
  if (st != MOA_OK) return st;
  if (!countable(*plan, *pages, batch)) return launched(who, kGridTooLarge);
  a.plan = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + decode_space(*plan, batch).plan);
  return launched(who, run_decode(*plan, *pages, a, hip_stream));
}

moa_status_t paged_decode_shared(const char* who, const moa_plan_t* plan, const Pool* pages, const int32_t* prefix_table,
                                     int64_t prefix_len, const void* q, void* o, const int32_t* positions,
                                     int32_t batch, void* workspace, size_t ws_bytes, void* hip_stream) {
  PagedArgs a;
  const moa_status_t st = attention_args(who, plan, pages, q, o, positions, batch, batch, workspace, ws_bytes, &a);
  if (st != MOA_OK) return st;
  if (!prefix_table || !aligned4(prefix_table)) return invalid(who, "null or misaligned prefix_table");
  if (prefix_len < 0 || prefix_len > int64_t(pages->max_pages) * pages->page_size)
    return invalid(who, "prefix_len must be in [0, max_pages * page_size]");
  const moa_desc_t& d = plan->desc;
  const size_t pb = sizeof(int32_t) * static_cast<size_t>(d.num_kv_heads) * pages->max_pages;
  if (overlaps(o, rows_bytes(*plan, batch, d.num_q_heads), prefix_table, pb) ||
      overlaps(workspace, moa_paged_workspace_bytes(plan, batch, batch), prefix_table, pb))
    return invalid(who, "o or the workspace overlaps prefix_table");
  if (!countable(*plan, *pages, batch)) return launched(who, kGridTooLarge);
  const DecodeSpace space = decode_space(*plan, batch);
  char* ws = static_cast<char*>(workspace);
  a.plan = reinterpret_cast<int32_t*>(ws + space.plan);
  if (prefix_len > 0) {
    a.prefix_table = prefix_table;
    a.prefix_len = static_cast<int32_t>(prefix_len);
    a.rows_part = reinterpret_cast<float*>(ws + space.rows);
    const int rows = paged_tile_rows(d.dtype);
    const int64_t tiles = (int64_t(batch) * plan->group + rows - 1) / rows;
    // Pieces of as few key tiles as give no more than `most` work-groups.
    int64_t keys[MOA_MAX_KV_HEADS], sum = 0, pieces = 0, widest = 0;
    for (int h = 0; h < d.num_kv_heads; ++h) {
      keys[h] = (std::min<int64_t>(prefix_len, int64_t(d.num_sink) + plan->window[h] + 63) + 63) / 64;
      sum += keys[h];
      widest = std::max(widest, keys[h]);
    }
    // fp32 at head_dim 128 has one work-group per compute unit, and half of them for each (16 x
    // 32/8 heads over 8,001 keys 54.6 -> 46.2 us, 3 over 5,000 40.5 -> 29.7, 32 over 2,000 with
    // up to 4,000 of their own 172.5 -> 175.8).
    const int32_t most = d.dtype == MOA_BF16 || d.head_dim == 64 ? kPagedPrefixItems : kPagedPrefixItems / 2;
    int64_t longest = std::max<int64_t>(2, (sum * tiles + most - 1) / most);
    for (int64_t end = widest; longest < end;) {      // at the widest head's keys there is one piece per head
      const int64_t mid = (longest + end) / 2;
      pieces = 0;
      for (int h = 0; h < d.num_kv_heads; ++h) pieces += (keys[h] + mid - 1) / mid;
      if (pieces * tiles <= most) end = mid;
      else longest = mid + 1;
    }
    pieces = 0;
    for (int h = 0; h < d.num_kv_heads; ++h) {
      a.prefix_piece[h] = static_cast<int32_t>(pieces);
      pieces += (keys[h] + longest - 1) / longest;
    }
    a.prefix_piece[d.num_kv_heads] = static_cast<int32_t>(pieces);
    a.prefix_items = static_cast<int32_t>(pieces * tiles);
    a.slots = most;
    return launched(who, pages->quant ? launch_quant_shared(a, d.head_dim, plan->group, hip_stream)
                                      : launch_paged_shared(a, d.dtype, d.head_dim, plan->group, hip_stream));
  }
  return launched(who, run_decode(*plan, *pages, a, hip_stream));
}

moa_status_t paged_assign(const char* who, const moa_plan_t* plan, const moa_page_tables_t* tables,
                          const moa_page_state_t* state, const int32_t* positions, const int32_t* seq_start,
                          const int32_t* fresh, int32_t* slots, int32_t batch, int64_t n_tokens, void* workspace,
                          size_t ws_bytes, void* hip_stream) {
  if (!plan || !tables) return invalid(who, "null plan or tables");
  if (!tables->table || !tables->free_pages || !tables->counts || !positions) return invalid(who, "null pointer");
  const void* const ints[] = {tables->table, tables->free_pages, tables->counts, positions, seq_start, fresh, slots};
  for (const void* p : ints)
    if (!aligned4(p)) return invalid(who, "tensors must be 4-byte aligned");
  const moa_status_t st = check_sizes(who, tables->page_size, tables->num_pages, tables->max_pages, batch, n_tokens);
  if (st != MOA_OK) return st;
  if (!seq_start && slots && n_tokens != batch) return invalid(who, "without seq_start there is one token per sequence");
  const moa_desc_t& d = plan->desc;
  float* const scales = state ? state->scales : nullptr;
  if (scales && d.dtype != MOA_BF16) return fail(MOA_ERR_UNSUPPORTED, std::string(who) + ": an 8-bit cache takes bf16 plans");
  if (!aligned8(scales)) return invalid(who, "misaligned scales (8-byte aligned)");
  int32_t* const lacked = state ? state->lacked : nullptr;
  if (!aligned4(lacked)) return invalid(who, "tensors must be 4-byte aligned");
  const size_t need = moa_paged_workspace_bytes(plan, batch, std::max<int64_t>(n_tokens, 1));
  if (!workspace || ws_bytes < need)
    return fail(MOA_ERR_WORKSPACE, std::string(who) + ": workspace missing or smaller than moa_paged_workspace_bytes (" +
                                       std::to_string(need) + " bytes)");
  if (reinterpret_cast<uintptr_t>(workspace) & 255u)
    return fail(MOA_ERR_WORKSPACE, std::string(who) + ": workspace must be 256-byte aligned");
  const size_t i4 = sizeof(int32_t), pairs = static_cast<size_t>(batch) * d.num_kv_heads;
  const struct { const void* p; size_t n; } args[] = {     // the first seven are written
      {tables->table, i4 * pairs * tables->max_pages},
      {tables->free_pages, i4 * static_cast<size_t>(tables->num_pages)},
      {tables->counts, i4 * 2},
      {slots, slots ? i4 * static_cast<size_t>(n_tokens) * d.num_kv_heads : 0},
      {workspace, need},
      {scales, scales ? sizeof(float) * 2 * static_cast<size_t>(tables->num_pages) * (tables->page_size / kQuantBlock) : 0},
      {lacked, lacked ? i4 * batch : 0},
      {positions, i4 * batch},
      {seq_start, seq_start ? i4 * (static_cast<size_t>(batch) + 1) : 0},
      {fresh, fresh ? i4 * batch : 0}};
  for (int i = 0; i < 7; ++i)
    for (int j = i + 1; j < 10; ++j)
      if (args[i].n && args[j].n && overlaps(args[i].p, args[i].n, args[j].p, args[j].n))
        return invalid(who, "an argument that is written overlaps another one");
  AssignArgs a;
  memset(&a, 0, sizeof(a));
  a.table = tables->table; a.free_pages = tables->free_pages; a.counts = tables->counts;
  a.positions = positions; a.seq_start = seq_start; a.fresh = fresh; a.slots = slots;
  a.plan = static_cast<int64_t*>(workspace);
  a.scales = scales;
  a.lacked = lacked;
  // The workspace has kPagedMaxWorkers rows of head_dim + 4 floats and as many more as there are pairs:
  // more than the 32 + 24 bytes a pair that the counts and their sums take.
  a.n_tokens = static_cast<int32_t>(n_tokens);
  a.batch = batch;
  a.hkv = d.num_kv_heads;
  a.num_pages = static_cast<int32_t>(std::min<int64_t>(tables->num_pages, INT32_MAX));
  a.page_shift = __builtin_ctz(static_cast<unsigned>(tables->page_size));
  a.max_pages = tables->max_pages;
  a.num_sink = d.num_sink;
  a.block_band = (d.flags & MOA_BLOCK_BAND) != 0;
  for (int h = 0; h < d.num_kv_heads; ++h) a.window[h] = plan->window[h];
  return launched(who, launch_paged_assign(a, need, hip_stream));
}

}  // namespace

}  // namespace moa

using namespace moa;

extern "C" {

moa_status_t moa_paged_append(const moa_plan_t* plan, const moa_pages_t* pages, const void* q, int64_t q_stride,
                              const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, void* q_out,
                              const moa_rope_t* rope, const int32_t* positions, const int32_t* seq_start,
                              int32_t batch, int64_t n_tokens, void* hip_stream) {
  Pool pool;
  return paged_append("moa_paged_append", plan, pool_of(pages, &pool), q, q_stride, k_new, k_stride, v_new, v_stride,
                      q_out, rope, positions, seq_start, batch, n_tokens, hip_stream);
}

moa_status_t moa_quant_append(const moa_plan_t* plan, const moa_quant_pages_t* pages, const void* q, int64_t q_stride,
                              const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, void* q_out,
                              const moa_rope_t* rope, const int32_t* positions, const int32_t* seq_start,
                              int32_t batch, int64_t n_tokens, void* hip_stream) {
  Pool pool;
  return paged_append("moa_quant_append", plan, pool_of(pages, &pool), q, q_stride, k_new, k_stride, v_new, v_stride,
                      q_out, rope, positions, seq_start, batch, n_tokens, hip_stream);
}

size_t moa_paged_workspace_bytes(const moa_plan_t* plan, int32_t batch, int64_t n_tokens) {
  if (!plan || batch < 1 || n_tokens < 1) return 0;
  return std::max(decode_space(*plan, batch).bytes, prefill_space(*plan).bytes);
}

moa_status_t moa_paged_prefill(const moa_plan_t* plan, const moa_pages_t* pages, const void* q, void* o,
                               const int32_t* positions, const int32_t* seq_start, int32_t batch, int64_t n_tokens,
                               void* workspace, size_t ws_bytes, void* hip_stream) {
  Pool pool;
  return paged_prefill("moa_paged_prefill", plan, pool_of(pages, &pool), q, o, positions, seq_start, batch, n_tokens,
                       workspace, ws_bytes, hip_stream);
}

moa_status_t moa_quant_prefill(const moa_plan_t* plan, const moa_quant_pages_t* pages, const void* q, void* o,
                               const int32_t* positions, const int32_t* seq_start, int32_t batch, int64_t n_tokens,
                               void* workspace, size_t ws_bytes, void* hip_stream) {
  Pool pool;
  return paged_prefill("moa_quant_prefill", plan, pool_of(pages, &pool), q, o, positions, seq_start, batch, n_tokens,
                       workspace, ws_bytes, hip_stream);
}

moa_status_t moa_paged_decode(const moa_plan_t* plan, const moa_pages_t* pages, const void* q, void* o,
                              const int32_t* positions, int32_t batch, void* workspace, size_t ws_bytes,
                              void* hip_stream) {
  Pool pool;
  return paged_decode("moa_paged_decode", plan, pool_of(pages, &pool), q, o, positions, batch, workspace, ws_bytes,
                      hip_stream);
}

moa_status_t moa_quant_decode(const moa_plan_t* plan, const moa_quant_pages_t* pages, const void* q, void* o,
                              const int32_t* positions, int32_t batch, void* workspace, size_t ws_bytes,
                              void* hip_stream) {
  Pool pool;
  return paged_decode("moa_quant_decode", plan, pool_of(pages, &pool), q, o, positions, batch, workspace, ws_bytes,
                      hip_stream);
}

moa_status_t moa_paged_decode_shared(const moa_plan_t* plan, const moa_pages_t* pages, const int32_t* prefix_table,
                                     int64_t prefix_len, const void* q, void* o, const int32_t* positions,
                                     int32_t batch, void* workspace, size_t ws_bytes, void* hip_stream) {
  Pool pool;
  return paged_decode_shared("moa_paged_decode_shared", plan, pool_of(pages, &pool), prefix_table, prefix_len, q, o,
                             positions, batch, workspace, ws_bytes, hip_stream);
}

moa_status_t moa_quant_decode_shared(const moa_plan_t* plan, const moa_quant_pages_t* pages, const int32_t* prefix_table,
                                     int64_t prefix_len, const void* q, void* o, const int32_t* positions,
                                     int32_t batch, void* workspace, size_t ws_bytes, void* hip_stream) {
  Pool pool;
  return paged_decode_shared("moa_quant_decode_shared", plan, pool_of(pages, &pool), prefix_table, prefix_len, q, o,
                             positions, batch, workspace, ws_bytes, hip_stream);
}

moa_status_t moa_paged_assign(const moa_plan_t* plan, const moa_page_tables_t* tables, const int32_t* positions,
                              const int32_t* seq_start, const int32_t* fresh, int32_t* slots, int32_t batch,
                              int64_t n_tokens, void* workspace, size_t ws_bytes, void* hip_stream) {
  return paged_assign("moa_paged_assign", plan, tables, nullptr, positions, seq_start, fresh, slots, batch, n_tokens,
                      workspace, ws_bytes, hip_stream);
}

moa_status_t moa_paged_assign_state(const moa_plan_t* plan, const moa_page_tables_t* tables,
                                    const moa_page_state_t* state, const int32_t* positions, const int32_t* seq_start,
                                    const int32_t* fresh, int32_t* slots, int32_t batch, int64_t n_tokens,
                                    void* workspace, size_t ws_bytes, void* hip_stream) {
  return paged_assign("moa_paged_assign_state", plan, tables, state, positions, seq_start, fresh, slots, batch, n_tokens,
                      workspace, ws_bytes, hip_stream);
}

}  // extern "C"

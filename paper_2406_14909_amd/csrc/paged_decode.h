// Decode over a paged cache: one query token per sequence, at a position of its own,
// over the keys that it sees: the sinks and the last w_g positions of each KV head, found
// through the page table.
//
// Bound by memory: each visible key and value row is read once, for all G query heads of
// its KV head.  The heads' windows differ by orders of magnitude, so the visible keys of
// all (sequence, KV head) pairs are laid end to end and cut into pieces of equal length,
// to one round, one per work-group ("worker", paged_split.h).  The lengths follow from
// positions on the device: every work-group adds up the rounds in front of its piece by
// itself (a prefix sum over the pairs, one trip to memory), which costs less than a
// launch of its own would.  Softmax statistics and sums are fp32 and kept relative to a
// running maximum; a cache that is cut leaves partial results that a second kernel merges.
// 16 sequences x 8 heads x 4 query heads, 0.36 GB: 62 us, 57 of them this kernel at
// 6.3 TB/s; one sequence x 32 heads, 35 MB: 13.8 us, most of them the start and the merge.
//
// Page numbers of a piece are fetched in one go into LDS, as rows of the pool; one lane
// per key forms the row of its key a tile ahead, and the lanes that load the row get it
// by a lane permutation.  A key on an absent page gets weight 0, and zeros for a value.
//
// Inner loops.  fp32: LPR lanes hold a row, products on the vector units.  bf16: 16x16x32
// matrix products (the G query heads padded to 16 columns),
//   S^T = K Q^T  (A = 16 keys x 32 dims, from whole rows turned in LDS),
//   O^T += V^T P^T  (B = P^T from the score registers, A = V^T by the transposing LDS
//   read, the keys of a step permuted alike on both sides).  P^T is in bf16: of a single
//   head in two columns, the second for what rounding left over, of groups in one each.
#pragma once

#include <type_traits>

#include "paged_rows.h"

namespace moa {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kPageRows = 1024;      // page numbers held in LDS
constexpr int kPlanHead = 4;         // plan: workers, per, rem, pad, then the rounds in front of each pair that has any

__device__ __forceinline__ f32x4 mma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
  (void)a;
  (void)b;
  return c;
#endif
}

// With a shared prefix: the keys behind it.  A sequence that is still inside the prefix has
// its keys read here, all of them, so that those that a tile of sequences reads of the
// prefix are one run without holes.
__device__ __forceinline__ VisibleKeys keys_of(const PagedArgs& a, int pos, int g) {
  return visible_keys(pos, a.window[g], 0, a.num_sink, pos < a.prefix_len - 1 ? 0 : a.prefix_len,
                      a.max_pages << a.page_shift);
}

__device__ __forceinline__ uint32_t rounds_of(const PagedArgs& a, int pos, int g, int round_shift) {
  return paged_rounds(pos, pos < 0 ? 0 : keys_of(a, pos, g).count, round_shift, a.rows_part != nullptr);
}

// Shared state of the walk over a worker's piece.
struct Walk {
  uint32_t wave_sum[kWaves], wave_max[kWaves];
  int pair, pos;                // where the piece begins, and its sequence's position
  uint32_t before;              // rounds in front of that pair
  int rows[kPageRows];
};

// Calls seg(b, g, keys, x0, x1, whole, pair) for each cache that this worker's piece
// touches: visible keys [x0, x1) of KV head g of sequence b, `whole` when these are all.
// Work-group uniform; every thread takes part.
template <class Seg>
__device__ __forceinline__ void for_each_piece(const PagedArgs& a, Walk& s, uint32_t w, int round_shift, Seg&& seg) {
  const int pairs = a.batch * a.hkv;
  const int each = (pairs + kThreads - 1) / kThreads;
  const int p0 = static_cast<int>(threadIdx.x) * each;
  const int p1 = min(pairs, p0 + each);
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  uint32_t sum = 0, longest = 0;
  int pos = -1;                                      // of the thread's last pair, of one the only one
  for (int p = p0; p < p1; ++p) {
    const int b = p / a.hkv;
    pos = a.positions[b];
    const uint32_t n = rounds_of(a, pos, p - b * a.hkv, round_shift);
    sum += n;
    longest = max(longest, n);
  }
  uint32_t incl = sum;
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const uint32_t other = __shfl_up(incl, off, 64);
    incl += lane >= off ? other : 0;
    longest = max(longest, static_cast<uint32_t>(__shfl_xor(longest, off, 64)));
  }
  if (lane == 63) {
    s.wave_sum[wave] = incl;
    s.wave_max[wave] = longest;
  }
  __syncthreads();
  uint32_t units = 0, before = 0;
  longest = 0;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    before += v < wave ? s.wave_sum[v] : 0;
    units += s.wave_sum[v];
    longest = max(longest, s.wave_max[v]);
  }
  before += incl - sum;
  const PagedSplit split = paged_split(units, longest, a.slots);
  if (w >= split.workers) return;
  if (w == 0 && threadIdx.x == 0) {
    a.plan[0] = split.workers;
    a.plan[1] = split.per;
    a.plan[2] = split.rem;
  }
  uint32_t x = split.start(w);
  const uint32_t x_end = split.start(w + 1);
  if (x >= before && x < before + sum) {             // one thread
    int p = p0;
    uint32_t at = before;
    for (; each > 1; ++p) {
      const int b = p / a.hkv;
      pos = a.positions[b];
      const uint32_t n = rounds_of(a, pos, p - b * a.hkv, round_shift);
      if (x < at + n) break;
      at += n;
    }
    s.pair = p;
    s.pos = pos;
    s.before = at;
  }
  __syncthreads();
  int pair = uniform(s.pair);
  uint32_t at = uniform(s.before);
  pos = uniform(s.pos);
  int b = pair / a.hkv, g = pair - b * a.hkv;
  while (true) {
    const uint32_t n = rounds_of(a, pos, g, round_shift);
    if (n > 0) {
      const VisibleKeys keys = keys_of(a, pos, g);
      const uint32_t lo = x - at, hi = min(n, lo + (x_end - x));
      if (lo == 0 && threadIdx.x == 0) a.plan[kPlanHead + pair] = static_cast<int32_t>(at);
      seg(b, g, keys, static_cast<int>(lo << round_shift),
          static_cast<int>(min(static_cast<uint32_t>(keys.count), hi << round_shift)), lo == 0 && hi == n, pair);
      x += hi - lo;
      if (x >= x_end) break;
    }
    at += n;
    ++pair;
    if (++g == a.hkv) {
      g = 0;
      pos = uniform(a.positions[++b]);
    }
  }
}

// The rows of a piece's keys: fetches page numbers into LDS in spans that fit there and
// calls part(x0, x1, row) for each, where row(x) is the pool's row of visible key x, or -1.
template <class Part>
__device__ __forceinline__ void for_each_span(const PagedArgs& a, Walk& s, int b, int g, const VisibleKeys& keys, int x0,
                                              int x1, int round_shift, Part&& part) {
  const VisiblePages pages(keys, a.page_shift);
  const int32_t* table = keys.from < a.prefix_len ? a.prefix_table + int64_t(g) * a.max_pages
                                                  : a.table + (int64_t(b) * a.hkv + g) * a.max_pages;
  const int span = ((kPageRows - 3) << a.page_shift) >> round_shift << round_shift;
  auto number = [&](int x) { return pages.number(x < keys.sinks, keys.at(x) >> a.page_shift); };
  for (int lo = x0; lo < x1; lo += span) {
    const int hi = min(x1, lo + span);
    const int first = number(lo), n = number(hi - 1) - first + 1;
    for (int i = threadIdx.x; i < n; i += kThreads)
      s.rows[i] = page_row(table[pages.index(first + i)], a.num_pages, a.page_shift);
    __syncthreads();
    part(lo, hi, [&](int x) {
      const int pos = keys.at(x);
      const int row = s.rows[pages.number(x < keys.sinks, pos >> a.page_shift) - first];
      return row < 0 ? -1 : row + (pos & ((1 << a.page_shift) - 1));
    });
    if (hi < x1) __syncthreads();                   // the numbers make room for the next ones
  }
}

// Merges the waves' states of one cache held in LDS (acc[w][h][d], ml[w][h] = (m, l), and with
// PARTS = 2 the sums of what the weights' rounding left over at h + G) and writes either o (all
// keys) or the worker's partial.  An infinite value makes NaN of the small parts' sums, which
// are left out there.
template <typename T, int D, int G, int PARTS>
__device__ __forceinline__ void merge_waves_and_store(const PagedArgs& a, const float* s_acc, const float* s_ml,
                                                      uint32_t w, int b, int g, int pair, bool whole) {
  constexpr int PS = D + kPagedPartPad;
  constexpr int H = PARTS * G;
  for (int idx = threadIdx.x; idx < G * D; idx += kThreads) {
    const int h = idx / D, d = idx % D;
    float mx = kNegBig;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) mx = fmaxf(mx, s_ml[(v * H + h) * 2]);
    float lsum = 0.0f, asum = 0.0f, low = 0.0f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const float f = fast_exp2(s_ml[(v * H + h) * 2] - mx);
      lsum += s_ml[(v * H + h) * 2 + 1] * f;
      asum += s_acc[(v * H + h) * D + d] * f;
      if constexpr (PARTS == 2) {
        lsum += s_ml[(v * H + G + h) * 2 + 1] * f;
        low += s_acc[(v * H + G + h) * D + d] * f;
      }
    }
    if constexpr (PARTS == 2) asum += finite(asum) ? low : 0.0f;
    if (whole) {
      // no key: zeros; a sum that is no number stays one, as in the merge of a cache that is cut
      static_cast<T*>(a.o)[(int64_t(b) * a.hq + g * G + h) * D + d] = static_cast<T>(lsum == 0.0f ? 0.0f : asum / lsum);
    } else {
      float* pp = a.part + ((int64_t(w) + pair) * G + h) * PS;
      pp[d] = asum;
      if (d == 0) {
        pp[D] = mx;
        pp[D + 1] = lsum;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Vector units (fp32): a wave's tile is U * RPW keys, RPW rows per load.
// ---------------------------------------------------------------------------
template <typename T, int D>
struct ValuTile {
  static constexpr int EPL = Vec16<T>::N;    // elements per lane
  static constexpr int LPR = D / EPL;        // lanes per row
  static constexpr int RPW = 64 / LPR;       // rows per load
  static constexpr int U = 8;                // loads of K and of V in flight
  static constexpr int KT = U * RPW;
  static constexpr int kRoundShift = __builtin_ctz(kWaves * KT);
};

template <int D, int G>
struct ValuLds {
  Walk walk;
  float acc[kWaves * G * D], ml[kWaves * G * 2];
};

template <typename T, int D, int G>
__device__ __forceinline__ void decode_valu(const PagedArgs& a, ValuLds<D, G>& lds, uint32_t w) {
  using TL = ValuTile<T, D>;
  constexpr int EPL = TL::EPL, LPR = TL::LPR, RPW = TL::RPW, U = TL::U, KT = TL::KT;
  Walk& s_walk = lds.walk;
  float* const s_acc = lds.acc;
  float* const s_ml = lds.ml;

  const int lane = threadIdx.x & 63;
  const int wave = uniform(threadIdx.x >> 6);
  const int rsub = lane / LPR;
  const int col = lane % LPR;

  for_each_piece(a, s_walk, w, TL::kRoundShift, [&](int b, int g, const VisibleKeys& keys, int x0, int x1, bool whole, int pair) {
    float qf[G][EPL];
    float m[G], l[G], acc[G][EPL];
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const Vec16<T> qv = load16(static_cast<const T*>(a.q) + (int64_t(b) * a.hq + g * G + h) * D + col * EPL);
      m[h] = kNegBig;
      l[h] = 0.0f;
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        qf[h][e] = qv.get(e) * a.scale_log2;
        acc[h][e] = 0.0f;
      }
    }
    const T* kbase = static_cast<const T*>(a.kp) + col * EPL;
    const T* vbase = static_cast<const T*>(a.vp) + col * EPL;
    for_each_span(a, s_walk, b, g, keys, x0, x1, TL::kRoundShift, [&](int lo, int hi, auto row_of) {
      auto rows_at = [&](int t) { return lane < KT && t + lane < hi ? row_of(t + lane) : -1; };
      int rows = rows_at(lo + wave * KT);
      for (int t0 = lo + wave * KT; t0 < hi; t0 += kWaves * KT) {
        Vec16<T> kv[U], vv[U];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = __shfl(rows, u * RPW + rsub, 64);
          in[u] = r >= 0;
          if (r >= 0) {
            kv[u] = load16_stream(kbase + int64_t(r) * D);
            vv[u] = load16_stream(vbase + int64_t(r) * D);
          } else {
            kv[u] = zero16<T>();
            vv[u] = zero16<T>();
          }
        }
        rows = rows_at(t0 + kWaves * KT);
#pragma unroll
        for (int h = 0; h < G; ++h) {
          float sc[U];
          float mb = kNegBig;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            float d = 0.0f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) d += qf[h][e] * kv[u].get(e);
            d = group_sum<LPR>(d);
            sc[u] = in[u] ? d : -INFINITY;
            mb = fmaxf(mb, sc[u]);
          }
          const float mn = fmaxf(m[h], mb);
          const float alpha = fast_exp2(m[h] - mn);
          m[h] = mn;
          l[h] *= alpha;
#pragma unroll
          for (int e = 0; e < EPL; ++e) acc[h][e] *= alpha;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const float p = fast_exp2(sc[u] - mn);
            l[h] += p;
#pragma unroll
            for (int e = 0; e < EPL; ++e) acc[h][e] += p * vv[u].get(e);
          }
        }
      }
    });

    // The lane groups of the wave (lanes with equal `col`) meet.
#pragma unroll
    for (int off = LPR; off < 64; off *= 2) {
#pragma unroll
      for (int h = 0; h < G; ++h) {
        const float m2 = __shfl_xor(m[h], off, 64);
        const float l2 = __shfl_xor(l[h], off, 64);
        const float mn = fmaxf(m[h], m2);
        const float f1 = fast_exp2(m[h] - mn), f2 = fast_exp2(m2 - mn);
        l[h] = l[h] * f1 + l2 * f2;
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          const float a2 = __shfl_xor(acc[h][e], off, 64);
          acc[h][e] = acc[h][e] * f1 + a2 * f2;
        }
        m[h] = mn;
      }
    }
    if (rsub == 0) {
#pragma unroll
      for (int h = 0; h < G; ++h) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) s_acc[(wave * G + h) * D + col * EPL + e] = acc[h][e];
        if (col == 0) {
          s_ml[(wave * G + h) * 2] = m[h];
          s_ml[(wave * G + h) * 2 + 1] = l[h];
        }
      }
    }
    __syncthreads();
    merge_waves_and_store<T, D, G, 1>(a, s_acc, s_ml, w, b, g, pair, whole && a.rows_part == nullptr);
    __syncthreads();                                // LDS is used by the next cache
  });
}

// ---------------------------------------------------------------------------
// Matrix units (bf16): a wave's tile is 32 keys.
// ---------------------------------------------------------------------------
template <int D>
struct MmaTile {
  static constexpr int KT = 32;
  static constexpr int KS = D / 32;           // steps over the head dimension
  static constexpr int DT = D / 16;           // 16-row tiles of O^T
  static constexpr int RB = D * 2;            // bytes per row
  static constexpr int CPR = RB / 16;         // 16-byte chunks per row
  static constexpr int LD = KT * CPR / 64;    // loads of K (of V) per lane
  static constexpr int kRoundShift = 7;
  static_assert(kWaves * KT == 1 << kRoundShift, "keys per round");
  // In LDS chunk c of a K row r sits at c ^ swk(r), and 32-byte block c of a V row at
  // c ^ swv(r), so that the rows that a part of the wave reads together hit distinct banks.
  __device__ __forceinline__ static int swk(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
  __device__ __forceinline__ static int swv(int r) { return D == 128 ? (r & 7) : ((r >> 1) & 3); }
};

template <int D>
struct MmaLds {
  char tile[kWaves][MmaTile<D>::KT * MmaTile<D>::RB];   // per-wave tiles; between caches the waves' states
  Walk walk;
};

template <int D, int G>
__device__ __forceinline__ void decode_mma(const PagedArgs& a, MmaLds<D>& lds, uint32_t w) {
  using TL = MmaTile<D>;
  constexpr int KT = TL::KT, KS = TL::KS, DT = TL::DT, RB = TL::RB, CPR = TL::CPR, LD = TL::LD;
  // Parts of a weight, each with columns of its own of the 16.  Of single heads, whose other
  // columns are empty anyway, a weight keeps 16 bits (is within 2^-16 of itself), so that a sum over
  // many keys is as good as moa_decode's, which keeps 32 (32 heads, 2,100 keys each 13.5 -> 13.7 us;
  // 32 x 32, 4,180 each, 320 -> 321).  Of groups it keeps 8, as in moa_decode (with 16, 23 x 8 KV
  // heads x 8 query heads 37.0 -> 38.4 us).
  constexpr int PARTS = G == 1 ? 2 : 1;
  static_assert(G >= 1 && PARTS * G <= 16, "query heads per KV head");
  static_assert((PARTS * G * D + PARTS * 2 * G) * 4 <= KT * RB, "the waves' states fit the tiles' LDS");
  Walk& s_walk = lds.walk;
  float* s_acc = reinterpret_cast<float*>(&lds.tile[0][0]);
  float* s_ml = s_acc + kWaves * PARTS * G * D;

  const int lane = threadIdx.x & 63;
  const int wave = uniform(threadIdx.x >> 6);
  const int n = lane & 15;        // column: query head n % G of part n / G
  const int q4 = lane >> 4;       // 16-lane group
  char* ts = &lds.tile[wave][0];

  // Transposing V reads: lane 16*q4 + 4e + a reads row 4*q4 + e (+ 16 for the upper half),
  // columns 16*dt + 4a .. +3.
  int rd_off[DT];
  {
    const int vr = 4 * q4 + ((lane >> 2) & 3);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) rd_off[dt] = vr * RB + ((dt ^ TL::swv(vr)) << 5) + 8 * (lane & 3);
  }

  // LDS places of a lane's chunks of a tile: those of load u repeat every 4 loads (K) and
  // every 2 (V), but for the u * 1024 bytes in front.
  int kw[4], vw[2];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int r = u * (64 / CPR) + lane / CPR, c = lane % CPR;
    kw[u] = r * RB + ((c ^ TL::swk(r)) << 4) - u * 1024;
    if (u < 2) vw[u] = r * RB + (((c >> 1) ^ TL::swv(r)) << 5) + ((c & 1) << 4) - u * 1024;
  }

  for_each_piece(a, s_walk, w, TL::kRoundShift, [&](int b, int g, const VisibleKeys& keys, int x0, int x1, bool whole, int pair) {
    // B = Q^T: lane holds column n, dims 32*kk + 8*q4 .. +7 (zero past the last part).
    bf16x8 qop[KS];
    if (n < PARTS * G) {
      const bf16* qp = static_cast<const bf16*>(a.q) + (int64_t(b) * a.hq + g * G + n % G) * D + 8 * q4;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) qop[kk] = *reinterpret_cast<const bf16x8*>(qp + 32 * kk);
    } else {
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) qop[kk] = bf16x8{};
    }
    f32x4 oacc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float m_run = kNegBig, l_run = 0.0f;
    const float c2 = a.scale_log2;
    const char* kbase = static_cast<const char*>(a.kp) + (lane % CPR) * 16;
    const char* vbase = static_cast<const char*>(a.vp) + (lane % CPR) * 16;

    for_each_span(a, s_walk, b, g, keys, x0, x1, TL::kRoundShift, [&](int lo, int hi, auto row_of) {
      auto rows_at = [&](int t) { return lane < KT && t + lane < hi ? row_of(t + lane) : -1; };
      // K and V in whole rows: chunk u * 64 + lane is row m / CPR, chunk m % CPR.  Keys that
      // are not there read row 0 of the pool, and are taken out below.  The next tile's K is
      // asked for as soon as this one's registers are free, its V likewise.
      bf16x8 kr[LD], vr[LD];
      auto load = [&](const char* base, int rows, bf16x8 (&x)[LD]) {
        const int row0 = max(rows, 0);
#pragma unroll
        for (int u = 0; u < LD; ++u) {
          const uint32_t r = __shfl(row0, u * (64 / CPR) + lane / CPR, 64);
          x[u] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(base + uint64_t(r) * RB));
        }
      };
      int rows = rows_at(lo + wave * KT);
      if (lo + wave * KT < hi) {
        load(kbase, rows, kr);
        load(vbase, rows, vr);
      }
      for (int t0 = lo + wave * KT; t0 < hi; t0 += kWaves * KT) {
        const uint32_t there = static_cast<uint32_t>(__ballot(rows >= 0));
        const bool more = t0 + kWaves * KT < hi;
        rows = rows_at(t0 + kWaves * KT);
#pragma unroll
        for (int u = 0; u < LD; ++u) *reinterpret_cast<bf16x8*>(ts + kw[u & 3] + u * 1024) = kr[u];
        if (more) load(kbase, rows, kr);
        sched_fence();
        f32x4 s[2];
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          const int r = 16 * st + n;
          bf16x8 kop[KS];
#pragma unroll
          for (int kk = 0; kk < KS; ++kk)
            kop[kk] = *reinterpret_cast<const bf16x8*>(ts + r * RB + (((4 * kk + q4) ^ TL::swk(r)) << 4));
          s[st] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int kk = 0; kk < KS; ++kk) s[st] = mma16(kop[kk], qop[kk], s[st]);
        }
        if (there != 0xffffffffu) {
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[st][i] = there >> (16 * st + 4 * q4 + i) & 1 ? s[st][i] : -INFINITY;
#pragma unroll
          for (int u = 0; u < LD; ++u)
            if (!(there >> ((u * 64 + lane) / CPR) & 1)) vr[u] = bf16x8{};
        }
        float tmax = -INFINITY;
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) tmax = fmaxf(tmax, s[st][i]);
        tmax = max_xor<16>(tmax);
        tmax = max_xor<32>(tmax);
        const float m_new = fmaxf(m_run, tmax * c2);
        const float alpha = fast_exp2(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;

        // P^T: score tiles 0 (keys 4*q4 + i) and 1 (keys 16 + 4*q4 + i).  Weights are rounded
        // to bf16 for the product, and what that leaves over, in the second part's columns, once
        // more; the sum is taken over the same parts.
        bf16x8 pop;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float p = fast_exp2(__builtin_fmaf(s[i >> 2][i & 3], c2, -m_new));
          pop[i] = static_cast<bf16>(p);
          if constexpr (PARTS == 2) pop[i] = n < G ? pop[i] : static_cast<bf16>(p - static_cast<float>(pop[i]));
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) l_run = dot2_ones(pop[i], pop[i + 1], l_run);
#pragma unroll
        for (int u = 0; u < LD; ++u) *reinterpret_cast<bf16x8*>(ts + vw[u & 1] + u * 1024) = vr[u];
        if (more) load(vbase, rows, vr);
        sched_fence();
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          const bf16x4 v0 = read_tr(ts + rd_off[dt]);
          const bf16x4 v1 = read_tr(ts + rd_off[dt] + 16 * RB);
          const bf16x8 va = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
          oacc[dt] = mma16(va, pop, oacc[dt]);
        }
      }
    });

    // Row sums of the four 16-lane groups; the running maximum is shared already.
    l_run = sum_xor<16>(l_run);
    l_run = sum_xor<32>(l_run);
    __syncthreads();                                // every wave is done with its tile
    if (n < PARTS * G) {
      const int at = wave * PARTS * G + n;
      float* sa = s_acc + at * D + 4 * q4;               // lane holds O^T rows 16*dt + 4*q4 + i
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4*>(sa + 16 * dt) = oacc[dt];
      if (q4 == 0) {
        s_ml[at * 2] = m_run;
        s_ml[at * 2 + 1] = l_run;
      }
    }
    __syncthreads();
    merge_waves_and_store<bf16, D, G, PARTS>(a, s_acc, s_ml, w, b, g, pair, whole && a.rows_part == nullptr);
    __syncthreads();                                // LDS is used by the next cache
  });
}

// The worker of a type: bf16 goes to the matrix units, of single heads too, as they leave the
// vector units to the rest (32 heads of 8,260 keys on average 29.0 -> 28.3 us, 32 x 32 of 4,180
// 326 -> 321).
template <typename T>
constexpr __host__ __device__ bool on_matrix_units() { return sizeof(T) == 2; }
template <typename T, int D, int G>
using DecodeLds = std::conditional_t<on_matrix_units<T>(), MmaLds<D>, ValuLds<D, G>>;
template <typename T, int D, int G>
constexpr __host__ __device__ int decode_round_shift() {
  return on_matrix_units<T>() ? MmaTile<D>::kRoundShift : ValuTile<T, D>::kRoundShift;
}
template <typename T, int D, int G>
__device__ __forceinline__ void decode_worker(const PagedArgs& a, DecodeLds<T, D, G>& lds, uint32_t w) {
  if constexpr (on_matrix_units<T>()) decode_mma<D, G>(a, lds, w);
  else decode_valu<T, D, G>(a, lds, w);
}

// ---------------------------------------------------------------------------
// Merge of the partial results of every cache that is cut:
// o = sum_p 2^(m_p - M) acc_p / sum_p 2^(m_p - M) l_p, M = max_p m_p.
// One work-group per (sequence, KV head, slice of at most 2 query heads); groups of TPR
// threads take every PG-th partial, MD of them in flight, and meet in LDS.  Bound by
// latency: a trip for the split, one per PG * MD partials.  Loads are unconditional with
// the number clamped, so that none waits for another.
// ---------------------------------------------------------------------------
template <int G>
constexpr int merge_heads() { return G <= 2 ? G : 2; }

template <typename T, int D, int G, bool kShared>
__global__ void __launch_bounds__(256) paged_combine_kernel(PagedArgs a) {
  constexpr int PS = D + kPagedPartPad;
  constexpr int V4 = D / 4;
  constexpr int HS = merge_heads<G>();       // query heads per work-group
  constexpr int TPR = HS * V4;               // threads per partial
  constexpr int PG = 256 / TPR;              // partials read at once
  constexpr int MD = 4;                      // in flight per thread
  constexpr int RT = sizeof(T) == 2 ? 128 : 64;   // rows of a prefix tile
  static_assert(TPR <= 256 && 256 % TPR == 0, "thread mapping");
  __shared__ f32x4 s_acc[256];
  __shared__ float s_m[256], s_l[256];
  const int pair = static_cast<int>(blockIdx.x) / (G / HS);
  const int h0 = (static_cast<int>(blockIdx.x) - pair * (G / HS)) * HS;
  const int b = pair / a.hkv, g = pair - b * a.hkv;
  const int pos = a.positions[b];
  const uint32_t x0 = a.plan[kPlanHead + pair];       // written by the worker that began with the pair, if one did
  const PagedSplit split = {static_cast<uint32_t>(a.plan[0]), static_cast<uint32_t>(a.plan[1]),
                            static_cast<uint32_t>(a.plan[2])};
  const int pg = static_cast<int>(threadIdx.x) / TPR, j = static_cast<int>(threadIdx.x) % TPR;
  const int h = j / V4, d4 = j % V4;
  // Partials 0 .. n_own - 1 are the workers', the others those of the shared prefix.
  int n_own = 0, np;
  const float *own = a.part, *prefix = nullptr;
  int64_t step = 0;                                   // from piece to piece of the prefix
  const uint32_t rounds = rounds_of(a, pos, g, decode_round_shift<T, D, G>());
  if (rounds > 0) {
    const uint32_t w0 = split.worker_of(x0), w1 = split.worker_of(x0 + rounds - 1);
    n_own = static_cast<int>(w1 - w0) + 1;
    own = a.part + ((int64_t(w0) + pair) * G + h0 + h) * PS;
  }
  np = n_own;
  if constexpr (kShared) {
    if (pos < 0) return;                              // idle
    const int row = b * G + h0 + h, tiles = prefix_row_tiles<RT>(a.batch, a.group_shift);
    const int first = a.prefix_piece[g];
    np += a.prefix_piece[g + 1] - first;
    step = int64_t(tiles) * RT * PS;
    prefix = a.rows_part + (int64_t(first) * tiles * RT + row) * PS - n_own * step;
  } else if (n_own <= 1) {
    return;                                           // idle, or its worker wrote the output
  }
  float m = kNegBig, l = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p0 = pg; p0 < np; p0 += PG * MD) {
    float mp[MD], lp[MD];
    f32x4 xp[MD];
#pragma unroll
    for (int u = 0; u < MD; ++u) {
      const int p = min(p0 + u * PG, np - 1);
      const float* q = own + int64_t(p) * G * PS;
      if constexpr (kShared) q = p < n_own ? q : prefix + p * step;
      mp[u] = q[D];
      lp[u] = q[D + 1];
      xp[u] = *reinterpret_cast<const f32x4*>(q + 4 * d4);
    }
    float mx = m;
#pragma unroll
    for (int u = 0; u < MD; ++u) mx = fmaxf(mx, mp[u]);
    const float f = fast_exp2(m - mx);
    l *= f;
    acc *= f;
    m = mx;
#pragma unroll
    for (int u = 0; u < MD; ++u) {
      const bool in = p0 + u * PG < np;
      const float wgt = in ? fast_exp2(mp[u] - mx) : 0.0f;
      l += wgt * lp[u];
      acc += (in ? xp[u] : f32x4{0.0f, 0.0f, 0.0f, 0.0f}) * wgt;
    }
  }
  if constexpr (PG > 1) {
    s_acc[threadIdx.x] = acc;
    s_m[threadIdx.x] = m;
    s_l[threadIdx.x] = l;
    __syncthreads();
    if (pg != 0) return;
    float mx = m;
#pragma unroll
    for (int v = 1; v < PG; ++v) mx = fmaxf(mx, s_m[v * TPR + j]);
    const float f = fast_exp2(m - mx);
    l *= f;
    acc *= f;
#pragma unroll
    for (int v = 1; v < PG; ++v) {
      const float wgt = fast_exp2(s_m[v * TPR + j] - mx);
      l += wgt * s_l[v * TPR + j];
      acc += s_acc[v * TPR + j] * wgt;
    }
  }
  acc *= l > 0.0f ? 1.0f / l : 0.0f;                  // no key: zeros
  T* op = static_cast<T*>(a.o) + (int64_t(b) * a.hq + g * G + h0 + h) * D + 4 * d4;
#pragma unroll
  for (int e = 0; e < 4; ++e) op[e] = static_cast<T>(acc[e]);
}

template <int G>
dim3 combine_grid(const PagedArgs& a) {
  return dim3(static_cast<unsigned>(a.batch) * a.hkv * (G / merge_heads<G>()));
}

}  // namespace

}  // namespace moa

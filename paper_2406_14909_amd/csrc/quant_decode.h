// Decode over an 8-bit paged cache: the split, the walk and the merge of paged_decode.h, over
// half the bytes.
//
// Keys and values are e4m3 numbers times a scale of their 16 rows: a lane that holds 16 of a row
// turns them into bf16, exactly and in 8 instructions, as it writes them to LDS, and from there on the
// products are those of bf16 pages: S^T = K Q^T and O^T += V^T P^T in 16x16x32 matrix instructions, query
// heads padded to 16 columns.  (The 8-bit matrix instructions take no bf16 queries; of queries in
// two 8-bit parts they need as long as bf16 ones, and add up less exactly: 1.4e-4 of a sum's magnitudes.)
//
// Bound by memory.  A wave's tile is 64 keys, so that as many bytes are on their way as of 32 keys in
// bf16, and a cache's start (positions, page numbers, rows: three trips) and end (the waves' merge) weigh
// twice as much against them: 16 sequences x 8 heads x 4 query heads, 179 MB, 38 us, 34 of them
// this kernel at 5.3 TB/s; 61 x 8 x 8, 0.67 GB, 121 us, 116 at 5.8 TB/s, of which a tenth goes into
// starts and ends; one sequence x 32 heads, 17 MB, 13 us, most of them start and merge.  Pieces are counted in
// steps of all four waves (the first two calls in pieces counted in 64, 128, 256 and 512 keys: 40.8, 40.3,
// 38.1 and 39.0 us; 128.8, 122.9, 122.8 and 121.3).  Of as many caches as workers and more, workers would
// differ in starts, so each counts as a round, too (48 x 32 heads of up to 4,200 keys 139.5 -> 125.5 us; of fewer
// caches it costs: the first call 38.2 -> 39.2; of caches of one round, 512 of up to 500 keys behind
// a prefix, 25.6 -> 27.1).
#pragma once

#include "paged_decode.h"
#include "quant_device.h"

namespace moa {

namespace {

template <int D>
struct QuantTile {
  static constexpr int KT = 64;
  static constexpr int KS = D / 32;           // steps over the head dimension
  static constexpr int DT = D / 16;           // 16-row tiles of O^T
  static constexpr int RB = D * 2;            // bytes per row in LDS
  static constexpr int CPR = D / 16;          // 16-byte chunks per stored row
  static constexpr int LD = KT * CPR / 64;    // loads of K (of V) per lane
  static constexpr int RPL = 64 / CPR;        // rows per load
  static constexpr int kRoundShift = 8;
  static_assert(kWaves * KT == 1 << kRoundShift, "keys per round");
};

template <int D>
struct QuantLds {
  char tile[kWaves][QuantTile<D>::KT * QuantTile<D>::RB];   // per-wave tiles; between caches the waves' states
  Walk walk;
};

template <int D, int G>
__device__ __forceinline__ void decode_quant(const PagedArgs& a, QuantLds<D>& lds, uint32_t w) {
  using TL = QuantTile<D>;
  using SW = MmaTile<D>;                      // the swizzles of its rows
  constexpr int KT = TL::KT, KS = TL::KS, DT = TL::DT, RB = TL::RB, CPR = TL::CPR, LD = TL::LD, RPL = TL::RPL;
  constexpr int PARTS = G == 1 ? 2 : 1;       // parts of a weight, as in decode_mma
  static_assert((PARTS * G * D + PARTS * 2 * G) * 4 <= KT * RB, "the waves' states fit the tiles' LDS");
  Walk& s_walk = lds.walk;
  float* s_acc = reinterpret_cast<float*>(&lds.tile[0][0]);
  float* s_ml = s_acc + kWaves * PARTS * G * D;

  const int lane = threadIdx.x & 63;
  const int wave = uniform(threadIdx.x >> 6);
  const int n = lane & 15;        // column: query head n % G of part n / G
  const int q4 = lane >> 4;       // 16-lane group
  char* ts = &lds.tile[wave][0];

  int rd_off[DT];                 // transposing V reads, as in decode_mma
  {
    const int vr = 4 * q4 + ((lane >> 2) & 3);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) rd_off[dt] = vr * RB + ((dt ^ SW::swv(vr)) << 5) + 8 * (lane & 3);
  }
  // LDS places of a lane's chunk of load u: its two halves of 8 keys' dimensions (K) or all of it (V), the
  // same every second load but for the rows in front.
  int kw[2][2];
  const int r8 = lane / CPR, c8 = lane % CPR;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int u = 0; u < 2; ++u) kw[u][h] = r8 * RB + (((2 * c8 + h) ^ SW::swk(u * RPL + r8)) << 4);
  }
  const int vw = r8 * RB + ((c8 ^ SW::swv(r8)) << 5);

  for_each_piece<true>(a, s_walk, w, TL::kRoundShift, [&](int b, int g, const VisibleKeys& keys, int x0, int x1, bool whole, int pair) {
    bf16x8 qop[KS];               // B = Q^T: lane holds column n, dims 32*kk + 8*q4 .. +7
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
      // A lane finds the row of one key of the tile and its scales; the lanes that load the row get
      // both by a permutation.  Keys that are not there read row 0 of the pool, and are taken out below;
      // its scale, which may be nothing, does not count.
      auto rows_at = [&](int t) { return t + lane < hi ? row_of(t + lane) : -1; };
      auto scales_at = [&](int rows) {
        const f32x2 x = reinterpret_cast<const f32x2*>(a.scales)[max(rows, 0) / kQuantBlock];
        return rows >= 0 ? x : f32x2{1.0f, 1.0f};
      };
      u32x4 kr[LD], vr[LD];
      auto load = [&](const char* base, int rows, u32x4 (&x)[LD]) {
        const int row0 = max(rows, 0);
#pragma unroll
        for (int u = 0; u < LD; ++u) {
          const uint32_t r = __shfl(row0, u * RPL + lane / CPR, 64);
          x[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base + uint64_t(r) * D));
        }
      };
      int rows = rows_at(lo + wave * KT);
      f32x2 scales = {0.0f, 0.0f};
      if (lo + wave * KT < hi) {
        scales = scales_at(rows);
        load(kbase, rows, kr);
        load(vbase, rows, vr);
      }
      for (int t0 = lo + wave * KT; t0 < hi; t0 += kWaves * KT) {
        const uint64_t there = __ballot(rows >= 0);
        const bool more = t0 + kWaves * KT < hi;
        const f32x2 sc = scales;
        rows = rows_at(t0 + kWaves * KT);
        if (more) scales = scales_at(rows);
#pragma unroll
        for (int u = 0; u < LD; ++u) {
          const float f = __shfl(sc[0], u * RPL + lane / CPR, 64);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            *reinterpret_cast<bf16x8*>(ts + kw[u & 1][h] + u * RPL * RB) = widen8(u32x2{kr[u][2 * h], kr[u][2 * h + 1]}, f);
        }
        if (more) load(kbase, rows, kr);
        sched_fence();
        f32x4 s[4];
#pragma unroll
        for (int st = 0; st < 4; ++st) {
          const int r = 16 * st + n;
          bf16x8 kop[KS];
#pragma unroll
          for (int kk = 0; kk < KS; ++kk)
            kop[kk] = *reinterpret_cast<const bf16x8*>(ts + r * RB + (((4 * kk + q4) ^ SW::swk(r)) << 4));
          s[st] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int kk = 0; kk < KS; ++kk) s[st] = mma16(kop[kk], qop[kk], s[st]);
        }
        if (there != ~uint64_t(0)) {
#pragma unroll
          for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[st][i] = there >> (16 * st + 4 * q4 + i) & 1 ? s[st][i] : -INFINITY;
#pragma unroll
          for (int u = 0; u < LD; ++u)
            if (!(there >> (u * RPL + lane / CPR) & 1)) vr[u] = u32x4{};
        }
        float tmax = -INFINITY;
#pragma unroll
        for (int st = 0; st < 4; ++st)
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

        // P^T of each 32 keys: score tiles 2h (keys 4*q4 + i) and 2h + 1 (keys 16 + 4*q4 + i),
        // rounded to bf16, in one part or two, as in decode_mma.
        bf16x8 pop[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float p = fast_exp2(__builtin_fmaf(s[2 * h + (i >> 2)][i & 3], c2, -m_new));
            pop[h][i] = static_cast<bf16>(p);
            if constexpr (PARTS == 2) pop[h][i] = n < G ? pop[h][i] : static_cast<bf16>(p - static_cast<float>(pop[h][i]));
          }
#pragma unroll
          for (int i = 0; i < 8; i += 2) l_run = dot2_ones(pop[h][i], pop[h][i + 1], l_run);
        }
#pragma unroll
        for (int u = 0; u < LD; ++u) {
          const float f = __shfl(sc[1], u * RPL + lane / CPR, 64);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            *reinterpret_cast<bf16x8*>(ts + vw + u * RPL * RB + 16 * h) = widen8(u32x2{vr[u][2 * h], vr[u][2 * h + 1]}, f);
        }
        if (more) load(vbase, rows, vr);
        sched_fence();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) {
            const bf16x4 v0 = read_tr(ts + rd_off[dt] + 32 * h * RB);
            const bf16x4 v1 = read_tr(ts + rd_off[dt] + (32 * h + 16) * RB);
            const bf16x8 va = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
            oacc[dt] = mma16(va, pop[h], oacc[dt]);
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

}  // namespace

}  // namespace moa

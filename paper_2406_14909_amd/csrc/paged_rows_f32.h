// Attention of many query rows over a paged cache in fp32: the work of paged_prefill.hip for
// fp32 plans, in tiles of 64 rows.
//
// Bound by the fp32 matrix units (32x32x2, a sixteenth of the bf16 rate; 32 heads of 64 x
// 2,048 tokens of one sequence behind 333: 192 us, 72 TFLOP/s, matrix units busy 48 %): operands come
// straight from memory, a tile's keys once per 32 rows.  Two waves share each 32 rows, and
// all four the rows of a tile that has no more: they take the 32-key tiles of the rows' span
// in turn and meet in LDS at the end.
//   S^T = K Q^T: a lane holds key lane % 32 and half of the dimensions, every other four of
//   them (which goes with which step of the product is free), so that the two halves' 16-byte
//   loads are neighbours.
//   O^T += V^T P^T: B = P^T from the score registers, a lane's A = V of one key of a pair,
//   dimension lane % 32 of 32.
// A lane looks up the page of its key two tiles ahead.  Keys that no row sees and keys on
// absent pages read the pool's first row instead, and count as zeros with weight 0.
#pragma once

#include <type_traits>

#include "paged_rows.h"

namespace moa {

namespace {

constexpr int kRowsF32 = 64;             // query rows per work-group
constexpr int kRowWaves = 4;

__device__ __forceinline__ f32x16 mma32f(float a, float b, const f32x16& c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
#else
  (void)a;
  (void)b;
  return c;
#endif
}

template <int D>
union RowsF32Lds {
  RowPlanLds plan;
  float state[(kRowWaves - 1) * (D / 2 + 2) * 64];
};

// Work-group w of a launch over ragged chunks, or (kShared) over a shared prefix.
template <int D, bool kShared>
__device__ __forceinline__ void rows_f32(const PagedArgs& a, RowsF32Lds<D>& lds, int w) {
  constexpr int PS = D + kPagedPartPad;
  constexpr int H = D / 2;                // dimensions of a half-wave
  constexpr int DT = D / 32;
  constexpr int kRegs = DT * 16 + 2;      // a lane's state
  const int lane = threadIdx.x & 63;
  const int wave = uniform(threadIdx.x >> 6);
  const int lrow = lane & 31;
  const int half = lane >> 5;
  const int gs = a.group_shift;
  auto tile = [&](const PagedItem& item) {
    const PagedItem it = uniform(item);
    __syncthreads();                      // the LDS of the tile before is free
    const int g = it.g;
    const int wband = a.window[g], bsh = a.band_shift, s = a.num_sink;
    auto band_start = [&](int i) { return ((i >> bsh) - wband + 1) * (1 << bsh); };

    const bool narrow = it.rows <= 32;
    const int row_block = narrow ? 0 : wave & 1;
    const int kg = narrow ? wave : wave >> 1, groups = narrow ? kRowWaves : kRowWaves / 2;   // of key tiles
    const int my_row = row_block * 32 + lrow;
    const bool in_tile = my_row < it.rows;
    const int token = it.token + (my_row >> gs);
    const int head = g * (1 << gs) + (my_row & ((1 << gs) - 1));
    int my_pos = -1;
    if (in_tile) my_pos = kShared ? a.positions[token] : it.pos + (my_row >> gs);
    if (kShared && my_pos < a.prefix_len - 1) my_pos = -1;   // idle, or inside the prefix: not read here
    int p_first = my_pos >= 0 ? my_pos : 0x7fffffff, p_last = my_pos;
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
      p_first = min(p_first, __shfl_xor(p_first, off, 64));
      p_last = max(p_last, __shfl_xor(p_last, off, 64));
    }
    p_first = uniform(p_first);
    p_last = uniform(p_last);
    const bool full = __ballot(my_pos >= 0) == ~0ull;

    // Keys that some row sees: [0, sinks) and [band_lo, key_end); 64-key tiles of this piece.
    const int cap = a.max_pages << a.page_shift;
    int key_end = min(p_last, cap - 1) + 1;
    if constexpr (kShared) key_end = min(key_end, a.prefix_len);
    const int sinks = min(s, key_end);
    const int band_lo = p_last < 0 ? key_end : min(max(0, band_start(p_first)), key_end);
    const int ta = (sinks + 63) / 64;
    const int tb = max(ta, band_lo / 64);
    const int ntiles = ta + (band_lo < key_end ? max(0, (key_end - 1) / 64 - tb + 1) : 0);
    const int t0 = uniform(row_part(ntiles, it.num0, it.den));
    const int t1 = uniform(row_part(ntiles, it.num1, it.den));
    const int32_t* const table = (kShared ? a.prefix_table : a.table) + it.table;

    // First key of the wave's u-th 32-key tile, and the pool's row of this lane's key there.
    auto tile_j0 = [&](int u) {
      const int t = t0 + (u >> 1);
      return (t < ta ? t : tb + (t - ta)) * 64 + 32 * (u & 1);
    };
    auto page_of = [&](int j0) {          // as the table has it
      const int j = j0 + lrow;
      return j >= key_end || (j >= sinks && j < band_lo) ? -1 : table[j >> a.page_shift];
    };
    auto row_of = [&](int j0, int page) {
      const int r = page_row(page, a.num_pages, a.page_shift);
      return r < 0 ? -1 : r + ((j0 + lrow) & ((1 << a.page_shift) - 1));
    };

    const int end = 2 * (t1 - t0);
    float qf[H];
#pragma unroll
    for (int i = 0; i < H; i += 4) {
      f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
      if (my_pos >= 0)
        x = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) + (int64_t(token) * a.hq + head) * D + 2 * i + half * 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) qf[i + e] = x[e];
    }
    f32x16 oacc[DT];
    float m_run, l_run;
    const float c2 = a.scale_log2;

    // Over the piece's keys.  `careful`: the second time, for values that are not finite.
    auto walk = [&](auto careful) {
      constexpr bool kCareful = decltype(careful)::value;
      int u = kg;
      auto page_at = [&](int v) { return v < end ? page_of(tile_j0(v)) : -1; };
      int row = row_of(tile_j0(u), page_at(u));
      // K of a tile is asked for behind the scores of the one before, V in front of its own
      // scores: each has a product's time to arrive, in one set of registers.
      f32x4 kf[H / 4];
      auto load_k = [&](int r) {
        const float* p = static_cast<const float*>(a.kp) + int64_t(max(r, 0)) * D + half * 4;
#pragma unroll
        for (int i = 0; i < H / 4; ++i) kf[i] = *reinterpret_cast<const f32x4*>(p + 8 * i);
      };
      if (u < end) load_k(row);
      int row_next = row_of(tile_j0(u + groups), page_at(u + groups));
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) oacc[dt] = f32x16{};
      m_run = kNegBig;
      l_run = 0.0f;
      for (; u < end; u += groups) {
        const int j0 = tile_j0(u);
        const uint32_t there = static_cast<uint32_t>(__ballot(row >= 0));
        // Asked for in front of V and used behind it: a wait for it is none for K.
        const int page_after = page_at(u + 2 * groups);
        sched_fence();
        float vf[16][DT];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int vrow = max(__shfl(row, (r >> 2) * 8 + half * 4 + (r & 3), 64), 0);
          const float* p = static_cast<const float*>(a.vp) + int64_t(vrow) * D + lrow;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) vf[r][dt] = p[dt * 32];
        }
        sched_fence();
        f32x16 sacc = f32x16{};
#pragma unroll
        for (int i = 0; i < H / 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) sacc = mma32f(kf[i][e], qf[4 * i + e], sacc);
        sched_fence();
        if (u + groups < end) load_k(row_next);
        sched_fence();
        if (there != 0xffffffffu) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
              vf[r][dt] = there >> ((r >> 2) * 8 + half * 4 + (r & 3)) & 1 ? vf[r][dt] : 0.0f;
        }
        if constexpr (kCareful) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vf[r][dt] = finite(vf[r][dt]) ? vf[r][dt] : 0.0f;
        }

        const bool all_vis = full && there == 0xffffffffu && j0 + 31 <= p_first && j0 + 32 <= key_end &&
                             (j0 + 32 <= s || band_start(p_last) <= j0);
        if (!all_vis) {
          const int jl = j0 + half * 4;                       // key of register 0 of this lane
          const int hi = min(my_pos, key_end - 1) - jl, band = band_start(my_pos) - jl, sink = s - jl;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int dj = (r >> 2) * 8 + (r & 3);
            const bool vis = (dj <= hi) & ((dj < sink) | (dj >= band)) & ((there >> (dj + half * 4) & 1) != 0);
            sacc[r] = vis ? sacc[r] : -INFINITY;
          }
        }
        float tmax = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, sacc[r]);
        tmax *= c2;
        if (__any(tmax > m_run + kRescaleSlack)) {
          const float m_new = fmaxf(m_run, max_xor<32>(tmax));
          const float alpha = fast_exp2(m_run - m_new);
          m_run = m_new;
          l_run *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) oacc[dt] *= alpha;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = fast_exp2(__builtin_fmaf(sacc[r], c2, -m_run));
          l_run += p;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) oacc[dt] = mma32f(vf[r][dt], p, oacc[dt]);
        }
        if constexpr (kCareful) {           // what is not finite goes to the rows that see its key
#pragma unroll 1
          for (int k = 0; k < 32; ++k) {
            const int r = __builtin_amdgcn_readlane(row, k);
            if (r < 0) continue;
            const int j = j0 + k;
            const bool vis = (j <= min(my_pos, key_end - 1)) & ((j < s) | (j >= band_start(my_pos)));
            const float* p = static_cast<const float*>(a.vp) + int64_t(r) * D + half * 4;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
              const f32x4 x = *reinterpret_cast<const f32x4*>(p + c * 8);
#pragma unroll
              for (int e = 0; e < 4; ++e) oacc[c / 4][c % 4 * 4 + e] += vis && !finite(x[e]) ? x[e] : 0.0f;
            }
          }
        }
        row = row_next;
        row_next = row_of(tile_j0(u + 2 * groups), page_after);
      }
    };
    walk(std::false_type{});
    // A weight of 0 times a value that is not finite is NaN, in a row that may not see it: the
    // sums of every row are looked at once, and the keys are taken again if need be.
    float zero = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) zero = __builtin_fmaf(oacc[dt][r], 0.0f, zero);
    if (__any(zero != 0.0f)) walk(std::true_type{});
    l_run = sum_xor<32>(l_run);

    // The waves' states of the same rows sit in the same lanes.
    if (kg > 0) {
      float* p = lds.state + (narrow ? kg - 1 : row_block) * kRegs * 64 + lane;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) p[(dt * 16 + r) * 64] = oacc[dt][r];
      p[(kRegs - 2) * 64] = m_run;
      p[(kRegs - 1) * 64] = l_run;
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll 1
    for (int v = 0; v < groups - 1; ++v) {
      const float* p = lds.state + (narrow ? v : row_block) * kRegs * 64 + lane;
      const float m2 = p[(kRegs - 2) * 64];
      const float m_new = fmaxf(m_run, m2);
      const float f1 = fast_exp2(m_run - m_new), f2 = fast_exp2(m2 - m_new);
      m_run = m_new;
      l_run = l_run * f1 + p[(kRegs - 1) * 64] * f2;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[dt][r] = oacc[dt][r] * f1 + p[(dt * 16 + r) * 64] * f2;
    }
    if (!in_tile) return;
    auto store = [&](float* out, int step, float f) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = oacc[dt][grp * 4 + e] * f;
          *reinterpret_cast<f32x4*>(out + (dt * 4 + grp) * step) = x;
        }
    };
    if (it.slot >= 0) {                   // by rows, or as the lanes hold them (see paged_prefill.hip)
      float* const pp = a.rows_part + int64_t(it.slot) * kRowsF32 * (kShared ? PS : D + 2);
      float* const st = kShared ? pp + my_row * PS + D : pp + kRowsF32 * D + my_row * 2;
      if (half == 0) {
        st[0] = m_run;
        st[1] = l_run;
      }
      if constexpr (kShared) store(pp + my_row * PS + half * 4, 8, 1.0f);
      else store(pp + (row_block * (D / 8) * 64 + lane) * 4, 256, 1.0f);
    } else {                              // a row that sees no key is 0
      store(static_cast<float*>(a.o) + (int64_t(token) * a.hq + head) * D + half * 4, 8, l_run > 0.0f ? 1.0f / l_run : 0.0f);
    }
  };
  if constexpr (kShared) {
    const PagedItem it = uniform(prefix_item<kRowsF32>(a, w));
    if (it.rows > 0) tile(it);
  } else {
    for_each_row_tile<kRowsF32, kRowWaves>(a, w, lds.plan, tile);
  }
}

}  // namespace

}  // namespace moa

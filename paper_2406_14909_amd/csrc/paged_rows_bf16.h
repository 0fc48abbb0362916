// Attention of many query rows over a paged cache (bf16): ragged chunks of new tokens over
// all that their sequences' pages hold (sinks and band of each KV head), and the tokens of
// a decode batch over a prefix that all its sequences share.
//
// Rows are (token, query head) pairs of one KV head, so that a key tile is read once for all
// the query heads that use it, and a short chunk or a batch of single tokens fills a tile of
// 128 rows.  What bounds it: in long prompts the matrix units and the board's power (32 heads,
// 16,384 tokens of 2 sequences: 849 us, 890 TFLOP/s, matrix units busy 41 % at 1.8 GHz; 6 chunks of
// 8 x 4 heads behind up to 16,000: 259 us, 652 TFLOP/s), memory and the chain of tiles where rows are few.
// Key tiles of few row tiles are cut into pieces for other work-groups (paged_rows.h).
//
// One work-group = 4 waves of 32 rows over the same 64-key tiles, which it stages in LDS by
// direct loads, K two tiles ahead and V one.  A wave loads the 16 keys of a tile that lie in
// one page: its number comes by a scalar load two tiles ahead of its use, and the page's
// address goes into the buffer descriptor.  Keys that no row sees (past the last token, in
// front of the band, in the gap behind the sinks) are replaced by a neighbour that one
// does, so that nothing unwritten is read; absent pages load as zeros and are masked.
//
// Products (32x32x16 bf16 matrix instructions):
//   S^T = K Q^T: A = keys, B = Q^T in registers; a lane holds one row's scores of 16 keys of 32.
//   O^T += V^T P^T: B = P^T straight from the score registers, rounded to bf16, A = V^T by
//   the transposing LDS read; the keys of a step are permuted alike on both sides.
// Softmax in base 2, relative to a running maximum that is raised only where a row would see
// exponents above 2^8; sums in fp32, of the rounded weights.  A weight is rounded to bf16, to within
// 2^-8 of itself, as in moa_prefill: what is left over would take a second product for V.
#pragma once

#include <type_traits>

#include "paged_rows.h"

namespace moa {

namespace {

constexpr int BN = 64;                  // keys per tile
constexpr int kRowsBf16 = 128;          // query rows per work-group: 4 waves of 32

__device__ __forceinline__ f32x16 mma32(const bf16x8& a, const bf16x8& b, const f32x16& c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
#else
  (void)a;
  (void)b;
  return c;
#endif
}

// Read through the scalar cache: the address is the same in all lanes, and nothing writes
// there during the call.
__device__ __forceinline__ int scalar_read(const int32_t* p, int i) {
#if defined(__HIP_DEVICE_COMPILE__)
  return *reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(reinterpret_cast<uintptr_t>(p + i));
#else
  return p[i];
#endif
}

template <int D>
struct RowTiles {
  static constexpr int RB = D * 2;                   // bytes per row
  static constexpr int CPR = RB / 16;                // 16-byte chunks per row
  static constexpr int TILE_BYTES = BN * RB;         // one K or V tile
  static constexpr int DPW = TILE_BYTES / 1024 / 4;   // 1 KB direct loads per wave and tile
  static constexpr int KSTAGES = 3;
  // Chunk c of K row r sits at chunk position c ^ swz_k(r), of V row r at c ^ swz_v(r): the
  // rows that one operand read takes together hit distinct banks.
  __device__ __forceinline__ static int swz_k(int r) { return CPR >= 16 ? (r & 15) : ((r >> 1) & 7); }
  __device__ __forceinline__ static int swz_v(int r) { return CPR >= 16 ? 4 * (r & 3) : 4 * ((r >> 1) & 1); }
};

// Of each key group K stages, then V stages; at first the plan.
template <int D, int KG>
struct RowsBf16Lds {
  static constexpr int GROUP = (RowTiles<D>::KSTAGES + 2) * RowTiles<D>::TILE_BYTES;
  char tiles[KG * GROUP];
};

// Work-group w of a launch over ragged chunks, or (kShared) over a shared prefix.  KG groups
// of 4 waves share its rows: group kg takes key tiles kg, kg + KG, ... through LDS stages of
// its own, and their states meet in LDS at the end.
template <int D, bool kShared, int KG>
__device__ __forceinline__ void rows_bf16(const PagedArgs& a, RowsBf16Lds<D, KG>& lds, int w) {
  using TL = RowTiles<D>;
  constexpr int KS = D / 16;              // steps over the head dimension
  constexpr int RB = TL::RB, CPR = TL::CPR, KST = TL::KSTAGES, DPW = TL::DPW;
  constexpr int PS = D + kPagedPartPad;
  const int wave_id = uniform(threadIdx.x >> 6);
  const int wave = KG == 1 ? wave_id : wave_id % 4;    // of the key group: rows
  const int kg = KG == 1 ? 0 : wave_id / 4;
  char* const sK = lds.tiles + kg * RowsBf16Lds<D, KG>::GROUP;
  char* const sV = sK + KST * TL::TILE_BYTES;

  const int lane = threadIdx.x & 63;
  const int lrow = lane & 31;
  const int half = lane >> 5;
  const int gs = a.group_shift;
  auto tile = [&](const PagedItem& item) {
    const PagedItem it = uniform(item);
    __syncthreads();                      // the LDS of the tile before is free
    const int g = it.g;
    const int wband = a.window[g], bsh = a.band_shift, s = a.num_sink;
    auto band_start = [&](int i) { return ((i >> bsh) - wband + 1) * (1 << bsh); };

    // This lane's row and its position (-1: no row, an idle sequence).
    const int row = wave * 32 + lrow;
    const bool in_tile = row < it.rows;
    const int token = it.token + (row >> gs);
    const int head = g * (1 << gs) + (row & ((1 << gs) - 1));
    int my_pos = -1;
    int p_first, p_last;                    // positions of the tile's rows, the idle ones left out
    if constexpr (kShared) {
      p_first = 0x7fffffff;
      p_last = -1;
      for (int i = lane; i < (it.rows + (1 << gs) - 1) >> gs; i += 64) {
        const int p = a.positions[it.token + i];
        if (p >= a.prefix_len - 1) {
          p_first = min(p_first, p);
          p_last = max(p_last, p);
        }
      }
#pragma unroll
      for (int off = 1; off < 64; off *= 2) {
        p_first = min(p_first, __shfl_xor(p_first, off, 64));
        p_last = max(p_last, __shfl_xor(p_last, off, 64));
      }
      p_first = uniform(p_first);
      p_last = uniform(p_last);
      if (in_tile) my_pos = a.positions[token];
      if (my_pos < a.prefix_len - 1) my_pos = -1;       // inside the prefix: not read here
    } else {
      p_first = it.pos;
      p_last = it.pos + ((it.rows - 1) >> gs);
      if (in_tile) my_pos = it.pos + (row >> gs);
    }
    const bool active = my_pos >= 0;
    int w_first = active ? my_pos : 0x7fffffff, w_last = active ? my_pos : -1;    // of the wave
#pragma unroll
    for (int off = 1; off < 32; off *= 2) {
      w_first = min(w_first, __shfl_xor(w_first, off, 64));
      w_last = max(w_last, __shfl_xor(w_last, off, 64));
    }
    w_first = uniform(w_first);
    w_last = uniform(w_last);
    const bool wave_full = __ballot(active) == ~0ull;

    // Keys that some row sees: [0, sinks) and [band_lo, key_end).
    const int cap = a.max_pages << a.page_shift;
    int key_end = min(p_last, cap - 1) + 1;
    if constexpr (kShared) key_end = min(key_end, a.prefix_len);
    const int sinks = min(s, key_end);
    const int band_lo = p_last < 0 ? key_end : min(max(0, band_start(p_first)), key_end);
    // Tiles: of the sinks [0, ta), of the band from tb on; this piece's are [t0, t1).
    const int ta = (sinks + BN - 1) / BN;
    const int tb = max(ta, band_lo / BN);
    const int ntiles = ta + (band_lo < key_end ? max(0, (key_end - 1) / BN - tb + 1) : 0);
    const int t0 = uniform(row_part(ntiles, it.num0, it.den));
    const int t1 = uniform(row_part(ntiles, it.num1, it.den));
    auto tile_j0 = [&](int t) { return (t < ta ? t : tb + (t - ta)) * BN; };

    const int ps_mask = (1 << a.page_shift) - 1;
    const int32_t* const table = (kShared ? a.prefix_table : a.table) + it.table;

    // Page numbers of a tile's four groups of 16 keys.
    struct Pages {
      int n0, n1, n2, n3;
    };
    auto fetch = [&](int j0) {
      auto page = [&](int i) { return scalar_read(table, uniform(min(j0 + 16 * i, key_end - 1) >> a.page_shift)); };
      return Pages{page(0), page(1), page(2), page(3)};
    };
    auto mine = [&](const Pages& p) {       // of the group that this wave loads
      const int lo = wave & 1 ? p.n1 : p.n0, hi = wave & 1 ? p.n3 : p.n2;
      return uniform(wave & 2 ? hi : lo);
    };
    auto present = [&](const Pages& p) {
      auto bit = [&](int n) { return static_cast<uint32_t>(n) < static_cast<uint32_t>(a.num_pages) ? 1 : 0; };
      return uniform(bit(p.n0) | bit(p.n1) << 1 | bit(p.n2) << 2 | bit(p.n3) << 3);
    };

    // Direct-to-LDS loads: instruction i of the wave writes rows 16 * wave + i * (1024 / RB) ..
    // of the tile; lane L's 16 bytes are chunk position L % CPR of row L / CPR of them.
    uint32_t k_src[DPW], v_src[DPW];        // row of the group * RB + chunk * 16
#pragma unroll
    for (int i = 0; i < DPW; ++i) {
      const int m = (wave * DPW + i) * 64 + lane;
      const int r = m / CPR, p = m % CPR;
      k_src[i] = uint32_t(r - 16 * wave) * RB + uint32_t(p ^ TL::swz_k(r)) * 16u;
      v_src[i] = uint32_t(r - 16 * wave) * RB + uint32_t(p ^ TL::swz_v(r)) * 16u;
    }
    // All 16 keys of this wave's group are seen by some row.
    auto group_full = [&](int kb) {
      return kb + 16 <= key_end && (kb + 16 <= sinks || kb >= band_lo || sinks >= band_lo);
    };
    auto group_desc = [&](const void* pool, int page, int kb) {
      const int r = page_row(page, a.num_pages, a.page_shift);
      return make_desc(static_cast<const char*>(pool) + int64_t(max(r, 0) + (kb & ps_mask)) * RB, r < 0 ? 0 : 16 * RB);
    };
    auto tile_dma = [&](const void* pool, const uint32_t (&src)[DPW], int j0, const Pages& pages, char* lds) {
      const int kb = j0 + 16 * wave;
      if (group_full(kb)) {
        const i32x4 rs = group_desc(pool, mine(pages), kb);
#pragma unroll
        for (int i = 0; i < DPW; ++i) dma16_async(rs, src[i], lds + (wave * DPW + i) * 1024);
        return;
      }
      // A key that no row sees takes a neighbour of its group, or, where there is none, of the
      // tile; so the whole group stays in one page.
      auto seen = [&](int j) {
        j = min(j, key_end - 1);
        if (j < sinks || j >= band_lo) return j;
        if (sinks > kb) return sinks - 1;
        if (band_lo < kb + 16 && band_lo < key_end) return band_lo;
        return sinks > j0 ? sinks - 1 : band_lo;
      };
      const int r = page_row(scalar_read(table, uniform(seen(kb)) >> a.page_shift), a.num_pages, a.page_shift);
      const i32x4 rs = make_desc(static_cast<const char*>(pool) + int64_t(max(r, 0)) * RB, r < 0 ? 0 : (ps_mask + 1) * RB);
#pragma unroll
      for (int i = 0; i < DPW; ++i) {
        const int c = seen(kb + static_cast<int>(src[i] / RB));
        dma16_async(rs, uint32_t(c & ps_mask) * RB + src[i] % RB, lds + (wave * DPW + i) * 1024);
      }
    };

    // Operand reads (tile independent).  K: row lrow (+ 32 * sub), elements 16 * kk + 8 * half ..;
    // V, transposing: lane 16G + 4e + a points at row (G/2)*4 + e, column 32*dt + 16*(G%2) + 4a.
    int k_off[KS];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) k_off[kk] = lrow * RB + (((2 * kk + half) ^ TL::swz_k(lrow)) * 16);
    int v_off[D / 32];
    {
      const int vr = (lane >> 5) * 4 + ((lane & 15) >> 2);
      const int a4 = lane & 3;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) {
        const int q = dt * 4 + ((lane >> 4) & 1) * 2 + (a4 >> 1);
        v_off[dt] = vr * RB + ((q ^ TL::swz_v(vr)) * 16) + (a4 & 1) * 8;
      }
    }

    f32x16 oacc[D / 32];
    float m_run, l_run;
    const float c2 = a.scale_log2;
    bf16x8 qf[KS];
    if (active) {
      const bf16* qrow = static_cast<const bf16*>(a.q) + (int64_t(token) * a.hq + head) * D + 8 * half;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) qf[kk] = *reinterpret_cast<const bf16x8*>(qrow + 16 * kk);
    } else {
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) qf[kk] = bf16x8{};
    }
    for (bool careful = false;; careful = true) {
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt) oacc[dt] = f32x16{};
      m_run = kNegBig;
      l_run = 0.0f;
      // During a group's tile t its V(t+1) and then K(t+2) stream in, and t+3's page numbers are read.
      int jt = 0, j1 = 0, j2 = 0;
      Pages pt = {}, p1 = {}, p2 = {};
      const int ts = t0 + kg;               // the group's first
      if (ts < t1) {
        jt = tile_j0(ts);
        pt = fetch(jt);
        tile_dma(a.vp, v_src, jt, pt, sV);
        tile_dma(a.kp, k_src, jt, pt, sK);
      }
      if (ts + KG < t1) {
        j1 = tile_j0(ts + KG);
        p1 = fetch(j1);
        tile_dma(a.kp, k_src, j1, p1, sK + TL::TILE_BYTES);
      }
      if (ts + 2 * KG < t1) {
        j2 = tile_j0(ts + 2 * KG);
        p2 = fetch(j2);
      }
      int k_now = 0, k_next = (KST - 1) * TL::TILE_BYTES, v_now = 0;      // byte offsets of stages
      // Wait for Q (and the first tiles) here, once: the compiler does not count the direct
      // loads and would otherwise wait for everything in flight inside the loop.
      __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
      for (int t = ts; t < t1 + kg; t += KG) {            // as many rounds for every group
        const int j0 = jt;
        const int ok = present(pt);
        if (t + KG < t1) __builtin_amdgcn_s_waitcnt(0x0F70 | DPW);  // the next K may be in flight
        else __builtin_amdgcn_s_waitcnt(0x0F70);
        if (__builtin_expect(careful && t < t1, 0)) {   // this wave's values of the tile: 0 in place of what is not finite
#pragma unroll 1
          for (int i = 0; i < DPW; ++i) {
            bf16x8* const at = reinterpret_cast<bf16x8*>(sV + v_now + (wave * DPW + i) * 1024 + lane * 16);
            bf16x8 v = *at;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = finite(static_cast<float>(v[e])) ? v[e] : static_cast<bf16>(0.0f);
            *at = v;
          }
        }
        __syncthreads();                      // K(t), V(t) are there for every wave; K(t-1), V(t-1) are free
        Pages p3 = {};
        int j3 = 0;
        if (t + 3 * KG < t1) {
          j3 = tile_j0(t + 3 * KG);
          p3 = fetch(j3);
        }

        // Does any (row, key) pair of this wave fall inside the mask?
        const bool any_vis = t < t1 && j0 <= w_last && (j0 < s || band_start(w_first) <= j0 + BN - 1);
        // At head_dim 128 the next tiles' loads go between the S products; issued at once they
        // would queue for the address unit with the waves standing still.
        constexpr bool kSpread = D == 128;
        const bool spread = kSpread && any_vis && t + 2 * KG < t1 && group_full(j1 + 16 * wave) && group_full(j2 + 16 * wave);
        if (!spread) {
          if (t + KG < t1) tile_dma(a.vp, v_src, j1, p1, sV + (v_now ^ TL::TILE_BYTES));
          if (t + 2 * KG < t1) tile_dma(a.kp, k_src, j2, p2, sK + k_next);
        }
        if (any_vis) {
          const bool all_vis = wave_full && ok == 15 && j0 + BN - 1 <= w_first && j0 + BN <= key_end &&
                               (j0 + BN <= s || band_start(w_last) <= j0);
          const char* kb = sK + k_now;
          auto kfrag = [&](int kk, int sub) {
            return *reinterpret_cast<const bf16x8*>(kb + sub * 32 * RB + k_off[kk]);
          };
          f32x16 sacc[2] = {f32x16{}, f32x16{}};
          bf16x8 kf[3][2];                    // read two steps ahead; the fence keeps that order
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            kf[kk][0] = kfrag(kk, 0);
            kf[kk][1] = kfrag(kk, 1);
          }
          auto products = [&](auto with_loads) {
            i32x4 rv = {}, rk = {};
            if constexpr (decltype(with_loads)::value) {
              rv = group_desc(a.vp, mine(p1), j1 + 16 * wave);
              rk = group_desc(a.kp, mine(p2), j2 + 16 * wave);
            }
#pragma unroll
            for (int kk = 0; kk < KS; ++kk) {
              if (kk + 2 < KS) {
                kf[(kk + 2) % 3][0] = kfrag(kk + 2, 0);
                kf[(kk + 2) % 3][1] = kfrag(kk + 2, 1);
              }
              sacc[0] = mma32(kf[kk % 3][0], qf[kk], sacc[0]);
              sacc[1] = mma32(kf[kk % 3][1], qf[kk], sacc[1]);
              if constexpr (decltype(with_loads)::value) {
                constexpr int kPerStep = 2 * DPW / KS;     // V(t+1) first: only K may be in flight at the next tile
#pragma unroll
                for (int e = 0; e < kPerStep; ++e) {
                  const int m = kk * kPerStep + e;
                  if (m < DPW) dma16_async(rv, v_src[m % DPW], sV + (v_now ^ TL::TILE_BYTES) + (wave * DPW + m) * 1024);
                  else dma16_async(rk, k_src[m % DPW], sK + k_next + (wave * DPW + m - DPW) * 1024);
                }
              }
              sched_fence();
            }
          };
          if constexpr (kSpread) {
            if (spread) products(std::true_type{});
            else products(std::false_type{});
          } else {
            products(std::false_type{});
          }

          const char* vb = sV + v_now;
          auto vfrag = [&](int step, int dt) {
            const int kb0 = (step >> 1) * 32 + 16 * (step & 1);
            const bf16x4 lo4 = read_tr(vb + kb0 * RB + v_off[dt]);
            const bf16x4 hi4 = read_tr(vb + (kb0 + 8) * RB + v_off[dt]);
            return __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7);
          };
          bf16x8 vf[2][D / 32];
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt) vf[0][dt] = vfrag(0, dt);
          sched_fence();

          if (!all_vis) {
            const int jl = j0 + half * 4;                       // key of register 0 of this lane
            const int hi = min(my_pos, key_end - 1) - jl;       // key offset <= hi (none for an idle row)
            const int band = band_start(my_pos) - jl;           // >= band
            const int sink = s - jl;                            // or < sink
#pragma unroll
            for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
              for (int r = 0; r < 16; ++r) {
                const int dj = sub * 32 + (r >> 2) * 8 + (r & 3);
                const bool vis = (dj <= hi) & ((dj < sink) | (dj >= band)) & ((ok >> (sub * 2 + (r >> 3)) & 1) != 0);
                sacc[sub][r] = vis ? sacc[sub][r] : -INFINITY;
              }
            }
          }
          float tmax = -INFINITY;
#pragma unroll
          for (int sub = 0; sub < 2; ++sub)
#pragma unroll
            for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, sacc[sub][r]);
          tmax *= c2;
          if (__any(tmax > m_run + kRescaleSlack)) {
            const float m_new = fmaxf(m_run, max_xor<32>(tmax));
            const float alpha = fast_exp2(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) oacc[dt] *= alpha;
          }
          bf16x8 pf[2][2];
          float psum = 0.0f;
#pragma unroll
          for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                pf[sub][c][e] = static_cast<bf16>(fast_exp2(__builtin_fmaf(sacc[sub][8 * c + e], c2, -m_run)));
#pragma unroll
              for (int e = 0; e < 8; e += 2) psum = dot2_ones(pf[sub][c][e], pf[sub][c][e + 1], psum);
            }
          }
          l_run += psum;
#pragma unroll
          for (int step = 0; step < 4; ++step) {
            if (step + 1 < 4) {
#pragma unroll
              for (int dt = 0; dt < D / 32; ++dt) vf[(step + 1) & 1][dt] = vfrag(step + 1, dt);
            }
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) oacc[dt] = mma32(vf[step & 1][dt], pf[step >> 1][step & 1], oacc[dt]);
          }
        }
        jt = j1;
        j1 = j2;
        j2 = j3;
        pt = p1;
        p1 = p2;
        p2 = p3;
        k_now = k_now == (KST - 1) * TL::TILE_BYTES ? 0 : k_now + TL::TILE_BYTES;
        k_next = k_next == (KST - 1) * TL::TILE_BYTES ? 0 : k_next + TL::TILE_BYTES;
        v_now ^= TL::TILE_BYTES;
      }
      if (careful) {
        // What is not finite goes to the rows that see its key.  16 keys, in one page, are
        // looked through at once.
#pragma unroll 1
        for (int i = 0; i < (t1 - ts + KG - 1) / KG * 4; ++i) {
          const int kb = tile_j0(ts + (i >> 2) * KG) + (i & 3) * 16;
          if (kb >= key_end) continue;
          const int r = page_row(scalar_read(table, uniform(kb >> a.page_shift)), a.num_pages, a.page_shift);
          if (r < 0) continue;
          const bf16* const rows = static_cast<const bf16*>(a.vp) + int64_t(r + (kb & ps_mask)) * D;
          uint32_t odd = 0;                   // keys with such a value
#pragma unroll
          for (int k = 0; k < 16; k += 64 / CPR) {
            const bf16x8 v = *reinterpret_cast<const bf16x8*>(rows + k * D + lane * 8);
            bool all = true;
#pragma unroll
            for (int e = 0; e < 8; ++e) all &= finite(static_cast<float>(v[e]));
#pragma unroll
            for (int h = 0; h < 64 / CPR; ++h) odd |= (__ballot(!all) >> (h * CPR) & ((uint64_t(1) << CPR) - 1)) ? 1u << (k + h) : 0;
          }
          while (odd != 0) {
            const int k = __builtin_ctz(odd), j = kb + k;
            odd &= odd - 1;
            const bool vis = (j <= min(my_pos, key_end - 1)) & ((j < s) | (j >= band_start(my_pos)));
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
              const bf16x4 v = *reinterpret_cast<const bf16x4*>(rows + k * D + c * 8 + half * 4);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float x = static_cast<float>(v[e]);
                oacc[c / 4][c % 4 * 4 + e] += vis && !finite(x) ? x : 0.0f;
              }
            }
          }
        }
        break;
      }
      // A weight of 0 times a value that is not finite is NaN, in a row that may not see it:
      // the sums of every row are looked at once, and the tile is taken again if need be (2 % of
      // 6 chunks behind 16,384, 1 us of a batch of 16 over 8,001 shared keys).
      float zero = 0.0f;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) zero = __builtin_fmaf(oacc[dt][r], 0.0f, zero);
      int* const bad = reinterpret_cast<int*>(lds.tiles);
      const int mine_bad = __any(zero != 0.0f);
      __syncthreads();                    // every tile has been read
      if (lane == 0) bad[wave_id] = mine_bad;
      __syncthreads();
      int any_bad = 0;
#pragma unroll
      for (int v = 0; v < 4 * KG; ++v) any_bad |= bad[v];
      if (!uniform(any_bad)) break;
      __syncthreads();                    // before the tiles are loaded again
    }
    l_run = sum_xor<32>(l_run);
    if constexpr (KG > 1) {
      // The groups' states of the same rows sit in the same lanes of waves 4 apart.
      constexpr int kRegs = D / 2 + 2;
      static_assert((KG - 1) * 4 * kRegs * 256 <= sizeof(lds.tiles), "the states fit the tiles' LDS");
      float* const st = reinterpret_cast<float*>(lds.tiles) + lane;
      __syncthreads();                    // every tile has been read
      if (kg > 0) {
        float* p = st + ((kg - 1) * 4 + wave) * kRegs * 64;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) p[(dt * 16 + r) * 64] = oacc[dt][r];
        p[(kRegs - 2) * 64] = m_run;
        p[(kRegs - 1) * 64] = l_run;
      }
      __syncthreads();
      if (kg > 0) return;
#pragma unroll 1
      for (int v = 0; v < KG - 1; ++v) {
        const float* p = st + (v * 4 + wave) * kRegs * 64;
        const float m2 = p[(kRegs - 2) * 64];
        const float m_new = fmaxf(m_run, m2);
        const float f1 = fast_exp2(m_run - m_new), f2 = fast_exp2(m2 - m_new);
        m_run = m_new;
        l_run = l_run * f1 + p[(kRegs - 1) * 64] * f2;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[dt][r] = oacc[dt][r] * f1 + p[(dt * 16 + r) * 64] * f2;
      }
    }

    if constexpr (kShared) {
      // By rows, for the merge of single tokens: turned in LDS, so that a store is whole rows.
      __syncthreads();                    // every tile has been read
      float* const turn = reinterpret_cast<float*>(lds.tiles) + wave * 32 * PS;
      static_assert(kRowsBf16 * PS * 4 <= sizeof(lds.tiles), "the rows fit the tiles' LDS");
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = oacc[dt][grp * 4 + e];
          *reinterpret_cast<f32x4*>(turn + lrow * PS + dt * 32 + grp * 8 + half * 4) = x;
        }
      __builtin_amdgcn_wave_barrier();    // the wave's own rows: in order in LDS
      float* const pp = a.rows_part + (int64_t(it.slot) * kRowsBf16 + wave * 32) * PS;
      const int rows = min(32, it.rows - wave * 32);
      constexpr int V4 = D / 4, AT = 64 / V4;              // lanes per row, rows per store
#pragma unroll
      for (int r0 = 0; r0 < 32; r0 += AT) {
        const int r = r0 + lane / V4;
        if (r < rows)
          *reinterpret_cast<f32x4*>(pp + r * PS + lane % V4 * 4) = *reinterpret_cast<const f32x4*>(turn + r * PS + lane % V4 * 4);
      }
      if (in_tile && half == 0) {
        pp[lrow * PS + D] = m_run;
        pp[lrow * PS + D + 1] = l_run;
      }
      return;
    }
    if (!in_tile) return;
    if (it.slot >= 0) {
      // As the lanes hold them, 1 KB per store (by rows, in 32-byte parts, the stores of 512
      // whole tiles took 12 us, and the merge's loads as long).
      float* const pp = a.rows_part + int64_t(it.slot) * kRowsBf16 * (D + 2);
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int grp = 0; grp < 4; ++grp) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = oacc[dt][grp * 4 + e];
          *reinterpret_cast<f32x4*>(pp + (((wave * (D / 32) + dt) * 4 + grp) * 64 + lane) * 4) = x;
        }
      if (half == 0) {
        pp[kRowsBf16 * D + row * 2] = m_run;
        pp[kRowsBf16 * D + row * 2 + 1] = l_run;
      }
      return;
    }
    const float inv_l = l_run > 0.0f ? 1.0f / l_run : 0.0f;   // a row that sees no key is 0
    bf16* orow = static_cast<bf16*>(a.o) + (int64_t(token) * a.hq + head) * D;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
#pragma unroll
      for (int grp = 0; grp < 4; ++grp) {
        bf16x4 outv;
#pragma unroll
        for (int e = 0; e < 4; ++e) outv[e] = static_cast<bf16>(oacc[dt][grp * 4 + e] * inv_l);
        *reinterpret_cast<bf16x4*>(orow + dt * 32 + grp * 8 + half * 4) = outv;
      }
    }
  };
  if constexpr (kShared) {
    const PagedItem it = uniform(prefix_item<kRowsBf16>(a, w));
    if (it.rows > 0) tile(it);
  } else {
    for_each_row_tile<kRowsBf16, 4 * KG>(a, w, *reinterpret_cast<RowPlanLds*>(lds.tiles), tile);
  }
}

}  // namespace

}  // namespace moa

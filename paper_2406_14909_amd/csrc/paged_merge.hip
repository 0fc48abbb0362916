// Merge of the partial results of row tiles whose keys were cut into pieces:
// o = sum_p 2^(m_p - M) acc_p / sum_p 2^(m_p - M) l_p, M = max_p m_p.
//
// Bound by latency, then by memory (400 row tiles in two or three pieces each, 54 MB: 14 us; with 8 loads
// in flight whatever the number of pieces, the last ones the same, 18.5).  Few tiles are cut into
// many pieces or many into few, and only the device knows: every work-group reads the notes of all workers and shares out what
// they left, 32 rows and 32 columns at a time.  Partial results lie as the lanes of the row
// kernels held them: 1 KB is 32 rows x 8 columns, lane l's float4 row l % 32, columns
// 4 * (l / 32) ..; so a wave reads whole blocks.  Each wave takes one of 4 such blocks, or,
// of more than kMany pieces, a quarter of the pieces of one, and they meet in LDS.
#include <type_traits>

#include "paged_rows.h"

namespace moa {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kGroups = 1024;    // work-groups
constexpr int kMany = 32;        // pieces above which the waves share them
constexpr int kFlight = 8;       // pieces in flight per thread

template <typename T, int D, int ROWS>
__global__ void __launch_bounds__(kThreads) paged_merge_kernel(PagedArgs a) {
  constexpr int SLOT = ROWS * (D + 2);     // floats of a partial result: accumulators, then (m, l) of each row
  constexpr int BLOCKS = D / 8;            // of 32 rows x 8 columns
  constexpr int PER = kPagedRowGroups / kThreads;
  static_assert(PER * kThreads == kPagedRowGroups && kPagedRowGroups % 64 == 0, "notes per thread");
  __shared__ PagedSeg s_seg[kPagedRowGroups];
  __shared__ uint32_t s_to[kPagedRowGroups];      // units up to and with each worker's
  __shared__ uint32_t s_wave[kWaves];
  __shared__ f32x4 s_acc[kThreads];
  __shared__ float s_m[kThreads], s_l[kThreads];
  const int thread = threadIdx.x, lane = thread & 63, wave = uniform(thread >> 6);
  // Units of a note: its blocks of 32 rows, in fours of 8 columns, or one by one.
  uint32_t n[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int w = thread * PER + i;
    PagedSeg seg = {0, 0, 0, 0};
    if (w < a.slots) seg = reinterpret_cast<const PagedSeg*>(a.plan)[w];
    s_seg[w] = seg;
    sum += seg.rows <= 0 ? 0 : (seg.rows + 31) / 32 * (seg.pieces > kMany ? BLOCKS : BLOCKS / kWaves);
    n[i] = sum;
  }
  uint32_t incl = sum;
#pragma unroll
  for (int off = 1; off < 64; off *= 2) {
    const uint32_t other = __shfl_up(incl, off, 64);
    incl += lane >= off ? other : 0;
  }
  if (lane == 63) s_wave[wave] = incl;
  __syncthreads();
  uint32_t before = incl - sum, all = 0;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    before += v < wave ? s_wave[v] : 0;
    all += s_wave[v];
  }
  if (blockIdx.x >= all) return;
#pragma unroll
  for (int i = 0; i < PER; ++i) s_to[thread * PER + i] = before + n[i];
  __syncthreads();

  for (uint32_t id = blockIdx.x; id < all; id += kGroups) {
    // the worker whose note has unit id: the first w with s_to[w] > id
    constexpr int kStride = kPagedRowGroups / 64;
    const int part = min(__builtin_popcountll(__ballot(s_to[lane * kStride + kStride - 1] <= id)), 63) * kStride;
    const int w = uniform(part + __builtin_popcountll(__ballot(lane < kStride && s_to[part + lane % kStride] <= id)));
    const PagedSeg seg = s_seg[w];
    const int k = static_cast<int>(id - (w > 0 ? s_to[w - 1] : 0));
    const bool many = seg.pieces > kMany;
    const int each = many ? BLOCKS : BLOCKS / kWaves;
    const int r32 = k / each;                                   // block of 32 rows
    const int c8 = many ? k - r32 * each : (k - r32 * each) * kWaves + wave;   // of 8 columns
    const int share = many ? wave : 0, step = many ? kWaves : 1;
    const int row = r32 * 32 + (lane & 31);
    const bool in = row < seg.rows;
    float m = kNegBig, l = 0.0f;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (in) {
      // slot 2 w + 1 of the first worker, 2 (w + p) of the others
      const float* base = a.rows_part + int64_t(2 * w) * SLOT;
      const float* block = base + ((r32 * BLOCKS + c8) * 64 + lane) * 4;
      const float* stat = base + ROWS * D + row * 2;
      // F pieces in flight, one after the other.
      auto add = [&](auto flight) {
        constexpr int F = decltype(flight)::value;
        for (int p0 = share; p0 < seg.pieces; p0 += F * step) {
          float mp[F], lp[F];
          f32x4 xp[F];
#pragma unroll
          for (int u = 0; u < F; ++u) {
            const int p = min(p0 + u * step, seg.pieces - 1);
            const int64_t at = int64_t(p == 0 ? 1 : 2 * p) * SLOT;
            mp[u] = stat[at];
            lp[u] = stat[at + 1];
            xp[u] = *reinterpret_cast<const f32x4*>(block + at);
          }
          float mx = m;
#pragma unroll
          for (int u = 0; u < F; ++u) mx = fmaxf(mx, mp[u]);
          const float f = fast_exp2(m - mx);
          l *= f;
          acc *= f;
          m = mx;
#pragma unroll
          for (int u = 0; u < F; ++u) {
            // past the last piece, which is read again there, sums count as zeros: they may be infinite
            const bool more = p0 + u * step < seg.pieces;
            const float wgt = more ? fast_exp2(mp[u] - mx) : 0.0f;
            l += wgt * lp[u];
            acc += (more ? xp[u] : f32x4{0.0f, 0.0f, 0.0f, 0.0f}) * wgt;
          }
        }
      };
      if (seg.pieces <= 2) add(std::integral_constant<int, 2>{});
      else if (seg.pieces <= 4) add(std::integral_constant<int, 4>{});
      else add(std::integral_constant<int, kFlight>{});
    }
    if (many) {
      __syncthreads();
      s_acc[thread] = acc;
      s_m[thread] = m;
      s_l[thread] = l;
      __syncthreads();
      if (wave == 0) {
        float mx = m;
#pragma unroll
        for (int v = 1; v < kWaves; ++v) mx = fmaxf(mx, s_m[thread + v * 64]);
        const float f = fast_exp2(m - mx);
        l *= f;
        acc *= f;
#pragma unroll
        for (int v = 1; v < kWaves; ++v) {
          const float wgt = fast_exp2(s_m[thread + v * 64] - mx);
          l += wgt * s_l[thread + v * 64];
          acc += s_acc[thread + v * 64] * wgt;
        }
      }
    }
    if (!in || share != 0) continue;
    acc *= l > 0.0f ? 1.0f / l : 0.0f;     // a row that sees no key is 0
    const int gs = a.group_shift;
    T* op = static_cast<T*>(a.o) + (int64_t(seg.token + (row >> gs)) * a.hq + (seg.head << gs) + (row & ((1 << gs) - 1))) * D +
            c8 * 8 + (lane >> 5) * 4;
    typedef T t4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<t4*>(op) = __builtin_convertvector(acc, t4);
  }
}

template <typename T, int D, int ROWS>
int launch_t(const PagedArgs& a, void* stream) {
  PagedArgs copy = a;
  void* args[] = {&copy};
  return static_cast<int>(hipLaunchKernel(reinterpret_cast<const void*>(&paged_merge_kernel<T, D, ROWS>), dim3(kGroups),
                                          dim3(kThreads), args, 0, static_cast<hipStream_t>(stream)));
}

}  // namespace

int launch_paged_merge(const PagedArgs& a, int dtype, int head_dim, void* stream) {
  if (dtype == MOA_BF16) return head_dim == 128 ? launch_t<bf16, 128, 128>(a, stream) : launch_t<bf16, 64, 128>(a, stream);
  return head_dim == 128 ? launch_t<float, 128, 64>(a, stream) : launch_t<float, 64, 64>(a, stream);
}

}  // namespace moa

// Merge of the partial results of row tiles whose keys were cut into pieces:
// o = sum_p 2^(m_p - M) acc_p / sum_p 2^(m_p - M) l_p, M = max_p m_p.
//
// Up to 16 work-groups per tile, of 8 rows at a time: with few pieces each row has its own
// threads (one float4 of it each); with many the threads of 4 rows share one row's pieces
// and meet in LDS, as one trip to memory per 4 pieces in a row would be what bounds it.
#include "paged_rows.h"

namespace moa {

namespace {

constexpr int kMany = 8;        // pieces from which on a row's pieces are shared out

template <typename T, int D>
__global__ void __launch_bounds__(256) paged_merge_kernel(PagedArgs a, int tile_rows) {
  constexpr int PS = D + kPagedPartPad;
  constexpr int V4 = D / 4;                // float4 per row
  constexpr int ROWS = 256 / V4;           // rows at once
  constexpr int SHARE = 4;                 // thread groups that share a row's pieces
  __shared__ f32x4 s_acc[256];
  __shared__ float s_m[256], s_l[256];
  const int blocks = tile_rows / 8;        // work-groups per tile
  const int seg_i = static_cast<int>(blockIdx.x) / blocks;
  if (seg_i >= a.plan[0]) return;
  const PagedSeg seg = reinterpret_cast<const PagedSeg*>(a.plan + 8)[seg_i];
  const int first = (static_cast<int>(blockIdx.x) % blocks) * 8;
  if (first >= seg.rows) return;
  const bool many = seg.pieces > kMany;
  const int thread = threadIdx.x, d4 = thread % V4, slot = thread / V4;
  const int share = many ? slot % SHARE : 0, step = many ? SHARE : 1, at_once = many ? ROWS / SHARE : ROWS;
  for (int r0 = first; r0 < min(first + 8, seg.rows); r0 += at_once) {
    const int row = r0 + (many ? slot / SHARE : slot);
    const bool in = row < min(first + 8, seg.rows);
    float m = kNegBig, l = 0.0f;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (in) {
      const float* base = a.rows_part + (int64_t(seg.slot) * tile_rows + row) * PS;
      for (int p0 = share; p0 < seg.pieces; p0 += 4 * step) {
        float mp[4], lp[4];
        f32x4 xp[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float* q = base + int64_t(min(p0 + u * step, seg.pieces - 1)) * tile_rows * PS;
          mp[u] = q[D];
          lp[u] = q[D + 1];
          xp[u] = *reinterpret_cast<const f32x4*>(q + 4 * d4);
        }
        float mx = m;
#pragma unroll
        for (int u = 0; u < 4; ++u) mx = fmaxf(mx, mp[u]);
        const float f = fast_exp2(m - mx);
        l *= f;
        acc *= f;
        m = mx;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float wgt = p0 + u * step < seg.pieces ? fast_exp2(mp[u] - mx) : 0.0f;
          l += wgt * lp[u];
          acc += xp[u] * wgt;
        }
      }
    }
    if (many) {
      __syncthreads();
      s_acc[thread] = acc;
      s_m[thread] = m;
      s_l[thread] = l;
      __syncthreads();
      if (share == 0) {
        float mx = m;
#pragma unroll
        for (int v = 1; v < SHARE; ++v) mx = fmaxf(mx, s_m[thread + v * V4]);
        const float f = fast_exp2(m - mx);
        l *= f;
        acc *= f;
#pragma unroll
        for (int v = 1; v < SHARE; ++v) {
          const float wgt = fast_exp2(s_m[thread + v * V4] - mx);
          l += wgt * s_l[thread + v * V4];
          acc += s_acc[thread + v * V4] * wgt;
        }
      }
    }
    if (!in || share != 0) continue;
    acc *= l > 0.0f ? 1.0f / l : 0.0f;     // a row that sees no key is 0
    const int group = a.hq / a.hkv;
    T* op = static_cast<T*>(a.o) +
            (int64_t(seg.token + row / group) * a.hq + seg.head * group + row % group) * D + 4 * d4;
#pragma unroll
    for (int e = 0; e < 4; ++e) op[e] = static_cast<T>(acc[e]);
  }
}

template <typename T, int D>
int launch_t(const PagedArgs& a, int tile_rows, int64_t segs, void* stream) {
  PagedArgs copy = a;
  void* args[] = {&copy, &tile_rows};
  return static_cast<int>(hipLaunchKernel(reinterpret_cast<const void*>(&paged_merge_kernel<T, D>),
                                          dim3(static_cast<unsigned>(segs * (tile_rows / 8))), dim3(256), args, 0,
                                          static_cast<hipStream_t>(stream)));
}

}  // namespace

int launch_paged_merge(const PagedArgs& a, int dtype, int head_dim, int tile_rows, int64_t segs, void* stream) {
  if (dtype == MOA_BF16)
    return head_dim == 128 ? launch_t<bf16, 128>(a, tile_rows, segs, stream) : launch_t<bf16, 64>(a, tile_rows, segs, stream);
  return head_dim == 128 ? launch_t<float, 128>(a, tile_rows, segs, stream) : launch_t<float, 64>(a, tile_rows, segs, stream);
}

}  // namespace moa

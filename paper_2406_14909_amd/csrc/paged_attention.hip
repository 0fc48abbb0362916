// Attention over a paged cache, one query head and token per wave: the form that the
// definitions give directly, for every type, length and mask.
#include "paged_device.h"

namespace moa {

namespace {

template <typename T, int D>
__global__ void __launch_bounds__(256) paged_attention_kernel(PagedArgs a) {
  constexpr int EPL = Vec16<T>::N;
  constexpr int LPR = D / EPL;        // lanes per key row
  constexpr int RPW = 64 / LPR;       // keys at once
  const int lane = threadIdx.x & 63;
  const int wave = uniform(threadIdx.x >> 6);
  const int t = static_cast<int>(blockIdx.x);
  const int h = static_cast<int>(blockIdx.y) * 4 + wave;
  if (h >= a.hq) return;
  const int g = h / (a.hq / a.hkv);
  int b = t;
  if (a.seq_start != nullptr) b = sequence_of(a.seq_start, a.batch, t);
  if (b < 0) return;
  const int pos = token_position(a.positions, a.seq_start, b, t);
  if (pos < 0) return;
  const int col = lane % LPR;
  const VisibleKeys vis =
      visible_keys(pos, a.window[g], a.band_shift, a.num_sink, 0, a.max_pages << a.page_shift);
  const int32_t* own = a.table + (int64_t(b) * a.hkv + g) * a.max_pages;
  const int32_t* pre = a.prefix_table + int64_t(g) * a.max_pages;
  const Vec16<T> qv = load16(static_cast<const T*>(a.q) + (int64_t(t) * a.hq + h) * D + col * EPL);
  float m = kNegBig, l = 0.0f, acc[EPL] = {};
  for (int x0 = 0; x0 < vis.count; x0 += RPW) {
    const int x = x0 + lane / LPR;
    int row = -1;
    if (x < vis.count) {
      const int p = vis.at(x);
      row = page_row(p < a.prefix_len ? pre[p >> a.page_shift] : own[p >> a.page_shift], a.num_pages, a.page_shift);
      if (row >= 0) row += p & ((1 << a.page_shift) - 1);
    }
    Vec16<T> k = zero16<T>(), v = zero16<T>();
    if (row >= 0) {
      k = load16(static_cast<const T*>(a.kp) + int64_t(row) * D + col * EPL);
      v = load16(static_cast<const T*>(a.vp) + int64_t(row) * D + col * EPL);
    }
    float sc = 0.0f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) sc += qv.get(e) * k.get(e);
    sc = group_sum<LPR>(sc);
    sc = row >= 0 ? sc * a.scale_log2 : -INFINITY;
    const float mn = fmaxf(m, sc);
    const float alpha = fast_exp2(m - mn), p = fast_exp2(sc - mn);
    m = mn;
    l = l * alpha + p;
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[e] = acc[e] * alpha + p * v.get(e);
  }
#pragma unroll
  for (int off = LPR; off < 64; off *= 2) {
    const float m2 = __shfl_xor(m, off, 64), l2 = __shfl_xor(l, off, 64);
    const float mn = fmaxf(m, m2);
    const float f1 = fast_exp2(m - mn), f2 = fast_exp2(m2 - mn);
    l = l * f1 + l2 * f2;
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[e] = acc[e] * f1 + __shfl_xor(acc[e], off, 64) * f2;
    m = mn;
  }
  if (lane >= LPR) return;
  Vec16<T> out;
#pragma unroll
  for (int e = 0; e < EPL; ++e) out.set(e, l > 0.0f ? acc[e] / l : 0.0f);   // a row that sees no key is 0
  *reinterpret_cast<decltype(out.v)*>(static_cast<T*>(a.o) + (int64_t(t) * a.hq + h) * D + col * EPL) = out.v;
}

template <typename T, int D>
int launch_t(const PagedArgs& a, void* stream) {
  PagedArgs copy = a;
  void* args[] = {&copy};
  return static_cast<int>(hipLaunchKernel(reinterpret_cast<const void*>(&paged_attention_kernel<T, D>),
                                          dim3(a.n_tokens, (a.hq + 3) / 4), dim3(256), args, 0,
                                          static_cast<hipStream_t>(stream)));
}

}  // namespace

int launch_paged_attention(const PagedArgs& a, int dtype, int head_dim, void* stream) {
  if (dtype == MOA_BF16) return head_dim == 128 ? launch_t<bf16, 128>(a, stream) : launch_t<bf16, 64>(a, stream);
  return head_dim == 128 ? launch_t<float, 128>(a, stream) : launch_t<float, 64>(a, stream);
}

}  // namespace moa

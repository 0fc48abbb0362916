// New tokens into a paged cache, with the rotation of their positions on the way.
//
// Token at position p, rotated dimensions R, frequency f_i of pair i (i < R / 2):
//   (x, y) -> (x cos(p f_i) - y sin(p f_i), y cos(p f_i) + x sin(p f_i))
// for the pairs (i, i + R/2), or (2i, 2i + 1) when interleaved; dimensions from R on
// stay.  Queries go to q_out, keys to the page of their position and head, values
// there unrotated.
//
// Bound by memory: every element is read once and written once (8,190 tokens of 64 + 16
// heads of 128, bf16, 0.34 GB: 74 us, 90 % of a copy's rate; single tokens of 16
// sequences 4.2 us, the launch and three trips to memory).  The angles are
// formed once per token, by the work-group, and used by all of its heads: p f_i in
// fp64 (a far position's angle has no correct digit behind the point in fp32), its
// fraction of a turn then in fp32.
#include "paged_device.h"

namespace moa {

namespace {

constexpr int kThreads = 256;

// TB tokens per work-group.  A thread moves two 16-byte chunks of a head that hold
// both elements of each of their pairs.
template <typename T, int D, int TB>
__global__ void __launch_bounds__(kThreads) paged_append_kernel(PagedAppendArgs a) {
  constexpr int EPL = Vec16<T>::N;            // elements per chunk
  constexpr int UNITS = D / (2 * EPL);        // threads per head
  constexpr int STEP = kThreads / UNITS;      // heads at once
  __shared__ float s_cos[TB][D / 2], s_sin[TB][D / 2];
  __shared__ int s_seq[TB], s_pos[TB];

  const int wave = uniform(threadIdx.x >> 6);
  const int t0 = static_cast<int>(blockIdx.x) * TB;
  for (int i = wave; i < TB; i += kThreads / 64) {
    const int t = t0 + i;
    int b = -1, pos = -1;
    if (t < a.n_tokens) {
      b = t;
      if (a.seq_start != nullptr) b = sequence_of(a.seq_start, a.batch, t);
      if (b >= 0) pos = token_position(a.positions, a.seq_start, b, t);
    }
    if ((threadIdx.x & 63) == 0) {
      s_seq[i] = b;
      s_pos[i] = pos;
    }
  }
  __syncthreads();
  const int half = a.rotary >> 1;
  for (int i = threadIdx.x; i < TB * half; i += kThreads) {
    const int tok = i / half, f = i - tok * half;
    const double turns = double(s_pos[tok]) * double(a.inv_freq[f]) * 0.15915494309189533577;   // 1 / (2 pi)
    float s, c;
    sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &s, &c);
    s_cos[tok][f] = c;
    s_sin[tok][f] = s;
  }
  __syncthreads();

  const int unit = threadIdx.x % UNITS;
  // The unit's chunks, as element offsets, and the first pair of its first chunk.
  const int rot_units = a.rotary / (2 * EPL);
  const bool rotate = unit < rot_units;
  const bool split = rotate && !a.interleaved;
  const int e0 = split ? unit * EPL : unit * 2 * EPL;
  const int e1 = split ? e0 + half : e0 + EPL;
  const int f0 = unit * EPL;
  const int heads = a.hq + 2 * a.hkv;
  for (int tok = 0; tok < TB; ++tok) {
    const int pos = s_pos[tok];
    if (pos < 0) continue;
    const int64_t t = t0 + tok;
    const int64_t page_index = pos >> a.page_shift;
    for (int h = threadIdx.x / UNITS; h < heads; h += STEP) {
      const char* src;
      T* dst = nullptr;
      if (h < a.hq) {
        src = static_cast<const char*>(a.q) + t * a.q_stride + int64_t(h) * D * sizeof(T);
        dst = static_cast<T*>(a.q_out) + (t * a.hq + h) * D;
      } else {
        const bool value = h >= a.hq + a.hkv;
        const int g = value ? h - a.hq - a.hkv : h - a.hq;
        src = (value ? static_cast<const char*>(a.vn) + t * a.v_stride : static_cast<const char*>(a.kn) + t * a.k_stride) +
              int64_t(g) * D * sizeof(T);
        if (page_index < a.max_pages) {
          const int64_t seq = s_seq[tok];
          const int row = page_row(a.table[(seq * a.hkv + g) * a.max_pages + page_index], a.num_pages, a.page_shift);
          const int64_t at = int64_t(row) + (pos & ((1 << a.page_shift) - 1));
          if (row >= 0) dst = static_cast<T*>(value ? a.vp : a.kp) + at * D;
        }
      }
      if (dst == nullptr) continue;
      const T* x = reinterpret_cast<const T*>(src);
      Vec16<T> x0 = load16(x + e0), x1 = load16(x + e1);
      if (rotate && h < a.hq + a.hkv) {
        if (split) {
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            const float u = x0.get(e), v = x1.get(e), c = s_cos[tok][f0 + e], s = s_sin[tok][f0 + e];
            x0.set(e, u * c - v * s);
            x1.set(e, v * c + u * s);
          }
        } else {
#pragma unroll
          for (int e = 0; e < EPL; e += 2) {
            const float c0 = s_cos[tok][f0 + e / 2], s0 = s_sin[tok][f0 + e / 2];
            const float c1 = s_cos[tok][f0 + (EPL + e) / 2], s1 = s_sin[tok][f0 + (EPL + e) / 2];
            const float u0 = x0.get(e), v0 = x0.get(e + 1), u1 = x1.get(e), v1 = x1.get(e + 1);
            x0.set(e, u0 * c0 - v0 * s0);
            x0.set(e + 1, v0 * c0 + u0 * s0);
            x1.set(e, u1 * c1 - v1 * s1);
            x1.set(e + 1, v1 * c1 + u1 * s1);
          }
        }
      }
      *reinterpret_cast<decltype(x0.v)*>(dst + e0) = x0.v;
      *reinterpret_cast<decltype(x1.v)*>(dst + e1) = x1.v;
    }
  }
}

template <typename T, int D, int TB>
int launch_t(const PagedAppendArgs& a, void* stream) {
  PagedAppendArgs copy = a;
  void* args[] = {&copy};
  const unsigned groups = static_cast<unsigned>((int64_t(a.n_tokens) + TB - 1) / TB);
  return static_cast<int>(hipLaunchKernel(reinterpret_cast<const void*>(&paged_append_kernel<T, D, TB>), dim3(groups),
                                          dim3(kThreads), args, 0, static_cast<hipStream_t>(stream)));
}

template <typename T, int D>
int launch_d(const PagedAppendArgs& a, void* stream) {
  return a.n_tokens >= 2048 ? launch_t<T, D, 4>(a, stream) : launch_t<T, D, 1>(a, stream);
}

}  // namespace

int launch_paged_append(const PagedAppendArgs& a, int dtype, int head_dim, void* stream) {
  if (dtype == MOA_BF16) return head_dim == 128 ? launch_d<bf16, 128>(a, stream) : launch_d<bf16, 64>(a, stream);
  return head_dim == 128 ? launch_d<float, 128>(a, stream) : launch_d<float, 64>(a, stream);
}

}  // namespace moa

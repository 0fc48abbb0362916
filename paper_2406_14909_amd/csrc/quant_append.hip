// New tokens into an 8-bit paged cache, with the rotation of their positions on the way.
//
// Rotation as in paged_append.hip, with sines and cosines formed in fp64 and rounded to fp32 (a code is a
// rounding to four bits, so that a key next to a border would else be another code than its definition's).
// Then, for the new tokens x of each block of 16 positions of each head, keys and values apart:
//   e = the smallest integer with max |x| <= 448 * 2^e, code = e4m3(x * 2^-e),
// and in a block that is entered behind its first position no less than the stored e; where
// that makes e grow, the rows in front are rounded to it.
//
// Bound by memory: every element is read and written once, keys and values to half their
// bytes (8,190 tokens of 64 + 16 heads of 128, 0.32 GB: 73 us, 87 % of a copy's rate; single tokens of 16
// sequences 4.4 us, the launch and three trips to memory).  A work-group takes the blocks that
// begin in a run of packed rows, with the angles of their tokens formed once; a wave holds the rows of
// one head's block in registers while their maximum is found (16 x 128 elements, 32 per lane).  Single
// tokens have 8 lanes (of heads of 128) each.
#include "quant_device.h"

namespace moa {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// A unit's 16 elements of a head: two chunks of 8 that hold both elements of each of their pairs.
struct Chunks {
  int e0, e1;       // element offsets
  int f0;           // first pair
  bool rotate;
};
template <bool kInterleaved>
__device__ __forceinline__ Chunks chunks_of(const PagedAppendArgs& a, int unit, bool turned) {
  Chunks c;
  c.rotate = turned && unit < a.rotary >> 4;
  const bool split = c.rotate && !kInterleaved;
  c.e0 = split ? unit * 8 : unit * 16;
  c.e1 = split ? c.e0 + (a.rotary >> 1) : c.e0 + 8;
  c.f0 = unit * 8;
  return c;
}

// Products and sums rounded one by one, as the definition has them.
template <bool kInterleaved>
__device__ __forceinline__ void turn(float (&x)[16], const Chunks& c, const float* cosines, const float* sines) {
#pragma clang fp contract(off)
  if (!c.rotate) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float &p = x[kInterleaved ? 2 * e : e], &q = x[kInterleaved ? 2 * e + 1 : 8 + e];
    const float u = p, v = q, co = cosines[c.f0 + e], si = sines[c.f0 + e];
    p = u * co - v * si;
    q = v * co + u * si;
  }
}

__device__ __forceinline__ void load_chunks(float (&x)[16], const bf16* row, const Chunks& c) {
  const Vec16<bf16> a = load16(row + c.e0), b = load16(row + c.e1);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = a.get(e);
    x[8 + e] = b.get(e);
  }
}

// Codes of a chunk of 8; what is past the largest number becomes that, what is not finite NaN.
__device__ __forceinline__ u32x2 codes8(const float* x, float inverse) {
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float s = fminf(fmaxf(x[e] * inverse, -kQuantMost), kQuantMost);
    y[e] = finite(x[e]) ? s : __builtin_nanf("");
  }
  return u32x2{narrow4(y[0], y[1], y[2], y[3]), narrow4(y[4], y[5], y[6], y[7])};
}

// ROWS = 16: blocks of a run of `span` packed rows; ROWS = 1: one token per sequence.
// Heads are shared out over gridDim.y work-groups.  Four work-groups per compute unit, in 128 registers
// (8,190 tokens of 64/8 heads: with as many registers as it likes, three, 76.0 us, with four 75.2,
// and with two query rows on their way instead of four 73.4).
template <int D, int ROWS, bool kInterleaved>
__global__ void __launch_bounds__(kThreads, 4) quant_append_kernel(QuantAppendArgs args, int span) {
  constexpr int UNITS = D / 16;                      // lanes per row
  constexpr int LPB = ROWS == 1 ? UNITS : 64;        // lanes per block of a head
  constexpr int RP = LPB / UNITS;                    // rows at once
  constexpr int NP = ROWS / RP;
  const PagedAppendArgs& a = args.a;
  __shared__ float s_cos[ROWS][D / 2], s_sin[ROWS][D / 2];
  const int half = a.rotary >> 1;
  const int part = blockIdx.y, parts = gridDim.y;
  const int q0 = a.hq * part / parts, q1 = a.hq * (part + 1) / parts;
  const int kv0 = 2 * a.hkv * part / parts, kv1 = 2 * a.hkv * (part + 1) / parts;

  // `len` tokens of sequence b from packed row t and position pos on, in one block.
  auto block = [&](int b, int t, int64_t pos, int len) {
    for (int i = threadIdx.x; i < len * half; i += kThreads) {
      const int tok = ROWS == 1 ? 0 : i / half, f = ROWS == 1 ? i : i - tok * half;
      const double turns = double(pos + tok) * double(a.inv_freq[f]) * 0.15915494309189533577;   // 1 / (2 pi)
      double s, c;
      sincospi(2.0 * (turns - rint(turns)), &s, &c);
      s_cos[tok][f] = static_cast<float>(c);
      s_sin[tok][f] = static_cast<float>(s);
    }
    __syncthreads();
    {
      const int unit = threadIdx.x % UNITS, heads = q1 - q0;
      const Chunks c = chunks_of<kInterleaved>(a, unit, true);
      // Two rows of a thread are on their way at once.
      constexpr int STEP = kThreads / UNITS, AHEAD = ROWS == 1 ? 1 : 2;
      for (int i0 = threadIdx.x / UNITS; i0 < heads * len; i0 += AHEAD * STEP) {
        Vec16<bf16> lo[AHEAD], hi[AHEAD];
        int tok[AHEAD], h[AHEAD];
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
          const int i = min(i0 + n * STEP, heads * len - 1);
          tok[n] = ROWS == 1 ? 0 : i / heads;
          h[n] = q0 + i - tok[n] * heads;
          const bf16* src = reinterpret_cast<const bf16*>(static_cast<const char*>(a.q) + (t + tok[n]) * a.q_stride) + h[n] * D;
          lo[n] = load16(src + c.e0);
          hi[n] = load16(src + c.e1);
        }
#pragma unroll
        for (int n = 0; n < AHEAD; ++n) {
          if (i0 + n * STEP >= heads * len) break;
          bf16* dst = static_cast<bf16*>(a.q_out) + (int64_t(t + tok[n]) * a.hq + h[n]) * D;
          float x[16];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = lo[n].get(e);
            x[8 + e] = hi[n].get(e);
          }
          turn<kInterleaved>(x, c, s_cos[tok[n]], s_sin[tok[n]]);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            lo[n].set(e, x[e]);
            hi[n].set(e, x[8 + e]);
          }
          *reinterpret_cast<bf16x8*>(dst + c.e0) = lo[n].v;
          *reinterpret_cast<bf16x8*>(dst + c.e1) = hi[n].v;
        }
      }
    }
    const int64_t page_index = pos >> a.page_shift;
    const int at = static_cast<int>(pos & ((1 << a.page_shift) - 1)), behind = at & (kQuantBlock - 1);
    const int lane = threadIdx.x % LPB, unit = lane % UNITS, sub = lane / UNITS;
    for (int i = kv0 + static_cast<int>(threadIdx.x) / LPB; i < kv1 && page_index < a.max_pages; i += kThreads / LPB) {
      const int g = i >> 1, value = i & 1;
      const int row0 = page_row(a.table[(int64_t(b) * a.hkv + g) * a.max_pages + page_index], a.num_pages, a.page_shift);
      if (row0 < 0) continue;
      const Chunks c = chunks_of<kInterleaved>(a, unit, !value);
      const char* src = value ? static_cast<const char*>(a.vn) + t * a.v_stride : static_cast<const char*>(a.kn) + t * a.k_stride;
      const int64_t stride = value ? a.v_stride : a.k_stride;
      float x[NP][16];
      float amax = 0.0f;
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        const int tok = n * RP + sub;
        if (tok < len) {
          load_chunks(x[n], reinterpret_cast<const bf16*>(src + tok * stride) + g * D, c);
          turn<kInterleaved>(x[n], c, s_cos[tok], s_sin[tok]);
#pragma unroll
          for (int e = 0; e < 16; ++e) amax = fmaxf(amax, finite(x[n][e]) ? fabsf(x[n][e]) : 0.0f);
        }
      }
#pragma unroll
      for (int off = 1; off < LPB; off *= 2) amax = fmaxf(amax, __shfl_xor(amax, off, 64));
      const int64_t row = int64_t(row0) + at;                           // of the first new token
      float* const scale = args.scales + (row / kQuantBlock) * 2 + value;
      uint8_t* const pool = static_cast<uint8_t*>(value ? a.vp : a.kp);
      int e = quant_exponent(amax);
      if (behind > 0) {
        const int old = quant_exponent_of(*scale);
        if (e > old) {
          const float by = pow2(max(old - e, -40));                     // of 2^-40 nothing is left either
          for (int r = sub; r < behind; r += RP) {
            uint8_t* const p = pool + (row - behind + r) * D + unit * 16;
            u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
#if defined(__HIP_DEVICE_COMPILE__)
              const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(v[w], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(v[w], true);
              v[w] = narrow4(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
#endif
            }
            *reinterpret_cast<u32x4*>(p) = v;
          }
        }
        e = max(e, old);
      }
      const float inverse = pow2(-e);
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        const int tok = n * RP + sub;
        if (tok < len) {
          uint8_t* const p = pool + (row + tok) * D;
          *reinterpret_cast<u32x2*>(p + c.e0) = codes8(x[n], inverse);
          *reinterpret_cast<u32x2*>(p + c.e1) = codes8(x[n] + 8, inverse);
        }
      }
      if (lane == 0) *scale = pow2(e);
    }
  };

  if constexpr (ROWS == 1) {
    const int64_t pos = a.positions[blockIdx.x];
    if (pos >= 0) block(blockIdx.x, blockIdx.x, pos, 1);
  } else {
    // The blocks whose first new token is in rows [t, end).
    int64_t t = int64_t(blockIdx.x) * span;
    const int64_t end = min(t + span, int64_t(a.n_tokens));
    int b = max(sequence_at(a.seq_start, a.batch, static_cast<int>(t)), 0);
    while (t < end && b < a.batch) {
      const int64_t first = a.seq_start[b], last = min(int64_t(a.seq_start[b + 1]), int64_t(a.n_tokens));
      t = max(t, first);
      const int64_t p0 = a.positions[b];
      if (p0 < 0 || t >= last) {                 // nothing of this sequence from here on
        if (p0 < 0) t = max(t, last);
        // the next with rows: there may be many without
        b = max(b + 1, t < end ? sequence_at(a.seq_start, a.batch, static_cast<int>(t)) : 0);
        continue;
      }
      if (t >= end) break;
      const int64_t pos = p0 + (t - first);
      const int in = static_cast<int>(pos & (kQuantBlock - 1));
      const int len = static_cast<int>(min(int64_t(kQuantBlock - in), last - t));
      if (t == max(first, int64_t(0)) || in == 0) {
        block(b, static_cast<int>(t), pos, len);
        __syncthreads();                         // the angles make room for the next block's
      }
      t += len;
    }
  }
}

template <int D, bool kInterleaved>
int launch_t(const QuantAppendArgs& args, void* stream) {
  QuantAppendArgs copy = args;
  const PagedAppendArgs& a = args.a;
  // Runs of 16 rows, or, where sequences have fewer on average, single ones, of which those in the
  // middle of a block leave at once.
  int span = a.seq_start != nullptr && a.n_tokens >= kQuantBlock * int64_t(a.batch) ? kQuantBlock : 1;
  const int64_t runs = (int64_t(a.n_tokens) + span - 1) / span;
  if (runs * kThreads >= kMaxGridThreads) return kGridTooLarge;
  // Heads over four work-groups (8,190 tokens of 64/8 heads: over 2, 4 and 8 79.7, 77.0 and 90.4 us
  // when this was chosen).
  const int parts = runs >= 2048 || a.hkv < 4 ? 1 : 4;
  void* params[] = {&copy, &span};
  const void* kernel = a.seq_start == nullptr ? reinterpret_cast<const void*>(&quant_append_kernel<D, 1, kInterleaved>)
                                              : reinterpret_cast<const void*>(&quant_append_kernel<D, 16, kInterleaved>);
  return static_cast<int>(hipLaunchKernel(kernel, dim3(static_cast<unsigned>(runs), parts), dim3(kThreads), params, 0,
                                          static_cast<hipStream_t>(stream)));
}

template <int D>
int launch_d(const QuantAppendArgs& a, void* stream) {
  return a.a.interleaved ? launch_t<D, true>(a, stream) : launch_t<D, false>(a, stream);
}

}  // namespace

int launch_quant_append(const QuantAppendArgs& a, int head_dim, void* stream) {
  return head_dim == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace moa

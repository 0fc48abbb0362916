// Device helpers of the paged kernels.
#pragma once

#include <algorithm>
#include <atomic>

#include "moa_device.h"
#include "paged.h"

namespace moa {

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The last b with seq_start[b] <= t, or -1.  All lanes of the wave search together, 64
// probes per trip to memory; whatever seq_start holds, only its batch + 1 entries are read.
__device__ __forceinline__ int sequence_at(const int32_t* seq_start, int batch, int t) {
  const int lane = threadIdx.x & 63;
  int b = 0, n = batch;
  while (true) {
    const int stride = (n + 63) >> 6;
    const bool below = lane * stride < n && seq_start[b + lane * stride] <= t;
    const int c = __builtin_popcountll(__ballot(below));
    if (c == 0) return -1;
    b += (c - 1) * stride;
    n = min(stride, n - (c - 1) * stride);
    if (stride == 1) break;
  }
  return uniform(b);
}

// The sequence of packed row t, or -1 where no sequence has the row.
__device__ __forceinline__ int sequence_of(const int32_t* seq_start, int batch, int t) {
  const int b = sequence_at(seq_start, batch, t);
  return b >= 0 && t < seq_start[b + 1] ? b : -1;
}

// Position of packed row t of sequence b, negative for an idle sequence.
__device__ __forceinline__ int token_position(const int32_t* positions, const int32_t* seq_start, int b, int t) {
  const int p0 = positions[b];
  if (p0 < 0 || seq_start == nullptr) return p0;
  return static_cast<int>(min(int64_t(p0) + t - seq_start[b], int64_t(0x7fffffff)));
}

// First row of a page in the pool, or -1 where the page is absent.
__device__ __forceinline__ int page_row(int page, int num_pages, int page_shift) {
  return static_cast<uint32_t>(page) < static_cast<uint32_t>(num_pages) ? page << page_shift : -1;
}

typedef short i16x4 __attribute__((ext_vector_type(4)));

// Transposing LDS read of four bf16: within each 16-lane group, lane 4a+b receives
// element b of the 8-byte reads issued by lanes 4e+a (e = 0..3), as its element e.
__device__ __forceinline__ bf16x4 read_tr(const void* p) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i16x4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) i16x4*)(const_cast<void*>(p)));
  return __builtin_bit_cast(bf16x4, r);
#else
  (void)p;
  return bf16x4{};
#endif
}

// acc + a + b with a, b in bf16.
__device__ __forceinline__ float dot2_ones(bf16 a, bf16 b, float acc) {
  typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
#if defined(__HIP_DEVICE_COMPILE__)
  const bf16x2 ab = {a, b};
  const bf16x2 ones = {bf16(1.0f), bf16(1.0f)};
  return __builtin_amdgcn_fdot2_f32_bf16(ab, ones, acc, false);
#else
  return acc + float(a) + float(b);
#endif
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// Resident work-groups of `kernel` on the current device (cached per device by the
// caller; threads that launch at once store the same value).
inline int resident_groups(const void* kernel, int threads, std::atomic<int>* cache) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) dev = 0;
  const int known = cache[dev].load(std::memory_order_relaxed);
  if (known > 0) return known;
  int cus = 0, per_cu = 0;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) cus = 1;
  if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kernel, threads, 0) != hipSuccess) per_cu = 1;
  const int groups = std::max(1, cus) * std::max(1, per_cu);
  cache[dev].store(groups, std::memory_order_relaxed);
  return groups;
}

}  // namespace moa

// Decode over a paged cache: launches (the kernels' work is in paged_decode.h).
#include "paged_decode.h"

namespace moa {

namespace {

// Two work-groups per compute unit where the matrix units do the work: a wave then has a whole
// tile on its way while it works on another (with three, in 168 registers, 16 sequences x 8 KV
// heads x 4 query heads, 357 MB: 82.2 us, without the loads ahead 76.2; with two 62.0).
template <typename T, int D, int G>
__global__ void __launch_bounds__(kThreads, (on_matrix_units<T>() ? 2 : 1)) paged_decode_kernel(PagedArgs a) {
  __shared__ __attribute__((aligned(1024))) DecodeLds<T, D, G> lds;
  decode_worker<T, D, G>(a, lds, blockIdx.x);
}

template <typename T, int D, int G>
int launch_t(PagedArgs a, void* stream) {
  const void* kernel = reinterpret_cast<const void*>(&paged_decode_kernel<T, D, G>);
  static std::atomic<int> group_cache[64];
  a.slots = std::min(resident_groups(kernel, kThreads, group_cache), kPagedMaxWorkers);
  void* args[] = {&a};
  hipError_t e = hipLaunchKernel(kernel, dim3(static_cast<unsigned>(a.slots)), dim3(kThreads), args, 0,
                                 static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return static_cast<int>(e);
  e = hipLaunchKernel(reinterpret_cast<const void*>(&paged_combine_kernel<T, D, G, false>), combine_grid<G>(a), dim3(256),
                      args, 0, static_cast<hipStream_t>(stream));
  return static_cast<int>(e);
}

template <typename T, int D>
int launch_g(const PagedArgs& a, int group, void* stream) {
  switch (group) {
    case 1: return launch_t<T, D, 1>(a, stream);
    case 2: return launch_t<T, D, 2>(a, stream);
    case 4: return launch_t<T, D, 4>(a, stream);
    case 8: return launch_t<T, D, 8>(a, stream);
    default: return static_cast<int>(hipErrorInvalidValue);
  }
}

}  // namespace

int launch_paged_decode(const PagedArgs& a, int dtype, int head_dim, int group, void* stream) {
  if (dtype == MOA_BF16) return head_dim == 128 ? launch_g<bf16, 128>(a, group, stream) : launch_g<bf16, 64>(a, group, stream);
  return head_dim == 128 ? launch_g<float, 128>(a, group, stream) : launch_g<float, 64>(a, group, stream);
}

}  // namespace moa

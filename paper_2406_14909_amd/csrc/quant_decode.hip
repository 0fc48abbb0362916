// Decode over an 8-bit paged cache: launches (the kernels' work is in quant_decode.h).
#include "quant_decode.h"

namespace moa {

namespace {

template <int D, int G>
__global__ void __launch_bounds__(kThreads, 2) quant_decode_kernel(PagedArgs a) {
  __shared__ __attribute__((aligned(1024))) QuantLds<D> lds;
  decode_quant<D, G>(a, lds, blockIdx.x);
}

template <int D, int G>
int launch_t(PagedArgs a, void* stream) {
  const void* kernel = reinterpret_cast<const void*>(&quant_decode_kernel<D, G>);
  static std::atomic<int> group_cache[64];
  a.slots = std::min(resident_groups(kernel, kThreads, group_cache), kPagedMaxWorkers);
  void* args[] = {&a};
  hipError_t e = hipLaunchKernel(kernel, dim3(static_cast<unsigned>(a.slots)), dim3(kThreads), args, 0,
                                 static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return static_cast<int>(e);
  e = hipLaunchKernel(reinterpret_cast<const void*>(&paged_combine_kernel<bf16, D, G, false, QuantTile<D>::kRoundShift, true>),
                      combine_grid<G>(a), dim3(256), args, 0, static_cast<hipStream_t>(stream));
  return static_cast<int>(e);
}

template <int D>
int launch_g(const PagedArgs& a, int group, void* stream) {
  switch (group) {
    case 1: return launch_t<D, 1>(a, stream);
    case 2: return launch_t<D, 2>(a, stream);
    case 4: return launch_t<D, 4>(a, stream);
    case 8: return launch_t<D, 8>(a, stream);
    default: return static_cast<int>(hipErrorInvalidValue);
  }
}

}  // namespace

int launch_quant_decode(const PagedArgs& a, int head_dim, int group, void* stream) {
  return head_dim == 128 ? launch_g<128>(a, group, stream) : launch_g<64>(a, group, stream);
}

}  // namespace moa

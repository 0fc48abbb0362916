// Prefill over an 8-bit paged cache: launches (the kernels' work is in paged_rows_bf16.h).
#include "paged_rows_bf16.h"

namespace moa {

namespace {

template <int D, int KG>
__global__ void __launch_bounds__(256 * KG, 2) quant_rows_kernel(PagedArgs a) {
  __shared__ __attribute__((aligned(1024))) RowsBf16Lds<D, KG> lds;
  rows_bf16<D, false, KG, true>(a, lds, blockIdx.x);
}

template <int D, int KG>
int launch_t(const PagedArgs& a, int64_t groups, void* stream) {
  if (groups >= kMaxGrid) return kGridTooLarge;
  PagedArgs copy = a;
  void* args[] = {&copy};
  return static_cast<int>(hipLaunchKernel(reinterpret_cast<const void*>(&quant_rows_kernel<D, KG>),
                                          dim3(static_cast<unsigned>(groups)), dim3(256 * KG), args, 0,
                                          static_cast<hipStream_t>(stream)));
}

}  // namespace

int launch_quant_rows(const PagedArgs& a, int head_dim, int key_groups, int64_t groups, void* stream) {
  if (key_groups == 1) return head_dim == 128 ? launch_t<128, 1>(a, groups, stream) : launch_t<64, 1>(a, groups, stream);
  return head_dim == 128 ? launch_t<128, 2>(a, groups, stream) : launch_t<64, 2>(a, groups, stream);
}

}  // namespace moa

// Prefill over a paged cache: launches (the kernels' work is in paged_rows_bf16.h and
// paged_rows_f32.h).
#include "paged_rows_bf16.h"
#include "paged_rows_f32.h"

namespace moa {

namespace {

// Two work-groups per compute unit; of fp32 at head_dim 128, whose operands take 400
// registers, one.
template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) == 4 && D == 128 ? 1 : 2) paged_rows_kernel(PagedArgs a) {
  if constexpr (sizeof(T) == 2) {
    __shared__ __attribute__((aligned(1024))) RowsBf16Lds<D> lds;
    rows_bf16<D, false>(a, lds, blockIdx.x);
  } else {
    __shared__ RowsF32Lds<D> lds;
    rows_f32<D, false>(a, lds, blockIdx.x);
  }
}

template <typename T, int D>
int launch_t(const PagedArgs& a, int64_t groups, void* stream) {
  if (groups >= kMaxGrid) return kGridTooLarge;
  PagedArgs copy = a;
  void* args[] = {&copy};
  return static_cast<int>(hipLaunchKernel(reinterpret_cast<const void*>(&paged_rows_kernel<T, D>),
                                          dim3(static_cast<unsigned>(groups)), dim3(256), args, 0,
                                          static_cast<hipStream_t>(stream)));
}

}  // namespace

int launch_paged_rows(const PagedArgs& a, int dtype, int head_dim, int64_t groups, void* stream) {
  if (dtype == MOA_BF16) return head_dim == 128 ? launch_t<bf16, 128>(a, groups, stream) : launch_t<bf16, 64>(a, groups, stream);
  return head_dim == 128 ? launch_t<float, 128>(a, groups, stream) : launch_t<float, 64>(a, groups, stream);
}

}  // namespace moa

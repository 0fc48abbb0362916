// Prefill over a paged cache: launches (the kernels' work is in paged_rows_bf16.h and
// paged_rows_f32.h).
#include "paged_rows_bf16.h"
#include "paged_rows_f32.h"

namespace moa {

namespace {

// bf16: KG groups of 4 waves.  Two work-groups of one per compute unit, or one of two at
// head_dim 128.  fp32: 4 waves, at head_dim 128, where operands take 400 registers, one
// work-group.
template <typename T, int D, int KG>
__global__ void __launch_bounds__(256 * KG, sizeof(T) == 4 && D == 128 ? 1 : 2) paged_rows_kernel(PagedArgs a) {
  if constexpr (sizeof(T) == 2) {
    __shared__ __attribute__((aligned(1024))) RowsBf16Lds<D, KG> lds;
    rows_bf16<D, false, KG>(a, lds, blockIdx.x);
  } else {
    __shared__ RowsF32Lds<D> lds;
    rows_f32<D, false>(a, lds, blockIdx.x);
  }
}

template <typename T, int D, int KG>
int launch_t(const PagedArgs& a, int64_t groups, void* stream) {
  if (groups >= kMaxGrid) return kGridTooLarge;
  PagedArgs copy = a;
  void* args[] = {&copy};
  return static_cast<int>(hipLaunchKernel(reinterpret_cast<const void*>(&paged_rows_kernel<T, D, KG>),
                                          dim3(static_cast<unsigned>(groups)), dim3(256 * KG), args, 0,
                                          static_cast<hipStream_t>(stream)));
}

}  // namespace

int launch_paged_rows(const PagedArgs& a, int dtype, int head_dim, int key_groups, int64_t groups, void* stream) {
  if (dtype != MOA_BF16)
    return head_dim == 128 ? launch_t<float, 128, 1>(a, groups, stream) : launch_t<float, 64, 1>(a, groups, stream);
  if (key_groups == 1)
    return head_dim == 128 ? launch_t<bf16, 128, 1>(a, groups, stream) : launch_t<bf16, 64, 1>(a, groups, stream);
  return head_dim == 128 ? launch_t<bf16, 128, 2>(a, groups, stream) : launch_t<bf16, 64, 2>(a, groups, stream);
}

}  // namespace moa

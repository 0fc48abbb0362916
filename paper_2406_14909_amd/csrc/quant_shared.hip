// Decode of a batch over a prefix that its sequences share, in an 8-bit cache, and over what each
// has behind it: the two kinds of work of one launch and the merge of paged_shared.hip.
#include "paged_rows_bf16.h"
#include "quant_decode.h"

namespace moa {

namespace {

template <int D, int G>
__global__ void __launch_bounds__(kThreads, 2) quant_shared_kernel(PagedArgs a) {
  __shared__ __attribute__((aligned(1024))) union {
    QuantLds<D> decode;
    RowsBf16Lds<D, 1> rows;
  } lds;
  const SharedWork work = shared_work(a, blockIdx.x);
  if (work.prefix) rows_bf16<D, true, 1, true>(a, lds.rows, work.index);
  else decode_quant<D, G>(a, lds.decode, work.index);
}

template <int D, int G>
int launch_t(const PagedArgs& a, void* stream) {
  PagedArgs copy = a;
  void* args[] = {&copy};
  hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&quant_shared_kernel<D, G>), dim3(shared_groups(a)),
                                 dim3(kThreads), args, 0, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return static_cast<int>(e);
  e = hipLaunchKernel(reinterpret_cast<const void*>(&paged_combine_kernel<bf16, D, G, true, QuantTile<D>::kRoundShift>),
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

int launch_quant_shared(const PagedArgs& a, int head_dim, int group, void* stream) {
  return head_dim == 128 ? launch_g<128>(a, group, stream) : launch_g<64>(a, group, stream);
}

}  // namespace moa

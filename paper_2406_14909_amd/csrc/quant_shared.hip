// Decode of a batch over a prefix that its sequences share, in an 8-bit cache, and over what each
// has behind it: the two kinds of work of one launch and the merge of paged_shared.hip, with a work-group of
// either kind on each compute unit.  Bound by the longest chain: a piece of the prefix is a dozen key tiles
// one after the other, at 3,600 cycles each (48 sequences x 8 heads x 8 query heads over 32,700 shared
// keys and up to 1,000 of their own: 41 us, 7 of them the merge; 46 with the kinds in turns).  More and
// shorter pieces, or more work-groups for either kind, help some batches and cost others (sequences x KV heads x
// query heads of each on a prefix, with up to so many keys of their own; work-groups for prefix and own keys; us of
// passes over two sets of inputs in turn, where the first call takes 43 for the 41 of more sets):
//                                   256 + 256   320 + 192   192 + 320   256 + 384
//   48 x 8 x 8 on 32,700, 1,000          43.2        44.5        48.9        47.3
//   16 x 8 x 4 on 8,001, 500             19.8        19.9        21.1        20.0
//   16 x 32 x 1 on 8,001, 500            37.4        32.6        42.6        37.4
//   48 x 32 x 1 on 8,001, 1,500          90.7       109.5        92.6       101.3
//   32 x 8 x 4 on 2,000, 4,000           38.4        42.8        42.1        37.1
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
  const SharedWork work = shared_work<true>(a, blockIdx.x);
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
  e = hipLaunchKernel(reinterpret_cast<const void*>(&paged_combine_kernel<bf16, D, G, true, QuantTile<D>::kRoundShift, true>),
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

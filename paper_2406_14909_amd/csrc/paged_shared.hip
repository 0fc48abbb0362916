// Decode of a batch over a prefix that its sequences share, and over what each has behind it.
//
// The prefix is read once for all: the batch's query rows against its keys are matrix
// products of up to 128 rows (paged_rows_bf16.h, paged_rows_f32.h), cut along the keys.  The
// keys behind it are read as in a decode call (paged_decode.h).  Both are work of the same
// launch, as both wait for memory much of the time: work-groups of the one kind and the
// other alternate, in eights, so that every die and most compute units have both.  All leave
// partial results, which one merge joins.  48 sequences x 8 heads x 8 query heads over 32,700
// shared keys (34 MB of those seen) and up to 1,000 of their own (103 MB): 50 us, 43 of them this
// kernel at 3.2 TB/s, matrix units busy 12 %.  Either part takes most of it alone: with one key of their
// own 42 us, as row tiles take a piece's key tiles one after the other; behind a prefix of 64 keys
// 39, as one work-group per compute unit reads what moa_paged_decode reads with two.
#include "paged_decode.h"
#include "paged_rows_bf16.h"
#include "paged_rows_f32.h"

namespace moa {

namespace {

template <typename T, int D, int G>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 && D == 128 ? 1 : 2) paged_shared_kernel(PagedArgs a) {
  using RowsLds = std::conditional_t<sizeof(T) == 2, RowsBf16Lds<D, 1>, RowsF32Lds<D>>;
  __shared__ __attribute__((aligned(1024))) union {
    DecodeLds<T, D, G> decode;
    RowsLds rows;
  } lds;
  const SharedWork work = shared_work(a, blockIdx.x);
  if (work.prefix) {
    if constexpr (sizeof(T) == 2) rows_bf16<D, true, 1>(a, lds.rows, work.index);
    else rows_f32<D, true>(a, lds.rows, work.index);
  } else {
    decode_worker<T, D, G>(a, lds.decode, work.index);
  }
}

template <typename T, int D, int G>
int launch_t(const PagedArgs& a, void* stream) {
  PagedArgs copy = a;
  void* args[] = {&copy};
  hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(&paged_shared_kernel<T, D, G>), dim3(shared_groups(a)),
                                 dim3(kThreads), args, 0, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return static_cast<int>(e);
  e = hipLaunchKernel(reinterpret_cast<const void*>(&paged_combine_kernel<T, D, G, true>), combine_grid<G>(a), dim3(256),
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

int launch_paged_shared(const PagedArgs& a, int dtype, int head_dim, int group, void* stream) {
  if (dtype == MOA_BF16) return head_dim == 128 ? launch_g<bf16, 128>(a, group, stream) : launch_g<bf16, 64>(a, group, stream);
  return head_dim == 128 ? launch_g<float, 128>(a, group, stream) : launch_g<float, 64>(a, group, stream);
}

}  // namespace moa

// pcs_attend_token_tree.cu -- attention of trees of drafted tokens, few query rows a
// key head, over a cache of 16-bit elements: the kernel of pcs_attend_token.cu, whose
// rows see what the tree says of the new tokens.  26 nodes of one session over a window of
// 1,024, 16 heads of 64: 16 us, the same as 26 tokens in a row; the bound is latency.
#include "pcs_attend_token_dev.h"

namespace pcs {
namespace {

template <typename T, int DP, int NT>
cudaError_t launch(const AttendArgs& a, cudaStream_t stream) {
  auto k = k_attend_token<T, DP, NT, true>;
  static SmemLimit limit;
  if (cudaError_t e = limit.set(k, kRingBytes<DP>)) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.batch.sessions) * a.cache.heads * a.splits);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kRingBytes<DP>;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, a);
}

template <typename T>
cudaError_t by_size(const AttendArgs& a, int rows, cudaStream_t stream) {
  if (a.cache.head_dim <= 64)
    return rows <= 8 ? launch<T, 64, 1>(a, stream) : rows <= 16 ? launch<T, 64, 2>(a, stream) : launch<T, 64, 4>(a, stream);
  return rows <= 8 ? launch<T, 128, 1>(a, stream) : rows <= 16 ? launch<T, 128, 2>(a, stream) : launch<T, 128, 4>(a, stream);
}

}  // namespace

cudaError_t launch_attend_token_tree(const AttendArgs& a, uint32_t dtype, int rows, cudaStream_t stream) {
  return dtype == PCS_DT_F16 ? by_size<__half>(a, rows, stream) : by_size<__nv_bfloat16>(a, rows, stream);
}

}  // namespace pcs

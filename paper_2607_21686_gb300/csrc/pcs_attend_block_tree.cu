// pcs_attend_block_tree.cu -- attention of trees of drafted tokens with many query rows
// a key head, over a cache of 16-bit elements: the kernel of pcs_attend_block.cu, whose
// rows see what the tree says of the new tokens.  60 nodes of each of 32 sessions over 500
// to 9,000 tokens, 32 query heads over 8 of 128, bfloat16: 136 us, of 96 us for its bytes
// (longest sessions first; as they came they took a seventh more); the bound is a block's
// loads, 44 GB/s an SM.
#include "pcs_attend_block_dev.h"

namespace pcs {
namespace {

template <typename T, int DP>
cudaError_t launch(const AttendArgs& a, int blocks, const TensorMaps& maps, cudaStream_t stream) {
  return a.box_rows == 0   ? launch_form<T, DP, 0, true>(a, blocks, maps, stream)
         : a.box_rows == 8 ? launch_form<T, DP, 2, true>(a, blocks, maps, stream)
                           : launch_form<T, DP, 1, true>(a, blocks, maps, stream);
}

}  // namespace

cudaError_t launch_attend_block_tree(const AttendArgs& a, uint32_t dtype, int blocks, const TensorMaps& maps,
                                     cudaStream_t stream) {
  if (dtype == PCS_DT_F16)
    return a.cache.head_dim <= 64 ? launch<__half, 64>(a, blocks, maps, stream) : launch<__half, 128>(a, blocks, maps, stream);
  return a.cache.head_dim <= 64 ? launch<__nv_bfloat16, 64>(a, blocks, maps, stream)
                                : launch<__nv_bfloat16, 128>(a, blocks, maps, stream);
}

}  // namespace pcs

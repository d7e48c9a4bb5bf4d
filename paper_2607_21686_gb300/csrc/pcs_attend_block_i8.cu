// pcs_attend_block_i8.cu -- the same as pcs_attend_block_e4m3.cu over a cache of 8-bit whole
// numbers.
#include "pcs_attend_block_dev.h"

namespace pcs {
namespace {

constexpr int kMakers = -2;

template <typename T, int DP>
cudaError_t launch(const AttendArgs& a, int blocks, const CodeMaps& maps, cudaStream_t stream) {
  return a.parent ? launch_form<T, DP, kMakers, true>(a, blocks, maps, stream)
                  : launch_form<T, DP, kMakers, false>(a, blocks, maps, stream);
}

}  // namespace

cudaError_t launch_attend_block_i8(const AttendArgs& a, uint32_t dtype, int blocks, const CodeMaps& maps, cudaStream_t stream) {
  if (dtype == PCS_DT_F16)
    return a.cache.head_dim <= 64 ? launch<__half, 64>(a, blocks, maps, stream) : launch<__half, 128>(a, blocks, maps, stream);
  return a.cache.head_dim <= 64 ? launch<__nv_bfloat16, 64>(a, blocks, maps, stream)
                                : launch<__nv_bfloat16, 128>(a, blocks, maps, stream);
}

}  // namespace pcs

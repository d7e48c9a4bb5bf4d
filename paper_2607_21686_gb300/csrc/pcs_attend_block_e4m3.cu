// pcs_attend_block_e4m3.cu -- attention of blocks of new tokens, trees among them, over a
// paged cache of 8-bit floats: the kernel of pcs_attend_block.cu, whose copying warps turn
// codes into elements of the queries' type on their way to the tiles.  That is exact
// in bfloat16, whose 8 bits hold every code and whose powers of two every scale, down to
// 2^-126; a float16 ends at 65504.  Trees of 60 nodes over contexts of 500 to 9,000 tokens of
// 32 sessions, 32 query heads over 8 of 128: 210 us, with queries in float16 204 us, over
// 16-bit pages 136 us.  The instructions of the conversion are not the bound: to float16 a
// code takes a third of what it takes to bfloat16.  What the form over 16 bits has beside it
// is a second tile of values (with heads of 128 there is room for one): here the next values
// are turned only when the products of both row tiles over the last ones are done, and the
// products wait for all 128 tokens of them.
#include "pcs_attend_block_dev.h"

namespace pcs {
namespace {

constexpr int kMakers = -1;

template <typename T, int DP>
cudaError_t launch(const AttendArgs& a, int blocks, const CodeMaps& maps, cudaStream_t stream) {
  return a.parent ? launch_form<T, DP, kMakers, true>(a, blocks, maps, stream)
                  : launch_form<T, DP, kMakers, false>(a, blocks, maps, stream);
}

}  // namespace

cudaError_t launch_attend_block_e4m3(const AttendArgs& a, uint32_t dtype, int blocks, const CodeMaps& maps, cudaStream_t stream) {
  if (dtype == PCS_DT_F16)
    return a.cache.head_dim <= 64 ? launch<__half, 64>(a, blocks, maps, stream) : launch<__half, 128>(a, blocks, maps, stream);
  return a.cache.head_dim <= 64 ? launch<__nv_bfloat16, 64>(a, blocks, maps, stream)
                                : launch<__nv_bfloat16, 128>(a, blocks, maps, stream);
}

}  // namespace pcs

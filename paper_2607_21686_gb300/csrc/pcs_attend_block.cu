// pcs_attend_block.cu -- attention of blocks of new tokens (frames, prompts)
// over a paged cache of keys and values.
//
// k_attend_block  The same one-pass softmax as the token kernel's, with enough
//                 query rows per key head that the matrix products bound it
//                 (4 head_dim flops per visible pair of row and token): they
//                 run on the fifth-generation tensor cores.  A block takes one
//                 session, key head and 256 rows (query heads of a key head
//                 side by side, then tokens) as two tiles of 128, and walks
//                 the tokens they see in tiles of 128.  Per tile and row tile
//                 S = Q K^T goes to tensor memory, four warps turn it into
//                 weights (a thread per row), write them back as the first
//                 operand of O += P V, which stays in tensor memory too; while
//                 one row tile is with its warps the other one has the matrix
//                 unit.  Keys and values come into rings in shared memory in
//                 the 128-byte swizzled layout the matrix unit reads: one warp
//                 sends tensor copies of boxes of 8 to 128 rows of a page
//                 (BOX), or three copy row by row, 16 bytes at a time, from
//                 pages whose size no such box divides.
//                 A tile that some rows see in part may hold infinities or NaN
//                 in values those rows must not see, and 0 * inf is NaN: there
//                 the copying warps replace them by zeros, and the rows that
//                 do see them take them up at the end.
//                 A prompt of 8,000 tokens, 32 query heads over 8 of 128 in
//                 bfloat16: 367 us, 1.43 PFLOP/s (75 % of the measured matrix
//                 rate), with inputs that come from memory; 349 us in a loop over
//                 three sets of them; by rows 867 us.  The matrix unit is busy
//                 52 % of a 4,096-token prompt's 111 us.  When that took 129 us,
//                 leaving out the warps' work on the scores saved 31 us, the products
//                 15 us and the exponentials 5 us: what bounds it is the chain
//                 of both with the hand-overs between them, and at windows and
//                 short sessions the 6 us a block takes to its first scores and
//                 from its last ones.  Some values of a thread spill (68 to 100
//                 bytes stored, 112 to 232 loaded, by form).
// k_attend_join   joins the parts of rows whose tokens were split over blocks.
#include "pcs_attend_block_dev.h"

namespace pcs {
namespace {

// Joins the parts of a row tile: a thread per row, 32 of its dims a block.
template <typename T, int DP>
__global__ void __launch_bounds__(kTile) k_attend_join(const __grid_constant__ AttendArgs a, int blocks) {
  attend_dependency();
  int b = blockIdx.x;
  const int d0 = b % (DP / 32) * 32;
  b /= DP / 32;
  const int t = b % 2;
  b /= 2;
  const int head = b % a.cache.heads;
  b /= a.cache.heads;
  const int s = b % a.batch.sessions, blk = blocks - 1 - b / a.batch.sessions;
  const SessionView v = session_rows(a, s);
  const int row = threadIdx.x, r = blk * 2 * kTile + t * kTile + row;
  if (!rows_there(a, v, false) || r >= v.m * a.group) return;
  // The parts of the blocks that the block kernel's numbering puts side by side.
  const int64_t first = static_cast<int64_t>(b) * a.splits * a.cache.heads + head;
  const int64_t step = static_cast<int64_t>(a.cache.heads) * 2 * (DP + 2) * kTile;
  const float* part = a.part + (first * 2 + t) * (DP + 2) * kTile + row;
  float top = -INFINITY;
  for (int w = 0; w < a.splits; ++w) top = fmaxf(top, __ldcg(part + w * step + DP * kTile));
  const float at = top == -INFINITY ? 0.0f : top;
  float o[32] = {}, total = 0.0f;
  for (int w = 0; w < a.splits; ++w) {
    const float f = exp2_fast(__ldcg(part + w * step + DP * kTile) - at);
    total = fmaf(__ldcg(part + w * step + (DP + 1) * kTile), f, total);
#pragma unroll
    for (int k = 0; k < 32; ++k) o[k] = fmaf(__ldcg(part + w * step + (d0 + k) * kTile), f, o[k]);
  }
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  const uint32_t tok = a.by_group.div(r);
  const int h = head * a.group + (r - static_cast<int>(tok) * a.group);
  uint8_t* out = a.out.data + (v.q0 + tok) * a.out.token_bytes + h * a.out.head_bytes + d0 * 2;
#pragma unroll
  for (int k = 0; k < 32; k += 8) {
    if (d0 + k >= a.cache.head_dim) continue;
    uint4 y;
    y.x = pack2<T>(o[k] * inv, o[k + 1] * inv);
    y.y = pack2<T>(o[k + 2] * inv, o[k + 3] * inv);
    y.z = pack2<T>(o[k + 4] * inv, o[k + 5] * inv);
    y.w = pack2<T>(o[k + 6] * inv, o[k + 7] * inv);
    *reinterpret_cast<uint4*>(out + 2 * k) = y;
  }
  if (d0 == 0 && a.lse)
    a.lse[(v.q0 + tok) * (static_cast<int64_t>(a.cache.heads) * a.group) + h] =
        total == 0.0f ? -INFINITY : fmaf(top - kLift<T>, 0.693147180559945309f, logf(total));
}

template <typename T, int DP>
cudaError_t launch(const AttendArgs& a, int blocks, const TensorMaps& maps, cudaStream_t stream) {
  return a.box_rows == 0   ? launch_form<T, DP, 0, false>(a, blocks, maps, stream)
         : a.box_rows == 8 ? launch_form<T, DP, 2, false>(a, blocks, maps, stream)
                           : launch_form<T, DP, 1, false>(a, blocks, maps, stream);
}

template <typename T, int DP>
cudaError_t launch_join(const AttendArgs& a, int blocks, cudaStream_t stream) {
  cudaLaunchAttribute attr;
  const cudaLaunchConfig_t cfg =
      config(static_cast<int64_t>(blocks) * a.batch.sessions * a.cache.heads * 2 * (DP / 32), kTile, 0, &attr, stream);
  return cudaLaunchKernelEx(&cfg, k_attend_join<T, DP>, a, blocks);
}

}  // namespace

cudaError_t launch_attend_block(const AttendArgs& a, uint32_t dtype, int blocks, const TensorMaps& maps,
                                cudaStream_t stream) {
  if (a.parent) return launch_attend_block_tree(a, dtype, blocks, maps, stream);
  if (dtype == PCS_DT_F16)
    return a.cache.head_dim <= 64 ? launch<__half, 64>(a, blocks, maps, stream) : launch<__half, 128>(a, blocks, maps, stream);
  return a.cache.head_dim <= 64 ? launch<__nv_bfloat16, 64>(a, blocks, maps, stream)
                                : launch<__nv_bfloat16, 128>(a, blocks, maps, stream);
}

cudaError_t launch_attend_join(const AttendArgs& a, uint32_t dtype, int blocks, cudaStream_t stream) {
  if (dtype == PCS_DT_F16)
    return a.cache.head_dim <= 64 ? launch_join<__half, 64>(a, blocks, stream) : launch_join<__half, 128>(a, blocks, stream);
  return a.cache.head_dim <= 64 ? launch_join<__nv_bfloat16, 64>(a, blocks, stream) : launch_join<__nv_bfloat16, 128>(a, blocks, stream);
}

}  // namespace pcs

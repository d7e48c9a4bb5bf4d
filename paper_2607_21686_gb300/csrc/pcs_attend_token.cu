// pcs_attend_token.cu -- attention of one new token, or of a few, of every
// session over a paged cache of keys and values.
//
// k_attend_token  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), s_j = scale
//                 q.k_j, over the tokens a new token sees, in one pass with
//                 running m and sums.  Every key and value row is used by the
//                 few query rows of its head alone (at most 32), so the bound
//                 is HBM.  A block takes one session, key head and part of the
//                 visible tokens; each of its warps walks tiles of 16 tokens
//                 through a ring of its own in shared memory, filled by
//                 16-byte asynchronous copies (pages of any size, no barrier
//                 between the warps), and the warps' and then the parts'
//                 results are joined by their maxima.
//                 Tokens are the rows of the matrix instruction (m16n8k16) and
//                 query rows its columns: keys and values come out of shared
//                 memory as the first operand, eight query rows cost one
//                 column tile, and the weights turn from result to operand
//                 with one transposing move per 8 x 8.  (That instruction is
//                 busy 6 % of the time while HBM is the bound: the fifth-
//                 generation tensor cores, which want 128 rows, have nothing to
//                 add here.)
//                 256 sessions over windows of 1,024 tokens, 16 heads of 64 in
//                 bfloat16: 170 us, 6.3 TB/s (95 % of the measured copy rate);
//                 four tokens over 200,001, 8 key heads of 128: 125 us, 6.6 TB/s.
//                 A second product with what the weights' rounding left of them
//                 took 175 us there, and 10 % more with 32 rows a key head: the
//                 weights stay in 16 bits.
//                 k_attend_token_join joins more parts than kTokenOwnJoin.
#include "pcs_attend_token_dev.h"

namespace pcs {
namespace {

// Joins many parts: a block per row, whose warps take every kWarps-th part.
template <typename T, int DP, int NT>
__global__ void __launch_bounds__(kThreads) k_attend_token_join(const __grid_constant__ AttendArgs a) {
  constexpr int kRows = 8 * NT;
  __shared__ float sums[kWarps][DP], tops[kWarps], totals[kWarps];
  attend_dependency();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t pair = blockIdx.x / kRows;
  const int row = static_cast<int>(blockIdx.x % kRows);
  const int s = static_cast<int>(pair / a.cache.heads), head = static_cast<int>(pair % a.cache.heads);
  const SessionView view = session_rows(a, s);
  if (row >= view.m * a.group || !rows_there(a, view, false)) return;
  const int64_t part_floats = static_cast<int64_t>(kRows) * (DP + 2);
  const float* part = a.part + pair * a.splits * part_floats;
  float m = -INFINITY;
  for (int w = threadIdx.x; w < a.splits; w += kThreads) m = fmaxf(m, __ldcg(part + w * part_floats + kRows * DP + row));
#pragma unroll
  for (int k = 16; k > 0; k /= 2) m = fmaxf(m, __shfl_xor_sync(kFull, m, k));
  if (lane == 0) tops[warp] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) m = fmaxf(m, tops[w]);
  const float at = m == -INFINITY ? 0.0f : m;
  float x[DP / 32] = {}, total = 0.0f;
#pragma unroll 8
  for (int w = warp; w < a.splits; w += kWarps) {
    const float* p = part + w * part_floats;
    const float f = exp2_fast(__ldcg(p + kRows * DP + row) - at);
    total = fmaf(__ldcg(p + kRows * DP + kRows + row), f, total);
#pragma unroll
    for (int k = 0; k < DP / 64; ++k) {
      const float2 y = __ldcg(reinterpret_cast<const float2*>(p + row * DP + 64 * k + 2 * lane));
      x[2 * k] = fmaf(y.x, f, x[2 * k]);
      x[2 * k + 1] = fmaf(y.y, f, x[2 * k + 1]);
    }
  }
#pragma unroll
  for (int k = 0; k < DP / 64; ++k)
    *reinterpret_cast<float2*>(&sums[warp][64 * k + 2 * lane]) = make_float2(x[2 * k], x[2 * k + 1]);
  if (lane == 0) totals[warp] = total;
  __syncthreads();
  total = 0.0f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) total += totals[w];
  const float inv = total == 0.0f ? 0.0f : 1.0f / total;
  const uint32_t tok = a.by_group.div(row);
  const int h = head * a.group + (row - static_cast<int>(tok) * a.group);
  for (int d = 2 * threadIdx.x; d < a.cache.head_dim; d += 2 * kThreads) {
    float2 y = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      y.x += sums[w][d];
      y.y += sums[w][d + 1];
    }
    *reinterpret_cast<uint32_t*>(a.out.data + (view.q0 + tok) * a.out.token_bytes + h * a.out.head_bytes + d * 2) =
        pack2<T>(y.x * inv, y.y * inv);
  }
  if (threadIdx.x == 0 && a.lse)
    a.lse[(view.q0 + tok) * (static_cast<int64_t>(a.cache.heads) * a.group) + h] =
        total == 0.0f ? -INFINITY : fmaf(m - kLift<T>, 0.693147180559945309f, logf(total));
}

template <typename T, int DP, int NT>
cudaError_t launch(const AttendArgs& a, bool join, cudaStream_t stream) {
  auto k = k_attend_token<T, DP, NT, false>;
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
  if (join) {  // (the parts of every form)
    cfg.gridDim = dim3(static_cast<unsigned>(static_cast<int64_t>(a.batch.sessions) * a.cache.heads * 8 * NT));
    cfg.dynamicSmemBytes = 0;
    return cudaLaunchKernelEx(&cfg, k_attend_token_join<T, DP, NT>, a);
  }
  return cudaLaunchKernelEx(&cfg, k, a);
}

template <typename T>
cudaError_t by_size(const AttendArgs& a, int rows, bool join, cudaStream_t stream) {
  if (a.cache.head_dim <= 64)
    return rows <= 8 ? launch<T, 64, 1>(a, join, stream) : rows <= 16 ? launch<T, 64, 2>(a, join, stream)
                                                               : launch<T, 64, 4>(a, join, stream);
  return rows <= 8 ? launch<T, 128, 1>(a, join, stream) : rows <= 16 ? launch<T, 128, 2>(a, join, stream)
                                                              : launch<T, 128, 4>(a, join, stream);
}

}  // namespace

int attend_token_blocks_per_sm(int head_dim, int rows) {
  if (head_dim <= 64) return rows <= 16 ? kResident<64, 2> : kResident<64, 4>;
  return kResident<128, 4>;
}

cudaError_t launch_attend_token(const AttendArgs& a, uint32_t dtype, int rows, bool join, cudaStream_t stream) {
  if (!join && a.parent) return launch_attend_token_tree(a, dtype, rows, stream);
  return dtype == PCS_DT_F16 ? by_size<__half>(a, rows, join, stream) : by_size<__nv_bfloat16>(a, rows, join, stream);
}

}  // namespace pcs

// pcs_kv_pages.cu -- tokens of a paged cache read out of their pages, and those of
// the new tokens that are kept moved next to the context.
//
// k_kv_read  y = code * 2^(b - 127), a head's tokens gathered from their pages;
//            16-bit elements as they are.  Each code is read once and each value
//            written once: the bound is HBM, two thirds of it the writes.  A block
//            takes a few tokens, whose rows its first warp looks up; a thread moves
//            units of eight elements, several of them in flight.
// k_kv_keep  rows to lower slots of the same session.  Kept row i comes from an index
//            of at least i, so what is read after row i is written lies further on: a
//            thread that takes a column of 16 bytes through all rows in their order
//            needs nobody else's.  A few rows a session: the bound is latency.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "pcs_attend.h"
#include "pcs_codes_dev.h"
#include "pcs_internal.h"
#include "pcs_place_dev.h"

namespace pcs {
namespace {

constexpr int kThreads = 256;
constexpr int kReadTokens = 8;   // tokens of a block at most
constexpr int kFlight = 4;       // units of a thread in flight

__device__ __forceinline__ void grid_dependency() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

struct ReadShape {
  FastDiv by_units, by_heads, by_tokens;
  int32_t per_block, tensors;
};

// Eight values of type T.
template <typename T>
struct alignas(16) Eight {
  T e[8];
};

template <int CODES, typename T>
__global__ void __launch_bounds__(kThreads) k_kv_read(const __grid_constant__ ReadArgs a, const __grid_constant__ ReadShape shape) {
  __shared__ Place place[kReadTokens];
  grid_dependency();
  const CacheDev& c = a.cache;
  const int tid = threadIdx.x;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * shape.per_block;
  const int nt = static_cast<int>(a.batch.tokens - t0 < shape.per_block ? a.batch.tokens - t0 : shape.per_block);
  if (tid < 32) {
    const int s = a.batch.q_off ? session_of(a.batch, t0, tid) : 0;
    if (tid < nt) place[tid] = place_of(c, a.batch, a.err, t0 + tid, s);
  }
  __syncthreads();
  const int total = shape.per_block * shape.tensors * c.heads * static_cast<int>(shape.by_units.d);
  for (int i0 = tid; i0 < total; i0 += kFlight * kThreads) {
    using Codes = std::conditional_t<CODES == kElements16, uint4, uint2>;
    Codes x[kFlight];
    uint32_t b[kFlight];
    uint8_t* to[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const int i = i0 + k * kThreads;
      x[k] = Codes{};
      b[k] = 127;
      to[k] = nullptr;
      if (i >= total) continue;
      // Unit u of head h of token t of tensor w.
      uint32_t q = shape.by_units.div(i);
      const uint32_t u = i - q * shape.by_units.d;
      uint32_t r = shape.by_heads.div(q);
      const uint32_t h = q - r * shape.by_heads.d;
      const uint32_t w = shape.by_tokens.div(r), t = r - w * shape.by_tokens.d;
      if (static_cast<int>(t) >= nt) continue;
      const int which = a.out[0].data == nullptr ? 1 : static_cast<int>(w);
      to[k] = a.out[which].data + (t0 + t) * a.out[which].token_bytes + h * a.out[which].head_bytes + u * 8 * sizeof(T);
      const int64_t at = which ? place[t].v : place[t].k;
      if (at < 0) continue;
      const uint8_t* row = (which ? c.v : c.k) + at;
      x[k] = __ldg(reinterpret_cast<const Codes*>(row + h * c.head_bytes + u * sizeof(Codes)));
      if (CODES != kElements16) b[k] = __ldg(row + c.scale_at + h);
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      if (to[k] == nullptr) continue;
      if constexpr (CODES == kElements16) {
        *reinterpret_cast<uint4*>(to[k]) = x[k];
      } else {
        const float s = scale_value(b[k]);
        float y[8];
        four_values<CODES>(x[k].x, y);
        four_values<CODES>(x[k].y, y + 4);
        Eight<T> z;
#pragma unroll
        for (int d = 0; d < 8; ++d) z.e[d] = rounded<T>(y[d] * s);
        if constexpr (sizeof(T) == 4) {
          reinterpret_cast<float4*>(to[k])[0] = make_float4(z.e[0], z.e[1], z.e[2], z.e[3]);
          reinterpret_cast<float4*>(to[k])[1] = make_float4(z.e[4], z.e[5], z.e[6], z.e[7]);
        } else {
          *reinterpret_cast<uint4*>(to[k]) = *reinterpret_cast<const uint4*>(&z);
        }
      }
    }
  }
}

template <int CODES, typename T>
cudaError_t read(const ReadArgs& a, const ReadShape& shape, cudaStream_t stream) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.batch.tokens + shape.per_block - 1) / shape.per_block));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_kv_read<CODES, T>, a, shape);
}

template <int CODES>
cudaError_t read_as(const ReadArgs& a, const ReadShape& shape, cudaStream_t stream) {
  switch (a.dtype) {
    case PCS_DT_F16: return read<CODES, __half>(a, shape, stream);
    case PCS_DT_BF16: return read<CODES, __nv_bfloat16>(a, shape, stream);
    default: return read<CODES, float>(a, shape, stream);
  }
}

// ---- Keep ------------------------------------------------------------------------------

constexpr int kKeepRows = 64;    // rows whose places are looked up at a time

// Where the row of position p is; -1: no page, and what is wrong goes to err.
__device__ __forceinline__ Place row_of(const CacheDev& c, uint32_t* err, int s, int64_t p) {
  const uint32_t slot = p < 0 || p > 0x7fffffff ? 0xffffffffu : c.slot_of(static_cast<uint32_t>(p));
  if (slot >= static_cast<uint32_t>(c.slots)) {
    atomicOr(err, kDevErrIndex);
    return {-1, -1};
  }
  const uint32_t page = c.page_rows.div(slot);
  const int64_t row = static_cast<int64_t>(slot - page * c.page_rows.d) * c.row_bytes;
  const int64_t e = s * c.table_stride + page;
  const int32_t kp = __ldg(c.table + e);
  const int32_t vp = c.v_table ? __ldg(c.v_table + e) : kp;
  if (kp < 0 || kp >= c.n_pages || vp < 0 || vp >= c.n_pages) {
    if (kp < -1 || kp >= c.n_pages || vp < -1 || vp >= c.n_pages) atomicOr(err, kDevErrIndex);
    return {-1, -1};
  }
  return {kp * c.page_bytes + row, vp * c.page_bytes + row};
}

template <typename U>
__device__ __forceinline__ void move_column(uint8_t* pool, int64_t column, const int64_t* from, const int64_t* to, int n) {
  for (int i = 0; i < n; i += 4) {
    U x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n && from[i + k] >= 0) x[k] = *reinterpret_cast<const U*>(pool + from[i + k] + column);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k < n && from[i + k] >= 0) *reinterpret_cast<U*>(pool + to[i + k] + column) = x[k];
  }
}

// A session's rows; a column is 16 bytes of a head, or with codes a scale byte.
__global__ void __launch_bounds__(kThreads) k_kv_keep(const __grid_constant__ KeepArgs a, FastDiv by_parts) {
  __shared__ int64_t from[2][kKeepRows], to[2][kKeepRows];
  grid_dependency();
  const CacheDev& c = a.cache;
  const int s = blockIdx.x, tid = threadIdx.x;
  const int m = a.batch.q_off ? __ldg(a.batch.q_off + s + 1) - __ldg(a.batch.q_off + s) : a.batch.each;
  const int32_t len = a.batch.lens[s], n = __ldg(a.count + s);
  const int64_t first = static_cast<int64_t>(len) - m;
  const int32_t* index = a.index + s * a.index_stride;
  bool bad = m < 0 || m > a.batch.max_new || first < 0 || n < 0 || n > a.most || n > m;
  if (!bad) {
    bool off = false;
    for (int i = tid; i < n; i += kThreads) {
      const int x = __ldg(index + i), before = i ? __ldg(index + i - 1) : -1;
      off |= x <= before || x >= m;
    }
    bad = __syncthreads_or(off) != 0;
  }
  if (bad && tid == 0) atomicOr(a.err, kDevErrIndex);
  const int parts = static_cast<int>(by_parts.d), columns = c.heads * parts;
  for (int i0 = 0; i0 < n && !bad; i0 += kKeepRows) {
    const int rows = min(kKeepRows, n - i0);
    for (int i = tid; i < rows; i += kThreads) {
      const int x = __ldg(index + i0 + i);
      Place src = {-1, -1}, dst = {-1, -1};
      if (x != i0 + i) {
        src = row_of(c, a.err, s, first + x);
        dst = row_of(c, a.err, s, first + i0 + i);
        if (src.k < 0 && dst.k >= 0) atomicOr(a.err, kDevErrIndex);
        if (src.k < 0 || dst.k < 0) src = {-1, -1};
      }
      from[0][i] = src.k, from[1][i] = src.v;
      to[0][i] = dst.k, to[1][i] = dst.v;
    }
    __syncthreads();
    for (int u = tid; u < 2 * columns; u += kThreads) {
      const int w = u >= columns, x = u - w * columns;
      const int h = by_parts.div(x);
      move_column<uint4>(w ? c.v : c.k, h * c.head_bytes + 16 * (x - h * parts), from[w], to[w], rows);
    }
    if (c.codes != kElements16)
      for (int u = tid; u < 2 * c.heads; u += kThreads) {
        const int w = u >= c.heads;
        move_column<uint8_t>(w ? c.v : c.k, c.scale_at + u - w * c.heads, from[w], to[w], rows);
      }
    __syncthreads();
  }
  // (lens_out may be lens: all threads have read that before they voted on the index,
  // and where they did not vote it stays as it is.)
  if (a.lens_out && tid == 0) a.lens_out[s] = bad ? len : static_cast<int32_t>(first + n);
}

}  // namespace

cudaError_t launch_read(const ReadArgs& a, int sm_count, cudaStream_t stream) {
  ReadShape shape;
  shape.by_units.set(a.cache.head_dim / 8);
  shape.by_heads.set(a.cache.heads);
  shape.tensors = (a.out[0].data != nullptr) + (a.out[1].data != nullptr);
  // Few tokens: a block for each; many: as many as keep four units a thread in flight.
  const int64_t share = a.batch.tokens / (2 * sm_count);
  const int64_t units = static_cast<int64_t>(shape.tensors) * a.cache.heads * (a.cache.head_dim / 8);
  int64_t most = (kFlight * kThreads + units - 1) / units;
  if (most > kReadTokens) most = kReadTokens;
  shape.per_block = static_cast<int32_t>(share < 1 ? 1 : share > most ? most : share);
  shape.by_tokens.set(shape.per_block);
  switch (a.cache.codes) {
    case kCodesE4M3: return read_as<kCodesE4M3>(a, shape, stream);
    case kCodesI8: return read_as<kCodesI8>(a, shape, stream);
    default: return read<kElements16, __half>(a, shape, stream);
  }
}

cudaError_t launch_keep(const KeepArgs& a, cudaStream_t stream) {
  FastDiv by_parts;
  const int element = a.cache.codes == kElements16 ? 2 : 1;
  by_parts.set(a.cache.head_dim * element / 16);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.batch.sessions);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_kv_keep, a, by_parts);
}

}  // namespace pcs

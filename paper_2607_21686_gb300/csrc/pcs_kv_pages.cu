// pcs_kv_pages.cu -- tokens of a paged cache read out of their pages, and those of
// the new tokens that are kept moved next to the context.
//
// k_kv_read  y = code * 2^(b - 127), a head's tokens gathered from their pages;
//            16-bit elements as they are.  Each code is read once and each value
//            written once: the bound is HBM, two thirds of it the writes.  A block
//            takes a few tokens, whose rows its first warp looks up; a thread takes
//            16 bytes of a row in several of them, so that what it computes of heads and
//            offsets serves all its tokens.
//            288,000 tokens of 48 sessions, 8 heads of 128, I8 to float16: 355 us, 6.6
//            TB/s (97 % of the measured copy rate); E4M3 345 us; 16-bit pages as they are
//            448 us, 6.9 TB/s (102 %).
// k_widen    the same into pages of 16-bit elements, slot by slot, of what the new tokens
//            of a call see: the cache that attention of many rows a key head goes over,
//            where every tile of codes would be converted once for each block of rows.
//            A prompt of 8,000 tokens, 8 heads of 128: 14 us, before 366 us of attention;
//            over the codes the call takes 675 us (I8), 632 us (E4M3).
// k_kv_keep  rows to lower slots of the same session.  Kept row i comes from an index
//            of at least i, so what is read after row i is written lies further on: a
//            thread that takes a column of 16 bytes through all rows in their order
//            needs nobody else's.  A few rows a session: the bound is latency (1 to 7 rows of
//            256 sessions, 8 heads of 128: 8 us on the device).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "pcs_attend.h"
#include "pcs_attend_dev.h"
#include "pcs_codes_dev.h"
#include "pcs_internal.h"
#include "pcs_place_dev.h"

namespace pcs {
namespace {

constexpr int kThreads = 256;
constexpr int kReadTokens = 128;  // tokens of a block at most
constexpr int kFlight = 4;       // units of a thread in flight
// What whole numbers take to become values fills more of the issue slots: more warps with
// fewer units each hide it better.  (288,000 tokens of 8 heads of 128: I8 381 us with four
// units and five blocks an SM, 356 us with two and seven; E4M3 345 and 350 us.)
template <int CODES>
constexpr int kReadFlight = CODES == kCodesI8 ? 2 : kFlight;
template <int CODES>
constexpr int kReadBlocks = CODES == kCodesI8 ? 7 : 5;

__device__ __forceinline__ void grid_dependency() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// A thread takes a unit of 16 bytes of a row -- of one head of the keys or of the values --
// in every `lanes`-th token of its block.
struct ReadShape {
  FastDiv by_units, by_row, by_threads;  // units of a head, of a row, threads a token lane
  int32_t per_block, units, lanes;       // tokens of a block, units of both rows, tokens at once
};

// 32 bytes at once, where their place is a multiple of that, else 16 and 16.
template <bool WIDE>
__device__ __forceinline__ void store32(uint8_t* to, const uint4& x, const uint4& y) {
  if constexpr (WIDE) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w),
                 "r"(y.x), "r"(y.y), "r"(y.z), "r"(y.w)
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(to)[0] = x;
    reinterpret_cast<uint4*>(to)[1] = y;
  }
}

template <int CODES, typename T, bool WIDE>
__device__ __forceinline__ void write_unit(uint8_t* to, const uint4& x, uint32_t b) {
  if constexpr (CODES == kElements16) {
    *reinterpret_cast<uint4*>(to) = x;
  } else if constexpr (sizeof(T) == 4) {
    const float s = scale_value(b);
    float y[16];
    four_values<CODES>(x.x, y);
    four_values<CODES>(x.y, y + 4);
    four_values<CODES>(x.z, y + 8);
    four_values<CODES>(x.w, y + 12);
    uint4 z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      z[i] = make_uint4(__float_as_uint(y[4 * i] * s), __float_as_uint(y[4 * i + 1] * s), __float_as_uint(y[4 * i + 2] * s),
                        __float_as_uint(y[4 * i + 3] * s));
    store32<WIDE>(to, z[0], z[1]);
    store32<WIDE>(to + 32, z[2], z[3]);
  } else {
    uint4 lo, hi;
    sixteen_elements<T, CODES>(x, b, lo, hi);
    store32<WIDE>(to, lo, hi);
  }
}

template <int CODES, typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads, kReadBlocks<CODES>) k_kv_read(const __grid_constant__ ReadArgs a, const __grid_constant__ ReadShape shape) {
  constexpr int kF = kReadFlight<CODES>;
  __shared__ Place place[kReadTokens];
  grid_dependency();
  const CacheDev& c = a.cache;
  const int tid = threadIdx.x;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * shape.per_block;
  // (Rows behind the last session's are nobody's: they stay as they are.)
  const int64_t end = a.batch.q_off ? min(a.batch.tokens, static_cast<int64_t>(__ldg(a.batch.q_off + a.batch.sessions))) : a.batch.tokens;
  const int nt = static_cast<int>(min(end - t0, static_cast<int64_t>(shape.per_block)));
  if ((tid & ~31) < nt) {  // a warp looks up 32 tokens
    const int s = a.batch.q_off ? session_of(a.batch, t0 + (tid & ~31), tid & 31) : 0;
    if (tid < nt) place[tid] = place_of(c, a.batch, a.err, t0 + tid, s);
  }
  __syncthreads();
  constexpr int kElements = CODES == kElements16 ? 8 : 16;  // of a unit
  const int lane = shape.by_threads.div(tid);
  for (int v = tid - lane * static_cast<int>(shape.by_threads.d); v < shape.units && lane < shape.lanes; v += kThreads) {
    // Unit u of head h of the keys (w 0) or the values.
    int w = shape.by_row.div(v);
    const uint32_t r = v - w * shape.by_row.d, h = shape.by_units.div(r), u = r - h * shape.by_units.d;
    if (a.out[0].data == nullptr) w = 1;
    const HeadsDev& out = a.out[w];
    const uint8_t* const from = (w ? c.v : c.k) + static_cast<int64_t>(h) * c.head_bytes + u * 16;
    const uint8_t* const scale = (w ? c.v : c.k) + c.scale_at + h;
    uint8_t* to = out.data + (t0 + lane) * out.token_bytes + static_cast<int64_t>(h) * out.head_bytes + u * (kElements * sizeof(T));
    const int64_t step = shape.lanes * out.token_bytes;
    for (int i = lane; i < nt; i += kF * shape.lanes) {
      uint4 x[kF];
      uint32_t b[kF];
#pragma unroll
      for (int k = 0; k < kF; ++k) {
        const int t = i + k * shape.lanes;
        x[k] = make_uint4(0, 0, 0, 0);
        b[k] = 127;
        if (t >= nt) continue;
        const int64_t at = w ? place[t].v : place[t].k;
        if (at < 0) continue;
        x[k] = __ldg(reinterpret_cast<const uint4*>(from + at));
        if (CODES != kElements16) b[k] = __ldg(scale + at);
      }
#pragma unroll
      for (int k = 0; k < kF; ++k) {
        if (i + k * shape.lanes < nt) write_unit<CODES, T, WIDE>(to, x[k], b[k]);
        to += step;
      }
    }
  }
}

template <int CODES, typename T, bool WIDE>
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
  return cudaLaunchKernelEx(&cfg, k_kv_read<CODES, T, WIDE>, a, shape);
}

template <int CODES, bool WIDE>
cudaError_t read_as(const ReadArgs& a, const ReadShape& shape, cudaStream_t stream) {
  switch (a.dtype) {
    case PCS_DT_F16: return read<CODES, __half, WIDE>(a, shape, stream);
    case PCS_DT_BF16: return read<CODES, __nv_bfloat16, WIDE>(a, shape, stream);
    default: return read<CODES, float, WIDE>(a, shape, stream);
  }
}

// ---- Codes to pages of elements -----------------------------------------------------------

constexpr int kWidenRows = 32;   // tokens of a block at a time at most

template <int CODES, typename T>
__global__ void __launch_bounds__(kThreads) k_widen(const __grid_constant__ AttendArgs a, const __grid_constant__ ReadShape shape,
                                                    const __grid_constant__ WidenTo to, int chunks) {
  __shared__ RowPlace place[kWidenRows];
  __shared__ int64_t row[kWidenRows];
  grid_dependency();
  const CacheDev& c = a.cache;
  const int tid = threadIdx.x, s = blockIdx.x / chunks, chunk = blockIdx.x - s * chunks;
  // Whole boxes of rows, as the kernel behind copies them: rows that nobody sees must not
  // hold what was in this memory before.
  SessionView view = session_rows(a, s);
  const int align = a.box_rows > 0 ? a.box_rows : 1;
  narrow(a, view, 0, view.m, align);
  if (view.m <= 0 || !rows_there(a, view, false)) return;  // nobody looks at the session
  const int places = (view.seen + align - 1) & -align;
  const int pages = c.slots / static_cast<int>(c.page_rows.d);
  if (chunk == 0)
    for (int p = tid; p < pages; p += kThreads) {
      const int32_t k = __ldg(c.table + s * c.table_stride + p), v = c.v_table ? __ldg(c.v_table + s * c.table_stride + p) : k;
      to.table[static_cast<int64_t>(s) * pages + p] = k < 0 || k >= c.n_pages || v < 0 || v >= c.n_pages ? -1 : s * pages + p;
    }
  const int lane = shape.by_threads.div(tid), v0 = tid - lane * static_cast<int>(shape.by_threads.d);
  const int rows = shape.per_block;
  for (int e0 = chunk * rows; e0 < places; e0 += chunks * rows) {
    __syncthreads();
    const int e = e0 + tid;
    if (tid < rows && e < places) {
      const uint32_t slot = align > 1 ? box_slot(a, view, e & -align) + (e & (align - 1)) : c.slot_of(static_cast<uint32_t>(seen_position(view, e)));
      place[tid] = slot_place(a, s, slot);
      row[tid] = static_cast<int64_t>(s) * c.slots + slot;
    }
    __syncthreads();
    const int nt = min(rows, places - e0);
    for (int v = v0; v < shape.units && lane < shape.lanes; v += kThreads) {
      const int w = shape.by_row.div(v);
      const uint32_t r = v - w * shape.by_row.d, h = shape.by_units.div(r), u = r - h * shape.by_units.d;
      const uint8_t* const pool = w ? c.v : c.k;
      const uint32_t from = h * static_cast<uint32_t>(c.head_bytes) + u * 16;
      uint8_t* const out = (w ? to.v : to.k) + r * 32;
      for (int i = lane; i < nt; i += kFlight * shape.lanes) {
        uint4 x[kFlight];
        uint32_t b[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
          const int t = i + k * shape.lanes;
          x[k] = make_uint4(0, 0, 0, 0);
          b[k] = 127;
          if (t >= nt) continue;
          const uint32_t at = w ? place[t].v : place[t].k;
          if (at == kNoRow) continue;
          const uint8_t* z = row_at(a, pool, at);
          x[k] = __ldg(reinterpret_cast<const uint4*>(z + from));
          b[k] = __ldg(z + c.scale_at + h);
        }
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
          const int t = i + k * shape.lanes;
          if (t < nt && place[t].k != kNoRow) write_unit<CODES, T, true>(out + row[t] * to.row_bytes, x[k], b[k]);
        }
      }
    }
  }
}

template <int CODES, typename T>
cudaError_t widen(const AttendArgs& a, const ReadShape& shape, const WidenTo& to, int chunks, cudaStream_t stream) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.batch.sessions) * chunks);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_widen<CODES, T>, a, shape, to, chunks);
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

namespace {
// Shares out the units of a row of `tensors` pools.
ReadShape shape_of(const CacheDev& c, int tensors) {
  ReadShape shape;
  const int head = c.head_dim / (c.codes == kElements16 ? 8 : 16), row = c.heads * head;
  shape.by_units.set(head);
  shape.by_row.set(row);
  shape.units = row * tensors;
  shape.lanes = shape.units >= kThreads ? 1 : kThreads / shape.units;
  shape.by_threads.set(kThreads / shape.lanes);
  shape.per_block = 0;
  return shape;
}
}  // namespace

cudaError_t launch_widen(const AttendArgs& a, const WidenTo& to, int64_t seen, cudaStream_t stream) {
  // As many tokens as a block's threads have in flight.  (A prompt of 8,000 tokens, 8 heads of
  // 128: 18 us in blocks of 32 tokens.)
  ReadShape shape = shape_of(a.cache, 2);
  shape.per_block = std::min(kWidenRows, kFlight * shape.lanes);
  const int64_t chunks =
      std::max<int64_t>(1, std::min<int64_t>((seen + shape.per_block - 1) / shape.per_block, 0x7fffffff / a.batch.sessions));
  const int n = static_cast<int>(chunks);
  const bool half = a.dtype == PCS_DT_F16;
  if (a.cache.codes == kCodesE4M3)
    return half ? widen<kCodesE4M3, __half>(a, shape, to, n, stream) : widen<kCodesE4M3, __nv_bfloat16>(a, shape, to, n, stream);
  return half ? widen<kCodesI8, __half>(a, shape, to, n, stream) : widen<kCodesI8, __nv_bfloat16>(a, shape, to, n, stream);
}

cudaError_t launch_read(const ReadArgs& a, int sm_count, cudaStream_t stream) {
  ReadShape shape = shape_of(a.cache, (a.out[0].data != nullptr) + (a.out[1].data != nullptr));
  // Few tokens: as many blocks as there are; many: blocks that look up as many tokens as
  // their threads take in a few rounds.
  const int flight = a.cache.codes == kCodesI8 ? kReadFlight<kCodesI8> : kReadFlight<kCodesE4M3>;
  const int64_t share = a.batch.tokens / (4 * sm_count), most = std::min<int64_t>(kReadTokens, 2 * flight * shape.lanes);
  shape.per_block = static_cast<int32_t>(std::max<int64_t>(1, std::min(share, most)));
  bool wide = true;
  for (const HeadsDev& o : a.out)
    wide = wide && reinterpret_cast<uintptr_t>(o.data) % 32 == 0 && o.token_bytes % 32 == 0 && o.head_bytes % 32 == 0;
  switch (a.cache.codes) {
    case kCodesE4M3: return wide ? read_as<kCodesE4M3, true>(a, shape, stream) : read_as<kCodesE4M3, false>(a, shape, stream);
    case kCodesI8: return wide ? read_as<kCodesI8, true>(a, shape, stream) : read_as<kCodesI8, false>(a, shape, stream);
    default: return read<kElements16, __half, false>(a, shape, stream);
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

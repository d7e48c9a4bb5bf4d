// pcs_attend_dev.h -- device code that the attention kernels share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstring>
#include <type_traits>
#include <cstdint>

#include "pcs_attend.h"
#include "pcs_attend_view.h"
#include "pcs_internal.h"

namespace pcs {

// Raises a kernel's limit of dynamic shared memory, once per device.
struct SmemLimit {
  std::atomic<uint64_t> done{0};
  template <typename K>
  cudaError_t set(K kernel, uint32_t bytes) {
    int dev = 0;
    if (cudaError_t e = cudaGetDevice(&dev)) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
  }
};

__device__ __forceinline__ void attend_dependency() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// 2^x; 0 for -inf.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two floats rounded to a pair of 16-bit elements, the first in the low half.
// The weights of a softmax are rounded to the cache's type for the matrix
// instruction, each by at most 2^-8 (bf16) or 2^-11 of itself, which is what
// the rounding of the result itself costs; their sum stays in 32 bits.
// float16 holds numbers below 2^-14 to 2^-25 and no better: many small weights
// beside a large one would be lost, while the total counts them.  So its weights
// are 2^kLift times exp(score - maximum) -- at most 2^15 with a maximum that is
// raised by steps of 2^8 -- and keep 11 bits down to 2^-21 of the largest, and
// 2^-32 below.  The total is taken over the same weights and takes the factor out.
template <typename T>
constexpr float kLift = std::is_same<T, __half>::value ? 7.0f : 0.0f;
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <>
__device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// 16 bytes from global to shared memory, zeros where there is no source.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
               "r"(there ? 16 : 0)
               : "memory");
}

// Whether a session's rows of the call's tensors are there, and no more than
// the call said; else an error is recorded.
__device__ __forceinline__ bool rows_there(const AttendArgs& a, const SessionView& v, bool tell) {
  const bool fine = v.m <= a.batch.max_new && v.q0 >= 0 && v.q0 + v.m <= a.batch.tokens;
  if (tell && (!fine || v.first < 0 || (a.cache.ring_rows == 0 && v.first + v.m > a.cache.slots)))
    atomicOr(a.err, kDevErrIndex);
  return fine;
}

// A session's new tokens; what they see is left to narrow().
__device__ __forceinline__ SessionView session_rows(const AttendArgs& a, int s) {
  SessionView v;
  const BatchDev& b = a.batch;
  if (b.q_off) {
    v.q0 = __ldg(b.q_off + s);
    v.m = __ldg(b.q_off + s + 1) - static_cast<int32_t>(v.q0);
  } else {
    v.q0 = static_cast<int64_t>(s) * b.each;
    v.m = b.each;
  }
  v.first = __ldg(b.lens + s) - v.m;
  return v;
}
// And what they see together.
__device__ __forceinline__ SessionView session_view(const AttendArgs& a, int s) {
  SessionView v = session_rows(a, s);
  narrow(a, v, 0, v.m, 1);
  return v;
}

// Where a slot of session s is in the cache (of head 0): offsets of its key and
// value in units, kNoRow if it is in no page; where position p is.
constexpr uint32_t kNoRow = 0xffffffffu;
struct RowPlace {
  uint32_t k, v;
};
__device__ __forceinline__ RowPlace slot_place(const AttendArgs& a, int s, uint32_t slot) {
  const CacheDev& c = a.cache;
  RowPlace r = {kNoRow, kNoRow};
  if (slot >= static_cast<uint32_t>(c.slots)) {
    atomicOr(a.err, kDevErrIndex);
    return r;
  }
  const uint32_t page = c.page_rows.div(slot);
  const uint32_t row = (slot - page * c.page_rows.d) * c.row_units;
  const int64_t e = s * c.table_stride + page;
  const int32_t kp = __ldg(c.table + e);
  const int32_t vp = c.v_table ? __ldg(c.v_table + e) : kp;
  if (kp < 0 || kp >= c.n_pages || vp < 0 || vp >= c.n_pages) {
    if (kp < -1 || kp >= c.n_pages || vp < -1 || vp >= c.n_pages) atomicOr(a.err, kDevErrIndex);
    return r;
  }
  r.k = kp * c.page_units + row;
  r.v = vp * c.page_units + row;
  return r;
}
__device__ __forceinline__ RowPlace row_place(const AttendArgs& a, int s, int32_t p) {
  return slot_place(a, s, a.cache.slot_of(static_cast<uint32_t>(p)));
}
__device__ __forceinline__ const uint8_t* row_at(const AttendArgs& a, const uint8_t* base, uint32_t off) {
  return base + static_cast<uint64_t>(off) * a.cache.unit;
}

// The session that is the r-th longest (of equal ones, and of those beyond four million
// tokens, the first comes first), for blocks that take sessions in that order: the last
// blocks of a launch are then short ones.  `scratch` holds kRankMost numbers, free again
// when this returns to all threads.
__device__ __forceinline__ int ranked_session(const BatchDev& b, int r, int tid, int threads, uint32_t* scratch) {
  __shared__ int found;
  const int n = (b.sessions + 3) & ~3;
  for (int i = tid; i < n; i += threads) {
    const int32_t len = i < b.sessions ? __ldg(b.lens + i) : 0;
    scratch[i] = i < b.sessions ? static_cast<uint32_t>(min(max(len, 0), 0x3ffffe) + 1) << 9 | (kRankMost - 1 - i) : 0u;
  }
  __syncthreads();
  for (int i = tid; i < b.sessions; i += threads) {
    const uint32_t mine = scratch[i];
    int ahead = 0;
    for (int k = 0; k < n; k += 4) {
      const uint4 x = *reinterpret_cast<const uint4*>(scratch + k);
      ahead += (x.x > mine) + (x.y > mine) + (x.z > mine) + (x.w > mine);
    }
    if (ahead == r) found = i;
  }
  __syncthreads();
  return found;
}

// A session's nodes into shared memory, by the block's threads (at least
// PCS_TREE_MAX of them): their parents first, then a thread a node.  (A parent that is
// not there or not before its child counts as the context and is reported.)
__device__ __forceinline__ void tree_nodes(const AttendArgs& a, const SessionView& v, int tid, TreeNode* nodes) {
  __shared__ int32_t parents[PCS_TREE_MAX];
  const int m = min(v.m, PCS_TREE_MAX);
  if (tid < m) {
    const int32_t p = __ldg(a.parent + v.q0 + tid);
    const bool fine = p >= -1 && p < tid;
    if (!fine) atomicOr(a.err, kDevErrIndex);
    parents[tid] = fine ? p : -1;
  }
  __syncthreads();
  if (tid < m) nodes[tid] = tree_node(a, v.first, [&](int k) { return parents[k]; }, tid);
}

// Whether some of eight elements are infinite or NaN: the lowest bit of an
// exponent added to one of all ones carries into the sign's place.
template <typename T>
__device__ __forceinline__ bool has_specials(const uint4& v) {
  constexpr uint32_t e = std::is_same<T, __half>::value ? 0x7c007c00u : 0x7f807f80u;
  constexpr uint32_t one = std::is_same<T, __half>::value ? 0x04000400u : 0x00800080u;
  return ((((v.x & e) + one) | ((v.y & e) + one) | ((v.z & e) + one) | ((v.w & e) + one)) & 0x80008000u) != 0;
}

// ---- Barriers in shared memory, boxes of rows ---------------------------------------------

constexpr long long kWaitCycles = 4000000000ll;
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait for the phase of the given parity; false: it gave up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  if (bar_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try(bar, parity))
    if (clock64() - t0 > kWaitCycles) return false;
  return true;
}

// A box of rows: pages of its keys and values as the table has them, the first
// row in them.  The page ids are on their way from memory until settle().
struct Box {
  int32_t k, v, row;
};
// The box at place e of a view.
__device__ __forceinline__ Box box_place(const AttendArgs& a, int s, const SessionView& w, int32_t e) {
  const CacheDev& c = a.cache;
  const uint32_t slot = box_slot(a, w, e);
  if (slot >= static_cast<uint32_t>(c.slots)) {
    atomicOr(a.err, kDevErrIndex);
    return {-1, -1, 0};
  }
  const uint32_t page = c.page_rows.div(slot);
  const int64_t at = s * c.table_stride + page;
  Box x;
  x.k = __ldg(c.table + at);
  x.v = __ldg((c.v_table ? c.v_table : c.table) + at);
  x.row = slot - page * c.page_rows.d;
  return x;
}
// Page n_pages, whose rows come out as zeros, for what is not in the cache.
__device__ __forceinline__ void settle(const AttendArgs& a, Box& x) {
  const int32_t n = a.cache.n_pages;
  if (x.k < 0 || x.k >= n || x.v < 0 || x.v >= n) {
    if (x.k < -1 || x.k >= n || x.v < -1 || x.v >= n) atomicOr(a.err, kDevErrIndex);
    x.k = x.v = n;
  }
}

}  // namespace pcs

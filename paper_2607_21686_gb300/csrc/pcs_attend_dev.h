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

// Where position p of session s is in the cache (of head 0): offsets of its
// key and value in units, kNoRow if it is in no page.
constexpr uint32_t kNoRow = 0xffffffffu;
struct RowPlace {
  uint32_t k, v;
};
__device__ __forceinline__ RowPlace row_place(const AttendArgs& a, int s, int32_t p) {
  const CacheDev& c = a.cache;
  RowPlace r = {kNoRow, kNoRow};
  const uint32_t slot = c.slot_of(static_cast<uint32_t>(p));
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
__device__ __forceinline__ const uint8_t* row_at(const AttendArgs& a, const uint8_t* base, uint32_t off) {
  return base + static_cast<uint64_t>(off) * a.cache.unit;
}

}  // namespace pcs

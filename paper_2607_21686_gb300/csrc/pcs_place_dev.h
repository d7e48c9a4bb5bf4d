// pcs_place_dev.h -- device code that finds the rows of the cache that a call's
// tokens lie in, for the kernels that write or read them token by token.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "pcs_attend.h"
#include "pcs_internal.h"

namespace pcs {

// Where a token's row of the cache is: byte offsets, or -1.
struct Place {
  int64_t k, v;
};

// The last of the sessions whose first token is at most t, by one warp: 32
// probes at a time.
__device__ __forceinline__ int session_of(const BatchDev& b, int64_t t, int lane) {
  int lo = 0, n = b.sessions;  // it is among [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int i = lo + lane * step;
    const unsigned m = __ballot_sync(0xffffffffu, lane * step < n && __ldg(b.q_off + i) <= t);
    const int k = m ? 31 - __clz(m) : 0;
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// Of row t of a call, of a session from s on; what is wrong with it goes to err.
__device__ __forceinline__ Place place_of(const CacheDev& c, const BatchDev& b, uint32_t* err, int64_t t, int s) {
  int at, m;
  if (b.q_off) {
    int32_t o = __ldg(b.q_off + s), end = __ldg(b.q_off + s + 1);
    while (t >= end && s + 1 < b.sessions) {
      ++s;
      o = end;
      end = __ldg(b.q_off + s + 1);
    }
    m = end - o;
    at = static_cast<int>(t - o);
    if (at < 0 || at >= m) return {-1, -1};
  } else {
    s = static_cast<int>(t / b.each);
    m = b.each;
    at = static_cast<int>(t - static_cast<int64_t>(s) * m);
  }
  const int64_t len = __ldg(b.lens + s), p = len - m + at;
  if (p < 0) {
    atomicOr(err, kDevErrIndex);
    return {-1, -1};
  }
  if (c.ring_rows && p >= c.sinks && p < len - c.ring_rows) return {-1, -1};
  const uint32_t slot = c.slot_of(static_cast<uint32_t>(p));
  if (slot >= static_cast<uint32_t>(c.slots)) {
    atomicOr(err, kDevErrIndex);
    return {-1, -1};
  }
  const uint32_t page = c.page_rows.div(slot);
  const int64_t row = static_cast<int64_t>(slot - page * c.page_rows.d) * c.row_bytes;
  const int64_t e = s * c.table_stride + page;
  const int32_t kp = __ldg(c.table + e);
  const int32_t vp = c.v_table ? __ldg(c.v_table + e) : kp;
  if (kp < 0 || kp >= c.n_pages || vp < 0 || vp >= c.n_pages) {  // neither of them is written
    if (kp < -1 || kp >= c.n_pages || vp < -1 || vp >= c.n_pages) atomicOr(err, kDevErrIndex);
    return {-1, -1};
  }
  return {kp * c.page_bytes + row, vp * c.page_bytes + row};
}

}  // namespace pcs

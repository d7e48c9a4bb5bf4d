// pcs_attend_view.h -- what the new tokens of a call see of their sessions: the
// places of the tokens they see together, and which of them each one sees.
// Arithmetic alone, for the kernels and for checks on the host.
#pragma once

#include <cstdint>

#include "pcs_attend.h"

namespace pcs {

__host__ __device__ __forceinline__ int32_t larger(int32_t x, int32_t y) { return x > y ? x : y; }
__host__ __device__ __forceinline__ int32_t smaller(int32_t x, int32_t y) { return x < y ? x : y; }

// The new tokens of a session, and the places of what some of them see together:
// [0, pad) the first `sinks` tokens (the last places are nobody's), then from
// position `lo` on; not apart, one run from position 0.
// Copies of whole boxes of `align` rows need a place's distance from its slot to
// be a multiple of align.  So the run begins at such a position, and where it
// goes over the end of a ring (position `wrap` has slot `sinks` again) the places
// [gap0, gap1) are nobody's.  With align 1 there is no gap (wrap: none).
struct SessionView {
  int64_t q0;       // the first new token's row
  int32_t m;        // new tokens
  int32_t first;    // position of the first one (negative: before the session)
  int32_t sinks, pad, lo, seen;
  int32_t slot;     // of place `pad`
  int32_t wrap, gap0, gap1;
  bool apart;
  __host__ __device__ __forceinline__ int32_t place(int32_t p) const { return p >= wrap ? gap1 + (p - wrap) : pad + (p - lo); }
};
constexpr int32_t kNever = 0x7fffffff;

// Narrows a view to what new tokens [t0, t1) see.
__host__ __device__ __forceinline__ void narrow(const AttendArgs& a, SessionView& v, int t0, int t1, int align) {
  const CacheDev& c = a.cache;
  const int32_t len = v.first + v.m;
  int32_t lo = a.window ? v.first + t0 - a.window + 1 : 0;
  if (c.ring_rows) lo = larger(lo, len - c.ring_rows);
  // (A session longer than its table sees what the table has room for.)
  const int32_t end = smaller(larger(v.first + t1, 0), c.ring_rows ? kNever : c.slots);
  v.apart = lo > c.sinks;
  v.sinks = v.apart ? smaller(c.sinks, end) : 0;
  v.pad = (v.sinks + align - 1) & -align;
  v.wrap = v.gap0 = v.gap1 = kNever;
  v.slot = 0;
  if (!v.apart) {
    v.lo = 0;
  } else if (align == 1) {
    v.lo = lo;
  } else {
    const int32_t slot = c.slot_of(lo);
    v.slot = slot & -align;
    v.lo = lo - (slot - v.slot);
    // (Differences, not positions: those may end at 2^31 - 1.)
    const int32_t left = c.sinks + c.ring_rows - slot;
    if (c.ring_rows && left < end - lo) {
      v.wrap = lo + left;
      v.gap0 = v.pad + (v.wrap - v.lo);
      v.gap1 = ((v.gap0 + align - 1) & -align) + (c.sinks & (align - 1));
    }
  }
  // (Rows that a ring has left behind see first tokens alone; those of one run
  // are places of it.)
  v.seen = end > (v.apart ? lo : 0) ? v.place(end - 1) + 1 : v.pad;
}

// Position of place e of a view, of a place that is somebody's.
__host__ __device__ __forceinline__ int32_t seen_position(const SessionView& v, int32_t e) {
  return e < v.pad ? e : e >= v.gap1 ? v.wrap + (e - v.gap1) : v.lo + (e - v.pad);
}

// The slot of place e of a view whose boxes are copied whole, e a box's first.
__host__ __device__ __forceinline__ uint32_t box_slot(const AttendArgs& a, const SessionView& w, int32_t e) {
  return e < w.pad ? e : e >= w.gap0 ? a.cache.sinks + (e - w.gap1) : w.slot + (e - w.pad);
}

// What a row at position p sees of a view's tokens: e with e <= hi and (e <
// first or e >= lo).
struct RowRange {
  int32_t hi, lo, first;
  // The tokens [b, b + 32) it sees, as bits.
  __host__ __device__ __forceinline__ uint32_t bits(int32_t b) const {
    return upto(hi + 1 - b) & (upto(first - b) | ~upto(lo - b));
  }
  static __host__ __device__ __forceinline__ uint32_t upto(int32_t n) {
    return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1;
  }
};
__host__ __device__ __forceinline__ RowRange row_range(const AttendArgs& a, const SessionView& v, int32_t p) {
  int32_t low = a.window ? larger(p - a.window + 1, 0) : 0;
  if (a.cache.ring_rows) low = larger(low, v.first + v.m - a.cache.ring_rows);
  RowRange r;
  // (A run of boxes may begin below `sinks`: a row of a first token sees no
  // further than itself all the same.)
  r.hi = p >= v.lo && !(v.apart && p < v.sinks) ? v.place(p) : smaller(p, v.pad - 1);
  r.first = v.apart ? v.sinks : a.cache.sinks;
  r.lo = v.apart ? v.place(larger(low, v.lo)) : larger(low, 0);
  return r;
}

// What the rows of a block or of a row tile see, at positions [pmin, pmax], in
// tiles: they all see all of tiles [.., all_to) from all_from on, or before
// all_first; some of them see some of tiles [.., some_to] from some_from on, or
// before some_first; tiles [gap_from, gap_to) have places that are nobody's.
struct RowsRange {
  int32_t all_to, all_from, all_first, some_to, some_from, some_first, gap_from, gap_to;
  // They all see all tokens of tile t that are in the cache.
  __host__ __device__ __forceinline__ bool whole(int t) const { return t < all_to && (t >= all_from || t < all_first); }
  __host__ __device__ __forceinline__ bool whole_and_filled(int t) const { return whole(t) && (t < gap_from || t >= gap_to); }
  // Some row sees some token of it.
  __host__ __device__ __forceinline__ bool some(int t) const { return t <= some_to && (t >= some_from || t < some_first); }
};
__host__ __device__ __forceinline__ RowsRange rows_range(const AttendArgs& a, const SessionView& v, int pmin, int pmax) {
  static_assert(kBlockTile == 128, "shifts");
  const RowRange x = row_range(a, v, pmin), y = row_range(a, v, pmax);
  return {(x.hi + 1) >> 7, static_cast<int32_t>((static_cast<uint32_t>(y.lo) + 127) >> 7), x.first >> 7, y.hi >> 7, x.lo >> 7,
          static_cast<int32_t>((static_cast<uint32_t>(x.first) + 127) >> 7), v.gap0 >> 7,
          static_cast<int32_t>((static_cast<uint32_t>(v.gap1) + 127) >> 7)};
}

// ---- Trees ---------------------------------------------------------------------------
// The new tokens of a session are nodes: node i lies where the new token i does, at
// place(first + i), but its position is first + depth.

// Of one node: those new tokens that it sees (itself, its ancestors), as bits.
struct TreeNode {
  uint64_t line;
  int32_t depth;
};

// `up`: the parents of a session's nodes, each -1 or smaller than its child.
template <typename Up>
__host__ __device__ __forceinline__ TreeNode tree_node(const AttendArgs& a, int32_t first, const Up& up, int i) {
  TreeNode n = {0, 0};
  for (int k = up(i); k >= 0; k = up(k)) ++n.depth;
  int behind = 0;  // positions from the ancestor on
  for (int k = i; k >= 0; k = up(k), ++behind)
    if (a.window == 0 || behind < a.window || first + n.depth - behind < a.cache.sinks) n.line |= 1ull << k;
  return n;
}

// The last place of the context (the tokens before the new ones); -1 or the last of
// the first tokens' places where it has none else.
__host__ __device__ __forceinline__ int32_t context_end(const SessionView& v) {
  const int32_t p = v.first - 1;
  return p >= v.lo && !(v.apart && p < v.sinks) ? v.place(p) : smaller(p, v.pad - 1);
}

// What a node sees of a view's tokens: a range of the context, and some new tokens,
// node k at place base + k, from `split` on (behind the end of a ring) at base2 + k.
struct TreeRow {
  RowRange context;
  uint64_t line;
  int32_t base, split, base2;
  static __host__ __device__ __forceinline__ uint32_t moved(uint64_t x, int32_t by) {
    return by >= 32 || by <= -64 ? 0u : by >= 0 ? static_cast<uint32_t>(x << by) : static_cast<uint32_t>(x >> -by);
  }
  // The tokens [b, b + 32) it sees, as bits.
  __host__ __device__ __forceinline__ uint32_t bits(int32_t b) const {
    const uint64_t low = split >= 64 ? ~0ull : (1ull << split) - 1;
    return context.bits(b) | moved(line & low, base - b) | moved(line & ~low, base2 - b);
  }
};
__host__ __device__ __forceinline__ TreeRow tree_row(const AttendArgs& a, const SessionView& v, const TreeNode& n) {
  TreeRow r;
  r.context = row_range(a, v, v.first + n.depth);
  r.context.hi = context_end(v);
  r.line = n.line;
  r.base = v.place(v.first);  // (below 0 for a session shorter than its new tokens: one run from place 0)
  r.split = 64;
  r.base2 = 0;
  if (v.wrap != kNever && v.wrap > v.first && v.wrap - v.first < 64) {
    r.split = v.wrap - v.first;
    r.base2 = v.gap1 - r.split;
  }
  return r;
}

// Of all nodes up to number t1, as rows_range has it; depths are not looked at: the
// deepest one may be anywhere up to t1.
__host__ __device__ __forceinline__ RowsRange tree_rows_range(const AttendArgs& a, const SessionView& v, int t1) {
  RowsRange r = rows_range(a, v, v.first, v.first + t1);
  r.all_to = (context_end(v) + 1) >> 7;
  return r;
}

}  // namespace pcs

// Checks of what a call's new tokens see (csrc/pcs_attend_view.h), run on the
// host: for random sessions, rings, first tokens, windows and boxes, every place
// that a row's masks let through has to be a token that it sees, in that token's
// slot, and every token that it sees has to be there once.
// Usage: view_check <seed> <geometries> <kind>
//          kind 0: sizes of a few tiles; 1: new tokens that lap the ring; 2: lengths up to 2^31 - 1
//        view_check <sinks> <ring> <window> <length> <new> <rows of a box> <group> <spare boxes>
// prints "ok" or the first failure.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "pcs_attend_view.h"

using namespace pcs;

namespace {

uint64_t state = 1;
uint32_t draw() {
  state = state * 6364136223846793005ull + 1442695040888963407ull;
  return static_cast<uint32_t>(state >> 33);
}
int32_t upto(int32_t n) { return static_cast<int32_t>(draw() % (static_cast<uint32_t>(n) + 1)); }

// The definition: the positions that the token at p of a session of n sees.
std::vector<int64_t> definition(const AttendArgs& a, int64_t n, int64_t p) {
  const int64_t sinks = a.cache.sinks, ring = a.cache.ring_rows, window = a.window;
  std::vector<int64_t> seen;
  auto there = [&](int64_t j) {
    if (j < 0 || j > p || j >= n) return false;
    if (window && j >= sinks && j <= p - window) return false;
    if (ring && j >= sinks && j < n - ring) return false;
    return ring || j < a.cache.slots;
  };
  int64_t from = 0;
  if (window) from = std::max(from, p - window);
  if (ring) from = std::max(from, n - ring);
  for (int64_t j = 0; j < std::min(sinks, from); ++j)
    if (there(j)) seen.push_back(j);
  for (int64_t j = std::max<int64_t>(from, 0); j <= p; ++j)
    if (there(j)) seen.push_back(j);
  return seen;
}

struct Checker {
  AttendArgs a = {};
  int align = 1, group = 1;
  int64_t len = 0;
  SessionView v;

  bool fail(const char* what, int64_t p, int64_t e) const {
    std::printf("%s: sinks %d ring %d window %d slots %d length %lld first %d new %d boxes of %d group %d, position %lld, place %lld\n",
                what, a.cache.sinks, a.cache.ring_rows, a.window, a.cache.slots, static_cast<long long>(len), v.first, v.m,
                align, group, static_cast<long long>(p), static_cast<long long>(e));
    return false;
  }
  // A place that is copied and is some token's.
  bool filled(int32_t e) const { return e / align * align < v.seen && !(e >= v.gap0 && e < v.gap1); }

  bool row(int32_t p) const {
    const RowRange r = row_range(a, v, p);
    std::vector<int64_t> got;
    const int32_t n = (v.seen + 127) / 128 * 128;
    for (int32_t b = 0; b < n; b += 32) {
      const uint32_t bits = r.bits(b);
      for (int32_t e = b; e < b + 32; ++e) {
        if (!(bits >> (e - b) & 1) || !filled(e)) continue;
        if (align > 1 && e >= v.seen) return fail("behind what is seen", p, e);
        const int32_t j = seen_position(v, e);
        const uint32_t slot = align > 1 ? box_slot(a, v, e / align * align) + e % align : a.cache.slot_of(j);
        if (slot != a.cache.slot_of(j) || slot >= static_cast<uint32_t>(a.cache.slots)) return fail("another slot", p, e);
        got.push_back(j);
      }
    }
    std::sort(got.begin(), got.end());
    const std::vector<int64_t> want = definition(a, len, p);
    if (got == want) return true;
    for (size_t i = 0; i < std::max(got.size(), want.size()); ++i)
      if (i >= got.size() || i >= want.size() || got[i] != want[i])
        return fail(i < want.size() && (i >= got.size() || want[i] < got[i]) ? "not seen" : "seen ahead or too long", p,
                    i < got.size() ? got[i] : -1);
    return true;
  }

  // Tiles that all or some of rows at [pmin, pmax] see, against their masks.
  bool tiles(int32_t pmin, int32_t pmax) const {
    const RowsRange range = rows_range(a, v, pmin, pmax);
    for (int32_t t = 0; t < (v.seen + 127) / 128; ++t) {
      bool all = true, some = false;
      for (int32_t p = pmin; p <= pmax; ++p) {
        const RowRange r = row_range(a, v, p);
        for (int k = 0; k < 4; ++k) {
          const uint32_t bits = r.bits(t * 128 + k * 32);
          all = all && bits == 0xffffffffu;
          some = some || bits != 0;
        }
      }
      bool gap = false;
      for (int32_t e = t * 128; e < (t + 1) * 128; ++e) gap = gap || (e >= v.gap0 && e < v.gap1);
      if (range.whole(t) && !all) return fail("a tile said to be whole", pmin, t * 128);
      if (range.whole_and_filled(t) && gap) return fail("a tile said to be filled", pmin, t * 128);
      if (some && !range.some(t)) return fail("a tile left out", pmin, t * 128);
    }
    return true;
  }

  // Rows [r0, r1) of the session and key head.
  bool block(const SessionView& all, int64_t r0, int64_t r1) {
    const int32_t t0 = static_cast<int32_t>(r0 / group), t1 = static_cast<int32_t>((r1 - 1) / group);
    v = all;
    narrow(a, v, t0, t1 + 1, align);
    for (int32_t t = t0; t <= t1; ++t)
      if (t == t0 || t == t1 || t1 - t0 < 12 || draw() % 16 == 0 || std::abs(v.first + t - a.cache.sinks) < 3)
        if (!row(v.first + t)) return false;
    if (!tiles(v.first + t0, v.first + t1)) return false;
    for (int64_t q = r0; q < r1; q += 128)
      if (!tiles(v.first + static_cast<int32_t>(q / group), v.first + static_cast<int32_t>((std::min(q + 128, r1) - 1) / group)))
        return false;
    return true;
  }
};

// A session of `len` tokens, the last m of them new; its table has `spare` boxes
// more than it needs.
bool session(Checker& c, int32_t len, int32_t m, int32_t rows, int32_t spare) {
  CacheDev& d = c.a.cache;
  if (d.ring_rows) d.ring.set(d.ring_rows);
  d.slots = (rows + c.align - 1) / c.align * c.align + c.align * spare;
  c.len = len;
  SessionView all = {};
  all.m = m;
  all.first = len - m;
  const int64_t count = static_cast<int64_t>(m) * c.group;
  // The whole session at once, as a few rows are taken; in blocks, all or some.
  if (c.align == 1 && !c.block(all, 0, count)) return false;
  const int64_t blocks = (count + kBlockRows - 1) / kBlockRows;
  for (int64_t b = 0; b < blocks; ++b)
    if (b < 3 || b + 3 > blocks || draw() % 4 == 0)
      if (!c.block(all, b * kBlockRows, std::min<int64_t>((b + 1) * kBlockRows, count))) return false;
  return true;
}

}  // namespace

int main(int argc, char** argv) {
  if (argc == 9) {
    int v[8];
    for (int i = 1; i < 9; ++i) v[i - 1] = std::atoi(argv[i]);
    Checker c;
    c.a.cache.sinks = v[0], c.a.cache.ring_rows = v[1], c.a.window = v[2];
    c.align = v[5], c.group = v[6];
    if (!session(c, v[3], v[4], v[1] ? v[0] + v[1] : v[3], v[7])) return 1;
    std::puts("ok");
    return 0;
  }
  if (argc != 4) return 2;
  state = std::strtoull(argv[1], nullptr, 10) * 7919 + 1;
  const int n = std::atoi(argv[2]), kind = std::atoi(argv[3]);
  for (int i = 0; i < n; ++i) {
    Checker c;
    c.align = 1 << (draw() % 6 ? 3 + draw() % 5 : 0);
    const int32_t groups[] = {1, 1, 2, 4, 5, 40, 64};
    c.group = groups[draw() % 7];
    CacheDev& d = c.a.cache;
    d.sinks = draw() % 3 ? upto(draw() % 2 ? 20 : 700) : 0;
    const bool ring = kind || draw() % 3;
    d.ring_rows = ring ? 1 + upto(draw() % 2 ? 100 : 900) : 0;
    c.a.window = draw() % 2 ? 1 + upto(draw() % 2 ? 40 : 800) : 0;
    int32_t len, m;
    if (kind == 2) {
      len = 0x7fffffff - upto(1 << (draw() % 12));
      m = 1 + upto(600);
    } else if (kind == 1) {  // and lengths around sinks + ring
      len = std::max(1, d.sinks + d.ring_rows - 5 + upto(draw() % 2 ? 20 : 1200));
      m = draw() % 2 ? len : 1 + upto(len - 1);
    } else {
      len = 1 + upto(1800);
      m = 1 + upto(draw() % 2 ? std::min(len, 300) - 1 : len - 1);
    }
    const int32_t rows = ring ? d.sinks + d.ring_rows : draw() % 8 ? len : std::max(1, len - upto(200));
    if (!session(c, len, m, rows, upto(2))) return 1;
  }
  std::puts("ok");
}

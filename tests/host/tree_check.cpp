// Checks of what the nodes of a tree of new tokens see (csrc/pcs_attend_view.h), run
// on the host: for random trees, sessions, rings, first tokens, windows and boxes,
// every place that a node's masks let through has to be a token that it sees, in that
// token's slot, and every token that it sees has to be there once.
// Usage: tree_check <seed> <geometries> <kind>    kind 0: sizes of a few tiles; 1: lengths up to 2^31 - 1
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

struct Session {
  AttendArgs a = {};
  int align = 1, group = 1;
  int64_t len = 0;
  SessionView v;
  std::vector<int32_t> parent;

  bool fail(const char* what, int64_t i, int64_t e) const {
    std::printf("%s: sinks %d ring %d window %d slots %d length %lld first %d new %d boxes of %d group %d, node %lld, place %lld\n",
                what, a.cache.sinks, a.cache.ring_rows, a.window, a.cache.slots, static_cast<long long>(len), v.first, v.m,
                align, group, static_cast<long long>(i), static_cast<long long>(e));
    return false;
  }
  TreeNode node(int i) const {
    return tree_node(a, v.first, [&](int k) { return parent[k]; }, i);
  }

  // The definition: slots' positions that node i sees.
  std::vector<int64_t> definition(int i) const {
    const int64_t sinks = a.cache.sinks, ring = a.cache.ring_rows, window = a.window, first = v.first;
    std::vector<int> line;
    for (int k = i; k >= 0; k = parent[k]) line.push_back(k);
    const int64_t pos = first + static_cast<int64_t>(line.size()) - 1;
    std::vector<int64_t> seen;
    auto there = [&](int64_t j) {
      if (j < 0 || j >= len) return false;
      if (ring && j >= sinks && j < len - ring) return false;
      return ring || j < a.cache.slots;
    };
    auto near = [&](int64_t p) { return !window || p > pos - window || p < sinks; };
    const int64_t from = std::max<int64_t>(0, first - (ring ? ring : first) - (window ? window : 0) - 70);
    for (int64_t j = 0; j < std::min(sinks, first); ++j)
      if (there(j) && near(j)) seen.push_back(j);
    for (int64_t j = std::max(std::min(sinks, first), from); j < first; ++j)
      if (there(j) && near(j)) seen.push_back(j);
    for (size_t k = 0; k < line.size(); ++k)
      if (there(first + line[k]) && near(pos - static_cast<int64_t>(k))) seen.push_back(first + line[k]);
    std::sort(seen.begin(), seen.end());
    return seen;
  }
  bool filled(int32_t e) const { return e / align * align < v.seen && !(e >= v.gap0 && e < v.gap1); }

  bool row(int i) const {
    const TreeRow r = tree_row(a, v, node(i));
    std::vector<int64_t> got;
    for (int32_t b = 0; b < (v.seen + 127) / 128 * 128; b += 32) {
      const uint32_t bits = r.bits(b);
      for (int32_t e = b; e < b + 32; ++e) {
        if (!(bits >> (e - b) & 1) || !filled(e)) continue;
        if (align > 1 && e >= v.seen) return fail("behind what is seen", i, e);
        const int32_t j = seen_position(v, e);
        const uint32_t slot = align > 1 ? box_slot(a, v, e / align * align) + e % align : a.cache.slot_of(j);
        if (slot != a.cache.slot_of(j) || slot >= static_cast<uint32_t>(a.cache.slots)) return fail("another slot", i, e);
        got.push_back(j);
      }
    }
    std::sort(got.begin(), got.end());
    const std::vector<int64_t> want = definition(i);
    if (got == want) return true;
    for (size_t k = 0; k < std::max(got.size(), want.size()); ++k)
      if (k >= got.size() || k >= want.size() || got[k] != want[k])
        return fail(k < want.size() && (k >= got.size() || want[k] < got[k]) ? "not seen" : "seen but not its own", i,
                    k < got.size() ? got[k] : -1);
    return true;
  }

  // Tiles that all or some of nodes [t0, t1] see, against their masks.
  bool tiles(int t0, int t1) const {
    const RowsRange range = tree_rows_range(a, v, t1);
    for (int32_t t = 0; t < (v.seen + 127) / 128; ++t) {
      bool all = true, some = false;
      for (int i = t0; i <= t1; ++i) {
        const TreeRow r = tree_row(a, v, node(i));
        for (int k = 0; k < 4; ++k) {
          const uint32_t bits = r.bits(t * 128 + k * 32);
          all = all && bits == 0xffffffffu;
          some = some || bits != 0;
        }
      }
      bool gap = false;
      for (int32_t e = t * 128; e < (t + 1) * 128; ++e) gap = gap || (e >= v.gap0 && e < v.gap1);
      if (range.whole(t) && !all) return fail("a tile said to be whole", t0, t * 128);
      if (range.whole_and_filled(t) && gap) return fail("a tile said to be filled", t0, t * 128);
      if (some && !range.some(t)) return fail("a tile left out", t0, t * 128);
    }
    return true;
  }

  bool block(const SessionView& all, int t0, int t1) {
    v = all;
    narrow(a, v, 0, t1 + 1, align);
    for (int i = t0; i <= t1; ++i)
      if (!row(i)) return false;
    return tiles(t0, t1);
  }
};

}  // namespace

int main(int argc, char** argv) {
  if (argc != 4) return 2;
  state = std::strtoull(argv[1], nullptr, 10) * 7919 + 1;
  const int n = std::atoi(argv[2]), kind = std::atoi(argv[3]);
  for (int g = 0; g < n; ++g) {
    Session c;
    c.align = 1 << (draw() % 4 ? 3 + draw() % 5 : 0);
    const int32_t groups[] = {1, 2, 4, 5, 8, 40};
    c.group = groups[draw() % 6];
    CacheDev& d = c.a.cache;
    const int32_t m = 1 + upto(63);
    d.sinks = draw() % 3 ? upto(draw() % 2 ? 20 : 500) : 0;
    d.ring_rows = kind || draw() % 2 ? m + upto(draw() % 2 ? 60 : 700) : 0;
    c.a.window = draw() % 2 ? 1 + upto(draw() % 2 ? 40 : 600) : 0;
    c.len = kind ? 0x7fffffff - upto(1 << (draw() % 12)) : m + upto(draw() % 3 ? 1500 : 30);
    if (!kind && draw() % 20 == 0) c.len = upto(m);  // shorter than its new tokens
    const int64_t rows = d.ring_rows ? d.sinks + d.ring_rows : draw() % 8 ? c.len : std::max<int64_t>(1, c.len - upto(100));
    if (d.ring_rows) d.ring.set(d.ring_rows);
    d.slots = static_cast<int32_t>((rows + c.align - 1) / c.align * c.align + c.align * upto(2));
    c.parent.resize(m);
    for (int i = 0; i < m; ++i) c.parent[i] = draw() % 2 ? i - 1 : upto(i) - 1;
    SessionView all = {};
    all.m = m;
    all.first = static_cast<int32_t>(c.len - m);
    if (c.align == 1 && !c.block(all, 0, m - 1)) return 1;
    for (int64_t r = 0; r < static_cast<int64_t>(m) * c.group; r += kBlockRows)
      if (!c.block(all, static_cast<int>(r / c.group),
                   static_cast<int>((std::min<int64_t>(r + kBlockRows, static_cast<int64_t>(m) * c.group) - 1) / c.group)))
        return 1;
  }
  std::puts("ok");
}

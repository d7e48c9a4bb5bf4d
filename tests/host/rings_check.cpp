// Check of what warps that send copies wait for before they end
// (csrc/pcs_attend_rounds.h): barriers of two phases told apart by parity, as the
// kernel has them.  After n fills, wherever the warps stopped, the waits return
// once all copies have landed, and not before.  And of the barriers' numbers.  Prints "ok" or the first failure.
#include <cstdio>
#include <vector>

#include "pcs_attend_rounds.h"

namespace {

template <int KEYS, int VALUES>
bool run(int step, int c, int sent) {
  using R = pcs::Rings<KEYS, VALUES>;
  // The warp's fills c, c + step, .. below `sent`; each buffer's, in order.
  std::vector<int> newest(KEYS + VALUES, -1), times(KEYS + VALUES, 0);
  int n = c;
  for (; n < sent; n += step) {
    if (R::use(n) != times[R::buffer(n)]) return false;
    newest[R::buffer(n)] = n;
    times[R::buffer(n)] += 1;
  }
  // A barrier whose phase x is in progress lets a wait for parity p through
  // where x and p differ in parity.
  for (int late = -1; late < KEYS + VALUES; ++late) {  // the buffer whose last copy has not landed
    if (late >= 0 && newest[late] < 0) continue;
    int waits = 0;
    const bool over = R::drain(c, step, n, [&](int i) {
      const int b = R::buffer(i), phase = times[b] - (b == late);
      ++waits;
      return ((phase ^ R::use(i)) & 1) != 0;
    });
    if (over != (late < 0) || waits > KEYS + VALUES) {
      std::printf("rings of %d and %d, step %d from %d, %d sent: buffer %d late, %d waits, %s\n", KEYS, VALUES, step, c, sent,
                  late, waits, over ? "over" : "not over");
      return false;
    }
  }
  return true;
}

template <int KEYS, int VALUES>
bool all() {
  for (int sent = 0; sent < 60; ++sent)
    if (!run<KEYS, VALUES>(1, 0, sent) || !run<KEYS, VALUES>(2, 0, sent) || !run<KEYS, VALUES>(2, 1, sent)) return false;
  return true;
}

// Every barrier is made once, and each name has one of its own.
template <int KEYS, int VALUES, bool LOOK>
bool barriers() {
  using B = pcs::Barriers<KEYS, VALUES, LOOK>;
  std::vector<int> made(B::kCount, 0), named(B::kCount, 0);
  bool fine = true;
  B::each(128, 256, 1, 64, [&](int i, int count) {
    if (i < 0 || i >= B::kCount || count < 1) fine = false;
    else made[i] += 1;
  });
  named[B::q_full()] += 1;
  named[B::drained()] += 1;
  for (int t = 0; t < 2; ++t)
    for (int i : {B::s_full(t), B::s_read(t), B::p_full(t), B::o_full(t)}) named[i] += 1;
  for (int i = 0; i < KEYS + VALUES; ++i) named[B::kv_full(i)] += 1, named[B::kv_empty(i)] += 1;
  for (int j = 0; LOOK && j < 3 * VALUES; ++j) named[B::v_fine(j)] += j < VALUES;
  for (int i = 0; i < B::kCount; ++i) fine = fine && made[i] == 1 && named[i] == 1;
  if (!fine) std::printf("barriers of rings of %d and %d are not made once each\n", KEYS, VALUES);
  return fine;
}

}  // namespace

int main() {
  if (!barriers<4, 4, true>() || !barriers<2, 3, true>() || !barriers<2, 2, false>() || !barriers<4, 4, false>()) return 1;
  if (!all<4, 4>() || !all<2, 3>() || !all<2, 2>() || !all<3, 2>()) return 1;
  std::puts("ok");
}

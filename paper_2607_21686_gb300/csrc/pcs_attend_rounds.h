// pcs_attend_rounds.h -- the rings of keys and values that warps fill: which
// buffer a fill goes to, what is waited for at the end, and how warps that fill
// one together give up.  Arithmetic and control flow alone, for the block kernel
// and for checks on the host.
#pragma once

#ifdef __CUDACC__
#define PCS_ROUNDS __device__ __forceinline__
#else
#define PCS_ROUNDS inline
#endif

namespace pcs {

// Fill i: keys of tile i / 2 (even), or its values; each has a ring of buffers.
template <int KEYS, int VALUES>
struct Rings {
  static PCS_ROUNDS constexpr int buffer(int i) { return i & 1 ? KEYS + (i >> 1) % VALUES : (i >> 1) % KEYS; }
  // How often its buffer has been filled before.
  static PCS_ROUNDS constexpr int use(int i) { return i & 1 ? (i >> 1) / VALUES : (i >> 1) / KEYS; }
  // A warp that sent fills c, c + step, .. below n waits for those that may still
  // be on their way: the last one of each buffer, for the ones before it had been
  // used by then.  Whether all of them came.
  template <typename Wait>
  static PCS_ROUNDS bool drain(int c, int step, int n, Wait&& wait) {
    bool ok = true;
#ifdef __CUDACC__
#pragma unroll 1
#endif
    for (int i = c; i < n; i += step)
      if (i + 2 * (i & 1 ? VALUES : KEYS) >= n) ok = ok && wait(i);
    return ok;
  }
};

// The block kernel's barriers, by number: of a ring's buffers (filled, free), of
// query rows, of row tiles' scores (made, in registers), weights and sums, of
// values that have been looked over (LOOK) and of the end.
template <int KEYS, int VALUES, bool LOOK>
struct Barriers {
  static constexpr int kRing = KEYS + VALUES;
  static constexpr int kCount = 10 + 2 * kRing + (LOOK ? VALUES : 0);
  static PCS_ROUNDS constexpr int q_full() { return 0; }
  static PCS_ROUNDS constexpr int drained() { return 1; }
  static PCS_ROUNDS constexpr int s_full(int t) { return 2 + t; }
  static PCS_ROUNDS constexpr int s_read(int t) { return 4 + t; }
  static PCS_ROUNDS constexpr int p_full(int t) { return 6 + t; }
  static PCS_ROUNDS constexpr int o_full(int t) { return 8 + t; }
  static PCS_ROUNDS constexpr int kv_full(int i) { return 10 + i; }
  static PCS_ROUNDS constexpr int kv_empty(int i) { return 10 + kRing + i; }
  static PCS_ROUNDS constexpr int v_fine(int j) { return 10 + 2 * kRing + j % VALUES; }
  // Each of them once, with how many arrivals end its phase: `rows` threads of a
  // row tile, `queries` that bring query rows, `fillers` of a buffer, `lookers`.
  template <typename Init>
  static PCS_ROUNDS void each(int rows, int queries, int fillers, int lookers, Init&& init) {
    init(q_full(), queries);
    init(drained(), 1);
    for (int t = 0; t < 2; ++t) {
      init(s_full(t), 1);
      init(s_read(t), rows);
      init(p_full(t), rows);
      init(o_full(t), 1);
    }
    for (int i = 0; i < kRing; ++i) {
      init(kv_full(i), fillers);
      init(kv_empty(i), 1);
    }
    for (int j = 0; LOOK && j < VALUES; ++j) init(v_fine(j), lookers);
  }
};

// Fills 0 .. n - 1, two a round.  Every warp waits for a fill's place (`wait`, with
// a limit; false: it ran out), and all meet at the beginning of each round.  A warp
// whose wait ran out fills and waits no more, but comes to every meeting, so that
// nobody waits for it in vain.  Whether all fills were made.
template <typename Wait, typename Meet, typename Fill>
PCS_ROUNDS bool in_rounds(int n, Wait&& wait, Meet&& meet, Fill&& fill) {
  bool ok = true;
  for (int i = 0; i < n; ++i) {
    ok = ok && wait(i);
    if ((i & 1) == 0) meet();
    if (ok) fill(i);
  }
  return ok;
}

}  // namespace pcs

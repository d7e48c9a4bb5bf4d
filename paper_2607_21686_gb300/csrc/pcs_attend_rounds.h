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

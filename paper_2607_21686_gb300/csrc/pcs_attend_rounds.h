// pcs_attend_rounds.h -- how several warps fill a ring together and give up
// together.  Control flow alone, for the block kernel and for checks on the host.
#pragma once

#ifdef __CUDACC__
#define PCS_ROUNDS __device__ __forceinline__
#else
#define PCS_ROUNDS inline
#endif

namespace pcs {

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

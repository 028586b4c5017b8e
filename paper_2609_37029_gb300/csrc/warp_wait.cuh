// A bounded wait that a whole warp makes together, apart from the machine so
// that it also compiles and runs on the host.
//
// Every lane tests the barrier, the other roles' flag and the clock for itself,
// and their answers may differ.  What follows a wait is executed by the whole
// warp (votes, tcgen05 .sync.aligned), so lanes that left on their own would
// leave the others waiting for them without a limit: the verdict is the warp's.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define LSP_WAIT_FN __device__ __forceinline__
#else
#define LSP_WAIT_FN inline
#endif

namespace lsp {

// W: ready()   this lane's test of the barrier (may take a while)
//    all(x)    whether x holds for every lane; any(x) for some lane
//    gone()    another role has given up
//    now()     nanoseconds
//    give_up(late)  called by every lane when the warp gives up; late: this lane's limit is over
// True once every lane has seen the barrier complete (one that has does not ask
// again: the phase may move on), false if some lane's limit is over or the flag
// is up before that; the same in every lane.
template <class W>
LSP_WAIT_FN bool warp_wait(W w, uint64_t limit_ns) {
  bool ok = w.ready();
  if (w.all(ok)) return true;
  const uint64_t t0 = w.now();
  for (uint32_t i = 1;; ++i) {
    ok = ok || w.ready();
    if (w.all(ok)) return true;
    if ((i & 31u) == 0) {
      const bool gone = w.gone(), late = !gone && w.now() - t0 > limit_ns;
      if (w.any(gone || late)) {
        w.give_up(late);
        return false;
      }
    }
  }
}

}  // namespace lsp

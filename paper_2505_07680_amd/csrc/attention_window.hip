// The attention kernel's forms with a window and sinks (see attention_split.h).

#include "attention_split.h"

namespace sr {

SplitKernel window_kernel(int D, int nq, int qg, int q_chunks, bool follow) {
  if (follow) return D == 64 ? pick_split<64, true, true>(nq, qg, q_chunks) : pick_split<128, true, true>(nq, qg, q_chunks);
  return D == 64 ? pick_split<64, false, true>(nq, qg, q_chunks) : pick_split<128, false, true>(nq, qg, q_chunks);
}

}  // namespace sr

// The attention kernel's forms with a window and sinks (see attention_split.h). Their
// softmax references stay lazy.

#include "attention_split.h"

namespace sr {

SplitKernel window_kernel(int D, int nq, int qg, int q_chunks) {
  return D == 64 ? pick_split<64, false, true>(nq, qg, q_chunks) : pick_split<128, false, true>(nq, qg, q_chunks);
}

}  // namespace sr

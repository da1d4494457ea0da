// Head norm and rotary positions (k_rope.cuh): heads that fit into one row of a warp, several tokens at a
// time, forward and gradients.

#include "k_rope.cuh"

namespace ress {

cudaError_t launch_rope_few(bool bwd, const RopeKind& kind, int type, RopeParams& p, int (&ctas)[2], cudaStream_t st) {
  return bwd ? launch_rope_kind<true, true>(kind, type, p, ctas, st) : launch_rope_kind<false, true>(kind, type, p, ctas, st);
}

}  // namespace ress

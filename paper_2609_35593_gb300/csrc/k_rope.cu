// Head norm and rotary positions (k_rope.cuh): the forward pass.

#include "k_rope.cuh"

namespace ress {

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st) {
  int first[3];
  return launch_rope_all<false>(a, first, st);
}

}  // namespace ress

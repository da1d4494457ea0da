// Head norm and rotary positions (k_rope.cuh): the forward pass.

#include "k_rope.cuh"

namespace ress {

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st) {
  int ctas[2];
  const cudaError_t e = launch_rope_part<true, false>(a, ctas, st);
  return e != cudaSuccess ? e : launch_rope_part<false, false>(a, ctas, st);
}

}  // namespace ress

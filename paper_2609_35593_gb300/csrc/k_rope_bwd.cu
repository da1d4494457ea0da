// Head norm and rotary positions (k_rope.cuh): the gradients, and the sums over CTAs of those of the
// norms' parameters.

#include "k_rope.cuh"

namespace ress {

namespace {

// Sums of the CTAs' partial rows in order, 32 channels of one parameter of one tensor per CTA.
constexpr int kRopeFoldWarps = 32;
struct RopeFoldParams {
  const float* partial;
  float* out[4];  // weight and bias of t[0], of t[1]
  int first[3];   // CTAs of t[0]: first[0]..first[1], of t[1]: first[1]..first[2]
  int hd;
};
__global__ void __launch_bounds__(32 * kRopeFoldWarps) k_rope_fold(const RopeFoldParams p) {
  __shared__ float acc[kRopeFoldWarps][33];
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  const int which = (int)blockIdx.y, a = which & 1, c = (int)blockIdx.x * 32 + lane;
  stream_acquire();
  float v = 0.f;
  if (c < p.hd) {
#pragma unroll 8
    for (int g = p.first[which >> 1] + warp; g < p.first[(which >> 1) + 1]; g += kRopeFoldWarps)
      v += p.partial[((int64_t)g * 2 + a) * p.hd + c];
  }
  acc[warp][lane] = v;
  __syncthreads();
  stream_release();
  if (warp == 0 && c < p.hd && p.out[which]) {
    v = 0.f;
#pragma unroll
    for (int q = 0; q < kRopeFoldWarps; ++q) v += acc[q][lane];
    p.out[which][c] = v;
  }
}

}  // namespace

cudaError_t launch_rope_bwd(const RopeArgs& a, cudaStream_t st) {
  RopeFoldParams f;
  const cudaError_t e = launch_rope_all<true>(a, f.first, st);
  if (e != cudaSuccess || !a.partial) return e;
  f.partial = a.partial;
  for (int i = 0; i < 2; ++i) {
    const bool norm = a.t[i].n_heads > 0 && a.t[i].norm.enabled;
    f.out[2 * i] = norm ? a.t[i].dweight : nullptr;
    f.out[2 * i + 1] = norm ? a.t[i].dbias : nullptr;
  }
  f.hd = a.plan.head_dim;
  return launch_pdl(k_rope_fold, dim3((f.hd + 31) / 32, 4), 32 * kRopeFoldWarps, 0, st, true, f);
}

}  // namespace ress

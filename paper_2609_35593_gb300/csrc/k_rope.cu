// Rotary positions over several axes on the heads of Q and K, after a layer norm over each head's
// channels where there is one, and the gradients of both.
//   forward   u = (x - m) r w + b over the head's channels (or u = x), then for each pair (i, j) of
//             channels with its angle t:  y_i = u_i cos t - u_j sin t,  y_j = u_j cos t + u_i sin t
//   backward  du = the same of dy with -t;  dx = du, or with h = (x - m) r and g = du w:
//             dx = r (g - avg(g) - h avg(g h)),  dw = sum over tokens and heads of du h,  db = of du
// Memory-bound: every element is read once and written once, whatever the norm and the rotation do
// in between.
//
// A head's channels lie on G lanes, 8 per lane, so a warp holds 32 / G heads of a token at a time,
// and takes K such rows at once to have enough bytes on the way.  An item is one token and up to
// K 32 / G of its heads, all of one tensor: a CTA stays with Q or K (shares of the grid by their
// heads), and its lanes keep the norm's parameters and their gradients' sums in registers.  The
// token's cosines and sines are formed once per item, one pair per lane, and handed out through
// shared memory.  A pair's two channels meet in one lane (interleaved pairs), by a shuffle between
// two lanes (the pairs' halves of a section are whole lanes), or through shared memory (any plan).
// Sums are float32 in a fixed order; the gradients of the parameters are summed per CTA and then
// over CTAs by a second kernel.

#include "row_ops.cuh"

namespace ress {
using namespace rows;

namespace {

constexpr int kRopeWarps = 4;
constexpr int kRopeThreads = 32 * kRopeWarps;

enum { kInLane = 0, kByShuffle = 1, kByShared = 2 };

struct RopeParams {
  ress_rope_plan plan;
  ress_rope_heads t[2];
  int64_t tokens;
  const int32_t* pos;
  float* partial;
  float eps;
  int first_ctas;  // CTAs of t[0]; the others have t[1]
  int param_type, meet;
  bool vec;        // 16-byte accesses
};

// A lane's 8 channels of one head, as float32; channels from n on are 0.
template <typename T>
__device__ __forceinline__ Vec<T, 8> load8(const T* p, int n, bool vec) {
  if (n <= 0) return zero_vec<T, 8>();
  if (vec) return load_vec<T, 8>(p);
  Vec<T, 8> r = zero_vec<T, 8>();
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) {
      if constexpr (sizeof(T) == 4)
        r.w[j] = reinterpret_cast<const uint32_t*>(p)[j];
      else
        r.w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
    }
  return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8], int n, bool vec) {
  if (n <= 0) return;
  if (vec) {
    store_vec<T, 8>(p, v);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) p[j] = from_f32<T>(v[j]);
}

template <typename T, int G, bool NORM, bool BWD, int K>
__global__ void __launch_bounds__(kRopeThreads) k_rope(const __grid_constant__ RopeParams p) {
  constexpr int kHeads = 32 / G;                     // heads of a warp's row
  constexpr int kPairs = G <= 8 ? 1 : G / 8;         // pairs per lane: 4 G pairs at most
  __shared__ float2 turn[kRopeWarps][32 * kPairs];
  __shared__ float swap[kRopeWarps][32 * 8];
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  const bool second = (int)blockIdx.x >= p.first_ctas;
  const ress_rope_heads& t = p.t[second];
  const ress_heads& out = BWD ? t.dx : t.y;
  const int hd = p.plan.head_dim, heads = t.n_heads;
  const int group = lane / G, c0 = lane % G * 8, n = hd - c0;  // n: the lane's channels, if below 8
  const float inv = 1.f / (float)hd;

  // The lane's channels in the rotation, one byte each: the pair, the other channel; bits: whether
  // it is rotated, whether it is the pair's second.
  uint32_t pair[2] = {0u, 0u}, other[2] = {0u, 0u}, turns = 0u, seconds = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const RopeChannel r = rope_channel(p.plan, min(c0 + j, hd - 1));
    if (c0 + j < hd && r.pair >= 0) {
      pair[j / 4] |= (uint32_t)r.pair << (8 * (j & 3));
      turns |= 1u << j;
      seconds |= (uint32_t)r.second << j;
    }
    other[j / 4] |= (uint32_t)(c0 + j < hd ? r.partner : c0 + j) << (8 * (j & 3));
  }
  const int from = (lane & ~(G - 1)) | (int)((other[0] & 255u) >> 3);  // the other channels' lane
  // The pairs whose angles this lane forms.
  uint64_t freq[kPairs];
  int axis[kPairs];
#pragma unroll
  for (int q = 0; q < kPairs; ++q) {
    const int k = min(lane + 32 * q, p.plan.n_pairs - 1);
    freq[q] = k < 0 ? 0ull : p.plan.turns[k];
    axis[q] = k < 0 ? 0 : rope_axis(p.plan, k);
  }

  stream_acquire();
  float w[8], b[8], dw[8], db[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    w[j] = NORM && j < n ? param_at(t.norm.weight, p.param_type, c0 + j, 1.f) : 0.f;
    b[j] = NORM && !BWD && j < n ? param_at(t.norm.bias, p.param_type, c0 + j, 0.f) : 0.f;
    dw[j] = db[j] = 0.f;
  }

  const int chunks = (heads + K * kHeads - 1) / (K * kHeads);  // items of a token
  const int64_t warps = (int64_t)(second ? gridDim.x - p.first_ctas : p.first_ctas) * kRopeWarps;
  const int64_t w0 = (int64_t)(blockIdx.x - (second ? p.first_ctas : 0)) * kRopeWarps + warp;
  const int64_t step = warps / chunks;
  const int step_rest = (int)(warps - step * chunks);
  int64_t token = w0 / chunks;
  int chunk = (int)(w0 - token * chunks);
  for (; token < p.tokens;) {
    Vec<T, 8> rx[K], ry[K];
    bool live[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int h = (chunk * K + k) * kHeads + group;
      live[k] = h < heads;
      if (!BWD || NORM)
        rx[k] = load8(static_cast<const T*>(t.x.data) + token * t.x.token_stride + h * t.x.head_stride + c0,
                      live[k] ? n : 0, p.vec);
      if (BWD)
        ry[k] = load8(static_cast<const T*>(t.y.data) + token * t.y.token_stride + h * t.y.head_stride + c0,
                      live[k] ? n : 0, p.vec);
    }
    // the token's angles
    __syncwarp();
#pragma unroll
    for (int q = 0; q < kPairs; ++q)
      if (lane + 32 * q < p.plan.n_pairs)
        turn[warp][lane + 32 * q] = rope_cos_sin(p.pos[token * p.plan.n_axes + axis[q]], freq[q]);
    __syncwarp();
    float cs[8], sn[8];  // y = u cs + (the other channel's u) sn
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 a = turn[warp][(pair[j / 4] >> (8 * (j & 3))) & 255u];
      cs[j] = a.x;
      sn[j] = ((seconds >> j & 1u) != 0u) != BWD ? a.y : -a.y;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float u[8], h[8], v[8], mean = 0.f, rstd = 1.f;
      if (NORM) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          h[j] = elem(rx[k], j);
          mean += h[j];
        }
        mean = segment_sum<G>(mean * inv);  // scaled first: the sum may overflow where its mean does not
        float sq = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          h[j] = j < n ? h[j] - mean : 0.f;
          sq = fmaf(h[j], h[j], sq);
        }
        rstd = rsqrtf(segment_sum<G>(sq * inv) + p.eps);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] *= rstd;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] = BWD ? elem(ry[k], j) : NORM ? fmaf(h[j], w[j], b[j]) : elem(rx[k], j);
      if (p.meet == kInLane) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = u[j ^ 1];
      } else if (p.meet == kByShuffle) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __shfl_sync(0xffffffffu, u[j], from);
      } else {
        float* row = &swap[warp][group * (8 * G)];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) row[c0 + j] = u[j];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = row[(other[j / 4] >> (8 * (j & 3))) & 255u];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = fmaf(u[j], cs[j], v[j] * sn[j]);
        u[j] = (turns >> j & 1u) ? y : u[j];
      }
      if constexpr (NORM && BWD) {
        float sg = 0.f, sgh = 0.f;
        if (live[k]) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            dw[j] = fmaf(u[j], h[j], dw[j]);
            db[j] += u[j];
            u[j] *= w[j];
            sg += u[j];
            sgh = fmaf(u[j], h[j], sgh);
          }
        }
        sg = segment_sum<G>(sg) * inv;
        sgh = segment_sum<G>(sgh) * inv;
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = rstd * (u[j] - sg - h[j] * sgh);
      }
      const int head = (chunk * K + k) * kHeads + group;
      store8(static_cast<T*>(out.data) + token * out.token_stride + head * out.head_stride + c0, u,
             live[k] ? n : 0, p.vec);
    }
    token += step;
    chunk += step_rest;
    if (chunk >= chunks) {
      chunk -= chunks;
      ++token;
    }
  }
  stream_release();
  if constexpr (NORM && BWD) {
    if (!p.partial) return;
    // the CTA's sums: a warp's groups, then its warps in order
    __shared__ float part[kRopeWarps][2][G * 8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
      for (int o = G; o < 32; o <<= 1) {
        dw[j] += __shfl_xor_sync(0xffffffffu, dw[j], o);
        db[j] += __shfl_xor_sync(0xffffffffu, db[j], o);
      }
      if (lane < G) {
        part[warp][0][c0 + j] = dw[j];
        part[warp][1][c0 + j] = db[j];
      }
    }
    __syncthreads();
    for (int k = (int)threadIdx.x; k < 2 * hd; k += kRopeThreads) {
      const int a = k >= hd, c = k - a * hd;
      float v = 0.f;
#pragma unroll
      for (int q = 0; q < kRopeWarps; ++q) v += part[q][a][c];
      p.partial[((int64_t)blockIdx.x * 2 + a) * hd + c] = v;
    }
  }
}

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

// How a pair's channels meet: see the top.
int meeting(const ress_rope_plan& plan) {
  if (plan.layout == RESS_ROPE_INTERLEAVED) return kInLane;
  if (plan.layout == RESS_ROPE_HALVES) return plan.n_pairs % 8 == 0 ? kByShuffle : kByShared;
  for (int a = 0; a < plan.n_axes; ++a)
    if (plan.axis_dims[a] % 16 != 0) return kByShared;
  return kByShuffle;
}

template <typename T, int G, bool NORM, bool BWD>
cudaError_t launch_rope_as(const RopeArgs& a, RopeParams& p, cudaStream_t st) {
  constexpr int K = sizeof(T) == 2 ? (BWD && NORM ? 2 : 4) : (BWD && NORM ? 1 : 2);
  auto kern = k_rope<T, G, NORM, BWD, K>;
  int resident = 1;
  if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kern, kRopeThreads, 0) != cudaSuccess || resident < 1)
    resident = 1;
  int64_t need[2], all = 0;  // CTAs at one item per warp
  for (int i = 0; i < 2; ++i) {
    const int64_t items = p.tokens * ((p.t[i].n_heads + K * (32 / G) - 1) / (K * (32 / G)));
    need[i] = (items + kRopeWarps - 1) / kRopeWarps;
    all += need[i];
  }
  const int64_t fit = min((int64_t)resident * sm_count(), (int64_t)kRopeParts - 2);
  const int64_t steps = max((all + fit - 1) / fit, (int64_t)1);
  const int first = (int)((need[0] + steps - 1) / steps), rest = (int)((need[1] + steps - 1) / steps);
  p.first_ctas = first;
  cudaError_t e = cudaSuccess;
  if (first + rest > 0) e = launch_pdl(kern, first + rest, kRopeThreads, 0, st, true, p);
  if (e != cudaSuccess || !p.partial) return e;
  RopeFoldParams f;
  f.partial = p.partial;
  for (int i = 0; i < 2; ++i) {
    const bool norm = p.t[i].n_heads > 0 && p.t[i].norm.enabled;
    f.out[2 * i] = norm ? p.t[i].dweight : nullptr;
    f.out[2 * i + 1] = norm ? p.t[i].dbias : nullptr;
  }
  f.first[0] = 0;
  f.first[1] = first;
  f.first[2] = first + rest;
  f.hd = p.plan.head_dim;
  return launch_pdl(k_rope_fold, dim3((f.hd + 31) / 32, 4), 32 * kRopeFoldWarps, 0, st, true, f);
}

template <typename T, bool NORM, bool BWD>
cudaError_t launch_rope_typed(const RopeArgs& a, RopeParams& p, cudaStream_t st) {
  const int hd = p.plan.head_dim;
  if (hd <= 32) return launch_rope_as<T, 4, NORM, BWD>(a, p, st);
  if (hd <= 64) return launch_rope_as<T, 8, NORM, BWD>(a, p, st);
  if (hd <= 128) return launch_rope_as<T, 16, NORM, BWD>(a, p, st);
  return launch_rope_as<T, 32, NORM, BWD>(a, p, st);
}

template <bool NORM, bool BWD>
cudaError_t launch_rope_norm(const RopeArgs& a, RopeParams& p, cudaStream_t st) {
  if (a.type == RESS_BF16) return launch_rope_typed<bf16, NORM, BWD>(a, p, st);
  if (a.type == RESS_F16) return launch_rope_typed<f16, NORM, BWD>(a, p, st);
  return launch_rope_typed<float, NORM, BWD>(a, p, st);
}

// The launch of the tensors whose norm is (not) enabled; the other's head count is 0 in it.
template <bool BWD>
cudaError_t launch_rope_part(const RopeArgs& a, bool norm, cudaStream_t st) {
  RopeParams p;
  p.plan = a.plan;
  p.tokens = a.n_tokens;
  p.pos = a.pos;
  p.eps = a.eps;
  p.param_type = a.param_type;
  p.meet = meeting(a.plan);
  p.partial = nullptr;
  const int bytes = a.type == RESS_F32 ? 4 : 2;
  p.vec = a.plan.head_dim % 8 == 0;
  bool any = false, grads = false;
  for (int i = 0; i < 2; ++i) {
    p.t[i] = a.t[i];
    ress_rope_heads& t = p.t[i];
    if (t.n_heads == 0 || (t.norm.enabled != 0) != norm) {
      t.n_heads = 0;
      continue;
    }
    any = true;
    grads = grads || (BWD && norm && (t.dweight || t.dbias));
    auto fits = [&](const ress_heads& h) {
      return reinterpret_cast<uintptr_t>(h.data) % 16 == 0 && (a.n_tokens == 1 || h.token_stride * bytes % 16 == 0) &&
             (t.n_heads == 1 || h.head_stride * bytes % 16 == 0);
    };
    p.vec = p.vec && fits(t.y) && ((BWD && !norm) || fits(t.x)) && (!BWD || fits(t.dx));
  }
  if (!any) return cudaSuccess;
  if (grads) p.partial = a.partial;
  if (p.tokens == 0 && !grads) return cudaSuccess;
  return norm ? launch_rope_norm<true, BWD>(a, p, st) : launch_rope_norm<false, BWD>(a, p, st);
}

template <bool BWD>
cudaError_t launch_rope_both(const RopeArgs& a, cudaStream_t st) {
  const cudaError_t e = launch_rope_part<BWD>(a, true, st);
  return e != cudaSuccess ? e : launch_rope_part<BWD>(a, false, st);
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, cudaStream_t st) { return launch_rope_both<false>(a, st); }
cudaError_t launch_rope_bwd(const RopeArgs& a, cudaStream_t st) { return launch_rope_both<true>(a, st); }

}  // namespace ress

// Layer norm over the rows of the residual stream, and its gradients.
//   forward   y = (x - m) r w + b,  m = avg(x),  r = 1 / sqrt(avg((x - m)^2) + eps)
//   backward  with h = (x - m) r and g = dy w:
//             dx = r (g - avg(g) - h avg(g h)) [+ dres],  dw = sum over rows of dy h,  db = of dy
// avg and the sums are over the row's channels.  One pass over the data: a row's elements stay in
// registers, as they lie in memory, between its sums and its result.
//
// A row belongs to a team: SEG lanes of a warp (rows of up to 64 or 128 channels), a warp, or a CTA
// of several warps, so that a thread has C = 8 channels and keeps their weight, bias and gradient sums
// in registers while its team goes through R rows at a time (above 4096 channels C = 32, and what is
// kept is in L1 and shared memory).  The
// mean is subtracted before squares are taken (two sums, one after the other): rows with an offset
// much larger than their spread keep their digits.  All sums are float32 in a fixed order.
//
// The gradients of the weight and the bias: each CTA adds up its rows in registers and shared memory
// and leaves one partial row of each in the workspace, and a second kernel adds the partial rows up
// in order, so that the result does not depend on the order in which CTAs finish.

#include "row_ops.cuh"

namespace ress {
using namespace rows;

namespace {

constexpr int kNormThreads = 128;     // CTA of teams of up to a warp
constexpr int kNormMaxThreads = 512;  // a team that is a CTA: at most 16 warps

struct NormParams {
  int64_t rows, x_stride, y_stride, dx_stride, dres_stride;
  const void *x, *y, *weight, *bias, *dres;  // y: backward dy
  void *out;                                 // forward y, backward dx
  float *mean, *rstd, *partial;
  float eps;
  int width, param_type, team;
};

// Sums over a team's threads of N values each: over the warp's segments, then over the CTA's warps
// through shared memory where the team has several.  The two halves of `red` take turns, so that one
// barrier per call is enough: a warp that writes a half again has passed the barrier of the call in
// between, which every warp reaches after reading.
template <int SEG, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float* red, int& turn, int warps) {
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = segment_sum<SEG>(v[k]);
  if (SEG < 32 || warps == 1) return;
  float* at = red + turn * (16 * N);
  turn ^= 1;
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int k = 0; k < N; ++k) at[(threadIdx.x >> 5) * N + k] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = 0.f;
  for (int w = 0; w < warps; ++w) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] += at[w * N + k];
  }
}

// The team of this thread: its index in the grid, the thread's place in it, its threads and warps.
template <int SEG>
struct Team {
  int64_t index, count;
  int t, threads, warps;
  __device__ explicit Team(int n) {  // n: threads of a team, SEG or a CTA's whole warps
    threads = SEG < 32 ? SEG : n;
    warps = SEG < 32 ? 1 : n / 32;
    t = (int)threadIdx.x % threads;
    const int per_cta = (int)blockDim.x / threads;
    index = (int64_t)blockIdx.x * per_cta + (int)threadIdx.x / threads;
    count = (int64_t)gridDim.x * per_cta;
  }
};

// A thread's weights or biases: in registers for the whole kernel where it has 8 channels, read
// where they are used (from L1) where it has 32.
template <int C>
constexpr bool kInRegisters = C == 8;
template <int E, int C>
struct Params {
  float v[kInRegisters<C> ? C : 1];
  const void* p;
  float none;
  int type, width, t, threads;
  __device__ Params(const void* p_, int type_, float none_, int width_, int t_, int threads_)
      : p(p_), none(none_), type(type_), width(width_), t(t_), threads(threads_) {
    if constexpr (kInRegisters<C>) {
#pragma unroll
      for (int c = 0; c < C; ++c) v[c] = load(c / E, c % E);
    }
  }
  __device__ float load(int i, int e) const {
    const int col = (t + i * threads) * E + e;
    return col < width ? param_at(p, type, col, none) : 0.f;
  }
  __device__ float at(int i, int e) const {
    if constexpr (kInRegisters<C>)
      return v[i * E + e];
    else
      return load(i, e);
  }
};

template <typename X, typename Y, int E, int C, int SEG, int R>
__global__ void __launch_bounds__(kNormMaxThreads) k_layer_norm(const NormParams p) {
  __shared__ float red[2 * 16 * R];
  constexpr int V = C / E;
  const Team<SEG> team(p.team);
  const float inv = 1.f / (float)p.width;
  int turn = 0;
  stream_acquire();
  Params<E, C> w(p.weight, p.param_type, 1.f, p.width, team.t, team.threads);
  Params<E, C> b(p.bias, p.param_type, 0.f, p.width, team.t, team.threads);
  bool in[V];
#pragma unroll
  for (int i = 0; i < V; ++i) in[i] = (team.t + i * team.threads) * E < p.width;
  const X* x = static_cast<const X*>(p.x) + (int64_t)team.t * E;
  Y* y = static_cast<Y*>(p.out) + (int64_t)team.t * E;
  const int step = team.threads * E;  // columns from one of the thread's vectors to the next
  // teams of a warp leave the loop together: their segments take part in each other's shuffles
  const int64_t first = SEG < 32 ? team.index / (32 / SEG) * (32 / SEG) : team.index;
  for (int64_t base = 0; (base + first) * R < p.rows; base += team.count) {
    const int64_t row0 = (base + team.index) * R;
    Vec<X, E> raw[R][V];
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i)
        raw[k][i] = in[i] && row0 + k < p.rows ? load_vec<X, E>(x + (row0 + k) * p.x_stride + i * step)
                                               : zero_vec<X, E>();
    float mean[R], rstd[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      mean[k] = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) mean[k] += elem(raw[k][i], e);
      mean[k] *= inv;  // before the threads' sums meet: a row's sum may overflow where its mean does not
    }
    team_sum<SEG>(mean, red, turn, team.warps);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      rstd[k] = 0.f;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float d = in[i] ? elem(raw[k][i], e) - mean[k] : 0.f;
          rstd[k] = fmaf(d, d, rstd[k]);
        }
      rstd[k] *= inv;
    }
    team_sum<SEG>(rstd, red, turn, team.warps);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (row0 + k >= p.rows) continue;
      const float r = rsqrtf(rstd[k] + p.eps);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!in[i]) continue;
        float out[E];
#pragma unroll
        for (int e = 0; e < E; ++e)
          out[e] = fmaf((elem(raw[k][i], e) - mean[k]) * r, w.at(i, e), b.at(i, e));
        store_vec<Y, E>(y + (row0 + k) * p.y_stride + i * step, out);
      }
      if (team.t == 0) {
        if (p.mean) p.mean[row0 + k] = mean[k];
        if (p.rstd) p.rstd[row0 + k] = r;
      }
    }
  }
  stream_release();
}

template <typename X, typename Y, int E, int C, int SEG, int R>
__global__ void __launch_bounds__(kNormMaxThreads) k_layer_norm_bwd(const NormParams p) {
  __shared__ float red[2 * 16 * 2 * R];
  constexpr int V = C / E;
  const Team<SEG> team(p.team);
  const float inv = 1.f / (float)p.width;
  int turn = 0;
  stream_acquire();
  Params<E, C> w(p.weight, p.param_type, 1.f, p.width, team.t, team.threads);
  // The thread's gradient sums: registers, or (C = 32) its own places in shared memory.
  extern __shared__ float wide[];
  float dw[kInRegisters<C> ? C : 1], db[kInRegisters<C> ? C : 1];
  bool in[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    in[i] = (team.t + i * team.threads) * E < p.width;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if constexpr (kInRegisters<C>) {
        dw[i * E + e] = 0.f;
        db[i * E + e] = 0.f;
      } else if (in[i]) {
        wide[(i * E + e) * team.threads + team.t] = 0.f;
        wide[(C + i * E + e) * team.threads + team.t] = 0.f;
      }
    }
  }
  const X* x = static_cast<const X*>(p.x) + (int64_t)team.t * E;
  const Y* dy = static_cast<const Y*>(p.y) + (int64_t)team.t * E;
  const X* dres = static_cast<const X*>(p.dres) + (p.dres ? (int64_t)team.t * E : 0);
  X* dx = static_cast<X*>(p.out) + (int64_t)team.t * E;
  const int step = team.threads * E;
  const int64_t first = SEG < 32 ? team.index / (32 / SEG) * (32 / SEG) : team.index;
  for (int64_t base = 0; (base + first) * R < p.rows; base += team.count) {
    const int64_t row0 = (base + team.index) * R;
    Vec<X, E> rx[R][V], rres[R][V];
    Vec<Y, E> rdy[R][V];
    float mean[R], rstd[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const bool live = row0 + k < p.rows;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int64_t row = row0 + k;
        rx[k][i] = in[i] && live ? load_vec<X, E>(x + row * p.x_stride + i * step) : zero_vec<X, E>();
        rdy[k][i] = in[i] && live ? load_vec<Y, E>(dy + row * p.y_stride + i * step) : zero_vec<Y, E>();
        rres[k][i] =
            p.dres && in[i] && live ? load_vec<X, E>(dres + row * p.dres_stride + i * step) : zero_vec<X, E>();
      }
      mean[k] = live ? p.mean[row0 + k] : 0.f;
      rstd[k] = live ? p.rstd[row0 + k] : 0.f;
    }
    float sums[2 * R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      float sg = 0.f, sgh = 0.f;
      if (row0 + k < p.rows) {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const int c = i * E + e;
            const float d = elem(rdy[k][i], e), h = in[i] ? (elem(rx[k][i], e) - mean[k]) * rstd[k] : 0.f;
            const float g = d * w.at(i, e);
            sg += g;
            sgh = fmaf(g, h, sgh);
            if constexpr (kInRegisters<C>) {
              dw[c] = fmaf(d, h, dw[c]);
              db[c] += d;
            } else if (in[i]) {
              wide[c * team.threads + team.t] += d * h;
              wide[(C + c) * team.threads + team.t] += d;
            }
          }
      }
      sums[2 * k] = sg;
      sums[2 * k + 1] = sgh;
    }
    team_sum<SEG>(sums, red, turn, team.warps);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (row0 + k >= p.rows) continue;
      const float ag = sums[2 * k] * inv, agh = sums[2 * k + 1] * inv;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!in[i]) continue;
        float out[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float h = (elem(rx[k][i], e) - mean[k]) * rstd[k];
          const float g = elem(rdy[k][i], e) * w.at(i, e);
          out[e] = rstd[k] * (g - ag - h * agh);
          if (p.dres) out[e] += elem(rres[k][i], e);
        }
        store_vec<X, E>(dx + (row0 + k) * p.dx_stride + i * step, out);
      }
    }
  }
  stream_release();
  if (!p.partial) return;
  // the CTA's partial rows: segments of a warp, then (teams of up to a warp) the CTA's warps in order
  float* out = p.partial + (int64_t)blockIdx.x * 2 * p.width;
  if (SEG == 32 && team.warps > 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (!in[i]) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int col = (team.t + i * team.threads) * E + e;
        const int c = i * E + e;
        out[col] = kInRegisters<C> ? dw[kInRegisters<C> ? c : 0] : wide[c * team.threads + team.t];
        out[p.width + col] = kInRegisters<C> ? db[kInRegisters<C> ? c : 0] : wide[(C + c) * team.threads + team.t];
      }
    }
    return;
  }
  // teams of up to a warp have at most 32 C = 256 channels
  __shared__ float part[kNormThreads / 32][2][32 * 8];
  if constexpr (kInRegisters<C>) {
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int o = SEG; o < 32; o <<= 1) {
        dw[c] += __shfl_xor_sync(0xffffffffu, dw[c], o);
        db[c] += __shfl_xor_sync(0xffffffffu, db[c], o);
      }
    if (lane < SEG) {
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int col = (team.t + i * team.threads) * E + e;
          part[warp][0][col] = dw[i * E + e];
          part[warp][1][col] = db[i * E + e];
        }
    }
    __syncthreads();
    for (int k = (int)threadIdx.x; k < 2 * p.width; k += kNormThreads) {
      const int a = k / p.width, col = k - a * p.width;
      float v = 0.f;
#pragma unroll
      for (int q = 0; q < kNormThreads / 32; ++q) v += part[q][a][col];
      out[k] = v;
    }
  }
}

// Column sums of `parts` rows of 2 `width` partial sums, in a fixed order: 32 columns per CTA, one
// warp per 32nd row, then the warps in order.
constexpr int kFoldWarps = 32;
__global__ void __launch_bounds__(32 * kFoldWarps)
    k_fold_parts(const float* partial, int parts, int width, float* dw, float* db) {
  __shared__ float acc[kFoldWarps][33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int col = blockIdx.x * 32 + lane;
  stream_acquire();
  float v = 0.f;
  if (col < 2 * width) {
#pragma unroll 8
    for (int g = warp; g < parts; g += kFoldWarps) v += partial[(int64_t)g * 2 * width + col];
  }
  acc[warp][lane] = v;
  __syncthreads();
  stream_release();
  if (warp == 0 && col < 2 * width) {
    v = 0.f;
#pragma unroll
    for (int q = 0; q < kFoldWarps; ++q) v += acc[q][lane];
    if (col < width) {
      if (dw) dw[col] = v;
    } else if (db) {
      db[col - width] = v;
    }
  }
}

// Teams of the launch: a multiple of a CTA's, as many as fit on the GPU at once at most, all with
// the same number of steps but for the last ones.
template <typename K>
int norm_ctas(K kern, int threads, size_t smem, int teams_per_cta, int64_t batches, int most) {
  int resident = 1;
  if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kern, threads, smem) != cudaSuccess || resident < 1)
    resident = 1;
  const int64_t ctas = (batches + teams_per_cta - 1) / teams_per_cta;
  const int64_t fit = min((int64_t)resident * sm_count(), (int64_t)most);
  const int64_t steps = (ctas + fit - 1) / fit;
  return (int)((ctas + steps - 1) / steps);
}

template <bool BWD, typename X, typename Y, int E, int C, int SEG>
cudaError_t launch_norm_as(const NormArgs& a, NormParams p, cudaStream_t st) {
  constexpr int R = C == 32 ? 1 : BWD ? (sizeof(X) == 2 && E > 1 ? 2 : 1) : (sizeof(X) == 2 && E > 1 ? 4 : 2);
  p.team = SEG < 32 ? SEG : ((p.width + C - 1) / C + 31) / 32 * 32;
  const int threads = p.team <= 32 ? kNormThreads : p.team;
  const int per_cta = threads / p.team;
  const int64_t batches = (p.rows + R - 1) / R;
  if constexpr (!BWD) {
    auto kern = k_layer_norm<X, Y, E, C, SEG, R>;
    const int ctas = norm_ctas(kern, threads, 0, per_cta, batches, INT32_MAX);
    return launch_pdl(kern, ctas, threads, 0, st, true, p);
  } else {
    auto kern = k_layer_norm_bwd<X, Y, E, C, SEG, R>;
    const size_t smem = kInRegisters<C> ? 0 : 2 * C * sizeof(float) * threads;
    cudaError_t e = cudaSuccess;
    if (smem > 0) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const int ctas = norm_ctas(kern, threads, smem, per_cta, batches, kNormParts);
    e = launch_pdl(kern, ctas, threads, smem, st, true, p);
    if (e != cudaSuccess || !p.partial) return e;
    return launch_pdl(k_fold_parts, (2 * p.width + 31) / 32, 32 * kFoldWarps, 0, st, true, p.partial, ctas,
                      p.width, a.dweight, a.dbias);
  }
}

template <bool BWD, typename X, typename Y>
cudaError_t launch_norm_typed(const NormArgs& a, const NormParams& p, bool vec, cudaStream_t st) {
  constexpr int E = 16 / (int)sizeof(X);
  if (vec && p.width <= 64) return launch_norm_as<BWD, X, Y, E, 8, 8>(a, p, st);
  if (vec && p.width <= 128) return launch_norm_as<BWD, X, Y, E, 8, 16>(a, p, st);
  if (p.width <= 8 * kNormMaxThreads)
    return vec ? launch_norm_as<BWD, X, Y, E, 8, 32>(a, p, st) : launch_norm_as<BWD, X, Y, 1, 8, 32>(a, p, st);
  return vec ? launch_norm_as<BWD, X, Y, E, 32, 32>(a, p, st) : launch_norm_as<BWD, X, Y, 1, 32, 32>(a, p, st);
}

template <bool BWD>
cudaError_t launch_norm(const NormArgs& a, cudaStream_t st) {
  NormParams p;
  p.rows = a.n.rows;
  p.x_stride = a.n.x_stride;
  p.y_stride = a.n.y_stride;
  p.dx_stride = a.n.dx_stride;
  p.dres_stride = a.n.dres_stride;
  p.x = a.x;
  p.y = a.dy;
  p.weight = a.weight;
  p.bias = a.bias;
  p.dres = a.dres;
  p.out = a.out;
  p.mean = a.mean;
  p.rstd = a.rstd;
  p.partial = a.partial;
  p.eps = a.n.eps;
  p.width = a.n.width;
  p.param_type = a.n.param_type;
  if (p.rows == 0) {  // nothing to do but the gradients of no rows
    if (!p.partial) return cudaSuccess;
    return launch_pdl(k_fold_parts, (2 * p.width + 31) / 32, 32 * kFoldWarps, 0, st, true, p.partial, 0, p.width,
                      a.dweight, a.dbias);
  }
  // 16-byte vectors of x: whole ones in a row, aligned in every row of every tensor (y's have as many
  // elements, so 16 or, narrower than x, 8 bytes)
  const int xb = a.n.x_type == RESS_F32 ? 4 : 2, yb = a.n.y_type == RESS_F32 ? 4 : 2, E = 16 / xb;
  auto fits = [&](const void* q, int64_t stride, int bytes) {
    return !q || (reinterpret_cast<uintptr_t>(q) % (E * bytes) == 0 && (p.rows == 1 || stride % E == 0));
  };
  const bool vec = p.width % E == 0 && fits(a.x, p.x_stride, xb) && fits(a.dy, p.y_stride, yb) &&
                   fits(a.dres, p.dres_stride, xb) &&
                   fits(a.out, BWD ? p.dx_stride : p.y_stride, BWD ? xb : yb);
  switch (a.n.x_type * 4 + a.n.y_type) {
    case RESS_BF16 * 4 + RESS_BF16: return launch_norm_typed<BWD, bf16, bf16>(a, p, vec, st);
    case RESS_F16 * 4 + RESS_F16: return launch_norm_typed<BWD, f16, f16>(a, p, vec, st);
    case RESS_F32 * 4 + RESS_BF16: return launch_norm_typed<BWD, float, bf16>(a, p, vec, st);
    case RESS_F32 * 4 + RESS_F16: return launch_norm_typed<BWD, float, f16>(a, p, vec, st);
    default: return launch_norm_typed<BWD, float, float>(a, p, vec, st);
  }
}

}  // namespace

cudaError_t launch_layer_norm(const NormArgs& a, cudaStream_t st) { return launch_norm<false>(a, st); }
cudaError_t launch_layer_norm_bwd(const NormArgs& a, cudaStream_t st) { return launch_norm<true>(a, st); }

}  // namespace ress

// Layer norm over the rows of the residual stream, and its gradients.
//   forward   y = (x - m) r w + b,  m = avg(x),  r = 1 / sqrt(avg((x - m)^2) + eps)
//   backward  with h = (x - m) r and g = dy w:
//             dx = r (g - avg(g) - h avg(g h)) [+ dres],  dw = sum over rows of dy h,  db = of dy
// avg and the sums are over the row's channels.  One pass over the data: a row's elements stay in
// registers, as they lie in memory, between its sums and its result.
//
// A row belongs to a team, 8 to 32 lanes of a warp or a CTA, each thread C channels of it, and a team
// takes R rows at a time, the next ones' elements on their way while it works on these:
//   forward   a warp has up to 1024 16-bit channels (C = 32), so that rows of that width need no barrier,
//             and keeps their weights and biases in registers (43,968 x 1024 bf16: 53 us with C = 8 on
//             four warps, 35 with the next rows under way, 33 with a warp per row; 36 where it reads
//             float32 parameters from L1 for each row; a device copy of the same bytes takes 31).
//             float32 elements take twice the registers: above 896 channels
//             C = 16;
//   backward  C = 8, because a thread keeps its channels' two gradient sums in registers: with C = 32
//             they leave room for 8 warps per SM (80 us), with C = 8 for 16 (63 us, and a barrier per
//             R = 2 rows).  Above 4096 channels C = 16, above 8192 C = 32 and the sums in shared memory.
// Rows that are no whole vectors of 16 bytes, or not aligned to them, are taken as the aligned vectors that they
// have and the elements at their two edges, one to a thread (EDGES: 20,000 x 1021 bf16 22.5 us, and 37 element by
// element; 3000 x 8191 28 and 123; 5003 x 1021 float32 to bf16 7.5 and 12.2; the gradient of the first 41 and 57;
// rows of whole vectors take 16, 21, 7 and 30).  A team's rows are then a whole number of vectors apart, so that
// its channels' parameters stay in registers all the same.  Up to 256 channels, for few rows, and where the tensors'
// rows start at different places of a vector they go element by element, C = 8 (32 above 4096 channels).
// The mean is subtracted before squares are taken (two sums, one after the other): rows with an offset
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
  int width, param_type;
};

// A team: TEAM lanes of a warp (8, 16 or 32), or all the warps of a CTA.
constexpr int kWholeCta = 0;
template <int TEAM>
constexpr int kLanes = TEAM == kWholeCta ? 32 : TEAM;  // that share a row in a warp

template <int TEAM>
struct Team {
  int64_t index, count;  // in the grid
  int t, threads;        // this thread's place in it, its threads
  __device__ Team() {
    threads = TEAM == kWholeCta ? (int)blockDim.x : TEAM;
    t = TEAM == kWholeCta ? (int)threadIdx.x : (int)threadIdx.x % kLanes<TEAM>;
    const int per_cta = TEAM == kWholeCta ? 1 : kNormThreads / kLanes<TEAM>;
    index = (int64_t)blockIdx.x * per_cta + (TEAM == kWholeCta ? 0 : (int)threadIdx.x / kLanes<TEAM>);
    count = (int64_t)gridDim.x * per_cta;
  }
  // The row that the first team of this warp is at: teams of a warp go through their loop together,
  // because their lanes take part in each other's shuffles.
  __device__ int64_t lead(int64_t row, int rows) const {
    if constexpr (kLanes<TEAM> == 32) return row;
    return row - (int)(threadIdx.x % 32) / kLanes<TEAM> * rows;
  }
};

// Sums over a team's threads of N values each: over the warp's lanes, then over the CTA's warps
// through shared memory.  The two halves of `red` take turns, so that one barrier per call is enough:
// a warp that writes a half again has passed the barrier of the call in between, which every warp
// reaches after reading.
template <int TEAM, int N>
__device__ __forceinline__ void team_sum(float (&v)[N], float* red, int& turn) {
  if constexpr (TEAM != kWholeCta) {
    if constexpr (N > 1 && N <= TEAM) {
      const float r = segment_sums<TEAM>(v);
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = __shfl_sync(0xffffffffu, r, k * (TEAM / N), TEAM);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] = segment_sum<TEAM>(v[k]);
    }
  } else {
    constexpr int kSpan = 32 / N;  // lanes that hold the same value's sum
    const float r = segment_sums<32>(v);
    float* at = red + turn * (16 * N);
    turn ^= 1;
    const int lane = (int)threadIdx.x & 31;
    if (lane % kSpan == 0) at[((int)threadIdx.x >> 5) * N + lane / kSpan] = r;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.f;
    for (int w = 0; w < (int)blockDim.x / 32; ++w) {
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += at[w * N + k];
    }
  }
}

// A thread's channels are vectors of E, a team's threads next to each other: vector i of thread t
// starts at channel (t + i threads) E.
// EDGES: rows that start between vectors and need not be whole ones.  The channels before the row's first
// aligned vector and after its last one, at most E - 1 each, go one to a thread beside its vectors.
template <int E, int TEAM, bool EDGES>
struct Place {
  int first, step, end;  // of the vectors
  int edge;              // this thread's channel at an edge, or -1
  __device__ Place(const Team<TEAM>& team, int width, int head) : first(team.t * E), step(team.threads * E), end(width), edge(-1) {
    if (EDGES) {
      const int tail = (width - head) % E, k = team.t - 8;
      first += head;
      end -= tail;
      edge = team.t < head ? team.t : k >= 0 && k < tail ? end + k : -1;
    }
  }
  __device__ int col(int i) const { return first + i * (TEAM == kWholeCta ? step : TEAM * E); }
  __device__ bool in(int i) const { return col(i) < end; }
};

// Elements before the first aligned vector of a row, the same for all rows of a team: they are team.count rows
// apart, whole vectors.
template <typename X, int E>
__device__ __forceinline__ int head_of(const void* x, int64_t row, int64_t stride) {
  return (int)(-(reinterpret_cast<uintptr_t>(x) / sizeof(X) + (uint64_t)(row * stride)) % E);
}

template <typename T, int E, int V, int TEAM, bool EDGES>
__device__ __forceinline__ void load_row(Vec<T, E> (&r)[V], Vec<T, 1>& edge, const void* p, int64_t row, int64_t stride,
                                         const Place<E, TEAM, EDGES>& at, bool live) {
  const T* x = static_cast<const T*>(p) + row * stride;
#pragma unroll
  for (int i = 0; i < V; ++i) r[i] = live && at.in(i) ? load_vec<T, E>(x + at.col(i)) : zero_vec<T, E>();
  if (EDGES) edge = live && at.edge >= 0 ? load_vec<T, 1>(x + at.edge) : zero_vec<T, 1>();
}

// E parameters at a channel that need not be a vector's.
template <typename T, int E>
__device__ __forceinline__ void params_each(const void* p, int col, float* out) {
  T v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = static_cast<const T*>(p)[col + e];
#pragma unroll
  for (int e = 0; e < E; ++e) out[e] = to_f32(v[e]);
}
template <int E, bool EDGES>
__device__ __forceinline__ void row_params(const void* p, int type, int col, float none, float* out) {
  if (!EDGES || !p)
    params_at<E>(p, type, col, none, out);
  else if (type == RESS_F32)
    params_each<float, E>(p, col, out);
  else if (type == RESS_BF16)
    params_each<bf16, E>(p, col, out);
  else
    params_each<f16, E>(p, col, out);
}

template <typename X, typename Y, int E, int C, int TEAM, int R, bool EDGES>
__global__ void __launch_bounds__(TEAM == kWholeCta ? kNormMaxThreads : kNormThreads, TEAM == kWholeCta ? 1 : 4)
    k_layer_norm(const NormParams p) {
  __shared__ float red[2 * 16 * R];
  constexpr int V = C / E, P = C / 2;
  // where elements take a register each, 32 channels leave no room for the next row and the parameters
  constexpr bool kKeep = C < 32 || (E > 1 && sizeof(X) == 2), kAhead = kKeep || E > 1;
  const Team<TEAM> team;
  // a team's R rows are next to each other or (EDGES) as far apart as its visits
  const int64_t start = EDGES ? team.index : team.index * R, gap = EDGES ? team.count : 1;
  const Place<E, TEAM, EDGES> at(team, p.width, EDGES ? head_of<X, E>(p.x, team.index, p.x_stride) : 0);
  const float inv = 1.f / (float)p.width;
  int turn = 0;
  stream_acquire();
  F2 w[kKeep ? P : 1], b[kKeep ? P : 1];
  if constexpr (kKeep) {
    float v[2][C];
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[0][i * E + e] = v[1][i * E + e] = 0.f;
      if (!at.in(i)) continue;
      row_params<E, EDGES>(p.weight, p.param_type, at.col(i), 1.f, v[0] + i * E);
      row_params<E, EDGES>(p.bias, p.param_type, at.col(i), 0.f, v[1] + i * E);
    }
#pragma unroll
    for (int j = 0; j < P; ++j) {
      w[j] = pack2(v[0][2 * j], v[0][2 * j + 1]);
      b[j] = pack2(v[1][2 * j], v[1][2 * j + 1]);
    }
  }
  float edge_w = 0.f, edge_b = 0.f;
  if (EDGES && at.edge >= 0) {
    edge_w = param_at(p.weight, p.param_type, at.edge, 1.f);
    edge_b = param_at(p.bias, p.param_type, at.edge, 0.f);
  }
  Vec<X, E> next[R][V];
  Vec<X, 1> next_edge[R];
  auto load = [&](int64_t row0) {
#pragma unroll
    for (int k = 0; k < R; ++k)
      load_row<X, E, V>(next[k], next_edge[k], p.x, row0 + k * gap, p.x_stride, at, row0 + k * gap < p.rows);
  };
  if (kAhead) load(start);
  for (int64_t row0 = start; team.lead(row0, EDGES ? 1 : R) < p.rows; row0 += team.count * R) {
    if (!kAhead) load(row0);
    Vec<X, E> raw[R][V];
    float edge[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
#pragma unroll
      for (int i = 0; i < V; ++i) raw[k][i] = next[k][i];
      if (EDGES) edge[k] = elem(next_edge[k], 0);
    }
    if (kAhead) load(row0 + team.count * R);
    // a thread's sums are scaled before the threads' meet: a row's sum may overflow where its average
    // does not
    float mean[R], rstd[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      F2 s = both(0.f);
#pragma unroll
      for (int j = 0; j < P; ++j) s = add2(s, pair_of(raw[k], j));
      mean[k] = (EDGES ? sum2(s) + edge[k] : sum2(s)) * inv;
    }
    team_sum<TEAM>(mean, red, turn);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if constexpr (E == 1) {
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float d = at.in(i) ? elem(raw[k][i], 0) - mean[k] : 0.f;
          sq = fmaf(d, d, sq);
        }
        rstd[k] = sq * inv;
      } else {
        const F2 m = both(-mean[k]);
        F2 s = both(0.f);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          if (!at.in(i)) continue;
#pragma unroll
          for (int j = i * E / 2; j < (i + 1) * E / 2; ++j) {
            const F2 d = add2(pair_of(raw[k], j), m);
            s = fma2(d, d, s);
          }
        }
        const float d = EDGES && at.edge >= 0 ? edge[k] - mean[k] : 0.f;
        rstd[k] = fmaf(d, d, sum2(s)) * inv;
      }
    }
    team_sum<TEAM>(rstd, red, turn);
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t row = row0 + k * gap;
      if (row >= p.rows) continue;
      const float r = rsqrtf(rstd[k] + p.eps);
      Y* y = static_cast<Y*>(p.out) + row * p.y_stride;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!at.in(i)) continue;
        float out[E];
        if constexpr (kKeep && E > 1) {
#pragma unroll
          for (int j = 0; j < E / 2; ++j) {
            const F2 h = mul2(add2(pair_of(raw[k], i * E / 2 + j), both(-mean[k])), both(r));
            unpack2(fma2(h, w[i * E / 2 + j], b[i * E / 2 + j]), out[2 * j], out[2 * j + 1]);
          }
        } else {
          float v[2][E];
          if constexpr (kKeep) {  // E = 1
            float a, c;
            unpack2(w[i / 2], a, c);
            v[0][0] = i % 2 ? c : a;
            unpack2(b[i / 2], a, c);
            v[1][0] = i % 2 ? c : a;
          } else {
            row_params<E, EDGES>(p.weight, p.param_type, at.col(i), 1.f, v[0]);
            row_params<E, EDGES>(p.bias, p.param_type, at.col(i), 0.f, v[1]);
          }
#pragma unroll
          for (int e = 0; e < E; ++e) out[e] = fmaf((elem(raw[k][i], e) - mean[k]) * r, v[0][e], v[1][e]);
        }
        store_vec<Y, E>(y + at.col(i), out);
      }
      if (EDGES && at.edge >= 0) y[at.edge] = from_f32<Y>(fmaf((edge[k] - mean[k]) * r, edge_w, edge_b));
      if (team.t == 0) {
        if (p.mean) p.mean[row] = mean[k];
        if (p.rstd) p.rstd[row] = r;
      }
    }
  }
  stream_release();
}

template <typename X, typename Y, int E, int C, int TEAM, int R, bool EDGES>
__global__ void __launch_bounds__(TEAM == kWholeCta ? kNormMaxThreads : kNormThreads, TEAM == kWholeCta ? 1 : 4)
    k_layer_norm_bwd(const NormParams p) {
  __shared__ float red[2 * 16 * 2 * R];
  extern __shared__ float wide[];  // C = 32: the threads' gradient sums, each at its own places
  constexpr int V = C / E, P = C / 2;
  constexpr bool kKeep = C <= 16;
  const Team<TEAM> team;
  // a team's R rows are next to each other or (EDGES) as far apart as its visits
  const int64_t start = EDGES ? team.index : team.index * R, gap = EDGES ? team.count : 1;
  const Place<E, TEAM, EDGES> at(team, p.width, EDGES ? head_of<X, E>(p.x, team.index, p.x_stride) : 0);
  const float inv = 1.f / (float)p.width;
  int turn = 0;
  stream_acquire();
  // Channels past the row's end have a weight, a dy and so every sum of the row of 0.
  float w[C];
  F2 dw[kKeep ? P : 1], db[kKeep ? P : 1];
  auto weights = [&](int i) {
#pragma unroll
    for (int e = 0; e < E; ++e) w[i * E + e] = 0.f;
    if (at.in(i)) row_params<E, EDGES>(p.weight, p.param_type, at.col(i), 1.f, w + i * E);
  };
  const float edge_w = EDGES && at.edge >= 0 ? param_at(p.weight, p.param_type, at.edge, 1.f) : 0.f;
  float edge_dw = 0.f, edge_db = 0.f;
  if (kKeep) {
#pragma unroll
    for (int i = 0; i < V; ++i) weights(i);
#pragma unroll
    for (int j = 0; j < (kKeep ? P : 1); ++j) dw[j] = db[j] = both(0.f);
  } else {
#pragma unroll
    for (int c = 0; c < 2 * C; ++c) wide[c * team.threads + team.t] = 0.f;
  }
  constexpr bool kAhead = kKeep;  // the next rows fit in the registers too
  Vec<X, E> next_x[R][V], next_res[R][V];
  Vec<Y, E> next_dy[R][V];
  Vec<X, 1> next_edge_x[R], next_edge_res[R];
  Vec<Y, 1> next_edge_dy[R];
  float next_mean[R], next_rstd[R];
  auto load = [&](int64_t row0) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t row = row0 + k * gap;
      const bool live = row < p.rows;
      load_row<X, E, V>(next_x[k], next_edge_x[k], p.x, row, p.x_stride, at, live);
      load_row<Y, E, V>(next_dy[k], next_edge_dy[k], p.y, row, p.y_stride, at, live);
      if (p.dres) load_row<X, E, V>(next_res[k], next_edge_res[k], p.dres, row, p.dres_stride, at, live);
      next_mean[k] = live ? p.mean[row] : 0.f;
      next_rstd[k] = live ? p.rstd[row] : 0.f;
    }
  };
  if (kAhead) load(start);
  for (int64_t row0 = start; team.lead(row0, EDGES ? 1 : R) < p.rows; row0 += team.count * R) {
    if (!kAhead) load(row0);
    Vec<X, E> x[R][V], res[R][V];
    Vec<Y, E> dy[R][V];
    float r[R], mr[R];  // 1 / standard deviation, mean
    float edge_x[R], edge_res[R], edge_dy[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[k][i] = next_x[k][i];
        dy[k][i] = next_dy[k][i];
        res[k][i] = next_res[k][i];
      }
      mr[k] = next_mean[k];
      r[k] = next_rstd[k];
      if (EDGES) {
        edge_x[k] = elem(next_edge_x[k], 0);
        edge_dy[k] = elem(next_edge_dy[k], 0);
        edge_res[k] = p.dres ? elem(next_edge_res[k], 0) : 0.f;
      }
    }
    if (kAhead) load(row0 + team.count * R);
    // h = (x - mean) r, in this order: the difference keeps the digits of rows far from 0
    auto centred = [&](int k, int j) { return add2(pair_of(x[k], j), both(-mr[k])); };
    auto h_of = [&](int k, int j) { return mul2(centred(k, j), both(r[k])); };
    float sums[2 * R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      // sum of g h as r times that of g (x - mean): past the row's end x, dy and g are 0, and (0 - mean) r may be
      // infinite, but mean is not
      F2 sg = both(0.f), sgc = both(0.f);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        if (!kKeep && 2 * j % E == 0) weights(2 * j / E);
        if (!kKeep && E == 1) weights(2 * j + 1);
        const F2 d = pair_of(dy[k], j), c = centred(k, j), h = mul2(c, both(r[k])), g = mul2(d, pack2(w[2 * j], w[2 * j + 1]));
        sg = add2(sg, g);
        sgc = fma2(g, c, sgc);
        if constexpr (kKeep) {
          dw[j] = fma2(d, h, dw[j]);
          db[j] = add2(db[j], d);
        } else {
          float v[4];
          unpack2(mul2(d, h), v[0], v[1]);
          unpack2(d, v[2], v[3]);
#pragma unroll
          for (int q = 0; q < 4; ++q) wide[(C * (q / 2) + 2 * j + q % 2) * team.threads + team.t] += v[q];
        }
      }
      float g = sum2(sg), gc = sum2(sgc);
      if (EDGES && at.edge >= 0) {
        const float c = edge_x[k] - mr[k], ge = edge_dy[k] * edge_w;
        g += ge;
        gc = fmaf(ge, c, gc);
        edge_dw = fmaf(edge_dy[k], c * r[k], edge_dw);
        edge_db += edge_dy[k];
      }
      sums[2 * k] = g * inv;
      sums[2 * k + 1] = gc * inv;
    }
    team_sum<TEAM>(sums, red, turn);
#pragma unroll
    for (int k = 0; k < R; ++k) sums[2 * k + 1] *= r[k];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const int64_t row = row0 + k * gap;
      if (row >= p.rows) continue;
      const F2 ag = both(-sums[2 * k]), agh = both(-sums[2 * k + 1]), r2 = both(r[k]);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!at.in(i)) continue;
        float out[E];
        if constexpr (E > 1) {
          if (!kKeep) weights(i);
#pragma unroll
          for (int j = i * E / 2; j < (i + 1) * E / 2; ++j) {
            const F2 g = fma2(pair_of(dy[k], j), pack2(w[2 * j], w[2 * j + 1]), ag);
            F2 d = mul2(fma2(h_of(k, j), agh, g), r2);
            if (p.dres) d = add2(d, pair_of(res[k], j));
            unpack2(d, out[2 * j - i * E], out[2 * j + 1 - i * E]);
          }
        } else {
          if (!kKeep) weights(i);
          const float h = (elem(x[k][i], 0) - mr[k]) * r[k], g = elem(dy[k][i], 0) * w[i];
          out[0] = r[k] * (g - sums[2 * k] - h * sums[2 * k + 1]);
          if (p.dres) out[0] += elem(res[k][i], 0);
        }
        store_vec<X, E>(static_cast<X*>(p.out) + row * p.dx_stride + at.col(i), out);
      }
      if (EDGES && at.edge >= 0) {
        const float h = (edge_x[k] - mr[k]) * r[k], g = edge_dy[k] * edge_w;
        const float d = r[k] * (g - sums[2 * k] - h * sums[2 * k + 1]);
        static_cast<X*>(p.out)[row * p.dx_stride + at.edge] = from_f32<X>(p.dres ? d + edge_res[k] : d);
      }
    }
  }
  stream_release();
  if (!p.partial) return;
  // the CTA's partial rows: segments of a warp, then (teams of up to a warp) the CTA's warps in order
  float* out = p.partial + (int64_t)blockIdx.x * 2 * p.width;
  if constexpr (TEAM == kWholeCta) {
    if (EDGES && at.edge >= 0) {
      out[at.edge] = edge_dw;
      out[p.width + at.edge] = edge_db;
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = at.col(c / E) + c % E;
      if (col >= at.end) continue;
      float v[2];
      if constexpr (kKeep) {
        float a, b;
        unpack2(dw[c / 2], a, b);
        v[0] = c % 2 ? b : a;
        unpack2(db[c / 2], a, b);
        v[1] = c % 2 ? b : a;
      } else {
        v[0] = wide[c * team.threads + team.t];
        v[1] = wide[(C + c) * team.threads + team.t];
      }
      out[col] = v[0];
      out[p.width + col] = v[1];
    }
  } else {
    static_assert(kKeep && !EDGES, "a lane's sums are in registers, of the same channels in every team");
    __shared__ float part[kNormThreads / 32][2][32 * C];
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float a, b, v[2];
      unpack2(dw[c / 2], a, b);
      v[0] = c % 2 ? b : a;
      unpack2(db[c / 2], a, b);
      v[1] = c % 2 ? b : a;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int o = TEAM; o < 32; o <<= 1) v[q] += __shfl_xor_sync(0xffffffffu, v[q], o);
        if (lane < TEAM) part[warp][q][at.col(c / E) + c % E] = v[q];
      }
    }
    __syncthreads();
    for (int k = (int)threadIdx.x; k < 2 * p.width; k += kNormThreads) {
      const int a = k >= p.width, col = k - a * p.width;
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

// CTAs of the launch: as many as fit on the GPU at once at most, all with the same number of steps but
// for the last ones.  (A team of a CTA has the threads its rows' width asks for: `resident` is for the
// threads at hand.)
int norm_ctas(int resident, int teams_per_cta, int64_t batches, int most) {
  const int64_t ctas = (batches + teams_per_cta - 1) / teams_per_cta;
  const int64_t fit = min((int64_t)resident * sm_count(), (int64_t)most);
  const int64_t steps = (ctas + fit - 1) / fit;
  return (int)((ctas + steps - 1) / steps);
}

// EDGES: a team's rows start at the same place of a vector if their distance, the teams of the grid, is a
// multiple of its elements, `of` CTAs'.  kEdgeRows make at least that many.
constexpr int kEdgeRows = 64;
int same_heads(int ctas, int of) { return of <= 1 ? ctas : ctas / of * of; }

template <bool BWD, typename X, typename Y, int E, int C, int TEAM, bool ONE = false, bool EDGES = false>
cudaError_t launch_norm_as(const NormArgs& a, const NormParams& p, cudaStream_t st) {
  constexpr bool wide = sizeof(X) == 4 || E == 1;  // elements that take a register each as they lie
  const int threads = TEAM == kWholeCta ? ((p.width + C - 1) / C + 31) / 32 * 32 : kNormThreads;
  const int per_cta = TEAM == kWholeCta ? 1 : kNormThreads / kLanes<TEAM>;
  if constexpr (!BWD) {
    constexpr int R = C == 32 || ONE ? 1 : wide ? 16 / C : 32 / C;
    constexpr auto kern = k_layer_norm<X, Y, E, C, TEAM, R, EDGES>;
    int fit = 0;
    const cudaError_t e = resident_ctas<kern>(threads, 0, fit);
    if (e != cudaSuccess) return e;
    int ctas = norm_ctas(fit, per_cta, (p.rows + R - 1) / R, INT32_MAX);
    if (EDGES) ctas = same_heads(ctas, E / per_cta);
    return launch_pdl(kern, ctas, threads, 0, st, true, p);
  } else {
    constexpr int R = C > 8 || wide ? 1 : 2;
    constexpr auto kern = k_layer_norm_bwd<X, Y, E, C, TEAM, R, EDGES>;
    // what the kernel may have is set for its largest CTA, the same by every call: the setting is the kernel's,
    // and calls of other widths on other host threads set it between this call's setting and its launch
    constexpr size_t kThreadSmem = C <= 16 ? 0 : 2 * C * sizeof(float), kMostSmem = kThreadSmem * kNormMaxThreads;
    const size_t smem = kThreadSmem * threads;
    cudaError_t e = cudaSuccess;
    if (kMostSmem > 0) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
    int fit = 0;
    if (e == cudaSuccess) e = resident_ctas<kern>(threads, smem, fit);
    if (e != cudaSuccess) return e;
    int ctas = norm_ctas(fit, per_cta, (p.rows + R - 1) / R, kNormParts);
    if (EDGES) ctas = same_heads(ctas, E / per_cta);
    e = launch_pdl(kern, ctas, threads, smem, st, true, p);
    if (e != cudaSuccess || !p.partial) return e;
    return launch_pdl(k_fold_parts, (2 * p.width + 31) / 32, 32 * kFoldWarps, 0, st, true, p.partial, ctas,
                      p.width, a.dweight, a.dbias);
  }
}

template <bool BWD, typename X, typename Y>
cudaError_t launch_norm_typed(const NormArgs& a, const NormParams& p, bool vec, bool edges, cudaStream_t st) {
  constexpr int E = 16 / (int)sizeof(X);
  const int D = p.width;
  if (!vec && edges && D > 256 && p.rows >= kEdgeRows) {
    if constexpr (BWD) {
      if (D <= 8 * kNormMaxThreads) return launch_norm_as<BWD, X, Y, E, 8, kWholeCta, false, true>(a, p, st);
      if (D <= 16 * kNormMaxThreads) return launch_norm_as<BWD, X, Y, E, 16, kWholeCta, false, true>(a, p, st);
    } else {
      if (D <= 512) return launch_norm_as<BWD, X, Y, E, 16, 32, false, true>(a, p, st);
      if constexpr (sizeof(X) == 4) {
        if (D <= 16 * kNormMaxThreads) return launch_norm_as<BWD, X, Y, E, 16, kWholeCta, false, true>(a, p, st);
      } else {
        if (D <= 1024) return launch_norm_as<BWD, X, Y, E, 32, 32, false, true>(a, p, st);
      }
    }
    return launch_norm_as<BWD, X, Y, E, 32, kWholeCta, false, true>(a, p, st);
  }
  if (!vec) {
    if (D <= 64) return launch_norm_as<BWD, X, Y, 1, 8, 8>(a, p, st);
    if (D <= 128) return launch_norm_as<BWD, X, Y, 1, 8, 16>(a, p, st);
    if (D <= 256) return launch_norm_as<BWD, X, Y, 1, 8, 32>(a, p, st);
    // one row at a time where the CTAs get large: rows of 2 leave one CTA of 9 warps per SM (21,961 x 2049
    // bf16: 141 us and 117 one at a time; 44,955 x 1001: 82 and 96)
    if (D <= 4 * kNormMaxThreads || (BWD && D <= 8 * kNormMaxThreads))
      return launch_norm_as<BWD, X, Y, 1, 8, kWholeCta>(a, p, st);
    if constexpr (!BWD)
      if (D <= 8 * kNormMaxThreads) return launch_norm_as<BWD, X, Y, 1, 8, kWholeCta, true>(a, p, st);
    return launch_norm_as<BWD, X, Y, 1, 32, kWholeCta>(a, p, st);
  }
  if (D <= 64) return launch_norm_as<BWD, X, Y, E, 8, 8>(a, p, st);
  if (D <= 128) return launch_norm_as<BWD, X, Y, E, 8, 16>(a, p, st);
  if (D <= 256) return launch_norm_as<BWD, X, Y, E, 8, 32>(a, p, st);
  if constexpr (BWD) {
    if (D <= 8 * kNormMaxThreads) return launch_norm_as<BWD, X, Y, E, 8, kWholeCta>(a, p, st);
    if (D <= 16 * kNormMaxThreads) return launch_norm_as<BWD, X, Y, E, 16, kWholeCta>(a, p, st);
  } else {
    if (D <= 512) return launch_norm_as<BWD, X, Y, E, 16, 32>(a, p, st);
    if constexpr (sizeof(X) == 4) {
      // a warp per row reads its parameters anew for each (20,000 x 1024 to bf16: 25.8 us, two warps per row that
      // keep them 23.8; x 640, where the second warp is mostly idle: 17.5 and 18.7)
      if (D <= 896) return launch_norm_as<BWD, X, Y, E, 32, 32>(a, p, st);
      if (D <= 16 * kNormMaxThreads) return launch_norm_as<BWD, X, Y, E, 16, kWholeCta>(a, p, st);
    } else if (D <= 1024) {
      return launch_norm_as<BWD, X, Y, E, 32, 32>(a, p, st);
    }
  }
  return launch_norm_as<BWD, X, Y, E, 32, kWholeCta>(a, p, st);
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
  auto fits_params = [&](const void* q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
  const bool vec = p.width % E == 0 && fits_params(a.weight) && fits_params(a.bias) && fits(a.x, p.x_stride, xb) && fits(a.dy, p.y_stride, yb) &&
                   fits(a.dres, p.dres_stride, xb) &&
                   fits(a.out, BWD ? p.dx_stride : p.y_stride, BWD ? xb : yb);
  // rows that start at any element, but all tensors' at the same one of a vector
  const uintptr_t place = reinterpret_cast<uintptr_t>(a.x) / xb % E;
  auto same = [&](const void* q, int64_t stride, int bytes) {
    return !q || (reinterpret_cast<uintptr_t>(q) / bytes % E == place && (stride - p.x_stride) % E == 0);
  };
  const bool edges = same(a.dy, p.y_stride, yb) && same(a.dres, p.dres_stride, xb) &&
                     same(a.out, BWD ? p.dx_stride : p.y_stride, BWD ? xb : yb);
  switch (a.n.x_type * 4 + a.n.y_type) {
    case RESS_BF16 * 4 + RESS_BF16: return launch_norm_typed<BWD, bf16, bf16>(a, p, vec, edges, st);
    case RESS_F16 * 4 + RESS_F16: return launch_norm_typed<BWD, f16, f16>(a, p, vec, edges, st);
    case RESS_F32 * 4 + RESS_BF16: return launch_norm_typed<BWD, float, bf16>(a, p, vec, edges, st);
    case RESS_F32 * 4 + RESS_F16: return launch_norm_typed<BWD, float, f16>(a, p, vec, edges, st);
    default: return launch_norm_typed<BWD, float, float>(a, p, vec, edges, st);
  }
}

}  // namespace

cudaError_t launch_layer_norm(const NormArgs& a, cudaStream_t st) { return launch_norm<false>(a, st); }
cudaError_t launch_layer_norm_bwd(const NormArgs& a, cudaStream_t st) { return launch_norm<true>(a, st); }

}  // namespace ress

// Rotary positions over several axes on the heads of Q and K, after a layer norm over each head's
// channels where there is one, and the gradients of both.
//   forward   u = (x - m) r w + b over the head's channels (or u = x), then for each pair (i, j) of
//             channels with its angle t:  y_i = u_i cos t - u_j sin t,  y_j = u_j cos t + u_i sin t
//   backward  du = the same of dy with -t;  dx = du, or with h = (x - m) r and g = du w:
//             dx = r (g - avg(g) - h avg(g h)),  dw = sum over tokens and heads of du h,  db = of du
// Memory-bound in bytes, but every element takes part in two sums and a rotation: with 248
// instructions per row of 4 heads of 64 the instructions took 111 us of the 53 that the bytes need
// (43,968 tokens, 16 + 16 heads, bf16), so the kernel is laid out for few of them.
//
// A lane holds S = 4 or 8 slots, each the two channels of a pair (or two channels without a pair), so
// that a rotation needs no other lane, and a head has G lanes.  Where the plan's pairs are S and S
// neighbouring channels (kChunks) or 2 S neighbours (kNeighbours) they are read and written as
// vectors, else one by one (kGather).  An item is one token and up to K rows of 32 / G of its heads
// of one tensor, and a warp has the next item's elements on their way while it works on one.  A CTA
// stays with Q or K (shares of the grid by their cost), and its lanes keep the norm's parameters
// and their gradients' sums in registers.  Where the heads fit into one row (FEW), a row has as
// many tokens as it has room for, and an item K such rows (1 head of 32 channels, a row of 8 for each: 13
// times the bytes' time).  The token's cosines and sines are formed once per item,
// one pair per lane, and handed out through shared memory.  Sums are float32 in a fixed order; the
// gradients of the parameters are summed per CTA and then over CTAs by a second kernel.
#pragma once

#include "row_ops.cuh"

namespace ress {
using namespace rows;

enum { kChunks = 0, kNeighbours = 1, kGather = 2 };

struct RopeTensor {
  int heads;
  const void *weight, *bias;
  const void *x, *y;  // y: backward dy
  void* out;          // forward y, backward dx
  int64_t x_token, x_head, y_token, y_head, out_token, out_head;  // strides in elements
};

struct RopeParams {
  ress_rope_plan plan;
  RopeTensor t[2];
  int64_t tokens;
  const int32_t* pos;
  float* partial;
  float eps;
  int most;           // CTAs at most
  int first_ctas;     // CTAs of t[0]; the others have t[1]
  int param_type;
  bool whole_tokens;  // a warp takes all of a token's items
  bool all;           // every channel has a pair
};

// Which kernel a tensor gets; tensors of one kind share a launch.
struct RopeKind {
  bool norm, few;   // few: several tokens per item
  int mode, slots;  // S
  int tokens;       // that fit into a row
  bool operator==(const RopeKind& k) const {
    return norm == k.norm && few == k.few && mode == k.mode && slots == k.slots;
  }
};

// The launches of tensors of one kind (p.t with 0 heads: absent); ctas: of each.  Few: k_rope_few.cu.
cudaError_t launch_rope_few(bool bwd, const RopeKind& kind, int type, RopeParams& p, int (&ctas)[2], cudaStream_t st);

namespace {

constexpr int kRopeWarps = 4;
constexpr int kRopeThreads = 32 * kRopeWarps;

// The channels of a slot.  Slots past the pairs have channels without one, if any are left: two
// neighbours, or (kChunks) those of a lane's S slots as S and S neighbours.
template <int MODE, int S>
__device__ __forceinline__ void slot_channels(const ress_rope_plan& p, int slot, int& a, int& b) {
  if (slot >= p.n_pairs) {
    const int i = slot - p.n_pairs;
    a = MODE == kChunks ? 2 * p.n_pairs + i / S * 2 * S + i % S : 2 * p.n_pairs + 2 * i;
    b = MODE == kChunks ? a + S : a + 1;
    return;
  }
  if (p.layout == RESS_ROPE_INTERLEAVED) {
    a = 2 * slot, b = 2 * slot + 1;
  } else if (p.layout == RESS_ROPE_HALVES) {
    a = slot, b = slot + p.n_pairs;
  } else {
    const int axis = rope_axis(p, slot);
    int start = 0;
    for (int i = 0; i < axis; ++i) start += p.axis_dims[i];
    a = start + slot - start / 2;
    b = a + p.axis_dims[axis] / 2;
  }
}

// A lane's 2 S elements: the first channels of its slots, then the second ones (kNeighbours: as they
// lie).
template <typename T, int MODE, int S>
struct Slots {
  const int *a, *b;  // kGather: the slots' channels
  bool in[S];        // the slots that exist
  bool any;          // (not kGather: all or none)
  int first, next;   // kChunks, kNeighbours: the lane's vectors

  __device__ Vec<T, 2 * S> load(const T* p, bool live) const {
    Vec<T, 2 * S> r = zero_vec<T, 2 * S>();
    if (!live || !any) return r;
    if constexpr (MODE == kNeighbours) {
      r = load_vec<T, 2 * S>(p + first);
    } else if constexpr (MODE == kChunks) {
      const Vec<T, S> u = load_vec<T, S>(p + first), v = load_vec<T, S>(p + next);
      constexpr int W = Vec<T, S>::kWords;
#pragma unroll
      for (int k = 0; k < W; ++k) r.w[k] = u.w[k], r.w[W + k] = v.w[k];
    } else {
#pragma unroll
      for (int j = 0; j < S; ++j)
        if (in[j]) {
          put(r, j, p[a[j]]);
          put(r, S + j, p[b[j]]);
        }
    }
    return r;
  }
  __device__ static void put(Vec<T, 2 * S>& r, int j, T v) {
    if constexpr (sizeof(T) == 4)
      r.w[j] = __float_as_uint(v);
    else
      r.w[j / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(&v) << (16 * (j & 1));
  }
  // Slots 2 q and 2 q + 1: their first (side 0) or second channels.
  __device__ static F2 get(const Vec<T, 2 * S>& r, int side, int q) {
    if constexpr (MODE == kNeighbours) return pack2(elem(r, 4 * q + side), elem(r, 4 * q + 2 + side));
    const Vec<T, 2 * S> one[1] = {r};
    return pair_of(one, side * (S / 2) + q);
  }
  __device__ void store(T* p, const F2 (&u)[2][S / 2], bool live) const {
    if (!live || !any) return;
    float v[2][S];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int q = 0; q < S / 2; ++q) unpack2(u[s][q], v[s][2 * q], v[s][2 * q + 1]);
    if constexpr (MODE == kNeighbours) {
      float o[2 * S];
#pragma unroll
      for (int j = 0; j < S; ++j) o[2 * j] = v[0][j], o[2 * j + 1] = v[1][j];
      store_vec<T, 2 * S>(p + first, o);
    } else if constexpr (MODE == kChunks) {
      store_vec<T, S>(p + first, v[0]);
      store_vec<T, S>(p + next, v[1]);
    } else {
#pragma unroll
      for (int j = 0; j < S; ++j)
        if (in[j]) {
          p[a[j]] = from_f32<T>(v[0][j]);
          p[b[j]] = from_f32<T>(v[1][j]);
        }
    }
  }
};

template <typename T, int G, int MODE, int S, bool NORM, bool BWD, bool FEW, int K>
__global__ void __launch_bounds__(kRopeThreads, (!NORM ? 6 : BWD ? 3 : 4) - (S == 8 ? 1 : 0)) k_rope(const __grid_constant__ RopeParams p) {
  constexpr int kHeads = 32 / G;              // heads of a warp's row
  constexpr int kPairs = G * S <= 32 ? 1 : G * S / 32;  // pairs per lane: G S pairs at most
  constexpr int Q = S / 2;
  constexpr bool kReadX = !BWD || NORM;
  constexpr int kMostTokens = FEW ? K * kHeads : 1;  // tokens of an item
  __shared__ __align__(16) float cosines[kRopeWarps][kMostTokens][G * S], sines[kRopeWarps][kMostTokens][G * S];
  const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
  const bool second = (int)blockIdx.x >= p.first_ctas;
  // (one field at a time: an index into the parameters would be looked up at each use)
  RopeTensor t;
  t.heads = second ? p.t[1].heads : p.t[0].heads;
  t.weight = second ? p.t[1].weight : p.t[0].weight;
  t.bias = second ? p.t[1].bias : p.t[0].bias;
  t.x = second ? p.t[1].x : p.t[0].x;
  t.y = second ? p.t[1].y : p.t[0].y;
  t.out = second ? p.t[1].out : p.t[0].out;
  t.x_token = second ? p.t[1].x_token : p.t[0].x_token;
  t.x_head = second ? p.t[1].x_head : p.t[0].x_head;
  t.y_token = second ? p.t[1].y_token : p.t[0].y_token;
  t.y_head = second ? p.t[1].y_head : p.t[0].y_head;
  t.out_token = second ? p.t[1].out_token : p.t[0].out_token;
  t.out_head = second ? p.t[1].out_head : p.t[0].out_head;
  const int hd = p.plan.head_dim, heads = t.heads;
  const int group = lane / G, slot = lane % G * S;
  const float inv = 1.f / (float)hd;

  int a[S], b[S];
  Slots<T, MODE, S> slots;
#pragma unroll
  for (int j = 0; j < S; ++j) {
    slots.in[j] = 2 * (slot + j) < hd;
    slot_channels<MODE, S>(p.plan, min(slot + j, hd / 2 - 1), a[j], b[j]);
  }
  slots.a = a;
  slots.b = b;
  slots.any = slots.in[0];
  slots.first = a[0];
  slots.next = b[0];
  const bool turns = slot < p.plan.n_pairs;  // kGather: slots turn one by one
  // FEW: a row has row_tokens tokens, this lane's group the head my_head of the one of number my_token,
  // and an item has K such rows.
  const int row_tokens = FEW ? kHeads / heads : 1, item_tokens = FEW ? K * row_tokens : 1;
  const int my_token = FEW ? group / heads : 0, my_head = FEW ? group % heads : group;
  // The pairs whose angles this lane forms: of one token at a time, or (fewer than 32 pairs) of several.
  int span_pairs = 32;
  while (FEW && kPairs == 1 && span_pairs / 2 >= p.plan.n_pairs) span_pairs /= 2;
  const int first_pair = lane % span_pairs;
  uint64_t freq[kPairs];
  int axis[kPairs];
#pragma unroll
  for (int q = 0; q < kPairs; ++q) {
    const int k = min(first_pair + 32 * q, p.plan.n_pairs - 1);
    freq[q] = p.plan.turns[k];
    axis[q] = rope_axis(p.plan, k);
  }
  auto angle = [&](int token, int q, int32_t at) {  // of a token of the item
    const float2 cs = rope_cos_sin(at, freq[q]);
    if (first_pair + 32 * q < p.plan.n_pairs) {
      cosines[warp][token][first_pair + 32 * q] = cs.x;
      sines[warp][token][first_pair + 32 * q] = BWD ? -cs.y : cs.y;
    }
  };

  // Slots without a pair, and lanes without channels, turn by nothing: their sums stay what they are.
  if (p.plan.n_pairs < G * S) {
    for (int i = lane; i < kMostTokens * G * S; i += 32) {
      cosines[warp][0][i] = 1.f;
      sines[warp][0][i] = 0.f;
    }
  }

  stream_acquire();
  // [side][slots 2q and 2q + 1]
  F2 w[2][Q], shift[2][Q], dw[2][Q], db[2][Q];
#pragma unroll
  for (int s = 0; s < 2; ++s)
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      float v[2][2] = {};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int j = 2 * q + e, c = s ? b[j] : a[j];
        if (NORM && slots.in[j]) {
          v[0][e] = param_at(t.weight, p.param_type, c, 1.f);
          if (!BWD) v[1][e] = param_at(t.bias, p.param_type, c, 0.f);
        }
      }
      w[s][q] = pack2(v[0][0], v[0][1]);
      shift[s][q] = pack2(v[1][0], v[1][1]);
      dw[s][q] = db[s][q] = both(0.f);
    }

  // A token's items one after the other, so that they share its angles, or (few tokens) each by itself.
  const int chunks = (heads + K * kHeads - 1) / (K * kHeads);  // items of a token
  const int span = p.whole_tokens ? chunks : 1, spans = chunks / span;
  const int64_t warps = (int64_t)(second ? gridDim.x - p.first_ctas : p.first_ctas) * kRopeWarps;
  const int64_t w0 = (int64_t)(blockIdx.x - (second ? p.first_ctas : 0)) * kRopeWarps + warp;
  const int64_t step = warps / spans * item_tokens;
  const int step_rest = (int)(warps % spans);
  int64_t token = w0 / spans * item_tokens;
  int chunk = (int)(w0 % spans) * span, left = span;  // left: items of the span from this one on
  // from row to row of an item, and to this lane's place in the first
  auto row_step = [&](int64_t token_stride, int64_t head_stride) {
    return FEW ? row_tokens * token_stride : kHeads * head_stride;
  };
  auto place = [&](int64_t token_stride, int64_t head_stride) {
    return (token + my_token) * token_stride + (chunk * K * kHeads + my_head) * head_stride;
  };
  // whether this lane's head of row k exists
  auto lives = [&](int64_t at, int ch, int k) {
    if (FEW) return my_token < row_tokens && at + k * row_tokens + my_token < p.tokens;
    return at < p.tokens && (ch * K + k) * kHeads + group < heads;
  };
  const int64_t x_step = row_step(t.x_token, t.x_head), y_step = row_step(t.y_token, t.y_head);
  const int64_t out_step = row_step(t.out_token, t.out_head);
  // the next item's rows (and, a token by itself, its positions) are on their way while this one is
  // worked on
  Vec<T, 2 * S> next_x[kReadX ? K : 1], next_y[BWD ? K : 1];
  constexpr int kAhead = FEW && kPairs == 1 ? K : kPairs;
  int32_t pos[kAhead];
  const int sweep = FEW ? 32 / span_pairs : 1, sweep_token = FEW ? lane / span_pairs : 0;  // tokens per sweep of the lanes
  auto position = [&](int64_t item, int i, int q) {  // of this lane's token of sweep i
    const int64_t at = item + i * sweep + sweep_token;
    return at < p.tokens ? p.pos[at * p.plan.n_axes + axis[q]] : 0;
  };
  auto load = [&]() {
    const T *px = nullptr, *py = nullptr;
    if constexpr (kReadX) px = static_cast<const T*>(t.x) + place(t.x_token, t.x_head);
    if constexpr (BWD) py = static_cast<const T*>(t.y) + place(t.y_token, t.y_head);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool live = lives(token, chunk, k);
      if constexpr (kReadX) next_x[k] = slots.load(px + k * x_step, live);
      if constexpr (BWD) next_y[k] = slots.load(py + k * y_step, live);
    }
    if constexpr (kPairs == 1) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i == 0 || i * sweep < item_tokens) pos[i] = position(token, i, 0);
    } else {
#pragma unroll
      for (int q = 0; q < kPairs; ++q) pos[q] = position(token, 0, q);
    }
  };
  load();
#pragma unroll 1
  while (token < p.tokens) {
    Vec<T, 2 * S> x[kReadX ? K : 1], y[BWD ? K : 1];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if constexpr (kReadX) x[k] = next_x[k];
      if constexpr (BWD) y[k] = next_y[k];
    }
    if (left == span) {  // the angles of the item's tokens, once the last one's are read
      __syncwarp();
      if constexpr (kPairs == 1) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
          if (i * sweep + sweep_token < item_tokens) angle(i * sweep + sweep_token, 0, pos[i]);
        for (int i = kAhead; i * sweep < item_tokens; ++i)
          if (i * sweep + sweep_token < item_tokens) angle(i * sweep + sweep_token, 0, position(token, i, 0));
      } else {
#pragma unroll
        for (int q = 0; q < kPairs; ++q) angle(0, q, pos[q]);
        for (int i = 1; i < item_tokens; ++i) {
#pragma unroll
          for (int q = 0; q < kPairs; ++q) angle(i, q, position(token, i, q));
        }
      }
      __syncwarp();
    }
    const int64_t token0 = token;
    const int chunk0 = chunk;
    T* const out = static_cast<T*>(t.out) + place(t.out_token, t.out_head);
    ++chunk;
    if (--left == 0) {
      left = span;
      chunk += step_rest * span - span;
      token += step;
      if (chunk >= chunks) {
        chunk -= chunks;
        token += item_tokens;
      }
    }
    load();
    F2 co[Q], si[Q], neg[Q];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      // no head of this row
      if (FEW ? token0 + k * row_tokens >= p.tokens : (chunk0 * K + k) * kHeads >= heads) break;
      if (FEW || k == 0) {
        const int at = FEW ? k * row_tokens + min(my_token, row_tokens - 1) : 0;
#pragma unroll
        for (int q = 0; q < Q; q += 2) {
          const float4 c = *reinterpret_cast<const float4*>(&cosines[warp][at][slot + 2 * q]);
          const float4 z = *reinterpret_cast<const float4*>(&sines[warp][at][slot + 2 * q]);
          co[q] = pack2(c.x, c.y), co[q + 1] = pack2(c.z, c.w);
          si[q] = pack2(z.x, z.y), si[q + 1] = pack2(z.z, z.w);
          neg[q] = pack2(-z.x, -z.y), neg[q + 1] = pack2(-z.z, -z.w);
        }
      }
      const bool live = lives(token0, chunk0, k);
      F2 h[2][Q], u[2][Q];
      float rstd = 1.f;
      if constexpr (NORM) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int q = 0; q < Q; ++q) h[s][q] = Slots<T, MODE, S>::get(x[k], s, q);
        // a lane's sum is scaled before the lanes' meet: the sum may overflow where its average does not
        F2 sum[2] = {h[0][0], h[1][0]};
#pragma unroll
        for (int q = 1; q < Q; ++q) sum[0] = add2(sum[0], h[0][q]), sum[1] = add2(sum[1], h[1][q]);
        const float mean = segment_sum<G>(sum2(add2(sum[0], sum[1])) * inv);
        // lanes without channels have h = 0: (0 - mean) rstd may be infinite, and times u = 0 it would enter the
        // gradient's sums
        const F2 m = both(slots.any ? -mean : 0.f);
        F2 sq = both(0.f);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int q = 0; q < Q; ++q) {
            h[s][q] = add2(h[s][q], m);
            if constexpr (MODE == kGather) {  // slots that do not exist
              float e0, e1;
              unpack2(h[s][q], e0, e1);
              h[s][q] = pack2(slots.in[2 * q] ? e0 : 0.f, slots.in[2 * q + 1] ? e1 : 0.f);
            }
            sq = fma2(h[s][q], h[s][q], sq);
          }
        rstd = rsqrtf(segment_sum<G>(sum2(sq) * inv) + p.eps);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int q = 0; q < Q; ++q) {
            h[s][q] = mul2(h[s][q], both(rstd));
            if (!BWD) u[s][q] = fma2(h[s][q], w[s][q], shift[s][q]);
          }
      }
      if constexpr (BWD || !NORM) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int q = 0; q < Q; ++q) u[s][q] = Slots<T, MODE, S>::get(BWD ? y[k] : x[k], s, q);
      }
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        F2 r0 = fma2(u[0][q], co[q], mul2(u[1][q], neg[q])), r1 = fma2(u[1][q], co[q], mul2(u[0][q], si[q]));
        if (!p.all) {  // channels without a pair keep their bits
          if constexpr (MODE == kGather) {
            float v[4], k[4];
            unpack2(r0, v[0], v[1]);
            unpack2(r1, v[2], v[3]);
            unpack2(u[0][q], k[0], k[1]);
            unpack2(u[1][q], k[2], k[3]);
            const bool t0 = slot + 2 * q < p.plan.n_pairs, t1 = slot + 2 * q + 1 < p.plan.n_pairs;
            r0 = pack2(t0 ? v[0] : k[0], t1 ? v[1] : k[1]);
            r1 = pack2(t0 ? v[2] : k[2], t1 ? v[3] : k[3]);
          } else if (!turns) {
            r0 = u[0][q], r1 = u[1][q];
          }
        }
        u[0][q] = r0, u[1][q] = r1;
      }
      if constexpr (NORM && BWD) {
        // rows past the last head and slots that do not exist have dy = 0 and add nothing, but h may
        // be anything where x is not read
        F2 sg = both(0.f), sgh = both(0.f);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int q = 0; q < Q; ++q) {
            if (live) {
              dw[s][q] = fma2(u[s][q], h[s][q], dw[s][q]);
              db[s][q] = add2(db[s][q], u[s][q]);
            }
            u[s][q] = mul2(u[s][q], w[s][q]);
            sg = add2(sg, u[s][q]);
            sgh = fma2(u[s][q], h[s][q], sgh);
          }
        const F2 ag = both(-segment_sum<G>(sum2(sg) * inv)), agh = both(-segment_sum<G>(sum2(sgh) * inv));
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int q = 0; q < Q; ++q) u[s][q] = mul2(fma2(h[s][q], agh, add2(u[s][q], ag)), both(rstd));
      }
      slots.store(out + k * out_step, u, live);
    }
  }
  stream_release();
  if constexpr (NORM && BWD) {
    if (!p.partial) return;
    // the CTA's sums: a warp's groups, then its warps in order
    __shared__ float part[kRopeWarps][2][G * 2 * S];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        float v[2][2];
        unpack2(dw[s][q], v[0][0], v[0][1]);
        unpack2(db[s][q], v[1][0], v[1][1]);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int o = G; o < 32; o <<= 1) v[k][e] += __shfl_xor_sync(0xffffffffu, v[k][e], o);
            if (lane < G && slots.in[2 * q + e]) part[warp][k][s ? b[2 * q + e] : a[2 * q + e]] = v[k][e];
          }
      }
    __syncthreads();
    for (int k = (int)threadIdx.x; k < 2 * hd; k += kRopeThreads) {
      const int which = k >= hd, c = k - which * hd;
      float v = 0.f;
#pragma unroll
      for (int q = 0; q < kRopeWarps; ++q) v += part[q][which][c];
      p.partial[((int64_t)blockIdx.x * 2 + which) * hd + c] = v;
    }
  }
}

template <typename T, int G, int MODE, int S, bool NORM, bool BWD, bool FEW>
cudaError_t launch_rope_as(RopeParams& p, int (&ctas)[2], cudaStream_t st) {
  // Rows of an item, their elements in registers twice (43,968 tokens, 16 + 16 heads of 64, bf16, with a
  // norm: S = 4 and K = 4 67 us, K = 2 73; S = 8 and K = 2 66, K = 1 76; without one, 20,011 tokens,
  // 12 + 4 heads, S = 4: K = 4 22, K = 2 20.5; gradient with a norm, 10,992 tokens, both launches: S = 4 and
  // K = 2 36.5, K = 1 45; S = 8 and K = 2 33, K = 1 40).
  constexpr int K = S == 8 ? 2 : sizeof(T) == 2 ? (NORM && !BWD ? 4 : 2) : (NORM && BWD ? 1 : 2);
  constexpr int kHeads = 32 / G;
  constexpr auto kern = k_rope<T, G, MODE, S, NORM, BWD, FEW, K>;
  int resident = 0;
  const cudaError_t e = resident_ctas<kern>(kRopeThreads, 0, resident);
  if (e != cudaSuccess) return e;
  const int64_t fit = min((int64_t)resident * sm_count(), (int64_t)p.most);
  p.whole_tokens = p.tokens * ((p.t[0].heads > 0) + (p.t[1].heads > 0)) >= fit * kRopeWarps;
  // CTAs at one visit (a token's items, or an item) per warp, and what a visit costs: an item about a row,
  // a lane's angle about half of one
  int64_t need[2], all = 0;
  double cost[2];
  for (int i = 0; i < 2; ++i) {
    const int heads = p.t[i].heads, rows = (heads + kHeads - 1) / kHeads, chunks = (rows + K - 1) / K;
    int64_t visits = 0;
    cost[i] = 0.0;
    if (heads > 0 && FEW) {
      const int tokens = K * (kHeads / heads);
      visits = (p.tokens + tokens - 1) / tokens;
      cost[i] = 1.0 + K + tokens * p.plan.n_pairs / 64.0;
    } else if (heads > 0) {
      visits = p.tokens * (p.whole_tokens ? 1 : chunks);
      cost[i] = p.whole_tokens ? chunks + rows + 0.5 : 1.5 + min(rows, K);
    }
    cost[i] *= visits;
    need[i] = (visits + kRopeWarps - 1) / kRopeWarps;
    all += need[i];
  }
  // shares of what fits at once by the tensors' costs, with the same number of visits for each warp of one
  for (int i = 0; i < 2; ++i) {
    const int64_t share = all <= fit ? need[i] : max((int64_t)(fit * (cost[i] / (cost[0] + cost[1]))), (int64_t)1);
    const int64_t steps = need[i] == 0 ? 1 : (need[i] + share - 1) / share;
    ctas[i] = (int)((need[i] + steps - 1) / steps);
  }
  p.first_ctas = ctas[0];
  if (ctas[0] + ctas[1] == 0) return cudaSuccess;
  return launch_pdl(kern, ctas[0] + ctas[1], kRopeThreads, 0, st, true, p);
}

template <typename T, int MODE, int S, bool NORM, bool BWD, bool FEW>
cudaError_t launch_rope_wide(RopeParams& p, int (&ctas)[2], cudaStream_t st) {
  const int lanes = (p.plan.head_dim + 2 * S - 1) / (2 * S);
  if constexpr (S == 8)
    if (lanes <= 2) return launch_rope_as<T, 2, MODE, S, NORM, BWD, FEW>(p, ctas, st);
  if (lanes <= 4) return launch_rope_as<T, 4, MODE, S, NORM, BWD, FEW>(p, ctas, st);
  if (lanes <= 8) return launch_rope_as<T, 8, MODE, S, NORM, BWD, FEW>(p, ctas, st);
  if constexpr (S == 4 && !FEW)
    if (lanes > 16) return launch_rope_as<T, 32, MODE, S, NORM, BWD, FEW>(p, ctas, st);
  return launch_rope_as<T, 16, MODE, S, NORM, BWD, FEW>(p, ctas, st);
}

template <typename T, bool NORM, bool BWD, bool FEW>
cudaError_t launch_rope_mode(const RopeKind& kind, RopeParams& p, int (&ctas)[2], cudaStream_t st) {
  if constexpr (sizeof(T) == 2 && !FEW)
    if (kind.slots == 8)
      return kind.mode == kNeighbours ? launch_rope_wide<T, kNeighbours, 8, NORM, BWD, FEW>(p, ctas, st)
                                      : launch_rope_wide<T, kChunks, 8, NORM, BWD, FEW>(p, ctas, st);
  if constexpr (!FEW)
    if (kind.mode == kGather) return launch_rope_wide<T, kGather, 4, NORM, BWD, FEW>(p, ctas, st);
  return kind.mode == kNeighbours ? launch_rope_wide<T, kNeighbours, 4, NORM, BWD, FEW>(p, ctas, st)
                                  : launch_rope_wide<T, kChunks, 4, NORM, BWD, FEW>(p, ctas, st);
}

template <bool BWD, bool FEW>
cudaError_t launch_rope_kind(const RopeKind& kind, int type, RopeParams& p, int (&ctas)[2], cudaStream_t st) {
  auto typed = [&](auto t) {
    using T = decltype(t);
    return kind.norm ? launch_rope_mode<T, true, BWD, FEW>(kind, p, ctas, st)
                     : launch_rope_mode<T, false, BWD, FEW>(kind, p, ctas, st);
  };
  return type == RESS_BF16 ? typed(bf16()) : type == RESS_F16 ? typed(f16()) : typed(0.f);
}

// How a tensor's channels lie on the lanes (see the top): 8 slots want 16-bit elements, vectors of 8, and
// heads that fill a warp's rows.
inline RopeKind rope_kind(const RopeArgs& a, const ress_rope_heads& t, bool bwd) {
  const ress_rope_plan& plan = a.plan;
  const int bytes = a.type == RESS_F32 ? 4 : 2;
  int run = 8;  // pairs of neighbouring channels that a lane can take as vectors: 8, 4 or 1
  auto fits = [&](const ress_heads& h) {
    const int align = min(run * bytes, 16);
    return reinterpret_cast<uintptr_t>(h.data) % align == 0 &&
           (a.n_tokens == 1 || h.token_stride * bytes % align == 0) &&
           (t.n_heads == 1 || h.head_stride * bytes % align == 0);
  };
  auto possible = [&] {
    if (plan.head_dim % (2 * run) != 0 || plan.n_pairs % run != 0) return false;
    if (plan.layout == RESS_ROPE_SECTIONS)
      for (int i = 0; i < plan.n_axes; ++i)
        if (plan.axis_dims[i] % (2 * run) != 0) return false;
    return ((bwd && !t.norm.enabled) || fits(t.x)) && fits(t.y) && (!bwd || fits(t.dx));
  };
  if (plan.layout == RESS_ROPE_INTERLEAVED) {  // a lane's vectors are as long as 8 channels all the same
    const bool aligned = ((bwd && !t.norm.enabled) || fits(t.x)) && fits(t.y) && (!bwd || fits(t.dx));
    while (run > 1 && (plan.head_dim % (2 * run) != 0 || plan.n_pairs % run != 0)) run = run == 8 ? 4 : 1;
    if (!aligned) run = 1;
  } else {
    while (run > 1 && !possible()) run = run == 8 ? 4 : 1;
  }
  RopeKind k;
  k.norm = t.norm.enabled != 0;
  k.mode = run == 1 ? kGather : plan.layout == RESS_ROPE_INTERLEAVED ? kNeighbours : kChunks;
  int lanes = 2;  // of 8 slots
  while (16 * lanes < plan.head_dim) lanes *= 2;
  k.slots = run == 8 && bytes == 2 && t.n_heads % (32 / lanes) == 0 ? 8 : 4;
  int row = 8;  // heads of a row, of lanes of 4 slots
  while (row > 1 && plan.head_dim > 256 / row) row /= 2;
  k.tokens = row / t.n_heads;
  k.few = k.slots == 4 && k.mode != kGather && row > 1 && k.tokens > 0;
  return k;
}

// All launches; first[i]..first[i + 1]: the CTAs of tensor i that leave partial sums of its norm's
// gradients.
template <bool BWD>
cudaError_t launch_rope_all(const RopeArgs& a, int (&first)[3], cudaStream_t st) {
  RopeParams p;
  p.plan = a.plan;
  p.tokens = a.n_tokens;
  p.pos = a.pos;
  p.eps = a.eps;
  p.param_type = a.param_type;
  p.all = 2 * a.plan.n_pairs == a.plan.head_dim;
  RopeTensor tensors[2];
  RopeKind kinds[2];
  for (int i = 0; i < 2; ++i) {
    const ress_rope_heads& t = a.t[i];
    const ress_heads& out = BWD ? t.dx : t.y;
    tensors[i] = RopeTensor{t.n_heads,        t.norm.weight,    t.norm.bias,     t.x.data,         t.y.data,
                            out.data,         t.x.token_stride, t.x.head_stride, t.y.token_stride, t.y.head_stride,
                            out.token_stride, out.head_stride};
    if (t.n_heads > 0) kinds[i] = rope_kind(a, t, BWD);
  }
  first[0] = first[1] = first[2] = 0;
  if (p.tokens == 0) return cudaSuccess;
  // One launch is worth more than several tokens per item with a token per row (20,011 tokens, 12 + 4 heads:
  // 22 us together, 31 apart).
  if (a.t[0].n_heads > 0 && a.t[1].n_heads > 0 && kinds[0].few != kinds[1].few) {
    RopeKind& few = kinds[kinds[0].few ? 0 : 1];
    if (few.tokens == 1) few.few = false;
  }
  const bool together = a.t[0].n_heads > 0 && a.t[1].n_heads > 0 && kinds[0] == kinds[1];
  p.most = together ? kRopeParts - 1 : kRopeParts / 2 - 1;
  for (int i = 0; i < 2; ++i) {
    first[i + 1] = max(first[i], first[i + 1]);
    if (a.t[i].n_heads == 0 || (together && i == 1)) continue;
    p.t[i] = tensors[i];
    p.t[1 - i] = together ? tensors[1 - i] : RopeTensor{};
    p.partial = BWD && kinds[i].norm && a.partial ? a.partial + (int64_t)first[i] * 2 * p.plan.head_dim : nullptr;
    int ctas[2] = {0, 0};
    const cudaError_t e = kinds[i].few ? launch_rope_few(BWD, kinds[i], a.type, p, ctas, st)
                                       : launch_rope_kind<BWD, false>(kinds[i], a.type, p, ctas, st);
    if (e != cudaSuccess) return e;
    if (!p.partial) continue;
    if (together) {
      first[1] = ctas[0];
      first[2] = ctas[0] + ctas[1];
    } else {
      first[i + 1] = first[i] + ctas[i];
    }
  }
  return cudaSuccess;
}

}  // namespace
}  // namespace ress

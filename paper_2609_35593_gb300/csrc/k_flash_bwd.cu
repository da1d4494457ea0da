// Gradient of dense attention (k_flash.cu): with p = exp(s - lse), dp = dO.V and delta = O.dO of each row,
//   ds = p (dp - delta) (1 - tanh^2),  dQ = sum_keys ds K / 8,  dK = sum_rows ds Q / 8,  dV = sum_rows p dO.
//
// Two passes of the same kernel, so that every sum is formed on chip in a fixed order: items of 128 rows with the keys
// streaming past them (dQ: three products a tile), and items of 128 keys with the rows streaming past (dK, dV:
// four).  One pass with five products would add dQ up from different CTAs: with atomics the bits change from run to
// run, in order the CTAs wait for one another.  The second pass works on the transposed scores
// S^T = K Q^T, so that in both what the element-wise warps write (P, dS; 16 bits, in TMEM over the scores they
// came from) is the A operand of the next product: nothing of the size of the scores touches shared memory.
// Heads of Q that share a head of K and V are rows of the same item (or columns of the same tile), which adds
// up their gradients.
//
// Roles (320 threads, one CTA per SM): producer, MMA issuer, and two groups of four warps that take every other
// tile: S and dP of the next tile are computed while a group works on the last one.  TMEM: S and dP of two tiles (256
// columns), two accumulators, two A operands (copied there once per item).  Shares of the work, partial results and
// waits are those of k_flash.cu (attn_work.cuh).
//
// In f16, P is kept times 2^8 and dS times a power of two that brings the largest |dO| to 1..2: probabilities of rows on
// thousands of keys are below f16's 2^-14, and so may gradients be.  dP is at most 64 max|dO| max|V|, so dS stays
// finite for |V| up to 250 whatever the values, and is taken back to scale in float32.
#include <cudaTypedefs.h>

#include "attn_work.cuh"

namespace ress {
using namespace ptx;
using namespace work;

namespace {

constexpr int kThreads = 320, kStages = 6, kItems = 4;
static_assert(kStages % 2 == 0, "a stage is always the same group's");
constexpr uint32_t kTileBytes = kTile * 128;
constexpr uint32_t kColP = 64, kColAcc1 = 256, kColAcc2 = 320, kColA1 = 384, kColA2 = 416;  // buffer b: 128 b
constexpr int kFirst = 1, kLast = 2, kTerm = 4, kMask = 8;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kPartFloats = 256 * 66;  // as k_flash.cu's: 128 rows of one or two gradients
constexpr float kPScale = 8.0f;            // log2 of P's scale in f16

struct Item {
  int q0, k0, nq, nk, d, p;
  int h, at;        // head of K; first token or key
  int from, t0, t1, g0;  // first row of the first tile (dK, dV); tiles; number of the first among all of the CTA's
  int part;
};

// What the columns of a tile are, where they are rows of Q (two of them next to each other are read together).
struct __align__(16) Cols {
  float lse[kTile], delta[kTile];  // -log2 of the sums, -delta (times the scale)
  int lim[kTile];                  // keys seen
  float pos[kTile], slope[kTile];
};

struct __align__(1024) Smem {
  uint8_t A1[128 * 128], A2[128 * 128];
  uint8_t B1[kStages][kTileBytes];
  uint8_t B2[kStages][kTileBytes];
  Cols cols[kStages];
  uint64_t kv_full[kStages], kv_empty[kStages];
  uint64_t q_full, q_empty, drain;
  uint64_t s_full[2], p_full[2], acc_full, acc_empty;
  uint64_t it_full[kItems], it_empty[kItems];
  int64_t scratch[34];
  Item item[kItems];
  int flags[kStages];
  uint32_t tmem_base;
  int abort;
};
static_assert(sizeof(Smem) + 1024 <= 227 * 1024, "one CTA's shared memory");

__device__ __forceinline__ void give_up(Smem& S, uint32_t* status) {
  flag_status(status, kStatusTimeout);
  *reinterpret_cast<volatile int*>(&S.abort) = 1;
}

__device__ __forceinline__ void mul2(float& d0, float& d1, float a0, float a1, float b0, float b1) {
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "mul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d0), "=f"(d1)
      : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

// The power of two that brings the largest |dO| to 1..2 (1 where there is none, or it is not finite).
__device__ __forceinline__ float grad_scale(const float* big, int n) {
  float m = 0.f;
  for (int i = threadIdx.x & 31; i < n; i += 32) m = fmaxf(m, big[i]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (!(m > 0.f) || m > 3e38f) return 1.f;
  return exp2f((float)-ilogbf(fmaxf(m, 1e-30f)));
}

// Items and the tiles of each.
template <bool kKeys>
struct Lines {
  const DenseArgs& a;
  int T;  // tokens of an item of rows
  __device__ Line operator()(const Seq& s) const { return kKeys ? key_line(a, s, 128) : row_line(a, s, T, [](int) { return 8; }); }
};
template <bool kKeys>
__device__ __forceinline__ int item_tiles(const DenseArgs& a, const Seq& s, int at, int T, int& from) {
  from = 0;
  if (kKeys) {
    from = first_row(a, s, at);
    const int per = kTile / a.group;
    return (s.nq - from + per - 1) / per;
  }
  return (max(0, row_limit(a, s, s.d + min(s.nq, at + T) - 1)) + kTile - 1) / kTile;
}

// 64 (or 32) channels of one row, scaled and rounded.
template <bool kF16, int N>
__device__ __forceinline__ void store_row(void* dst, const uint32_t (&o)[N], float by) {
  uint4* p = static_cast<uint4*>(dst);
#pragma unroll
  for (int k = 0; k < N / 8; ++k) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = pack2<kF16>(__uint_as_float(o[8 * k + 2 * e]) * by, __uint_as_float(o[8 * k + 2 * e + 1]) * by);
    p[k] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

}  // namespace

// Per row: log2 of its sum and delta = O . dO, laid out as the tiles of rows read them ([kv_heads, rows, group]), and
// in f16 the largest |dO| of each CTA's rows.  Eight lanes a row; bound by HBM (O and dO once).
template <bool kF16>
__global__ void __launch_bounds__(256) k_flash_rows(const __grid_constant__ DenseArgs a) {
  __shared__ float tops[8];
  rows::stream_acquire();
  const int sub = threadIdx.x & 7, heads = a.kv_heads * a.group;
  // rows of no sequence do not count
  const int64_t lo = a.q_start ? max(0, a.q_start[0]) : 0;
  const int64_t hi = a.q_start ? min(a.rows, (int64_t)a.q_start[a.n_seqs]) : a.rows;
  float top = 0.f;
  for (int64_t i = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3); i < a.rows * heads; i += (int64_t)gridDim.x * 32) {
    const int64_t t = i / heads;
    const int head = (int)(i - t * heads);
    if (t < lo || t >= hi) continue;  // (all eight lanes)
    const uint4 o = ld_stream(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.o.data) + t * a.o.token_stride +
                                                              head * a.o.head_stride) + sub);
    const uint4 g = ld_stream(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.d_o.data) +
                                                              t * a.d_o.token_stride + head * a.d_o.head_stride) + sub);
    const uint32_t ow[4] = {o.x, o.y, o.z, o.w}, gw[4] = {g.x, g.y, g.z, g.w};
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 x = unpack2<kF16>(ow[e]), y = unpack2<kF16>(gw[e]);
      sum = fmaf(x.x, y.x, fmaf(x.y, y.y, sum));
      if (kF16) top = fmaxf(top, fmaxf(fabsf(y.x), fabsf(y.y)));
    }
    const uint32_t lanes = 0xffu << (threadIdx.x & 24);
#pragma unroll
    for (int s = 4; s > 0; s >>= 1) sum += __shfl_xor_sync(lanes, sum, s);
    if (sub == 0) {
      const float lse = a.lse[head * a.rows + t];
      // a row that sees nothing: 2^(s - inf) = 0
      a.stat[((int64_t)(head / a.group) * a.rows + t) * a.group + head % a.group] =
          make_float2(lse == -INFINITY ? INFINITY : lse * kLog2e, sum);
    }
  }
  if (kF16) {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < 8; ++w) top = fmaxf(top, tops[w]);
      a.big[blockIdx.x] = top;
    }
  }
}

// kKeys: items of keys (dK, dV); else of rows (dQ).
template <bool kF16, bool kGen, bool kKeys>
__global__ void __launch_bounds__(kThreads, 1)
    k_flash_bwd(const __grid_constant__ CUtensorMap tmA1, const __grid_constant__ CUtensorMap tmA2,
                const __grid_constant__ CUtensorMap tmB1, const __grid_constant__ CUtensorMap tmB2,
                const __grid_constant__ DenseArgs a) {
  extern __shared__ uint8_t smem_raw[];
  Smem& S = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort = &S.abort;
  const int G = a.group, T = 128 / G, per = kTile / G;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&S.kv_full[s], 1);
      mbar_init(&S.kv_empty[s], 1);
    }
    mbar_init(&S.q_full, 1);
    mbar_init(&S.q_empty, 1);
    mbar_init(&S.drain, 1);
    for (int b = 0; b < 2; ++b) {
      mbar_init(&S.s_full[b], 1);
      mbar_init(&S.p_full[b], 4);
    }
    mbar_init(&S.acc_full, 1);
    mbar_init(&S.acc_empty, 8);
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&S.it_full[i], 1);
      mbar_init(&S.it_empty[i], 8);
    }
    S.abort = 0;
    fence_barrier_init();
    prefetch_tensormap(&tmA1);
    prefetch_tensormap(&tmA2);
    prefetch_tensormap(&tmB1);
    prefetch_tensormap(&tmB2);
  }
  if (kKeys && per * G < kTile) {  // rows of a tile that no box reaches are summed over, times 0
    for (int f = threadIdx.x; f < (int)(2 * kStages * kTileBytes / 16); f += kThreads)
      reinterpret_cast<uint4*>(S.B1)[f] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
  }
  if (warp == 1) tmem_alloc(&S.tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = S.tmem_base;
  rows::stream_acquire();
  const Lines<kKeys> line_of{a, T};
  const Range range = find_range(a, line_of, gridDim.x, blockIdx.x, S.scratch, blockIdx.x == 0 ? a.status : nullptr);

  if (warp == 0) {
    // =============================== producer ====================================
    int g = 0, it = 0, pub = 0;
    bool failed = false, a_loaded = false;
    const float f = kF16 ? grad_scale(a.big, a.n_big) * exp2f(-kPScale) : 1.f;
    if (lane == 0) a.share[2 * blockIdx.x].n = a.share[2 * blockIdx.x + 1].n = -1;
    __syncwarp();
    auto publish = [&](const Item* item) -> bool {
      const int i = pub % kItems, u = pub / kItems;
      if (u > 0 && !wait(&S.it_empty[i], (u - 1) & 1, abort)) return false;
      if (lane == 0) {
        if (item)
          S.item[i] = *item;
        else
          S.item[i].h = -1;
        mbar_arrive(&S.it_full[i]);
      }
      __syncwarp();
      ++pub;
      return true;
    };
    if (range.x0 < range.x1) {
      Cursor c;
      seek(a, line_of, range.x0, range.b0, range.base, c);
      do {
        Item item;
        item.q0 = c.s.q0, item.k0 = c.s.k0, item.nq = c.s.nq, item.nk = c.s.nk, item.d = c.s.d, item.p = c.s.p;
        item.h = c.h, item.at = c.j * (kKeys ? 128 : T);
        const int n = item_tiles<kKeys>(a, c.s, item.at, T, item.from);
        tiles_of(c, range.x0, range.x1, n, item.t0, item.t1);
        item.g0 = g;
        item.part = item.t0 == 0 && item.t1 == n ? -1 : share_slot(c, range.x0);
        if (item.t0 == item.t1 && (n > 0 || c.start < range.x0)) continue;
        if (item.part >= 0 && lane == 0)
          a.share[item.part] = DenseShare{item.t0, item.t1, n, c.h, (kKeys ? c.s.k0 : c.s.q0) + item.at,
                                          min((kKeys ? c.s.nk : c.s.nq) - item.at, kKeys ? 128 : T), {}};
        if (!publish(&item)) {
          failed = true;
          break;
        }
        if (n == 0) continue;
        if (it > 0 && !wait(&S.q_empty, (it - 1) & 1, abort)) {
          failed = true;
          break;
        }
        if (lane == 0) {
          mbar_arrive_expect_tx(&S.q_full, kKeys ? 2 * 128 * 128 : 2 * T * G * 128);
          if (kKeys) {
            tma_load_4d(S.A1, &tmA1, &S.q_full, 0, c.h, item.k0 + item.at, 0);
            tma_load_4d(S.A2, &tmA2, &S.q_full, 0, c.h, item.k0 + item.at, 0);
          } else {
            tma_load_4d(S.A1, &tmA1, &S.q_full, 0, 0, c.h, item.q0 + item.at);
            tma_load_4d(S.A2, &tmA2, &S.q_full, 0, 0, c.h, item.q0 + item.at);
          }
        }
        __syncwarp();
        a_loaded = true;
        // columns lane and lane + 32 of a tile of rows; the next tile's are loaded ahead
        auto stats = [&](int t, float2 (&x)[2]) {
          const int tok = item.from + t * per;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int col = lane + 32 * e;
            x[e] = make_float2(INFINITY, 0.f);
            if (col < per * G && tok + col / G < item.nq)
              x[e] = a.stat[((int64_t)c.h * a.rows + item.q0 + tok) * G + col];
          }
        };
        float2 now[2], ahead[2];
        if (kKeys) stats(item.t0, now);
        for (int t = item.t0; t < item.t1; ++t) {
          const int s = g % kStages, u = g / kStages;
          if (kKeys && t + 1 < item.t1) stats(t + 1, ahead);
          if (u > 0 && !wait(&S.kv_empty[s], (u - 1) & 1, abort)) {
            failed = true;
            break;
          }
          int flags = (t == item.t0 ? kFirst : 0) | (t == item.t1 - 1 ? kLast : 0);
          const int tok = item.from + t * per;
          if (kKeys) {
            bool whole = true;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int col = lane + 32 * e, row = tok + col / G, pos = item.d + row;
              const bool exists = col < per * G && row < item.nq;
              const int lim = !exists ? 0 : a.causal ? max(0, max(item.p, pos + 1)) : item.nk;
              whole = whole && lim >= min(item.nk, item.at + 128);
              S.cols[s].lse[col] = (kF16 ? kPScale : 0.f) - now[e].x;
              S.cols[s].delta[col] = -now[e].y * f;
              S.cols[s].lim[col] = lim;
              if (kGen) {
                S.cols[s].pos[col] = (float)pos;
                S.cols[s].slope[col] = a.slopes && exists ? a.slopes[c.h * G + col % G] * kLog2e : 0.f;
              }
            }
            if (!__all_sync(0xffffffffu, whole)) flags |= kMask;
          }
          __syncwarp();
          if (lane == 0) {
            S.flags[s] = flags;
            mbar_arrive_expect_tx(&S.kv_full[s], kKeys ? 2 * per * G * 128 : 2 * kTileBytes);
            if (kKeys) {
              tma_load_4d(S.B1[s], &tmB1, &S.kv_full[s], 0, 0, c.h, item.q0 + tok);
              tma_load_4d(S.B2[s], &tmB2, &S.kv_full[s], 0, 0, c.h, item.q0 + tok);
            } else {
              tma_load_4d(S.B1[s], &tmB1, &S.kv_full[s], 0, c.h, item.k0 + t * kTile, 0);
              tma_load_4d(S.B2[s], &tmB2, &S.kv_full[s], 0, c.h, item.k0 + t * kTile, 0);
            }
          }
          __syncwarp();
          now[0] = ahead[0], now[1] = ahead[1];
          ++g;
        }
        if (failed) break;
        ++it;
        a_loaded = false;
      } while (next(a, line_of, c) && c.start < range.x1);
    }
    rows::stream_release();
    if (!failed) {
      const int s = g % kStages, u = g / kStages;
      if (u > 0 && !wait(&S.kv_empty[s], (u - 1) & 1, abort)) {
        failed = true;
      } else if (lane == 0) {
        S.flags[s] = kTerm;
        mbar_arrive(&S.kv_full[s]);
      }
      if (!failed && !publish(nullptr)) failed = true;
    }
    if (failed && lane == 0) {
      give_up(S, a.status);
      // let every copy already issued land before the CTA's shared memory goes away
      volatile int no_abort = 0;
      for (int back = 1; back <= kStages && g - back >= 0; ++back)
        mbar_wait(&S.kv_full[(g - back) % kStages], ((g - back) / kStages) & 1, &no_abort, kDrainNs);
      if (a_loaded) mbar_wait(&S.q_full, it & 1, &no_abort, kDrainNs);
    }
  } else if (warp == 1) {
    // ================================ MMA issuer ===================================
    const bool leader = elect_one();
    bool failed = false;
    constexpr uint32_t kRow = idesc16<kF16>(128, kTile, false), kSum = idesc16<kF16>(128, 64, true);
    constexpr uint64_t kStageUnits = kTileBytes >> 4;
    const uint64_t b10 = sdesc_sw128(smem_u32(S.B1[0])), b20 = sdesc_sw128(smem_u32(S.B2[0]));
    int it = 0, sums = 0;  // items whose A operands are in TMEM, and whose sums were begun
    auto fetch = [&](int t, int& flags) -> bool {
      if (!wait(&S.kv_full[t % kStages], (t / kStages) & 1, abort)) return false;
      flags = S.flags[t % kStages];
      return true;
    };
    auto issue_sums = [&](int t, int flags) -> bool {
      const int st = t % kStages, b = t & 1;
      if (!wait(&S.p_full[b], (t >> 1) & 1, abort)) return false;
      if (flags & kFirst) {  // the item before has been read
        if (sums > 0 && !wait(&S.acc_empty, (sums - 1) & 1, abort)) return false;
        ++sums;
      }
      tc_fence_after();
      if (leader) {
        const uint64_t d1 = b10 + (uint64_t)st * kStageUnits, d2 = b20 + (uint64_t)st * kStageUnits;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t more = k > 0 || !(flags & kFirst) ? 1u : 0u;
          if (kKeys) mma_bf16_ts(tmem + kColAcc2, tmem + 128 * b + 8 * k, d2 + 128 * k, kSum, more);
          mma_bf16_ts(tmem + kColAcc1, tmem + 128 * b + kColP + 8 * k, d1 + 128 * k, kSum, more);
        }
        mma_commit(&S.kv_empty[st]);
        if (flags & kLast) mma_commit(&S.acc_full);
      }
      __syncwarp();
      return true;
    };
    // Per tile: S and dP, then the sums over the tile before it.  The last sums of an item do not wait for a tile
    // to come: the producer may be waiting for the element-wise warps to end the item.
    int flags = kTerm, held = -1, held_flags = 0;
    if (!fetch(0, flags)) failed = true;
    for (int g = 0; !failed && !(flags & kTerm); ++g) {
      if (flags & kFirst) {
        if (!wait(&S.q_full, it & 1, abort)) {
          failed = true;
          break;
        }
        tc_fence_after();
        if (leader) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            tmem_cp_128x256b(tmem + kColA1 + 8 * k, sdesc_sw128(smem_u32(S.A1) + 32 * k));
            tmem_cp_128x256b(tmem + kColA2 + 8 * k, sdesc_sw128(smem_u32(S.A2) + 32 * k));
          }
          mma_commit(&S.q_empty);
        }
        __syncwarp();
        ++it;
      }
      const uint64_t at = (uint64_t)(g % kStages) * kStageUnits;
      const int b = g & 1;
      if (leader) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_bf16_ts(tmem + 128 * b, tmem + kColA1 + 8 * k, b10 + at + 2 * k, kRow, k > 0 ? 1u : 0u);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma_bf16_ts(tmem + 128 * b + kColP, tmem + kColA2 + 8 * k, b20 + at + 2 * k, kRow, k > 0 ? 1u : 0u);
        mma_commit(&S.s_full[b]);
      }
      __syncwarp();
      if (held >= 0 && !issue_sums(held, held_flags)) {
        failed = true;
        break;
      }
      held = g, held_flags = flags;
      if ((flags & kLast) && !mbar_ready(&S.kv_full[(g + 1) % kStages], ((g + 1) / kStages) & 1)) {
        if (!issue_sums(held, held_flags)) {
          failed = true;
          break;
        }
        held = -1;
      }
      if (!fetch(g + 1, flags) || ((flags & kTerm) && held >= 0 && !issue_sums(held, held_flags))) {
        failed = true;
        break;
      }
    }
    if (failed && lane == 0) give_up(S, a.status);
    // wait for every MMA issued so far before TMEM is released
    if (leader) {
      mma_commit(&S.drain);
      volatile int no_abort = 0;
      mbar_wait(&S.drain, 0, &no_abort, kDrainNs);
    }
    __syncwarp();
  } else {
    // ============================ element-wise groups ==============================
    const int group = (warp - 2) >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;
    const int tid = (warp - 2 - 4 * group) * 32 + lane;  // 0..127, for the zeroing
    const uint32_t tm = tmem + ((uint32_t)(quarter * 32) << 16), tS = tm + 128 * group, tP = tS + kColP;
    const float kScale = kLog2e * 0.125f;
    const float cap = a.cap, in = a.cap > 0.f ? 0.25f * kLog2e / a.cap : 0.125f * kLog2e, out = a.cap * kLog2e;
    const float back = a.cap > 0.f ? 1.0f / out : 0.f;
    const float scale = kF16 ? grad_scale(a.big, a.n_big) : 1.f, f = kF16 ? scale * exp2f(-kPScale) : 1.f;
    const float undo = 0.125f / scale;
    int it = 0;
    bool stop = false;
    for (int pub = 0; !stop; ++pub) {
      const int i = pub % kItems;
      if (!wait(&S.it_full[i], (pub / kItems) & 1, abort)) {
        give_up(S, a.status);
        break;
      }
      const Item item = S.item[i];
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.it_empty[i]);
      if (item.h < 0) break;
      // this thread's row: a key, or a row of Q
      const int tok = item.at + (kKeys ? r : r / G);
      const bool exists = kKeys ? tok < item.nk : r / G < T && tok < item.nq;
      const int pos = item.d + tok, head = item.h * G + r % G;  // (of a row of Q)
      float nlse = -INFINITY, ndelta = 0.f, slope = 0.f;
      int lim = 0, least = 0;
      if (!kKeys) {
        if (exists) {
          const float2 x = a.stat[((int64_t)item.h * a.rows + item.q0 + tok) * G + r % G];
          nlse = (kF16 ? kPScale : 0.f) - x.x, ndelta = -x.y * f;
          lim = a.causal ? min(item.nk, max(item.p, pos + 1)) : item.nk;
          if (kGen && a.slopes) slope = a.slopes[head] * kLog2e;
        }
        least = __reduce_min_sync(0xffffffffu, exists ? max(lim, 0) : INT32_MAX);
      }
      const int g1 = item.g0 + item.t1 - item.t0;
      for (int g = item.g0 + ((item.g0 & 1) != group); g < g1; g += 2) {
        const int st = g % kStages;
        if (!wait(&S.kv_full[st], (g / kStages) & 1, abort) || !wait(&S.s_full[group], (g >> 1) & 1, abort)) {
          give_up(S, a.status);
          stop = true;
          break;
        }
        tc_fence_after();
        const int t = item.t0 + g - item.g0, key = t * kTile;
        const Cols& cols = S.cols[st];
        const bool masked = kKeys ? (S.flags[st] & kMask) != 0 : key + kTile > least;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint32_t s[32], dp[32], w1[16], w2[16];
          RESS_TMEM_LD32(tS + 32 * hf, s);
          RESS_TMEM_LD32(tP + 32 * hf, dp);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const int col = 32 * hf + e;
            float l0 = nlse, l1 = nlse, n0 = ndelta, n1 = ndelta;
            if (kKeys) {
              const float2 l = *reinterpret_cast<const float2*>(&cols.lse[col]);
              const float2 n = *reinterpret_cast<const float2*>(&cols.delta[col]);
              l0 = l.x, l1 = l.y, n0 = n.x, n1 = n.y;
            }
            float x0 = __uint_as_float(s[e]), x1 = __uint_as_float(s[e + 1]);
            float y0 = __uint_as_float(dp[e]), y1 = __uint_as_float(dp[e + 1]);
            float c0 = 1.f, c1 = 1.f;
            if (kGen) {
              if (cap > 0.f) {
                capped2(x0, x1, in, out);
                float u0, u1;
                mul2(u0, u1, x0, x1, back, back);
                fma2(c0, c1, -u0, -u1, u0, u1, 1.f, 1.f);
              } else {
                x0 *= in, x1 *= in;
              }
              if (a.slopes) {
                if (kKeys) {
                  const float2 q = *reinterpret_cast<const float2*>(&cols.pos[col]);
                  const float2 m = *reinterpret_cast<const float2*>(&cols.slope[col]);
                  x0 = fmaf(-m.x, fabsf(q.x - (float)tok), x0);
                  x1 = fmaf(-m.y, fabsf(q.y - (float)tok), x1);
                } else {
                  x0 = fmaf(-slope, fabsf((float)(pos - key - col)), x0);
                  x1 = fmaf(-slope, fabsf((float)(pos - key - col - 1)), x1);
                }
              }
              add2(x0, x1, x0, x1, l0, l1);
            } else {
              fma2(x0, x1, x0, x1, kScale, kScale, l0, l1);
            }
            x0 = ex2(x0), x1 = ex2(x1);
            if (kF16)
              fma2(y0, y1, y0, y1, f, f, n0, n1);
            else
              add2(y0, y1, y0, y1, n0, n1);
            if (kGen) mul2(y0, y1, y0, y1, c0, c1);
            mul2(y0, y1, y0, y1, x0, x1);
            if (masked) {
              bool s0, s1;
              if (kKeys) {
                const int2 m = *reinterpret_cast<const int2*>(&cols.lim[col]);
                s0 = tok < m.x, s1 = tok < m.y;
              } else {
                s0 = key + col < lim, s1 = key + col + 1 < lim;
              }
              x0 = s0 ? x0 : 0.f, x1 = s1 ? x1 : 0.f;
              y0 = s0 ? y0 : 0.f, y1 = s1 ? y1 : 0.f;
            }
            w1[e >> 1] = pack2<kF16>(x0, x1);
            w2[e >> 1] = pack2<kF16>(y0, y1);
          }
          if (kKeys) RESS_TMEM_ST16(tS + 16 * hf, w1);
          RESS_TMEM_ST16(tP + 16 * hf, w2);
        }
        // rows of the tile that are not this sequence's, which the sums run over
        const int valid = kKeys ? (item.nq - item.from - t * per) * G : item.nk - key;
        if (valid < (kKeys ? per * G : kTile)) {
          zero_rows(S.B1[st], valid, tid);
          if (kKeys) zero_rows(S.B2[st], valid, tid);
          fence_proxy_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.p_full[group]);
      }
      if (stop) break;
      // group 0 takes dK, or half of the channels of dQ; group 1 dV, or the other half
      constexpr int N = kKeys ? 64 : 32;
      uint32_t o[N];
      if (item.t1 > item.t0) {
        if (!wait(&S.acc_full, it & 1, abort)) {
          give_up(S, a.status);
          break;
        }
        ++it;
        tc_fence_after();
        if constexpr (kKeys)
          RESS_TMEM_LD64(tm + (group ? kColAcc2 : kColAcc1), o);
        else
          RESS_TMEM_LD32(tm + kColAcc1 + 32 * group, o);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.acc_empty);
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) o[e] = 0u;
      }
      if (!exists) continue;
      const float by = kKeys && group ? (kF16 ? exp2f(-kPScale) : 1.f) : undo;
      if (item.part >= 0) {
        float4* dst = reinterpret_cast<float4*>(a.part + item.part * kPartFloats + (kKeys ? (group * 128 + r) * 64 : r * 64 + 32 * group));
#pragma unroll
        for (int e = 0; e < N / 4; ++e)
          dst[e] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]),
                               __uint_as_float(o[4 * e + 3]));
      } else if (kKeys) {
        const ress_heads& d = group ? a.dv : a.dk;
        store_row<kF16>(static_cast<uint16_t*>(d.data) + ((int64_t)item.k0 + tok) * d.token_stride + item.h * d.head_stride, o, by);
      } else {
        store_row<kF16>(static_cast<uint16_t*>(a.dq.data) + ((int64_t)item.q0 + tok) * a.dq.token_stride +
                            head * a.dq.head_stride + 32 * group, o, by);
      }
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Gradients of items that several CTAs had shares of: the shares' sums, in their order.  Blocks as in k_flash_join: 32
// rows each (of dK, then of dV), half a warp per row.
template <bool kF16, bool kKeys>
__global__ void __launch_bounds__(256) k_flash_bwd_join(const __grid_constant__ DenseArgs a, int ctas) {
  rows::stream_acquire();
  const DenseShare item = a.share[blockIdx.x];
  if (item.n < 0 || item.t0 != 0) return;
  const int G = a.group, T = 128 / G, sub = threadIdx.x & 15;
  const float undo = 0.125f / (kF16 ? grad_scale(a.big, a.n_big) : 1.f);
  for (int i = threadIdx.x >> 4; i < 32; i += 16) {
    const int row = blockIdx.y * 32 + i, which = row >> 7, rr = row & 127;
    if (kKeys ? rr >= item.count : rr >= T * G || rr / G >= item.count) continue;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = blockIdx.x, t1 = item.t1;;) {
      const float4 v = reinterpret_cast<const float4*>(a.part + s * kPartFloats + row * 64)[sub];
      o.x += v.x, o.y += v.y, o.z += v.z, o.w += v.w;
      if (t1 >= item.n || (s = next_share(a, s, ctas)) < 0) break;
      t1 = a.share[s].t1;
    }
    const float by = kKeys && which ? (kF16 ? exp2f(-kPScale) : 1.f) : undo;
    const ress_heads& d = kKeys ? (which ? a.dv : a.dk) : a.dq;
    const int64_t token = (int64_t)item.first + (kKeys ? rr : rr / G);
    const int head = kKeys ? item.head : item.head * G + rr % G;
    reinterpret_cast<uint2*>(static_cast<uint16_t*>(d.data) + token * d.token_stride + head * d.head_stride)[sub] =
        make_uint2(pack2<kF16>(o.x * by, o.y * by), pack2<kF16>(o.z * by, o.w * by));
  }
}

template <bool kF16, bool kGen, bool kKeys>
static cudaError_t launch_pass(const DenseArgs& a, const CUtensorMap (&m)[4], int ctas, cudaStream_t st) {
  auto kern = k_flash_bwd<kF16, kGen, kKeys>;
  const size_t smem = sizeof(Smem) + 1024;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  if ((e = launch_pdl(kern, ctas, kThreads, smem, st, true, m[0], m[1], m[2], m[3], a)) != cudaSuccess || ctas == 1) return e;
  return launch_pdl(k_flash_bwd_join<kF16, kKeys>, dim3(2 * ctas, kKeys ? 8 : 4), 256, 0, st, true, a, ctas);
}

template <bool kF16>
static cudaError_t launch_type(DenseArgs a, cudaStream_t st) {
  const int ctas = dense_ctas();
  cudaError_t e;
  if (a.rows > 0) {
    const int64_t rows = a.rows * a.kv_heads * a.group;
    a.n_big = (int)(rows / 32 < kBigParts ? (rows + 31) / 32 : kBigParts);
    if ((e = launch_pdl(k_flash_rows<kF16>, dim3(a.n_big), 256, 0, st, true, a)) != cudaSuccess) return e;
  }
  const bool gen = a.cap > 0.f || a.slopes;
  // a tensor without rows or keys is not read, but its map needs some memory
  ress_heads q = a.q, g = a.d_o, k = a.k, v = a.v;
  if (a.rows == 0) q = g = k, q.head_stride = g.head_stride = 64;
  if (a.keys == 0) k = v = q, k.head_stride = v.head_stride = 64;
  const int64_t rows = a.rows > 0 ? a.rows : 1, keys = a.keys > 0 ? a.keys : 1;
  CUtensorMap m[4];
  if (a.keys > 0) {
    const int per = kTile / a.group;
    if (!make_key_map(&m[0], k, a.type, keys, 1, 0, a.kv_heads, 128) || !make_key_map(&m[1], v, a.type, keys, 1, 0, a.kv_heads, 128) ||
        !make_row_map(&m[2], q, a.type, rows, a.kv_heads, a.group, per) ||
        !make_row_map(&m[3], g, a.type, rows, a.kv_heads, a.group, per))
      return cudaErrorInvalidValue;
    if ((e = gen ? launch_pass<kF16, true, true>(a, m, ctas, st) : launch_pass<kF16, false, true>(a, m, ctas, st)) != cudaSuccess)
      return e;
  }
  if (a.rows > 0) {
    const int T = 128 / a.group;
    if (!make_row_map(&m[0], q, a.type, rows, a.kv_heads, a.group, T) || !make_row_map(&m[1], g, a.type, rows, a.kv_heads, a.group, T) ||
        !make_key_map(&m[2], k, a.type, keys, 1, 0, a.kv_heads, kTile) || !make_key_map(&m[3], v, a.type, keys, 1, 0, a.kv_heads, kTile))
      return cudaErrorInvalidValue;
    if ((e = gen ? launch_pass<kF16, true, false>(a, m, ctas, st) : launch_pass<kF16, false, false>(a, m, ctas, st)) != cudaSuccess)
      return e;
  }
  return cudaSuccess;
}

cudaError_t launch_flash_bwd(const DenseArgs& a, cudaStream_t st) {
  return a.type == RESS_F16 ? launch_type<true>(a, st) : launch_type<false>(a, st);
}

}  // namespace ress

// Gradient of dense attention (k_flash.cu): with p = exp(s - lse), dp = dO.V and delta = O.dO of each row,
//   ds = p (dp - delta) (1 - tanh^2),  dQ = sum_keys ds K / 8,  dK = sum_rows ds Q / 8,  dV = sum_rows p dO.
//
// Two passes of the same kernel, so that every sum is formed on chip in a fixed order: items of 128 rows with the keys
// streaming past them (dQ: three products a tile), and items of 128 keys with the rows streaming past (dK, dV:
// four).  One pass with five products would add dQ up from different CTAs: with atomics the bits change from run to
// run, in order the CTAs wait for one another.  The second pass works on the transposed scores
// S^T = K Q^T, so that in both what the element-wise warps write (P, dS; 16 bits, in TMEM) is the A operand of the
// next product: nothing of the size of the scores touches shared memory.  Heads of Q that share a head of K and V are
// rows of the same item (or columns of the same tile), which adds up their gradients.
//
// Roles (640 threads, one CTA per SM): warp 0 producer, warp 1 issuer of S and dP (M128 N128 K64, operands in shared
// memory, each as soon as the last one's values are in registers), warps 2 and 3 issuers of the sums over P and over dS,
// warps 4-19 element-wise: 16 rows x 64 columns of a tile of 128 x 128 each.  S and dP (256 columns of TMEM) are free for the next tile as soon as they are in registers, P and
// dS (128) have columns of their own, so the products of the next tile run meanwhile; two accumulators (128).  With
// eight element-wise warps on tiles of 64 columns and one issuer a tile of 128 x 64 took 1,700 cycles, its four
// products 512 (8 images at once, 10,992 rows and keys of 16 heads: 2,200 us; now 1,405 to 1,497, 0.83 to 0.88 PFLOP/s of five products'
// work or 1.16 to 1.23 of the seven formed).  What bounds it is the chain of a tile from scores to dS and back.  Shares of the work, partial results and waits are those of k_flash.cu.
//
// In f16, P is kept times 2^8 and dS times a power of two: probabilities of rows on thousands of keys are below f16's 2^-14,
// and so may gradients be.  |dP - delta| is at most 2 |dO| max|V| over the sequence's keys (norms over channels: O is a mean of
// rows of V), so the power that brings this to 2^14..2^15 keeps dS finite whatever the values are, and what is lost of it below
// 2^-39 of that bound.  |dO| is that of the row where rows are the accumulators' rows (dQ), and the sequence's largest where the rows are
// summed over (dK): no row and no sequence takes digits from others.  The largest come from chunks of 16 rows or keys that
// k_flash_rows leaves, once per sequence and head (k_flash_steps: a launch of some 4 us; looked up by the producers instead,
// f16 documents took 255 us where 230, 32 images 1,148 where 1,005).  Gradients are taken back to scale in float32.
#include <cudaTypedefs.h>

#include <type_traits>

#include "attn_work.cuh"

namespace ress {
using namespace ptx;
using namespace work;

namespace {

constexpr int kThreads = 640, kStages = 4, kItems = 4, kCols = 128;
constexpr int kProducer = 0, kIssueS = 1, kIssueDs = 3, kElem = 4;  // warps (2: issuer of the sums over P)
constexpr uint32_t kTileBytes = kCols * 128;
constexpr uint32_t kColDp = 128, kColP = 256, kColDs = 320, kColAcc1 = 384, kColAcc2 = 448;  // TMEM; S at 0
constexpr int kFirst = 1, kLast = 2, kTerm = 4, kMask = 8;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kPartFloats = 256 * 66;  // as k_flash.cu's: 128 rows of one or two gradients
constexpr float kPScale = 8.0f;            // log2 of P's scale in f16

struct Item {
  int q0, k0, nq, nk, d, p;
  int h, at;        // head of K (-1: no more items); first token or key
  int from, t0, t1, g0;  // first row of the first tile (dK, dV); tiles; number of the first among all of the CTA's
  int part;
  float step;  // f16: the power of two of dS (dK), the largest |V|^2 (dQ)
};

// What the columns of a tile are, where they are rows of Q (two next to each other are read together).
struct __align__(16) Cols {
  float lse[kCols], delta[kCols];  // -log2 of the sums, -delta (times the scale)
  int lim[kCols];                  // keys seen
  float pos[kCols], slope[kCols];  // position after the item's first key (exact where it matters, however long the sequence)
};

struct __align__(1024) Smem {
  uint8_t A[2][2][128 * 128];  // of two items
  uint8_t B1[kStages][kTileBytes];
  uint8_t B2[kStages][kTileBytes];
  Cols cols[kStages];
  uint8_t row_token[128], row_head[128];  // of 128 rows of Q
  uint64_t kv_full[kStages], kv_empty[kStages];
  uint64_t a_full[2], a_empty[2], drain[3];
  uint64_t s_full, s_free, dp_full, dp_free, p_full, p_done, acc_full, acc_empty;
  uint64_t it_full[kItems], it_empty[kItems];
  int64_t scratch[34];
  Item item[kItems], next;
  Cursor cursor;
  int flags[kStages];
  uint32_t tmem_base;
  int abort;
};
static_assert(sizeof(Smem) + 1024 <= 227 * 1024, "one CTA's shared memory");

__device__ __forceinline__ void give_up(Smem& S, uint32_t* status) {
  flag_status(status, kStatusTimeout);
  *reinterpret_cast<volatile int*>(&S.abort) = 1;
}

// The power of two that brings 2 |dO| |V|, by their squares, to 2^14..2^15 (1 where there is none, or they are not finite).
__device__ __forceinline__ float step_scale(float do2, float v2) {
  const float b = do2 * v2;
  if (!(b > 0.f && b < 3e38f)) return 1.f;
  const int e = (__float_as_int(b) >> 23) - 127;  // sqrt(b) is below 2^((e + 1) / 2)
  return __int_as_float((127 + 14 - ((e + 2) >> 1)) << 23);
}
__device__ __forceinline__ float inverse2(float p) { return __int_as_float((254 << 23) - __float_as_int(p)); }  // of a power of two

__device__ __forceinline__ float square8(uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 x = unpack2<true>(w[e]);
    s = fmaf(x.x, x.x, fmaf(x.y, x.y, s));
  }
  return s;
}
__device__ __forceinline__ const uint4* row_at(const ress_heads& h, int64_t token, int head, int chunk) {
  return reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(h.data) + token * h.token_stride + head * h.head_stride) + chunk;
}

// Rows [lo, hi) of a head as whole chunks [c0, c1) and what is left of them at both ends: [lo, e0) and [e1, hi).
struct Chunks {
  int c0, c1, e0, e1;
  __device__ Chunks(int lo, int hi, int chunk) {
    c0 = (int)(((int64_t)lo + chunk - 1) / chunk), c1 = hi / chunk;
    e0 = c0 < c1 ? c0 * chunk : hi, e1 = c0 < c1 ? c1 * chunk : hi;
  }
};
__device__ __forceinline__ float warp_max(float m) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
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
    return (s.nq - from + T - 1) / T;
  }
  return (max(0, row_limit(a, s, s.d + min(s.nq, at + T) - 1)) + kCols - 1) / kCols;
}

}  // namespace

// Per row: log2 of its sum and delta = O . dO, laid out as the tiles of rows read them ([kv_heads, rows, group]), and
// in f16 |dO|^2 and the largest of it, and of |V|^2, in chunks.  A chunk of a head per warp, eight lanes a row; bound by HBM
// (O and dO once; in f16 V too).
template <bool kF16>
__global__ void __launch_bounds__(256) k_flash_rows(const __grid_constant__ DenseArgs a) {
  rows::stream_acquire();
  const int lane = threadIdx.x & 31, sub = lane & 7;
  // Rows behind the last sequence are left out: those from the largest start on (the last one, unless some are bad: the sequences
  // around a bad one are as ever).
  int64_t hi = a.rows;
  if (a.q_start) {
    __shared__ int ends[8];
    int end = 0;
    for (int b = threadIdx.x; b <= a.n_seqs; b += 256) end = max(end, a.q_start[b]);
    end = __reduce_max_sync(0xffffffffu, end);
    if (lane == 0) ends[threadIdx.x >> 5] = end;
    __syncthreads();
    for (int w = 0; w < 8; ++w) end = max(end, ends[w]);
    hi = min(hi, (int64_t)end);
  }
  auto total = [](float x) {
#pragma unroll
    for (int s = 4; s > 0; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
    return x;
  };
  constexpr int kAtOnce = kTopRows / 4;
  const int heads = a.kv_heads * a.group;
  const int64_t q_chunks = (a.rows + kTopRows - 1) / kTopRows, v_chunks = kF16 ? (a.keys + a.v_chunk - 1) / a.v_chunk : 0;
  const int64_t q_units = q_chunks * heads, units = q_units + v_chunks * a.kv_heads;
  for (int64_t u = blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += gridDim.x * 8) {
    // the heads of a chunk next to each other, as they are in memory
    float top = 0.f;
    if (u < q_units) {
      const int64_t c = quotient(u, heads), t0 = c * kTopRows + (lane >> 3);
      const int head = (int)(u - c * heads), h = head / a.group, g = head - h * a.group;
      uint4 o[kAtOnce], d[kAtOnce];
      float lse[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        o[i] = d[i] = make_uint4(0u, 0u, 0u, 0u);
        lse[i] = 0.f;
        const int64_t t = t0 + 4 * i;
        if (t < hi) {
          o[i] = ld_stream(row_at(a.o, t, head, sub)), d[i] = ld_stream(row_at(a.d_o, t, head, sub));
          lse[i] = a.lse[head * a.rows + t];
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const uint32_t ow[4] = {o[i].x, o[i].y, o[i].z, o[i].w}, dw[4] = {d[i].x, d[i].y, d[i].z, d[i].w};
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 x = unpack2<kF16>(ow[e]), y = unpack2<kF16>(dw[e]);
          sum = fmaf(x.x, y.x, fmaf(x.y, y.y, sum));
        }
        sum = total(sum);
        const float square = kF16 ? total(square8(d[i])) : 0.f;
        top = fmaxf(top, square);
        const int64_t t = t0 + 4 * i;
        if (sub == 0 && t < hi) {
          const int64_t at = ((int64_t)h * a.rows + t) * a.group + g;
          // a row that sees nothing: 2^(s - inf) = 0
          a.stat[at] = make_float2(lse[i] == -INFINITY ? INFINITY : lse[i] * kLog2e, sum);
          if (kF16) a.norm[at] = square;
        }
      }
      if (kF16) {
        top = warp_max(top);
        if (lane == 0) a.q_top[head * q_chunks + c] = top;
      }
    } else {
      const int64_t c = quotient(u - q_units, a.kv_heads), k1 = min(a.keys, (c + 1) * a.v_chunk);
      const int h = (int)(u - q_units - c * a.kv_heads);
#pragma unroll 1
      for (int64_t k0 = c * a.v_chunk + (lane >> 3); k0 - (lane >> 3) < k1; k0 += 4 * kAtOnce) {
        uint4 v[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          v[i] = make_uint4(0u, 0u, 0u, 0u);
          if (k0 + 4 * i < k1) v[i] = ld_stream(row_at(a.v, k0 + 4 * i, h, sub));
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, total(square8(v[i])));
      }
      top = warp_max(top);
      if (lane == 0) a.v_top[h * v_chunks + c] = top;
    }
  }
}

// In f16, of each sequence and head of K, laid out by the sequence's first row ([kv_heads, rows]): the largest |V|^2 of its keys,
// and the power of two of dS with the largest |dO|^2 of its rows.  A CTA each; bound by latency (two rounds of loads for
// sequences of some thousand rows).
constexpr int kStepThreads = 128;
__global__ void __launch_bounds__(kStepThreads) k_flash_steps(const __grid_constant__ DenseArgs a) {
  __shared__ float tops[2][kStepThreads / 32];
  rows::stream_acquire();
  const int tid = threadIdx.x, G = a.group;
  const int64_t q_chunks = (a.rows + kTopRows - 1) / kTopRows, v_chunks = (a.keys + a.v_chunk - 1) / a.v_chunk;
  for (int64_t u = blockIdx.x; u < (int64_t)a.n_seqs * a.kv_heads; u += gridDim.x) {
    const int b = (int)(u / a.kv_heads), h = (int)(u - (int64_t)b * a.kv_heads);
    const Seq s = load_seq(a, b, nullptr);
    if (s.nq == 0) continue;
    float v2 = 0.f, d2 = 0.f;
    {
      const Chunks r(s.k0, s.k0 + s.nk, a.v_chunk);
#pragma unroll 8
      for (int c = r.c0 + tid; c < r.c1; c += kStepThreads) v2 = fmaxf(v2, a.v_top[h * v_chunks + c]);
      const int first = r.e0 - s.k0, n = first + s.k0 + s.nk - r.e1;
#pragma unroll 4
      for (int i = 0; i < n; i += kStepThreads / 8) {  // eight lanes a row
        const int k = i + (tid >> 3);
        float x = k < n ? square8(*row_at(a.v, k < first ? s.k0 + k : r.e1 + k - first, h, tid & 7)) : 0.f;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        v2 = fmaxf(v2, x);
      }
    }
    {
      const Chunks r(s.q0, s.q0 + s.nq, kTopRows);
      for (int c = r.c0 + tid; c < r.c1; c += kStepThreads)
#pragma unroll 4
        for (int g = 0; g < G; ++g) d2 = fmaxf(d2, a.q_top[((int64_t)h * G + g) * q_chunks + c]);
      const float* norm = a.norm + (int64_t)h * a.rows * G;
      const int first = (r.e0 - s.q0) * G, n = first + (s.q0 + s.nq - r.e1) * G;
#pragma unroll 4
      for (int i = tid; i < n; i += kStepThreads)
        d2 = fmaxf(d2, norm[i < first ? (int64_t)s.q0 * G + i : (int64_t)r.e1 * G + i - first]);
    }
    v2 = warp_max(v2), d2 = warp_max(d2);
    if ((tid & 31) == 0) tops[0][tid >> 5] = v2, tops[1][tid >> 5] = d2;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kStepThreads / 32; ++w) v2 = fmaxf(v2, tops[0][w]), d2 = fmaxf(d2, tops[1][w]);
      a.steps[(int64_t)h * a.rows + s.q0] = make_float2(v2, step_scale(d2, v2));
    }
    __syncthreads();
  }
}

// kKeys: items of keys (dK, dV); else of rows (dQ).
template <bool kF16, int kGen, bool kKeys>
__global__ void __launch_bounds__(kThreads, 1)
    k_flash_bwd(const __grid_constant__ CUtensorMap tmA1, const __grid_constant__ CUtensorMap tmA2,
                const __grid_constant__ CUtensorMap tmB1, const __grid_constant__ CUtensorMap tmB2,
                const __grid_constant__ DenseArgs a) {
  extern __shared__ uint8_t smem_raw[];
  Smem& S = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort = &S.abort;
  const int G = a.group, T = 128 / G;
  constexpr int kSums = kKeys ? 2 : 1;  // issuers of sums
  constexpr bool kSlopes = kGen >= 2, kCap = kGen & 1;  // (kGen as in k_flash)
  static_assert(offsetof(Smem, B2) == offsetof(Smem, B1) + kStages * kTileBytes && kTileBytes == sizeof S.A[0][0], "tiles one after another");

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&S.kv_full[s], 1);
      mbar_init(&S.kv_empty[s], 1 + kSums);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&S.a_full[b], 1);
      mbar_init(&S.a_empty[b], 1);
    }
    for (int i = 0; i < 3; ++i) mbar_init(&S.drain[i], 1);
    mbar_init(&S.s_full, 1);
    mbar_init(&S.s_free, 16);
    mbar_init(&S.dp_full, 1);
    mbar_init(&S.dp_free, 16);
    mbar_init(&S.p_full, 16);
    mbar_init(&S.p_done, kSums);
    mbar_init(&S.acc_full, kSums);
    mbar_init(&S.acc_empty, 16);
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&S.it_full[i], 1);
      mbar_init(&S.it_empty[i], 16);
    }
    S.abort = 0;
    fence_barrier_init();
    prefetch_tensormap(&tmA1);
    prefetch_tensormap(&tmA2);
    prefetch_tensormap(&tmB1);
    prefetch_tensormap(&tmB2);
  }
  if (const int r = (int)threadIdx.x - 512; r >= 0) {
    S.row_token[r] = r / G, S.row_head[r] = r % G;
    // rows that no token fills stay 0, as in k_flash (where they are rows of a streamed tile they are summed over, times 0)
    if (r >= T * G) {
#pragma unroll 1
      for (int i = 0; i < (kKeys ? 2 * kStages : 4) * 8; ++i)
        reinterpret_cast<uint4*>((kKeys ? S.B1[0] : S.A[0][0]) + (i >> 3) * kTileBytes + r * 128)[i & 7] = make_uint4(0u, 0u, 0u, 0u);
      fence_proxy_async_smem();
    }
  }
  if (warp == kIssueS) tmem_alloc(&S.tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = S.tmem_base;
  rows::stream_acquire();
  const Lines<kKeys> line_of{a, T};
  Range range;  // (of the producer)
  if (a.n_seqs > 32) range = find_range(a, line_of, gridDim.x, blockIdx.x, S.scratch, blockIdx.x == 0 ? a.status : nullptr);

  // registers as in k_flash
  if (warp < kElem) {
    regs_dec<64>();
    if (warp == kProducer) {
      // =============================== producer ====================================
      int g = 0, it = 0, pub = 0;
      bool failed = false;
      if (a.n_seqs <= 32)
        range = find_range_warp(a, line_of, gridDim.x, blockIdx.x, blockIdx.x == 0 ? a.status : nullptr);
      if (lane == 0) a.share[2 * blockIdx.x].n = a.share[2 * blockIdx.x + 1].n = -1;
      int col_tok[4];  // token of this lane's columns lane, lane + 32, .. of a tile of rows (past it: never one)
#pragma unroll
      for (int e = 0; e < 4; ++e) col_tok[e] = lane + 32 * e < T * G ? (lane + 32 * e) / G : INT32_MAX / 2;
      // The next item that this share has tiles of, to S.next (see k_flash).
      auto advance = [&](bool first) {
        __syncwarp();
        if (lane == 0) {
          Cursor& c = S.cursor;
          Item& item = S.next;
          item.h = -1;
          if (first) seek(a, line_of, range.x0, range.b0, range.base, c);
          while (first || (next(a, line_of, c) && c.start < range.x1)) {
            first = false;
            int from, t0, t1;
            const int at = c.j * (kKeys ? 128 : T), n = item_tiles<kKeys>(a, c.s, at, T, from);
            tiles_of(c, range.x0, range.x1, n, t0, t1);
            if (t0 == t1 && (n > 0 || c.start < range.x0)) continue;
            item.q0 = c.s.q0, item.k0 = c.s.k0, item.nq = c.s.nq, item.nk = c.s.nk, item.d = c.s.d, item.p = c.s.p;
            item.h = c.h, item.at = at, item.from = from, item.t0 = t0, item.t1 = t1;
            item.part = t0 == 0 && t1 == n ? -1 : share_slot(c, range.x0);
            if (kF16) {
              item.step = 1.f;
              if (t0 < t1) item.step = reinterpret_cast<const float*>(a.steps + (int64_t)c.h * a.rows + c.s.q0)[kKeys];
            }
            if (item.part >= 0)
              a.share[item.part] = DenseShare{t0, t1, n, c.h, (kKeys ? c.s.k0 : c.s.q0) + at,
                                              min((kKeys ? c.s.nk : c.s.nq) - at, kKeys ? 128 : T), {}};
            break;
          }
        }
        __syncwarp();
      };
      auto publish = [&]() -> bool {
        const int i = pub % kItems, u = pub / kItems;
        if (u > 0 && !wait(&S.it_empty[i], (u - 1) & 1, abort)) return false;
        if (lane == 0) {
          S.next.g0 = g;
          S.item[i] = S.next;
          mbar_arrive(&S.it_full[i]);
        }
        __syncwarp();
        ++pub;
        return true;
      };
      if (range.x0 < range.x1) {
        for (advance(true); S.next.h >= 0 && !failed; advance(false)) {
          if (!publish()) {
            failed = true;
            break;
          }
          const Item& item = S.next;
          if (item.t0 == item.t1) continue;  // nothing to add up
          const int buf = it & 1, h = item.h, t0 = item.t0, t1 = item.t1;
          if (it > 1 && !wait(&S.a_empty[buf], ((it >> 1) - 1) & 1, abort)) {
            failed = true;
            break;
          }
          if (lane == 0) {
            mbar_arrive_expect_tx(&S.a_full[buf], kKeys ? 2 * 128 * 128 : 2 * T * G * 128);
            if (kKeys) {
              tma_load_4d(S.A[buf][0], &tmA1, &S.a_full[buf], 0, h, item.k0 + item.at, 0);
              tma_load_4d(S.A[buf][1], &tmA2, &S.a_full[buf], 0, h, item.k0 + item.at, 0);
            } else {
              tma_load_4d(S.A[buf][0], &tmA1, &S.a_full[buf], 0, 0, h, item.q0 + item.at);
              tma_load_4d(S.A[buf][1], &tmA2, &S.a_full[buf], 0, 0, h, item.q0 + item.at);
            }
          }
          __syncwarp();
          ++it;
          // the next tile's columns are loaded ahead
          const float2* stat = a.stat + ((int64_t)h * a.rows + item.q0 + item.from) * G + lane;
          const int left = item.nq - item.from, pos0 = item.d + item.from, base = kKeys ? item.q0 + item.from : item.k0;
          const int nk = item.nk, p = item.p, last_key = min(nk, item.at + 128);
          const float f = kF16 && kKeys ? item.step * exp2f(-kPScale) : 1.f;
          float slope[4] = {0.f, 0.f, 0.f, 0.f};
          if (kKeys && kSlopes) {
#pragma unroll
            for (int e = 0; e < 4; ++e) slope[e] = a.slopes[h * G + (lane + 32 * e) % G] * kLog2e;
          }
          auto stats = [&](int t, float2 (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[e] = make_float2(INFINITY, 0.f);
              if (t * T + col_tok[e] < left) x[e] = stat[(int64_t)t * T * G + 32 * e];
            }
          };
          float2 now[4], ahead[4];
          if (kKeys) stats(t0, now);
          for (int t = t0; t < t1; ++t) {
            const int s = g % kStages, u = g / kStages;
            if (kKeys && t + 1 < t1) stats(t + 1, ahead);
            if (u > 0 && !wait(&S.kv_empty[s], (u - 1) & 1, abort)) {
              failed = true;
              break;
            }
            int flags = (t == t0 ? kFirst : 0) | (t == t1 - 1 ? kLast : 0);
            if (kKeys) {
              bool whole = true;
              Cols& cols = S.cols[s];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int col = lane + 32 * e, row = t * T + col_tok[e];
                const int lim = row >= left ? 0 : a.causal ? max(p, pos0 + row + 1) : nk;
                whole = whole && lim >= last_key;
                cols.lse[col] = (kF16 ? kPScale : 0.f) - now[e].x;
                cols.delta[col] = -now[e].y * f;
                cols.lim[col] = lim;
                if (kSlopes) cols.pos[col] = (float)(pos0 + row - item.at), cols.slope[col] = slope[e];
                now[e] = ahead[e];
              }
              if (!__all_sync(0xffffffffu, whole)) flags |= kMask;
            }
            __syncwarp();
            if (lane == 0) {
              S.flags[s] = flags;
              mbar_arrive_expect_tx(&S.kv_full[s], kKeys ? 2 * T * G * 128 : 2 * kTileBytes);
              if (kKeys) {
                tma_load_4d(S.B1[s], &tmB1, &S.kv_full[s], 0, 0, h, base + t * T);
                tma_load_4d(S.B2[s], &tmB2, &S.kv_full[s], 0, 0, h, base + t * T);
              } else {
                tma_load_4d(S.B1[s], &tmB1, &S.kv_full[s], 0, h, base + t * kCols, 0);
                tma_load_4d(S.B2[s], &tmB2, &S.kv_full[s], 0, h, base + t * kCols, 0);
              }
            }
            __syncwarp();
            ++g;
          }
        }
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
        __syncwarp();
        if (lane == 0) S.next.h = -1;
        __syncwarp();
        if (!failed && !publish()) failed = true;
      }
      if (failed && lane == 0) {
        give_up(S, a.status);
        // let every copy already issued land before the CTA's shared memory goes away
        volatile int no_abort = 0;
        for (int back = 1; back <= kStages && g - back >= 0; ++back)
          mbar_wait(&S.kv_full[(g - back) % kStages], ((g - back) / kStages) & 1, &no_abort, kDrainNs);
        for (int back = 1; back <= 2 && it - back >= 0; ++back)
          mbar_wait(&S.a_full[(it - back) & 1], ((it - back) >> 1) & 1, &no_abort, kDrainNs);
      }
    } else {
      // ================================ MMA issuers ==================================
      const bool leader = elect_one();
      bool failed = false;
      constexpr uint32_t kRow = idesc16<kF16>(128, kCols, false), kSum = idesc16<kF16>(128, 64, true);
      constexpr uint64_t kStageUnits = kTileBytes >> 4, kAUnits = (128 * 128) >> 4;
      uint32_t phase = 0;
      if (warp == kIssueS) {
        const uint64_t b1 = sdesc_sw128(smem_u32(S.B1[0])), b2 = sdesc_sw128(smem_u32(S.B2[0]));
        const uint64_t a0 = sdesc_sw128(smem_u32(S.A[0][0]));
        uint32_t s_phase = 1, items = 0;
        for (int st = 0;;) {
          if (!wait(&S.kv_full[st], phase, abort)) {
            failed = true;
            break;
          }
          const int flags = S.flags[st];
          if (flags & kTerm) break;
          if (flags & kFirst) {
            if (!wait(&S.a_full[items & 1], (items >> 1) & 1, abort)) {
              failed = true;
              break;
            }
            ++items;
          }
          const uint32_t buf = (items - 1) & 1;
          const uint64_t ad = a0 + 2 * buf * kAUnits, at = (uint64_t)st * kStageUnits;
          if (!wait(&S.s_free, s_phase, abort)) {  // (the first time: at once)
            failed = true;
            break;
          }
          tc_fence_after();
          if (leader) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_bf16_ss(tmem, ad + 2 * k, b1 + at + 2 * k, kRow, k > 0 ? 1u : 0u);
            mma_commit(&S.s_full);
          }
          __syncwarp();
          if (!wait(&S.dp_free, s_phase, abort)) {
            failed = true;
            break;
          }
          s_phase ^= 1;
          tc_fence_after();
          if (leader) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_bf16_ss(tmem + kColDp, ad + kAUnits + 2 * k, b2 + at + 2 * k, kRow, k > 0 ? 1u : 0u);
            mma_commit(&S.dp_full);
            if (flags & kLast) mma_commit(&S.a_empty[buf]);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&S.kv_empty[st]);
          __syncwarp();
          if (++st == kStages) st = 0, phase ^= 1;
        }
      } else if (kKeys || warp == kIssueDs) {
        // dQ, dK += dS B1; dV += P B2
        const bool ds = warp == kIssueDs;
        const uint64_t b0 = sdesc_sw128(smem_u32(ds ? S.B1[0] : S.B2[0]));
        const uint32_t acc = tmem + (ds ? kColAcc1 : kColAcc2), from = tmem + (ds ? kColDs : kColP);
        uint32_t p_phase = 0, e_phase = 1;
        for (int st = 0;;) {
          if (!wait(&S.kv_full[st], phase, abort)) {
            failed = true;
            break;
          }
          const int flags = S.flags[st];
          if (flags & kTerm) break;
          if (!wait(&S.p_full, p_phase, abort)) {
            failed = true;
            break;
          }
          p_phase ^= 1;
          if (flags & kFirst) {  // the item before has been read (the first time: at once)
            if (!wait(&S.acc_empty, e_phase, abort)) {
              failed = true;
              break;
            }
            e_phase ^= 1;
          }
          tc_fence_after();
          if (leader) {
            const uint64_t bd = b0 + (uint64_t)st * kStageUnits;
            mma_bf16_ts(acc, from, bd, kSum, flags & kFirst ? 0u : 1u);
#pragma unroll
            for (int k = 1; k < 8; ++k) mma_bf16_ts(acc, from + 8 * k, bd + 128 * k, kSum, 1u);
            mma_commit(&S.p_done);
            mma_commit(&S.kv_empty[st]);
            if (flags & kLast) mma_commit(&S.acc_full);
          }
          __syncwarp();
          if (++st == kStages) st = 0, phase ^= 1;
        }
      }
      if (failed && lane == 0) give_up(S, a.status);
      // wait for every MMA issued so far before TMEM is released
      if (leader) {
        mma_commit(&S.drain[warp - kIssueS]);
        volatile int no_abort = 0;
        mbar_wait(&S.drain[warp - kIssueS], 0, &no_abort, kDrainNs);
      }
      __syncwarp();
    }
  } else {
    regs_inc<104>();
    // ============================ element-wise warps ===============================
    const int idx = warp - kElem, side = idx >> 3, half = idx >> 2 & 1, quarter = warp & 3;  // side: columns 64 side ..
    const int r0 = quarter * 32 + half * 16 + (lane >> 2), two = 2 * (lane & 3);  // this lane's rows: r0, r0 + 8; columns
    const uint32_t tm = tmem + ((uint32_t)(quarter * 32 + half * 16) << 16);
    const float kScale = kLog2e * 0.125f;
    const float in = kCap ? 0.25f * kLog2e / a.cap : 0.125f * kLog2e, out = a.cap * kLog2e;
    const float back = kCap ? 1.0f / out : 0.f;
    uint32_t c = 0, it = 0;  // tiles, and items with any, so far
    bool stop = false;
    for (int pub = 0; !stop; ++pub) {
      const int i = pub % kItems;
      if (!wait(&S.it_full[i], (pub / kItems) & 1, abort)) {
        give_up(S, a.status);
        break;
      }
      const Item& item = S.item[i];
      if (item.h < 0) break;
      // this lane's rows: keys, or rows of Q
      const int tiles = item.t1 - item.t0;
      auto token_of = [&](int j) { return item.at + (kKeys ? r0 + 8 * j : S.row_token[r0 + 8 * j]); };
      auto exists = [&](int j) {
        return kKeys ? token_of(j) < item.nk : S.row_token[r0 + 8 * j] < T && token_of(j) < item.nq;
      };
      int tok[2], pos[2], lim[2] = {0, 0}, least = item.nk;
      float nlse[2] = {-INFINITY, -INFINITY}, ndelta[2] = {0.f, 0.f}, slope[2] = {0.f, 0.f};
      float f[2];  // dS's power of two, over that of P (of both rows the same in the pass over keys)
      f[0] = f[1] = kF16 && kKeys ? item.step * exp2f(-kPScale) : 1.f;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = r0 + 8 * j;
        tok[j] = token_of(j);
        pos[j] = item.d + tok[j];
        if (!kKeys && exists(j)) {
          const int64_t at = ((int64_t)item.h * a.rows + item.q0 + tok[j]) * G + S.row_head[r];
          const float2 x = a.stat[at];
          if (kF16) f[j] = step_scale(a.norm[at], item.step) * exp2f(-kPScale);
          nlse[j] = (kF16 ? kPScale : 0.f) - x.x, ndelta[j] = -x.y * f[j];
          lim[j] = a.causal ? max(0, min(item.nk, max(item.p, pos[j] + 1))) : item.nk;
          least = min(least, lim[j]);
          if (kSlopes) slope[j] = a.slopes[item.h * G + S.row_head[r]] * kLog2e;
        }
      }
      if (!kKeys) least = __reduce_min_sync(0xffffffffu, least);
      // (In registers: read from the item in shared memory in every tile they cost 40 of 1,434 us on 8 images at once.)
      const int full = kKeys ? T * G : kCols;  // rows of a tile
      int g = item.g0, key = kKeys ? 0 : item.t0 * kCols, left = kKeys ? (item.nq - item.from - item.t0 * T) * G : 0;
      for (int n = tiles; n > 0; --n, ++c, ++g, key += kCols, left -= full) {
        const int st = g % kStages;
        // (the columns' numbers are there, and in the other pass nothing but S is looked at before the tail)
        if ((kKeys && !wait(&S.kv_full[st], (g / kStages) & 1, abort)) || !wait(&S.s_full, c & 1, abort)) {
          give_up(S, a.status);
          stop = true;
          break;
        }
        tc_fence_after();
        const Cols& cols = S.cols[st];
        const bool masked = kKeys ? (S.flags[st] & kMask) != 0 : key + kCols > least;  // (warp's rows: at least at the last key)
        float x[32];
        uint32_t w[16];
        {
          uint32_t v[32];
          RESS_TMEM_LD16X64(tm + 64 * side, v);
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(v[e]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.s_free);  // S is in registers: that of the next tile may come
        __syncwarp();
        // p and dP of masked scores become 0, whatever they were.  The votes keep this a branch: as selects in the loops it
        // took three quarters of the ALU's cycles in all tiles, 1,830 us on 8 images at once.
        auto masks = [&](auto&& at) {
          if (__any_sync(0xffffffffu, masked)) {
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const int j = e >> 1 & 1, col = 64 * side + 8 * (e >> 2) + two;
              if (kKeys) {
                const int2 m = *reinterpret_cast<const int2*>(&cols.lim[col]);
                at(e, tok[j] < m.x), at(e + 1, tok[j] < m.y);
              } else {
                at(e, key + col < lim[j]), at(e + 1, key + col + 1 < lim[j]);
              }
            }
          }
        };
        // P; kLarge: a product may be above half of the cap
        auto probabilities = [&](auto large) {
          constexpr bool kLarge = decltype(large)::value;
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const int j = e >> 1 & 1, col = 64 * side + 8 * (e >> 2) + two;  // row, columns col and col + 1
            float l0 = nlse[j], l1 = nlse[j];
            if (kKeys) {
              const float2 l = *reinterpret_cast<const float2*>(&cols.lse[col]);
              l0 = l.x, l1 = l.y;
            }
            float x0 = x[e], x1 = x[e + 1];
            float c0 = 1.f, c1 = 1.f;
            if (kGen) {
              if (kCap)
                cap_slope2<kLarge>(x0, x1, c0, c1, a, in, out, back);
              else
                x0 *= in, x1 *= in;
              if (kSlopes) {
                if (kKeys) {
                  const float2 q = *reinterpret_cast<const float2*>(&cols.pos[col]);
                  const float2 m = *reinterpret_cast<const float2*>(&cols.slope[col]);
                  x0 = fmaf(-m.x, fabsf(q.x - (float)(r0 + 8 * j)), x0);
                  x1 = fmaf(-m.y, fabsf(q.y - (float)(r0 + 8 * j)), x1);
                } else {
                  x0 = fmaf(-slope[j], fabsf((float)(pos[j] - key - col)), x0);
                  x1 = fmaf(-slope[j], fabsf((float)(pos[j] - key - col - 1)), x1);
                }
              }
              add2(x0, x1, x0, x1, l0, l1);
            } else {
              fma2(x0, x1, x0, x1, kScale, kScale, l0, l1);
            }
            x0 = ex2(x0), x1 = ex2(x1);
            if (kKeys) w[e >> 1] = pack2<kF16>(x0, x1);
            if (kCap) mul2(x0, x1, x0, x1, c0, c1);
            x[e] = x0, x[e + 1] = x1;  // p, times the cap's slope
          }
        };
        if (!kCap || !any_above_cap(x, a))
          probabilities(std::false_type());
        else
          probabilities(std::integral_constant<bool, kCap>());
        masks([&](int e, bool seen) {
          x[e] = seen ? x[e] : 0.f;
          w[e >> 1] &= seen ? 0xffffffffu : e & 1 ? 0x0000ffffu : 0xffff0000u;
        });
        // the sums over the tile before this one have read P and dS
        if ((c > 0 && !wait(&S.p_done, (c - 1) & 1, abort)) || !wait(&S.dp_full, c & 1, abort)) {
          give_up(S, a.status);
          stop = true;
          break;
        }
        tc_fence_after();
        if (kKeys) RESS_TMEM_ST16X32P_NOWAIT(tm + kColP + 32 * side, w);
        uint32_t v[32];
        RESS_TMEM_LD16X64(tm + kColDp + 64 * side, v);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.dp_free);
        __syncwarp();
        // dS
        masks([&](int e, bool seen) { v[e] = seen ? v[e] : 0u; });
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const int j = e >> 1 & 1, col = 64 * side + 8 * (e >> 2) + two;
          float n0 = ndelta[j], n1 = ndelta[j];
          if (kKeys) {
            const float2 n = *reinterpret_cast<const float2*>(&cols.delta[col]);
            n0 = n.x, n1 = n.y;
          }
          float y0 = __uint_as_float(v[e]), y1 = __uint_as_float(v[e + 1]);
          if (kF16)
            fma2(y0, y1, y0, y1, f[j], f[j], n0, n1);
          else
            add2(y0, y1, y0, y1, n0, n1);
          mul2(y0, y1, y0, y1, x[e], x[e + 1]);
          w[e >> 1] = pack2<kF16>(y0, y1);
        }
        if (kKeys) tmem_wait_st();
        RESS_TMEM_ST16X32P_NOWAIT(tm + kColDs + 32 * side, w);
        // rows of the tile that are not this sequence's, which the sums run over
        const int valid = kKeys ? left : masked ? item.nk - key : kCols;
        if (valid < full) {
          if (!kKeys && !wait(&S.kv_full[st], (g / kStages) & 1, abort)) {
            give_up(S, a.status);
            stop = true;
            break;
          }
          if (side == 0)
            zero_rows(S.B1[st], valid, (idx & 7) * 32 + lane);
          else if (kKeys)
            zero_rows(S.B2[st], valid, (idx & 7) * 32 + lane);
          fence_proxy_async_smem();
        }
        __syncwarp();
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.p_full);
        __syncwarp();
      }
      if (stop) break;
      // side 0 takes dK or dQ, side 1 dV
      float o[32];
#pragma unroll
      for (int e = 0; e < 32; ++e) o[e] = 0.f;
      if (tiles > 0) {
        if (!wait(&S.acc_full, it & 1, abort)) {
          give_up(S, a.status);
          break;
        }
        ++it;
        tc_fence_after();
        uint32_t v[32];
        RESS_TMEM_LD16X64(tm + (kKeys && side ? kColAcc2 : kColAcc1), v);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.acc_empty);
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(v[e]);
      }
      const ress_heads& to = kKeys ? (side ? a.dv : a.dk) : a.dq;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = r0 + 8 * j;
        if (!kKeys && side) break;
        const float by = (kKeys && side ? 1.f : kF16 ? 0.125f * inverse2(f[j]) : 0.125f) * (kF16 ? exp2f(-kPScale) : 1.f);
        if (item.part >= 0) {
          float2* dst = reinterpret_cast<float2*>(a.part + item.part * kPartFloats + (side * 128 + r) * 64 + two);
          if (exists(j)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) dst[4 * e] = make_float2(o[4 * e + 2 * j] * by, o[4 * e + 2 * j + 1] * by);
          }
        } else {
          uint32_t w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float y0, y1;
            mul2(y0, y1, o[4 * e + 2 * j], o[4 * e + 2 * j + 1], by, by);
            w[e] = pack2<kF16>(y0, y1);
          }
          // a row's four lanes: from two channels of every eight to eight of every 32
          transpose4(w[0], w[1], w[2], w[3], lane);
          transpose4(w[4], w[5], w[6], w[7], lane);
          if (exists(j)) {
            const int64_t token = (int64_t)(kKeys ? item.k0 : item.q0) + token_of(j);
            const int head = kKeys ? item.h : item.h * G + S.row_head[r];
            uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(to.data) + token * to.token_stride +
                                                  head * to.head_stride) + (lane & 3);
            dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
            dst[4] = make_uint4(w[4], w[5], w[6], w[7]);
          }
        }
        __syncwarp();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.it_empty[i]);
      __syncwarp();
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kIssueS) {
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
    const ress_heads& d = kKeys ? (which ? a.dv : a.dk) : a.dq;
    const int64_t token = (int64_t)item.first + (kKeys ? rr : rr / G);
    const int head = kKeys ? item.head : item.head * G + rr % G;
    reinterpret_cast<uint2*>(static_cast<uint16_t*>(d.data) + token * d.token_stride + head * d.head_stride)[sub] =
        make_uint2(pack2<kF16>(o.x, o.y), pack2<kF16>(o.z, o.w));
  }
}

template <bool kF16, int kGen, bool kKeys>
static cudaError_t launch_pass(const DenseArgs& a, const CUtensorMap (&m)[4], int ctas, cudaStream_t st) {
  auto kern = k_flash_bwd<kF16, kGen, kKeys>;
  const size_t smem = sizeof(Smem) + 1024;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  if ((e = launch_pdl(kern, ctas, kThreads, smem, st, true, m[0], m[1], m[2], m[3], a)) != cudaSuccess || ctas == 1) return e;
  return launch_pdl(k_flash_bwd_join<kF16, kKeys>, dim3(2 * ctas, kKeys ? 8 : 4), 256, 0, st, true, a, ctas);
}

template <bool kF16, bool kKeys>
static cudaError_t launch_gen(const DenseArgs& a, const CUtensorMap (&m)[4], int ctas, cudaStream_t st) {
  switch (dense_gen(a)) {
    case 0: return launch_pass<kF16, 0, kKeys>(a, m, ctas, st);
    case 1: return launch_pass<kF16, 1, kKeys>(a, m, ctas, st);
    case 2: return launch_pass<kF16, 2, kKeys>(a, m, ctas, st);
    default: return launch_pass<kF16, 3, kKeys>(a, m, ctas, st);
  }
}

template <bool kF16>
static cudaError_t launch_type(DenseArgs a, cudaStream_t st) {
  const int ctas = dense_ctas();
  cudaError_t e;
  a.v_chunk = kTopRows;
  const auto v_chunks = [&] { return (a.keys + a.v_chunk - 1) / a.v_chunk; };
  while (v_chunks() > kHeadTops || v_chunks() * a.kv_heads > kVTops) a.v_chunk *= 2;
  if (a.rows > 0) {
    const int64_t chunks = a.kv_heads * ((a.rows + kTopRows - 1) / kTopRows * a.group + (kF16 ? v_chunks() : 0));
    const int64_t units = (chunks + 7) / 8, full = 8 * (int64_t)ctas;
    if ((e = launch_pdl(k_flash_rows<kF16>, dim3((unsigned)(units < full ? units : full)), 256, 0, st, true, a)) != cudaSuccess)
      return e;
    const int64_t pairs = (int64_t)a.n_seqs * a.kv_heads, most = 16 * (int64_t)ctas;
    if (kF16 && (e = launch_pdl(k_flash_steps, dim3((unsigned)(pairs < most ? pairs : most)), kStepThreads, 0, st, true, a)) != cudaSuccess)
      return e;
  }
  if (a.cap > 0.f) set_cap(a);
  // a tensor without rows or keys is not read, but its map needs some memory
  ress_heads q = a.q, g = a.d_o, k = a.k, v = a.v;
  if (a.rows == 0) q = g = k, q.head_stride = g.head_stride = 64;
  if (a.keys == 0) k = v = q, k.head_stride = v.head_stride = 64;
  const int64_t rows = a.rows > 0 ? a.rows : 1, keys = a.keys > 0 ? a.keys : 1;
  CUtensorMap m[4];
  if (a.keys > 0) {
    const int per = 128 / a.group;
    if (!make_key_map(&m[0], k, a.type, keys, 1, 0, a.kv_heads, 128) || !make_key_map(&m[1], v, a.type, keys, 1, 0, a.kv_heads, 128) ||
        !make_row_map(&m[2], q, a.type, rows, a.kv_heads, a.group, per) ||
        !make_row_map(&m[3], g, a.type, rows, a.kv_heads, a.group, per))
      return cudaErrorInvalidValue;
    e = launch_gen<kF16, true>(a, m, ctas, st);
    if (e != cudaSuccess) return e;
  }
  if (a.rows > 0) {
    const int T = 128 / a.group;
    if (!make_row_map(&m[0], q, a.type, rows, a.kv_heads, a.group, T) || !make_row_map(&m[1], g, a.type, rows, a.kv_heads, a.group, T) ||
        !make_key_map(&m[2], k, a.type, keys, 1, 0, a.kv_heads, kCols) || !make_key_map(&m[3], v, a.type, keys, 1, 0, a.kv_heads, kCols))
      return cudaErrorInvalidValue;
    e = launch_gen<kF16, false>(a, m, ctas, st);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_flash_bwd(const DenseArgs& a, cudaStream_t st) {
  return a.type == RESS_F16 ? launch_type<true>(a, st) : launch_type<false>(a, st);
}

}  // namespace ress

// The projection of a layer's input to Q, K and V on the tensor cores, with what comes between the
// product and the attention in its epilogue:
//   [Q | K | V] = x [W_q | W_k | W_v]^T + bias, and on the heads of Q and K, before the one rounding
//   to bf16, a layer norm over the head's 64 channels (where the backbone has one) and the rotary
//   positions.
// x is [N, D], the weights are [H * 64, D] (Linear weights, out x in), Q, K and V [N, H, 64].  On
// their own the norm and the rotation would read and write Q and K once more.
//
// The product is tiled as the output projection's (k_oproj.cu): 256 tokens x up to 256 channels, that
// is 4 heads of one of Q, K, V, per CTA pair (cta_group::2, M256 N256 K16), over D in 64-wide slices
// through a TMA ring, persistent pairs with two TMEM accumulators.  Per CTA 320 threads:
//   warp 0     TMA of its half of the x and W slices;
//   warp 1     TMEM owner; in the rank-0 CTA one elected lane issues the pair's MMAs;
//   warps 2-9  epilogue in two groups of four warps that take the tile's heads in turn, one thread
//              per token: a head's 64 channels are 64 columns of the thread's TMEM lane, all of them in
//              its registers, so that neither the norm's sums nor the rotation need another thread.
//              Plans that pair channel c with c xor h and turn all of them (h = 1, 16, 32: neighbours,
//              two sections of 32, halves) are unrolled; any other plan's pairs are read from TMEM
//              once more, one by one, over the head without rotation.  The cosines and sines of the
//              CTA's 128 tokens are formed in shared memory while the tile's MMAs run.  The epilogue
//              has to stay below the MMAs' 8,270 cycles per tile (D = 1024): read and worked on 8
//              channels at a time, with every parameter looked up on its own, it took 19,000 (243 us
//              for 43,968 tokens, 16 heads, D = 1024).
// Waits are bounded as in k_oproj.cu.

#include <cudaTypedefs.h>

#include "row_ops.cuh"

namespace ress {
using namespace ptx;
using rows::F2;

PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder();

namespace {

constexpr int kQThreads = 320;
constexpr int kQEpilogue = 256;                  // threads of the epilogue: two groups of four warps
constexpr int kQM = 128;                         // tokens per tile and CTA
constexpr int kQHeads = 4;                       // heads per tile
constexpr int kQStages = 4;
constexpr uint32_t kQABytes = kQM * 128;         // 128 x 64 bf16
constexpr uint32_t kQBBytes = kQHeads * 32 * 128;  // this CTA's half of the tile's 256 weight rows
constexpr uint32_t kQStage = kQABytes + kQBBytes;
constexpr uint32_t kQBox = kQM * 128;            // one head of 128 tokens
constexpr uint32_t kQCols = 512;                 // TMEM: two 128 x 256 fp32 accumulators
constexpr uint64_t kQWaitNs = 2000000000ull;
constexpr uint64_t kQDrainNs = 200000000ull;

constexpr uint32_t kQOffOut = kQStages * kQStage;          // two boxes per epilogue group
constexpr uint32_t kQOffTurn = kQOffOut + kQHeads * kQBox;  // float4 [16][128 tokens]: of pairs 2q and
                                                           // 2q + 1 both cosines, both sines
constexpr uint32_t kQOffCtl = kQOffTurn + 32 * kQM * 8;

struct QCtl {
  __align__(16) float gain[2][64], shift[2][64];  // the norms of Q and K
  uint64_t full[kQStages], empty[kQStages], acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort;
};

// Which of a plan's rotations are unrolled: by the distance h of pairs (c, c xor h); the others pair
// by pair.
enum { kNoTurn = 0, kByPairs = -1 };

struct QParams {
  int N, K, H;
  int step, units;         // heads of a unit, units
  int turn, pairs, axes;   // turn: h, kNoTurn or kByPairs
  uint8_t lo[32], hi[32];  // channels of each pair
  uint8_t axis[32];
  uint64_t turns[32];
  const int32_t* pos;
  const uint16_t* bias[3];
  ress_head_norm norm[2];
  int param_type;
  float eps;
  uint32_t* status;
};

struct QMaps {
  CUtensorMap x, w[3], w_part[3], out[3];  // w: 128 weight rows at a time, w_part: 32
};

__device__ __forceinline__ bool q_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  int ok = 1;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity, abort, kQWaitNs) ? 1 : 0;
  ok = __shfl_sync(0xffffffffu, ok, 0);
  __syncwarp();
  return ok != 0;
}

__device__ __forceinline__ void q_give_up(QCtl& C, uint32_t* status) {
  flag_status(status, kStatusTimeout);
  *reinterpret_cast<volatile int*>(&C.abort) = 1;
}

// Barriers of all epilogue warps (the second also ANDs a flag across them) and of one group of
// four, in the form that does not ask for a converged warp.
__device__ __forceinline__ void q_epi_sync() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(kQEpilogue) : "memory"); }
__device__ __forceinline__ bool q_epi_sync_and(bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.pred q, 2, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(v ? 1u : 0u), "n"(kQEpilogue)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void q_group_sync(int group) {
  asm volatile("barrier.cta.sync %0, 128;" ::"r"(3 + group) : "memory");
}

// One column at each of two places of this warp's lanes, waited for in the same asm block so that no
// register is read before it is valid.
#define RESS_TMEM_LD1_TWICE(at0, a, at1, b)                 \
  asm volatile(                                             \
      "tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%2];\n\t" \
      "tcgen05.ld.sync.aligned.32x32b.x1.b32 {%1}, [%3];\n\t" \
      "tcgen05.wait::ld.sync.aligned;"                      \
      : "=&r"(a), "=&r"(b)                                  \
      : "r"(at0), "r"(at1)                                  \
      : "memory")

// A unit is up to `step` heads of one of Q, K, V of one token stripe: one tile.  The units of all
// stripes stand in a row (stripe, then Q, K, V, then head), and a pair's share is a range of them, so that
// a pair goes through its stripes' tiles one after the other: their x slices come from L2 and their
// cosines and sines are formed once.  step is 4, or fewer where each pair then still has one unit at
// most: a call on few tokens has single heads on many SMs.
struct QUnit {
  int mt, which, head, heads;
};
struct QCursor {
  int at, end;
  __device__ explicit QCursor(const QParams& p) {
    const int pairs = (int)gridDim.x >> 1, i = (int)blockIdx.x >> 1, rest = p.units % pairs;
    at = p.units / pairs * i + min(i, rest);
    end = at + p.units / pairs + (i < rest);
  }
  __device__ bool more() const { return at < end; }
  __device__ QUnit unit(const QParams& p) const {
    const int per = (p.H + p.step - 1) / p.step, in_stripe = at % (3 * per);
    QUnit t;
    t.mt = at / (3 * per);
    t.which = in_stripe / per;
    t.head = in_stripe % per * p.step;
    t.heads = min(p.step, p.H - t.head);
    return t;
  }
  __device__ void next() { ++at; }
};

// One head of one token: 64 columns of this thread's TMEM lane, to its row of an output box.
struct QHead {
  const uint16_t* bias;         // of the head, or NULL
  const float *gain, *shift;    // of the norm, or NULL
  float eps;
  const float4* turn;           // the token's entry of the cosines and sines
};

// The accumulators plus the bias.
__device__ __forceinline__ void q_add_bias(const uint16_t* bias, F2 (&u)[32]) {
  if (!bias) return;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const uint4 v = reinterpret_cast<const uint4*>(bias)[c];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) u[4 * c + j] = rows::add2(u[4 * c + j], rows::pack2(bf16_lo(w[j]), bf16_hi(w[j])));
  }
}

// The head's row: bias, norm and the unrolled rotation of pairs H apart (H = 0: none).  With a norm, mean and rstd
// are left for the pairs that are turned one by one afterwards (else 0 and 1).
template <int H>
__device__ __forceinline__ void q_head(uint32_t acc, const QHead& a, uint8_t* row, int r, float& mean, float& rstd) {
  using rows::add2;
  using rows::both;
  using rows::fma2;
  using rows::mul2;
  using rows::pack2;
  F2 u[32];  // channels 2j and 2j + 1
  {
    uint32_t v[64];
    __syncwarp();
    RESS_TMEM_LD64(acc, v);
#pragma unroll
    for (int j = 0; j < 32; ++j) u[j] = pack2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
  }
  q_add_bias(a.bias, u);
  mean = 0.f;
  rstd = 1.f;
  if (a.gain) {
    F2 s[2] = {both(0.f), both(0.f)};
#pragma unroll
    for (int j = 0; j < 32; ++j) s[j & 1] = add2(s[j & 1], u[j]);
    mean = rows::sum2(add2(s[0], s[1])) * (1.f / 64.f);
    const F2 m = both(-mean);
    s[0] = s[1] = both(0.f);
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      u[j] = add2(u[j], m);
      s[j & 1] = fma2(u[j], u[j], s[j & 1]);
    }
    rstd = rsqrtf(fmaf(rows::sum2(add2(s[0], s[1])), 1.f / 64.f, a.eps));
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      const float4 g = reinterpret_cast<const float4*>(a.gain)[c], b = reinterpret_cast<const float4*>(a.shift)[c];
      u[2 * c] = fma2(mul2(u[2 * c], both(rstd)), pack2(g.x, g.y), pack2(b.x, b.y));
      u[2 * c + 1] = fma2(mul2(u[2 * c + 1], both(rstd)), pack2(g.z, g.w), pack2(b.z, b.w));
    }
  }
  if constexpr (H > 0) {
#pragma unroll
    for (int q = 0; q < 16; ++q) {  // pairs 2q and 2q + 1
      const float4 t = a.turn[q * kQM];
      if constexpr (H == 1) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float c = e ? t.y : t.x, s = e ? t.w : t.z;
          float x, y;
          rows::unpack2(u[2 * q + e], x, y);
          u[2 * q + e] = pack2(fmaf(x, c, -y * s), fmaf(y, c, x * s));
        }
      } else {
        const int lo = (2 * q / H * 2 * H + 2 * q % H) / 2, hi = lo + H / 2;
        const F2 c = pack2(t.x, t.y), s = pack2(t.z, t.w), x = u[lo], y = u[hi];
        u[lo] = fma2(x, c, mul2(y, pack2(-t.z, -t.w)));
        u[hi] = fma2(y, c, mul2(x, s));
      }
    }
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x, y;
      rows::unpack2(u[4 * c + j], x, y);
      w[j] = cvt_bf16x2(x, y);
    }
    *reinterpret_cast<uint4*>(row + ((c ^ (r & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

__global__ void __launch_bounds__(kQThreads, 1)
    k_qkv(const __grid_constant__ QMaps maps, const __grid_constant__ QParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  QCtl& C = *reinterpret_cast<QCtl*>(base + kQOffCtl);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort = &C.abort;
  const int ksteps = p.K / 64;
  const int rank = (int)cluster_rank() & 1, lead = (int)cluster_rank() & ~1;
  const uint32_t both = 3u << lead;
  auto A = [&](int s) { return base + s * kQStage; };
  auto B = [&](int s) { return A(s) + kQABytes; };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kQStages; ++s) {
      mbar_init(&C.full[s], 1);
      mbar_init(&C.empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&C.acc_full[b], 1);
      mbar_init(&C.acc_empty[b], 2 * kQEpilogue / 32);  // the epilogue warps of both CTAs
    }
    C.abort = 0;
    fence_barrier_init();
    prefetch_tensormap(&maps.x);
    for (int i = 0; i < 3; ++i) {
      prefetch_tensormap(&maps.w[i]);
      prefetch_tensormap(&maps.out[i]);
    }
  }
  if (warp == 1) tmem_alloc_pair(&C.tmem_base, kQCols);
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers exist
  tc_fence_after();
  const uint32_t tmem = C.tmem_base;
  rows::stream_acquire();

  if (warp == 0) {
    // ================================ loads ==========================================
    int it = 0;
    bool failed = false;
    for (QCursor c(p); c.more() && !failed;) {
      const QUnit t = c.unit(p);
      c.next();
      const bool ahead = c.more() && c.unit(p).mt != t.mt;  // the next stripe into L2 meanwhile
      for (int ks = 0; ks < ksteps; ++ks, ++it) {
        const int s = it % kQStages, u = it / kQStages;
        if (u > 0 && !q_wait(&C.empty[s], (u - 1) & 1, abort)) {
          failed = true;
          break;
        }
        if (lane == 0) {
          if (rank == 0) mbar_arrive_expect_tx(&C.full[s], 2 * (kQABytes + t.heads * 32 * 128));
          const uint32_t full = cluster_addr(&C.full[s], lead);
          tma_load_3d_pair(A(s), &maps.x, full, 64 * ks, kQM * (2 * t.mt + rank), 0);
          const int row = 64 * t.head + 32 * t.heads * rank;  // this CTA's half of the unit's weight rows
          if (t.heads == kQHeads) {
            tma_load_3d_pair(B(s), &maps.w[t.which], full, 64 * ks, row, 0);
          } else {
            for (int h = 0; h < t.heads; ++h)
              tma_load_3d_pair(B(s) + h * 32 * 128, &maps.w_part[t.which], full, 64 * ks, row + 32 * h, 0);
          }
          if (ahead) tma_prefetch_3d(&maps.x, 64 * ks, kQM * (2 * t.mt + 2 + rank), 0);
        }
        __syncwarp();
      }
    }
    rows::stream_release();  // every slice of the CTA's tiles is on its way
    // the pair's MMAs release every stage in both CTAs: nothing arrives here after the end
    for (int q = max(0, it - kQStages); q < it && !failed; ++q)
      if (!q_wait(&C.empty[q % kQStages], (q / kQStages) & 1, abort)) failed = true;
    if (failed && lane == 0) {
      q_give_up(C, p.status);
      volatile int no_abort = 0;  // copies already issued land before the memory goes away
      for (int q = max(0, it - kQStages); q < it; ++q)
        mbar_wait(&C.full[q % kQStages], (q / kQStages) & 1, &no_abort, kQDrainNs);
    }
    __syncwarp();
  } else if (warp == 1 && rank == 0) {
    // ================================ MMAs ===========================================
    const bool leader = elect_one();
    int it = 0, n = 0;
    bool failed = false;
    if (__popc(__ballot_sync(0xffffffffu, leader)) != 1) {  // exactly one issuing lane
      if (lane == 0) {
        flag_status(p.status, kStatusBadRow);
        *abort = 1;
      }
      failed = true;
    }
    for (QCursor c(p); c.more() && !failed;) {
      const QUnit t = c.unit(p);
      c.next();
      const uint32_t idesc = idesc_bf16_f32(2 * kQM, 64 * t.heads, false);
      const int b = n & 1, use = n >> 1;  // the accumulator, its earlier uses
      ++n;
      if (use > 0 && !q_wait(&C.acc_empty[b], (use - 1) & 1, abort)) {
        failed = true;
        break;
      }
      tc_fence_after();
      const uint32_t acc = tmem + 256u * b;
      for (int ks = 0; ks < ksteps; ++ks, ++it) {
        const int s = it % kQStages;
        if (!q_wait(&C.full[s], (it / kQStages) & 1, abort)) {
          failed = true;
          break;
        }
        tc_fence_after();
        if (leader) {
          const uint32_t a = smem_u32(A(s)), bb = smem_u32(B(s));
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_bf16_ss_pair(acc, sdesc_sw128(a + 32 * kk), sdesc_sw128(bb + 32 * kk), idesc,
                             (ks > 0 || kk > 0) ? 1u : 0u);
          mma_commit_pair(&C.empty[s], both);
          if (ks + 1 == ksteps) mma_commit_pair(&C.acc_full[b], both);
        }
        __syncwarp();
      }
    }
    if (failed && lane == 0) {
      q_give_up(C, p.status);
      if (it > 0) {  // MMAs still running must finish before TMEM is freed
        volatile int no_abort = 0;
        const int q = it - 1;
        mbar_wait(&C.empty[q % kQStages], (q / kQStages) & 1, &no_abort, kQDrainNs);
      }
    }
    __syncwarp();
  } else if (warp > 1) {
    // ================================ epilogue =======================================
    const int group = (warp - 2) >> 2, quarter = warp & 3;
    const int r = 32 * quarter + lane;  // token of the CTA's tile = TMEM lane
    const int et = (int)threadIdx.x - 64;
    const bool leader = (warp - 2) % 4 == 0 && lane == 0;
    uint8_t* out = base + kQOffOut + 2 * group * kQBox;
    float4* turn = reinterpret_cast<float4*>(base + kQOffTurn);
    if (et < 64) {
      for (int i = 0; i < 2; ++i) {
        C.gain[i][et] = rows::param_at(p.norm[i].weight, p.param_type, et, 1.f);
        C.shift[i][et] = rows::param_at(p.norm[i].bias, p.param_type, et, 0.f);
      }
    }
    int n = 0, boxes = 0, table = -1;  // units done; boxes this group has stored; the table's stripe
    for (QCursor c(p); c.more();) {
      const QUnit t = c.unit(p);
      c.next();
      const int b = n & 1, use = n >> 1;
      ++n;
      const int row0 = kQM * (2 * t.mt + rank), which = t.which, mode = which < 2 ? p.turn : kNoTurn;
      if (mode != kNoTurn && table != t.mt) {  // the stripe's cosines and sines, while the unit's MMAs run
        table = t.mt;
        q_epi_sync();  // nobody reads the last stripe's any more
        const int64_t token = min(row0 + r, p.N - 1);
        for (int q = group; 2 * q < p.pairs; q += 2) {
          float2 cs[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int pair = min(2 * q + e, p.pairs - 1);
            cs[e] = rows::rope_cos_sin(p.pos[token * p.axes + p.axis[pair]], p.turns[pair]);
          }
          turn[q * kQM + r] = make_float4(cs[0].x, cs[1].x, cs[0].y, cs[1].y);
        }
      }
      const bool ok = q_wait(&C.acc_full[b], use & 1, abort);
      if (!q_epi_sync_and(ok)) {  // all leave together
        if (!ok && lane == 0) q_give_up(C, p.status);
        break;
      }
      tc_fence_after();
      QHead a;
      const bool norm = which < 2 && p.norm[which & 1].enabled;
      a.gain = norm ? C.gain[which & 1] : nullptr;
      a.shift = C.shift[which & 1];
      a.eps = p.eps;
      a.turn = turn + r;
      for (int h = group; h < t.heads; h += 2) {
        const uint32_t acc = tmem + ((uint32_t)(32 * quarter) << 16) + 256u * b + 64 * h;
        a.bias = p.bias[which] ? p.bias[which] + 64 * (t.head + h) : nullptr;
        // the box is free when the store before the last has read it
        uint8_t* box = out + (boxes & 1) * kQBox;
        ++boxes;
        if (leader) bulk_wait_read_but1();
        q_group_sync(group);
        uint8_t* row = box + r * 128;
        float mean, rstd;
        if (mode == 16)
          q_head<16>(acc, a, row, r, mean, rstd);
        else if (mode == 32)
          q_head<32>(acc, a, row, r, mean, rstd);
        else if (mode == 1)
          q_head<1>(acc, a, row, r, mean, rstd);
        else
          q_head<0>(acc, a, row, r, mean, rstd);
        if (mode == kByPairs) {
#pragma unroll 1
          for (int q = 0; q < p.pairs; ++q) {
            const int c[2] = {p.lo[q], p.hi[q]};
            uint32_t v[2];
            __syncwarp();
            RESS_TMEM_LD1_TWICE(acc + c[0], v[0], acc + c[1], v[1]);
            const float4 t4 = a.turn[q / 2 * kQM];
            const float cs = q % 2 ? t4.y : t4.x, sn = q % 2 ? t4.w : t4.z;
            float u[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              u[e] = __uint_as_float(v[e]) + (a.bias ? __uint_as_float((uint32_t)a.bias[c[e]] << 16) : 0.f);
              if (norm) u[e] = fmaf((u[e] - mean) * rstd, a.gain[c[e]], a.shift[c[e]]);
            }
            const float y[2] = {fmaf(u[0], cs, -u[1] * sn), fmaf(u[1], cs, u[0] * sn)};
#pragma unroll
            for (int e = 0; e < 2; ++e)
              reinterpret_cast<uint16_t*>(row + (((c[e] >> 3) ^ (r & 7)) << 4))[c[e] & 7] = cvt_bf16(y[e]);
          }
        }
        fence_proxy_async_smem();
        q_group_sync(group);
        if (leader) {
          if (row0 < p.N) tma_store_3d(&maps.out[which], box, 64 * (t.head + h), row0, 0);
          bulk_commit();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(cluster_addr(&C.acc_empty[b], lead));  // may be reused
    }
    if (leader) bulk_wait_read_all();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // the pair's MMAs and barrier arrivals are over in both CTAs
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, kQCols);
  }
}

// A row-major bf16 matrix [rows, cols] as a 3-D tensor {cols, rows, 1}; box {64, box_rows, 1},
// 128-byte swizzle.  Loads past the edges read zeros; stores past them are dropped.
bool make_map(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int box_rows) {
  auto fn = tensor_map_encoder();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, 1};
  cuuint64_t strides[2] = {(cuuint64_t)cols * 2, (cuuint64_t)rows * cols * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t launch_qkv_proj(const QkvArgs& a, cudaStream_t st) {
  QParams p{};
  p.N = a.N;
  p.K = a.Dm;
  p.H = a.H;
  const int pairs = max(1, rows::sm_count() / 2);
  for (p.step = 1; p.step <= kQHeads; p.step *= 2) {
    p.units = (a.N + 2 * kQM - 1) / (2 * kQM) * 3 * ((a.H + p.step - 1) / p.step);
    if (p.step == kQHeads || p.units <= pairs) break;
  }
  // a map takes the host a good part of what the GPU needs for a few tokens: those that the units use
  QMaps m;
  const int64_t out = (int64_t)a.H * 64;
  const bool whole = p.step == kQHeads && a.H >= kQHeads, part = p.step < kQHeads || a.H % kQHeads != 0;
  bool made = make_map(&m.x, a.x, a.N, a.Dm, kQM);
  for (int i = 0; i < 3; ++i) {
    if (whole) made = made && make_map(&m.w[i], a.W[i], out, a.Dm, 32 * kQHeads);
    if (part) made = made && make_map(&m.w_part[i], a.W[i], out, a.Dm, 32);
    if (!whole) m.w[i] = m.w_part[i];
    if (!part) m.w_part[i] = m.w[i];
    made = made && make_map(&m.out[i], a.out[i], a.N, out, kQM);
  }
  if (!made) return cudaErrorInvalidValue;
  p.turn = kNoTurn;
  if (a.rotate) {
    const ress_rope_plan& plan = a.plan;
    p.pairs = plan.n_pairs;
    p.axes = plan.n_axes;
    int first = 0, k = 0;  // of the axis: its first channel, its first pair
    for (int t = 0; t < plan.n_axes; ++t) {
      const int half = plan.axis_dims[t] / 2;
      for (int i = 0; i < half; ++i, ++k) {
        p.axis[k] = (uint8_t)t;
        p.turns[k] = plan.turns[k];
        p.lo[k] = (uint8_t)(plan.layout == RESS_ROPE_SECTIONS ? first + i : plan.layout == RESS_ROPE_HALVES ? k : 2 * k);
        p.hi[k] = (uint8_t)(p.lo[k] + (plan.layout == RESS_ROPE_SECTIONS ? half
                                       : plan.layout == RESS_ROPE_HALVES ? plan.n_pairs : 1));
      }
      first += 2 * half;
    }
    // all channels turn, pair k at distance h where an unrolled rotation has it
    p.turn = kByPairs;
    for (int h : {1, 16, 32}) {
      bool fits = p.pairs == 32;
      for (k = 0; fits && k < p.pairs; ++k) fits = p.lo[k] == k / h * 2 * h + k % h && p.hi[k] == p.lo[k] + h;
      if (fits) p.turn = h;
    }
  }
  p.pos = a.pos;
  for (int i = 0; i < 3; ++i) p.bias[i] = a.b[i];
  for (int i = 0; i < 2; ++i) p.norm[i] = a.norm[i];
  p.param_type = a.param_type;
  p.eps = a.eps;
  p.status = a.status;
  const size_t smem = kQOffCtl + sizeof(QCtl) + 1024;
  static_assert(kQOffCtl + sizeof(QCtl) + 1024 <= 227 * 1024, "shared memory of a CTA");
  cudaError_t e = cudaFuncSetAttribute(k_qkv, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_with(k_qkv, 2 * min(p.units, pairs), kQThreads, smem, st, true, 2, m, p);
}

}  // namespace ress

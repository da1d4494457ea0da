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
//              per token: a head's 64 channels are 64 columns of the thread's TMEM lane, so the norm's
//              two sums need no other thread, and the two channels of a pair, wherever the plan has
//              them, are columns of the same lane, read 8 at a time.  The cosines and sines of the
//              CTA's 128 tokens are formed in shared memory while the tile's MMAs run.
// Waits are bounded as in k_oproj.cu.

#include <cudaTypedefs.h>

#include "row_ops.cuh"

namespace ress {
using namespace ptx;

PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder();

namespace {

constexpr int kQThreads = 320;
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
constexpr uint32_t kQOffTurn = kQOffOut + 4 * kQBox;       // float2 [32 pairs][128 tokens]
constexpr uint32_t kQOffCtl = kQOffTurn + 32 * kQM * 8;

struct QCtl {
  uint16_t bias[kQHeads * 64];
  float weight[2][64], shift[2][64];  // the norms of Q and K
  uint64_t full[kQStages], empty[kQStages], acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort;
};

// How the epilogue walks a head's channels.
enum { kPlain = 0, kBlocks = 1, kNeighbours = 2, kSingle = 3 };

struct QParams {
  int N, K, H, mtiles;
  int tiles_of;            // tiles of one of Q, K, V: ceil(H / 4)
  int whole, parts;        // the first `whole` tiles run whole, the others as `parts` units each
  int walk, pairs, axes;
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

// Barriers of the eight epilogue warps (the second also ANDs a flag across them) and of one group of
// four, in the form that does not ask for a converged warp.
__device__ __forceinline__ void q_epi_sync() { asm volatile("barrier.cta.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ bool q_epi_sync_and(bool v) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "barrier.cta.red.and.pred q, 2, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(v ? 1u : 0u)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void q_group_sync(int group) {
  asm volatile("barrier.cta.sync %0, 128;" ::"r"(3 + group) : "memory");
}

// 8 (or 1) columns at each of two places, or 8 at one, of this warp's lanes, waited for in the same asm
// block so that no register is read before it is valid.
#define RESS_TMEM_LD8_TWICE(at0, a, at1, b)                                                          \
  asm volatile(                                                                                      \
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%16];\n\t"                  \
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%8,%9,%10,%11,%12,%13,%14,%15}, [%17];\n\t"            \
      "tcgen05.wait::ld.sync.aligned;"                                                               \
      : "=&r"(a[0]), "=&r"(a[1]), "=&r"(a[2]), "=&r"(a[3]), "=&r"(a[4]), "=&r"(a[5]), "=&r"(a[6]),   \
        "=&r"(a[7]), "=&r"(b[0]), "=&r"(b[1]), "=&r"(b[2]), "=&r"(b[3]), "=&r"(b[4]), "=&r"(b[5]),   \
        "=&r"(b[6]), "=&r"(b[7])                                                                     \
      : "r"(at0), "r"(at1)                                                                           \
      : "memory")
#define RESS_TMEM_LD8(at, a)                                                                         \
  asm volatile(                                                                                      \
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\t"                   \
      "tcgen05.wait::ld.sync.aligned;"                                                               \
      : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]), "=r"(a[4]), "=r"(a[5]), "=r"(a[6]), "=r"(a[7]) \
      : "r"(at)                                                                                      \
      : "memory")
#define RESS_TMEM_LD1_TWICE(at0, a, at1, b)                                                          \
  asm volatile(                                                                                      \
      "tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%2];\n\t"                                        \
      "tcgen05.ld.sync.aligned.32x32b.x1.b32 {%1}, [%3];\n\t"                                        \
      "tcgen05.wait::ld.sync.aligned;"                                                               \
      : "=&r"(a), "=&r"(b)                                                                           \
      : "r"(at0), "r"(at1)                                                                           \
      : "memory")

// One unit of work of a pair: token stripe mt, `heads` heads from `head` on of Q, K or V (which).
struct QUnit {
  int mt, which, head, heads;
};
__device__ __forceinline__ int q_units(const QParams& p) {
  const int units = p.whole + (p.mtiles * 3 * p.tiles_of - p.whole) * p.parts;
  return (units - 1 - (int)(blockIdx.x >> 1)) / (int)(gridDim.x >> 1) + 1;
}
__device__ __forceinline__ QUnit q_unit(const QParams& p, int k) {
  const int u = (int)(blockIdx.x >> 1) + k * (int)(gridDim.x >> 1);
  int tile = u, part = 0, parts = 1;
  if (u >= p.whole) {
    parts = p.parts;
    tile = p.whole + (u - p.whole) / parts;
    part = (u - p.whole) % parts;
  }
  // consecutive tiles share their token stripe, so x slices are re-read from L2
  const int per = 3 * p.tiles_of, j = tile % per, heads = kQHeads / parts;
  QUnit t;
  t.mt = tile / per;
  t.which = j / p.tiles_of;
  t.head = kQHeads * (j % p.tiles_of) + heads * part;
  t.heads = max(0, min(heads, p.H - t.head));  // a part past the last head has none
  return t;
}

__global__ void __launch_bounds__(kQThreads, 1)
    k_qkv(const __grid_constant__ QMaps maps, const __grid_constant__ QParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  QCtl& C = *reinterpret_cast<QCtl*>(base + kQOffCtl);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort = &C.abort;
  const int ksteps = p.K / 64, nunits = q_units(p);
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
      mbar_init(&C.acc_empty[b], 16);  // the epilogue warps of both CTAs
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
    for (int k = 0; k < nunits && !failed; ++k) {
      const QUnit t = q_unit(p, k);
      if (t.heads == 0) continue;
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
    for (int k = 0; k < nunits && !failed; ++k) {
      const QUnit t = q_unit(p, k);
      if (t.heads == 0) continue;
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
    float2* turn = reinterpret_cast<float2*>(base + kQOffTurn);
    if (et < 64) {
      for (int i = 0; i < 2; ++i) {
        const ress_head_norm& m = p.norm[i];
        C.weight[i][et] = m.enabled ? rows::param_at(m.weight, p.param_type, et, 1.f) : 1.f;
        C.shift[i][et] = m.enabled ? rows::param_at(m.bias, p.param_type, et, 0.f) : 0.f;
      }
    }
    int n = 0, boxes = 0, table = -1;  // units done; boxes this group has stored; the table's stripe
    for (int k = 0; k < nunits; ++k) {
      const QUnit t = q_unit(p, k);
      if (t.heads == 0) continue;
      const int b = n & 1, use = n >> 1;
      ++n;
      const int row0 = kQM * (2 * t.mt + rank), which = t.which;
      // the unit's bias and the stripe's cosines and sines, while its MMAs run
      q_epi_sync();  // nobody reads the last unit's any more
      if (et < 64 * t.heads)
        C.bias[et] = p.bias[which] ? p.bias[which][64 * t.head + et] : (uint16_t)0;
      if (which < 2 && p.walk != kPlain && table != t.mt) {
        table = t.mt;
        const int64_t token = min(row0 + r, p.N - 1);
        for (int q = group; q < p.pairs; q += 2)
          turn[q * kQM + r] = rows::rope_cos_sin(p.pos[token * p.axes + p.axis[q]], p.turns[q]);
      }
      const bool ok = q_wait(&C.acc_full[b], use & 1, abort);
      if (!q_epi_sync_and(ok)) {  // all leave together
        if (!ok && lane == 0) q_give_up(C, p.status);
        break;
      }
      tc_fence_after();
      for (int h = group; h < t.heads; h += 2) {
        const uint32_t acc = tmem + ((uint32_t)(32 * quarter) << 16) + 256u * b + 64 * h;
        const uint16_t* bias_bits = C.bias + 64 * h;
        auto bias = [&](int c) { return __uint_as_float((uint32_t)bias_bits[c] << 16); };
        const int side = which & 1;
        float mean = 0.f, rstd = 1.f;
        if (which < 2 && p.norm[side].enabled) {
          uint32_t v[64];
          __syncwarp();
          RESS_TMEM_LD64(acc, v);
          float sum = 0.f;
#pragma unroll
          for (int c = 0; c < 64; ++c) {
            const float u = __uint_as_float(v[c]) + bias(c);
            v[c] = __float_as_uint(u);
            sum += u;
          }
          mean = sum * (1.f / 64.f);
          float sq = 0.f;
#pragma unroll
          for (int c = 0; c < 64; ++c) {
            const float u = __uint_as_float(v[c]) - mean;
            sq = fmaf(u, u, sq);
          }
          rstd = rsqrtf(fmaf(sq, 1.f / 64.f, p.eps));
        }
        // the box is free when the store before the last has read it
        uint8_t* box = out + (boxes & 1) * kQBox;
        ++boxes;
        if (leader) bulk_wait_read_but1();
        q_group_sync(group);
        uint8_t* row = box + r * 128;
        const float* gain = C.weight[side];
        const float* shift = C.shift[side];
        // a channel's value from its accumulator: bias, norm
        auto value = [&](uint32_t bits, int c) {
          const float u = __uint_as_float(bits) + bias(c);
          return which < 2 ? fmaf((u - mean) * rstd, gain[c], shift[c]) : u;
        };
        auto chunk = [&](int c) { return reinterpret_cast<uint4*>(row + (((c >> 3) ^ (r & 7)) << 4)); };
        const int walk = which < 2 ? p.walk : kPlain;
        int done = 0;  // channels below this one are written
        if (walk == kBlocks) {
#pragma unroll 1
          for (int q = 0; q < p.pairs; q += 8) {
            const int lo = p.lo[q], hi = p.hi[q];
            uint32_t a[8], c[8];
            float ya[8], yc[8];
            __syncwarp();
            RESS_TMEM_LD8_TWICE(acc + lo, a, acc + hi, c);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float2 cs = turn[(q + j) * kQM + r];
              const float ua = value(a[j], lo + j), uc = value(c[j], hi + j);
              ya[j] = fmaf(ua, cs.x, -uc * cs.y);
              yc[j] = fmaf(uc, cs.x, ua * cs.y);
            }
            *chunk(lo) = make_uint4(cvt_bf16x2(ya[0], ya[1]), cvt_bf16x2(ya[2], ya[3]),
                                    cvt_bf16x2(ya[4], ya[5]), cvt_bf16x2(ya[6], ya[7]));
            *chunk(hi) = make_uint4(cvt_bf16x2(yc[0], yc[1]), cvt_bf16x2(yc[2], yc[3]),
                                    cvt_bf16x2(yc[4], yc[5]), cvt_bf16x2(yc[6], yc[7]));
          }
          done = 2 * p.pairs;
        } else if (walk == kNeighbours) {
          // 8 channels at a time; a last block may have fewer than 4 pairs
#pragma unroll 1
          for (int q = 0; q < p.pairs; q += 4) {
            uint32_t a[8];
            float y[8];
            __syncwarp();
            RESS_TMEM_LD8(acc + 2 * q, a);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float u = value(a[2 * j], 2 * (q + j)), v = value(a[2 * j + 1], 2 * (q + j) + 1);
              const float2 cs = q + j < p.pairs ? turn[(q + j) * kQM + r] : make_float2(1.f, 0.f);
              y[2 * j] = q + j < p.pairs ? fmaf(u, cs.x, -v * cs.y) : u;
              y[2 * j + 1] = q + j < p.pairs ? fmaf(v, cs.x, u * cs.y) : v;
            }
            *chunk(2 * q) = make_uint4(cvt_bf16x2(y[0], y[1]), cvt_bf16x2(y[2], y[3]), cvt_bf16x2(y[4], y[5]),
                                       cvt_bf16x2(y[6], y[7]));
          }
          done = (2 * p.pairs + 7) & ~7;
        } else if (walk == kSingle) {
          // the whole head without rotation first (below), then the pairs one by one over it
          done = 0;
        }
#pragma unroll 1
        for (; done < 64; done += 8) {
          uint32_t a[8];
          float y[8];
          __syncwarp();
          RESS_TMEM_LD8(acc + done, a);
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = value(a[j], done + j);
          *chunk(done) = make_uint4(cvt_bf16x2(y[0], y[1]), cvt_bf16x2(y[2], y[3]), cvt_bf16x2(y[4], y[5]),
                                    cvt_bf16x2(y[6], y[7]));
        }
        if (walk == kSingle) {
#pragma unroll 1
          for (int q = 0; q < p.pairs; ++q) {
            const int lo = p.lo[q], hi = p.hi[q];
            uint32_t a, c;
            __syncwarp();
            RESS_TMEM_LD1_TWICE(acc + lo, a, acc + hi, c);
            const float2 cs = turn[q * kQM + r];
            const float ua = value(a, lo), uc = value(c, hi);
            reinterpret_cast<uint16_t*>(chunk(lo))[lo & 7] = cvt_bf16(fmaf(ua, cs.x, -uc * cs.y));
            reinterpret_cast<uint16_t*>(chunk(hi))[hi & 7] = cvt_bf16(fmaf(uc, cs.x, ua * cs.y));
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
  QMaps m;
  const int64_t out = (int64_t)a.H * 64;
  if (!make_map(&m.x, a.x, a.N, a.Dm, kQM)) return cudaErrorInvalidValue;
  for (int i = 0; i < 3; ++i)
    if (!make_map(&m.w[i], a.W[i], out, a.Dm, 32 * kQHeads) || !make_map(&m.w_part[i], a.W[i], out, a.Dm, 32) ||
        !make_map(&m.out[i], a.out[i], a.N, out, kQM))
      return cudaErrorInvalidValue;
  QParams p{};
  p.N = a.N;
  p.K = a.Dm;
  p.H = a.H;
  p.mtiles = (a.N + 2 * kQM - 1) / (2 * kQM);
  p.tiles_of = (a.H + kQHeads - 1) / kQHeads;
  p.walk = kPlain;
  if (a.rotate) {
    const ress_rope_plan& plan = a.plan;
    p.pairs = plan.n_pairs;
    p.axes = plan.n_axes;
    bool blocks = plan.layout != RESS_ROPE_INTERLEAVED;  // whole blocks of 8 pairs
    for (int c = 0; c < 2 * plan.n_pairs; ++c) {
      const rows::RopeChannel r = rows::rope_channel(plan, c);
      (r.second ? p.hi : p.lo)[r.pair] = (uint8_t)c;
    }
    for (int q = 0; q < plan.n_pairs; ++q) {
      p.axis[q] = (uint8_t)rows::rope_axis(plan, q);
      p.turns[q] = plan.turns[q];
    }
    blocks = blocks && plan.n_pairs % 8 == 0;
    for (int q = 0; blocks && q < plan.n_pairs; q += 8)
      blocks = p.lo[q] % 8 == 0 && p.hi[q] % 8 == 0 && p.lo[q + 7] == p.lo[q] + 7 && p.hi[q + 7] == p.hi[q] + 7;
    p.walk = plan.layout == RESS_ROPE_INTERLEAVED ? kNeighbours : blocks ? kBlocks : kSingle;
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
  const int tiles = p.mtiles * 3 * p.tiles_of, slots = max(1, rows::sm_count() / 2);
  // tiles past the last whole wave of pairs run as 2 or 4 units of fewer heads where those fit into one
  p.whole = tiles;
  p.parts = 1;
  const int left = tiles % slots;
  if (left > 0 && 2 * left <= slots) {
    p.whole = tiles - left;
    p.parts = 4 * left <= slots ? 4 : 2;
  }
  const int units = p.whole + (tiles - p.whole) * p.parts;
  return launch_with(k_qkv, 2 * min(units, slots), kQThreads, smem, st, true, 2, m, p);
}

}  // namespace ress

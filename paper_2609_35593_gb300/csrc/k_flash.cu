// Dense attention over packed sequences or a paged cache: O = softmax(s) V for the keys that each row sees,
// with s = cap tanh(q.k / 8 / cap) - slope |distance|, and log sum exp(s) of each row.
//
// One CTA per SM walks its share of the work (attn_work.cuh).  An item is 2 x 128 rows of one head of K and V:
// floor(128 / group) tokens, each with its `group` heads of Q, make 128 rows, so that heads which share K read it
// once and single tokens still fill rows.  The two halves ("slots") share the 64-key tiles that TMA brings
// in, which halves what comes from L2: at the tensor cores' peak a tile of 16 KB per 128 rows would need 64 bytes
// per cycle and SM.  Warp roles (320 threads):
//   warp 0      item and tile producer: TMA of Q, K and V (128-byte swizzle), 10 stages of 16 KB, so that single
//               tokens, which only stream the cache, keep 160 KB per SM in flight
//   warp 1      TMEM owner and MMA issuer, per tile and slot: S = Q K^T (M128 N64 K64, Q copied to TMEM) and,
//               one tile later, O += P V (P from TMEM, V MN-major); S is double-buffered
//   warps 2-5, 6-9  one row of slot 0, 1 per thread: online softmax in the exp2 domain.  The reference maximum is only
//               raised when a tile exceeds it by 2^8 (what P's 16 bits and O's 32 hold easily), so O in TMEM is
//               rescaled seldom; sums are float32, of the exponentials before they are rounded to 16 bits.
// Rows of V behind a sequence's last key are zeroed in shared memory (0 x NaN of a cache page never written
// would be NaN); keys there and masked ones are -inf by selection, whatever their scores are.
// Every mbarrier wait is bounded; one that gives up records RESS_ETIMEOUT and the CTA leaves, see k_attn.cu.
#include <cudaTypedefs.h>

#include "attn_work.cuh"

namespace ress {
using namespace ptx;
using namespace work;

namespace {

constexpr int kThreads = 320, kStages = 10, kSlots = 2, kItems = 4;
constexpr uint32_t kTileBytes = kTile * 128;
constexpr uint32_t kColSlot = 256, kColO = 128, kColQ = 192;  // TMEM: per slot S x 2, O, Q
constexpr int kFirst = 1, kTerm = 2, kHas = 4;
constexpr float kLazy = 8.0f;  // log2 units
// Lowest reference maximum: finite, so that rows that have seen no key yet give exponentials of 0.
constexpr float kMinRef = -2147483648.0f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int64_t kPartFloats = 256 * 66;  // a slot of partial results: 256 rows of 64, maxima, sums

struct Item {
  int q0, nq, nk, d, p;      // the sequence
  int h, tok;                // head of K, first token (of the sequence)
  int t0, t1, g0;            // tiles; number of the first among all of the CTA's
  int n[kSlots];             // tiles of each slot's keys
  int part;                  // slot of partial results, or -1: whole
};

struct __align__(1024) Smem {
  uint8_t Q[kSlots][128 * 128];
  uint8_t K[kStages][kTileBytes];
  uint8_t V[kStages][kTileBytes];
  uint64_t kv_full[kStages], kv_empty[kStages];
  uint64_t q_full, q_empty, drain;
  uint64_t s_full[kSlots][2], p_full[kSlots][2], o_full[kSlots][2];
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

// Tokens of slot s of an item, and the tiles of the keys that any of them sees.
__device__ __forceinline__ int slot_tokens(int nq, int tok, int s, int T) { return max(0, min(T, nq - tok - s * T)); }
__device__ __forceinline__ int slot_tiles(const DenseArgs& a, const Seq& q, int tok, int s, int T) {
  const int n = slot_tokens(q.nq, tok, s, T);
  if (n == 0) return 0;
  return (max(0, row_limit(a, q, q.d + tok + s * T + n - 1)) + kTile - 1) / kTile;
}

template <bool kF16>
__device__ __forceinline__ void store_row(void* dst, const uint32_t (&o)[2][32], float by) {
  uint4* p = static_cast<uint4*>(dst);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = 8 * k + 2 * e;
      w[e] = pack2<kF16>(__uint_as_float(o[c >> 5][c & 31]) * by, __uint_as_float(o[c >> 5][(c & 31) + 1]) * by);
    }
    p[k] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

}  // namespace

// kGen: scores with a cap or slopes.
template <bool kF16, bool kGen>
__global__ void __launch_bounds__(kThreads, 1)
    k_flash(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
            const __grid_constant__ CUtensorMap tmV, const __grid_constant__ DenseArgs a) {
  extern __shared__ uint8_t smem_raw[];
  Smem& S = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort = &S.abort;
  const int G = a.group, T = 128 / G;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&S.kv_full[s], 1);
      mbar_init(&S.kv_empty[s], 1);
    }
    mbar_init(&S.q_full, 1);
    mbar_init(&S.q_empty, 1);
    mbar_init(&S.drain, 1);
    for (int s = 0; s < kSlots; ++s) {
      for (int b = 0; b < 2; ++b) {
        mbar_init(&S.s_full[s][b], 1);
        mbar_init(&S.p_full[s][b], 4);
        mbar_init(&S.o_full[s][b], 1);
      }
    }
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&S.it_full[i], 1);
      mbar_init(&S.it_empty[i], 8);
    }
    S.abort = 0;
    fence_barrier_init();
    prefetch_tensormap(&tmQ);
    prefetch_tensormap(&tmK);
    prefetch_tensormap(&tmV);
  }
  if (warp == 1) tmem_alloc(&S.tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = S.tmem_base;
  rows::stream_acquire();
  auto line_of = [&](const Seq& s) { return row_line(a, s, kSlots * T, T); };
  const Range range = find_range(a, line_of, gridDim.x, blockIdx.x, S.scratch, blockIdx.x == 0 ? a.status : nullptr);

  if (warp == 0) {
    // =============================== producer ====================================
    int g = 0, it = 0, pub = 0;
    bool failed = false, q_loaded = false;
    const int box = a.table ? min(kTile, a.page & -a.page) : kTile;  // the page's power of two
    const int boxes = kTile / box;
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
        item.q0 = c.s.q0, item.nq = c.s.nq, item.nk = c.s.nk, item.d = c.s.d, item.p = c.s.p;
        item.h = c.h, item.tok = c.j * kSlots * T;
        int n = 0;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) n = max(n, item.n[s] = slot_tiles(a, c.s, item.tok, s, T));
        tiles_of(c, range.x0, range.x1, n, item.t0, item.t1);
        item.g0 = g;
        item.part = item.t0 == 0 && item.t1 == n ? -1 : 2 * (int)blockIdx.x + (c.start >= range.x0 ? 1 : 0);
        if (item.t0 == item.t1 && (n > 0 || c.start < range.x0)) continue;
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
          const bool two = item.n[1] > item.t0, one = item.n[0] > item.t0;
          mbar_arrive_expect_tx(&S.q_full, T * G * 128 * ((one ? 1 : 0) + (two ? 1 : 0)));
          if (one) tma_load_4d(S.Q[0], &tmQ, &S.q_full, 0, 0, c.h, item.q0 + item.tok);
          if (two) tma_load_4d(S.Q[1], &tmQ, &S.q_full, 0, 0, c.h, item.q0 + item.tok + T);
        }
        __syncwarp();
        q_loaded = true;
        // where this lane's box of a tile is: lanes 0..boxes-1 load K, the next ones V
        const bool mine = lane < 2 * boxes;
        const int at = (lane < boxes ? lane : lane - boxes) * box;  // its first key in the tile
        auto place = [&](int t, int& row, int& page) {
          row = c.s.k0 + t * kTile + at, page = 0;
          if (!a.table) return;
          const int key = t * kTile + at;
          row = key % a.page, page = (int)a.n_pages;  // no such page: TMA fills in zeros
          if (mine && key < item.nk) {
            const int id = a.table[c.b * a.table_stride + key / a.page];
            if (id >= 0 && id < a.n_pages)
              page = id;
            else
              flag_status(a.status, kStatusBadIndex);
          }
        };
        int row, page;
        place(item.t0, row, page);
        for (int t = item.t0; t < item.t1; ++t) {
          const int s = g % kStages, u = g / kStages;
          int next_row = 0, next_page = 0;
          if (t + 1 < item.t1) place(t + 1, next_row, next_page);
          if (u > 0 && !wait(&S.kv_empty[s], (u - 1) & 1, abort)) {
            failed = true;
            break;
          }
          if (lane == 0) {
            S.flags[s] = (t == item.t0 ? kFirst : 0) | (t < item.n[0] ? kHas : 0) | (t < item.n[1] ? 2 * kHas : 0);
            mbar_arrive_expect_tx(&S.kv_full[s], 2 * kTileBytes);
          }
          __syncwarp();
          if (mine)
            tma_load_4d((lane < boxes ? S.K[s] : S.V[s]) + at * 128, lane < boxes ? &tmK : &tmV, &S.kv_full[s], 0,
                        c.h, row, page);
          __syncwarp();
          row = next_row, page = next_page;
          ++g;
        }
        if (failed) break;
        ++it;
        q_loaded = false;
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
      if (q_loaded) mbar_wait(&S.q_full, it & 1, &no_abort, kDrainNs);
    }
  } else if (warp == 1) {
    // ================================ MMA issuer ===================================
    const bool leader = elect_one();
    bool failed = false;
    constexpr uint32_t kQk = idesc16<kF16>(128, kTile, false), kPv = idesc16<kF16>(128, 64, true);
    constexpr uint64_t kStageUnits = kTileBytes >> 4;
    const uint64_t kd0 = sdesc_sw128(smem_u32(S.K[0])), vd0 = sdesc_sw128(smem_u32(S.V[0]));
    int it = 0, ns[kSlots] = {0, 0}, np[kSlots] = {0, 0};  // S and P V of each slot so far
    auto fetch = [&](int t, int& flags) -> bool {
      if (!wait(&S.kv_full[t % kStages], (t / kStages) & 1, abort)) return false;
      flags = S.flags[t % kStages];
      return true;
    };
    auto issue_pv = [&](int t, int flags) -> bool {
      const int st = t % kStages;
      const uint64_t vd = vd0 + (uint64_t)st * kStageUnits;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        if (!(flags & (kHas << s))) continue;
        const int b = np[s] & 1;
        if (!wait(&S.p_full[s][b], (np[s] >> 1) & 1, abort)) return false;
        tc_fence_after();
        if (leader) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma_bf16_ts(tmem + s * kColSlot + kColO, tmem + s * kColSlot + 64 * b + 8 * k, vd + 128 * k, kPv,
                        (k > 0 || !(flags & kFirst)) ? 1u : 0u);
          mma_commit(&S.o_full[s][b]);
        }
        __syncwarp();
        ++np[s];
      }
      if (leader) mma_commit(&S.kv_empty[st]);
      __syncwarp();
      return true;
    };
    int flags = kTerm, prev = 0;
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
          for (int s = 0; s < kSlots; ++s)
            if (flags & (kHas << s))
#pragma unroll
              for (int k = 0; k < 4; ++k)
                tmem_cp_128x256b(tmem + s * kColSlot + kColQ + 8 * k, sdesc_sw128(smem_u32(S.Q[s]) + 32 * k));
          mma_commit(&S.q_empty);
        }
        __syncwarp();
        ++it;
      }
      const uint64_t kd = kd0 + (uint64_t)(g % kStages) * kStageUnits;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) {
        if (!(flags & (kHas << s))) continue;
        const int b = ns[s] & 1;
        if (leader) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mma_bf16_ts(tmem + s * kColSlot + 64 * b, tmem + s * kColSlot + kColQ + 8 * k, kd + 2 * k, kQk, k > 0 ? 1u : 0u);
          mma_commit(&S.s_full[s][b]);
        }
        __syncwarp();
        ++ns[s];
      }
      const int cur = flags;
      if (!fetch(g + 1, flags) || (g > 0 && !issue_pv(g - 1, prev)) || ((flags & kTerm) && !issue_pv(g, cur))) {
        failed = true;
        break;
      }
      prev = cur;
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
    // ================================ softmax =====================================
    const int slot = (warp - 2) >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;             // row within the slot
    const int tid = (warp - 2 - 4 * slot) * 32 + lane;  // 0..127, for the zeroing of V
    const uint32_t tm = tmem + slot * kColSlot + ((uint32_t)(quarter * 32) << 16);
    const float kScale = kGen ? 1.0f : kLog2e * 0.125f;
    const float cap = a.cap, in = a.cap > 0.f ? 0.125f / a.cap : 0.125f * kLog2e, out = a.cap * kLog2e;
    // p = 2^(x kScale - m) of this row's 64 columns, packed; returns their sum
    auto exps = [&](const float (&x)[64], float m, uint32_t (&w)[32]) -> float {
      const float nm = -m;
      float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        float t0, t1;
        fma2(t0, t1, x[2 * e], x[2 * e + 1], kScale, kScale, nm, nm);
        t0 = ex2(t0), t1 = ex2(t1);
        w[e] = pack2<kF16>(t0, t1);
        if (e & 1)
          add2(s2, s3, s2, s3, t0, t1);
        else
          add2(s0, s1, s0, s1, t0, t1);
      }
      return (s0 + s2) + (s1 + s3);
    };
    auto row_max = [&](const float (&x)[64]) -> float {
      float m1[22];
#pragma unroll
      for (int k = 0; k < 21; ++k) m1[k] = fmax3(x[3 * k], x[3 * k + 1], x[3 * k + 2]);
      m1[21] = x[63];
      float m2[8];
#pragma unroll
      for (int k = 0; k < 7; ++k) m2[k] = fmax3(m1[3 * k], m1[3 * k + 1], m1[3 * k + 2]);
      m2[7] = m1[21];
      return fmax3(fmax3(m2[0], m2[1], m2[2]), fmax3(m2[3], m2[4], m2[5]), fmaxf(m2[6], m2[7]));
    };
    int c = 0;  // tiles of this slot so far
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
      const int ntok = slot_tokens(item.nq, item.tok, slot, T);
      const int tiles = max(0, min(item.t1, item.n[slot]) - item.t0);
      const int tok = item.tok + slot * T + r / G;  // of the sequence
      const bool exists = r / G < ntok;
      const int pos = item.d + tok;
      const int lim = !exists ? 0 : a.causal ? min(item.nk, max(item.p, pos + 1)) : item.nk;
      // rows that do not exist see what the last one does: no tile is masked for them alone
      const int least = __reduce_min_sync(0xffffffffu, exists ? max(lim, 0) : INT32_MAX);
      const bool any = __any_sync(0xffffffffu, exists);
      const int head = item.h * G + r % G;
      float slope = 0.f;
      if (kGen && a.slopes && exists) slope = a.slopes[head] * kLog2e;
      float m = -INFINITY, l = 0.f;  // reference maximum (log2 units), sum of the exponentials against it
      for (int k = 0; k < tiles; ++k, ++c) {
        const int b = c & 1, key = (item.t0 + k) * kTile;
        if (!wait(&S.s_full[slot][b], (c >> 1) & 1, abort)) {
          give_up(S, a.status);
          stop = true;
          break;
        }
        tc_fence_after();
        if (any) {  // rows of a warp without any are garbage that nothing reads
          const uint32_t tS = tm + 64 * b;
          float x[64];
          {
            uint32_t v[64];
            RESS_TMEM_LD64(tS, v);
#pragma unroll
            for (int e = 0; e < 64; ++e) x[e] = __uint_as_float(v[e]);
          }
          if (kGen) {
            if (cap > 0.f) {
#pragma unroll
              for (int e = 0; e < 64; ++e) x[e] = out * tanh_of(x[e] * in);
            } else {
#pragma unroll
              for (int e = 0; e < 64; ++e) x[e] *= in;
            }
            if (a.slopes) {
              const float dist = (float)(pos - key);
#pragma unroll
              for (int e = 0; e < 64; ++e) x[e] = fmaf(-slope, fabsf(dist - (float)e), x[e]);
            }
          }
          if (key + kTile > least) {
#pragma unroll
            for (int e = 0; e < 64; ++e) x[e] = key + e < lim ? x[e] : -INFINITY;
          }
          uint32_t w[32];
          float alpha = 1.f;
          bool rescale = false;
          if (k == 0) {
            m = fmaxf(row_max(x) * kScale, kMinRef);
            l = exps(x, m, w);
          } else {
            // against the reference so far, while the tile's maximum is formed; redone in the rare case that
            // this grew too far past it
            float sum = exps(x, m, w);
            const float mt = row_max(x) * kScale;
            const bool grow = mt > m + kLazy;
            if (__any_sync(0xffffffffu, grow)) {
              if (grow) {
                alpha = ex2(m - mt);
                m = mt;
                rescale = true;
              }
              __syncwarp();
              sum = exps(x, m, w);
            }
            l = fmaf(l, alpha, sum);
          }
          RESS_TMEM_ST32(tS, w);
          if (__any_sync(0xffffffffu, rescale)) {
            // the P V before this one (the one before that is done: S of this tile was issued after it)
            if (!wait(&S.o_full[slot][b ^ 1], ((c - 1) >> 1) & 1, abort)) {
              give_up(S, a.status);
              stop = true;
              break;
            }
            tc_fence_after();
#pragma unroll
            for (int hc = 0; hc < 2; ++hc) {
              uint32_t v[32];
              RESS_TMEM_LD32(tm + kColO + 32 * hc, v);
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * alpha);
              RESS_TMEM_ST32(tm + kColO + 32 * hc, v);
            }
          }
        }
        if (key + kTile > item.nk) {  // V's rows behind the last key
          const int st = (item.g0 + k) % kStages;
          if (!wait(&S.kv_full[st], ((item.g0 + k) / kStages) & 1, abort)) {
            give_up(S, a.status);
            stop = true;
            break;
          }
          zero_rows(S.V[st], item.nk - key, tid);
          fence_proxy_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.p_full[slot][b]);
      }
      if (stop) break;
      uint32_t o[2][32];
      if (tiles > 0) {
        if (!wait(&S.o_full[slot][(c - 1) & 1], ((c - 1) >> 1) & 1, abort)) {
          give_up(S, a.status);
          break;
        }
        tc_fence_after();
        if (any) {
          RESS_TMEM_LD32(tm + kColO, o[0]);
          RESS_TMEM_LD32(tm + kColO + 32, o[1]);
        }
        tc_fence_before();
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) o[0][e] = o[1][e] = 0u;
      }
      if (!exists) continue;
      if (item.part >= 0) {
        float* part = a.part + item.part * kPartFloats;
        const int row = slot * 128 + r;
        float4* dst = reinterpret_cast<float4*>(part + row * 64);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          dst[e] = make_float4(__uint_as_float(o[e >> 3][(4 * e) & 31]), __uint_as_float(o[e >> 3][(4 * e + 1) & 31]),
                               __uint_as_float(o[e >> 3][(4 * e + 2) & 31]), __uint_as_float(o[e >> 3][(4 * e + 3) & 31]));
        part[256 * 64 + row] = l == 0.f ? -INFINITY : m;
        part[256 * 65 + row] = l;
      } else {
        const int64_t q = (int64_t)item.q0 + tok;
        store_row<kF16>(static_cast<uint16_t*>(a.o.data) + q * a.o.token_stride + head * a.o.head_stride, o,
                        l == 0.f ? 0.f : 1.0f / l);
        if (a.lse) a.lse[head * a.rows + q] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
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

// ------------------------------------------------------------------------------------
// Items that several CTAs had shares of: with m the largest of their maxima,
// O = sum_s 2^(m_s - m) O_s / l and l = sum_s 2^(m_s - m) l_s.  Block (c, y) takes the item that the end of share
// c is inside of, if no earlier share ends there: 32 of its rows, half a warp per row and step.
// ------------------------------------------------------------------------------------
template <bool kF16>
__global__ void __launch_bounds__(256) k_flash_join(const __grid_constant__ DenseArgs a, int ctas) {
  __shared__ int64_t scratch[34];
  rows::stream_acquire();
  const int G = a.group, T = 128 / G;
  auto line_of = [&](const Seq& s) { return row_line(a, s, kSlots * T, T); };
  const int first = blockIdx.x;
  const Range r = find_range(a, line_of, ctas, first + 1, scratch, nullptr);
  if (first + 1 >= r.active || r.total == 0) return;
  Cursor c;
  seek(a, line_of, r.x0, r.b0, r.base, c);
  const int64_t end = c.start + c.weight;
  if (c.start == r.x0 || (first > 0 && bound(r.total, r.active, first) > c.start)) return;
  const int tok0 = c.j * kSlots * T;
  int n = 0;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) n = max(n, slot_tiles(a, c.s, tok0, s, T));
  if (n == 0) return;
  int parts = 1;  // shares first .. first + parts - 1 touch the item
  while (first + parts < r.active && bound(r.total, r.active, first + parts) < end) ++parts;
  auto share = [&](int k, int& t0, int& t1) {
    tiles_of(c, bound(r.total, r.active, first + k), bound(r.total, r.active, first + k + 1), n, t0, t1);
  };
  auto slot_of = [&](int k) -> const float* {
    return a.part + (2 * (int64_t)(first + k) + (c.start >= bound(r.total, r.active, first + k) ? 1 : 0)) * kPartFloats;
  };
  for (int k = 0; k < parts; ++k) {
    int t0, t1;
    share(k, t0, t1);
    if (t0 == 0 && t1 == n) return;  // one of them has it all
  }
  const int half = threadIdx.x >> 4, sub = threadIdx.x & 15;
  for (int i = half; i < 32; i += 16) {
    const int row = blockIdx.y * 32 + i, slot = row >> 7, rr = row & 127;
    if (rr / G >= slot_tokens(c.s.nq, tok0, slot, T)) continue;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < parts; ++k) {
      int t0, t1;
      share(k, t0, t1);
      if (t0 == t1) continue;
      const float* p = slot_of(k);
      const float mk = p[256 * 64 + row];
      if (mk == -INFINITY) continue;
      const float4 v = reinterpret_cast<const float4*>(p + row * 64)[sub];
      const float lk = p[256 * 65 + row], top = fmaxf(m, mk);
      const float wa = m == -INFINITY ? 0.f : ex2(m - top), wb = ex2(mk - top);
      m = top;
      l = fmaf(l, wa, lk * wb);
      o.x = fmaf(o.x, wa, v.x * wb), o.y = fmaf(o.y, wa, v.y * wb);
      o.z = fmaf(o.z, wa, v.z * wb), o.w = fmaf(o.w, wa, v.w * wb);
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const int64_t q = (int64_t)c.s.q0 + tok0 + slot * T + rr / G;
    const int head = c.h * G + rr % G;
    uint2* dst = reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o.data) + q * a.o.token_stride + head * a.o.head_stride);
    dst[sub] = make_uint2(pack2<kF16>(o.x * inv, o.y * inv), pack2<kF16>(o.z * inv, o.w * inv));
    if (a.lse && sub == 0) a.lse[head * a.rows + q] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
  }
}

// ------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------
static PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  }();
  return fn;
}

static bool encode(void* map, const void* base, int type, const cuuint64_t (&dims)[4], const cuuint64_t (&strides)[3],
                   const cuuint32_t (&box)[4]) {
  auto fn = encode_fn();
  cuuint32_t one[4] = {1, 1, 1, 1};
  return fn && fn(static_cast<CUtensorMap*>(map),
                  type == RESS_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                  const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A dimension of one element is never stepped over: any stride will do for it.
static cuuint64_t step_bytes(int64_t n, int64_t stride) { return n > 1 ? (cuuint64_t)stride * 2 : 128; }

bool make_row_map(void* map, const ress_heads& h, int type, int64_t rows, int kv_heads, int group, int tokens) {
  return encode(map, h.data, type, {64, (cuuint64_t)group, (cuuint64_t)kv_heads, (cuuint64_t)rows},
                {step_bytes(group, h.head_stride), step_bytes(kv_heads, group * h.head_stride), step_bytes(rows, h.token_stride)},
                {64, (cuuint32_t)group, 1, (cuuint32_t)tokens});
}

bool make_key_map(void* map, const ress_heads& h, int type, int64_t keys, int64_t pages, int64_t page_stride, int kv_heads,
                  int box) {
  return encode(map, h.data, type, {64, (cuuint64_t)kv_heads, (cuuint64_t)keys, (cuuint64_t)pages},
                {step_bytes(kv_heads, h.head_stride), step_bytes(keys, h.token_stride), step_bytes(pages, page_stride)},
                {64, 1, (cuuint32_t)box, 1});
}

int dense_ctas() {
  int dev = 0, n = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
  return n < 1 ? 1 : n < kMaxCtas ? n : kMaxCtas;
}

size_t dense_part_bytes() { return (size_t)kMaxCtas * 2 * kPartFloats * 4; }

cudaError_t launch_flash(const DenseArgs& a, cudaStream_t st) {
  CUtensorMap tq, tk, tv;
  // a tensor without keys is not read, but needs a map
  const int64_t keys = a.table ? a.page : a.keys > 0 ? a.keys : 1, pages = a.table ? a.n_pages : 1;
  ress_heads k = a.k, v = a.v;
  if (!a.table && a.keys == 0) k = v = a.q, k.head_stride = v.head_stride = 64;
  const int box = a.table && (a.page & -a.page) < kTile ? (a.page & -a.page) : kTile;
  if (!make_row_map(&tq, a.q, a.type, a.rows, a.kv_heads, a.group, 128 / a.group) ||
      !make_key_map(&tk, k, a.type, keys, pages, a.k_page_stride, a.kv_heads, box) ||
      !make_key_map(&tv, v, a.type, keys, pages, a.v_page_stride, a.kv_heads, box))
    return cudaErrorInvalidValue;
  const bool f16 = a.type == RESS_F16, gen = a.cap > 0.f || a.slopes;
  auto kern = f16 ? (gen ? k_flash<true, true> : k_flash<true, false>) : gen ? k_flash<false, true> : k_flash<false, false>;
  const size_t smem = sizeof(Smem) + 1024;
  const int ctas = dense_ctas();
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  if ((e = launch_pdl(kern, ctas, kThreads, smem, st, true, tq, tk, tv, a)) != cudaSuccess) return e;
  if (ctas == 1) return e;
  return launch_pdl(f16 ? k_flash_join<true> : k_flash_join<false>, dim3(ctas - 1, 8), 256, 0, st, true, a, ctas);
}

}  // namespace ress

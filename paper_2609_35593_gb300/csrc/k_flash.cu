// Dense attention over packed sequences or a paged cache: O = softmax(s) V for the keys that each row sees,
// with s = cap tanh(q.k / 8 / cap) - slope |distance|, and log sum exp(s) of each row.
//
// One CTA per SM walks its share of the work (attn_work.cuh).  An item is 4 x 128 rows of one head of K and V:
// floor(128 / group) tokens, each with its `group` heads of Q, make 128 rows, so that heads which share K read it
// once and single tokens still fill rows.  Its four parts ("slots") share the 64-key tiles that TMA brings in, a
// quarter of what 128 rows at a time would take from L2.  An item with rows for one slot (single tokens) or two gives
// its tiles to the slots in turn, which join their sums on chip.  Warp roles (640 threads):
//   warps 0-15  one row of a slot per thread: online softmax in the exp2 domain.  The reference maximum is that of
//               an item's first tile, and only raised where 64 exponentials against it add up to more than 2^13
//               (what P's 16 bits and O's 32 hold easily): O in TMEM is rescaled seldom, and no maximum is formed
//               otherwise.  Sums are float32, of the exponentials before they are rounded to 16 bits.
//   warp 16     item and tile producer: TMA of Q, K and V (128-byte swizzle), 9 stages of 16 KB, so that single
//               tokens, which only stream the cache, keep about 100 KB per SM in flight
//   warps 17, 18  MMA issuers of two slots each, per tile and slot: O += P V of the tile before (M128 N64 K64, P from
//               TMEM, V MN-major), then S = Q K^T (M128 N64 K64, both from shared memory) over P's columns
// Four slots because the softmax warps' chain (scores from TMEM, exponentials, P to TMEM, hand-over) is latency:
// with two, S double-buffered or in columns of its own, a sub-partition's two warps kept its SFU busy a third of the time
// (8 images at once 636 and 618 us).
// Rows of V behind a sequence's last key are zeroed in shared memory (0 x NaN of a cache page never written
// would be NaN); keys there and masked ones are -inf by selection, whatever their scores are.
// Every mbarrier wait is bounded; one that gives up records RESS_ETIMEOUT and the CTA leaves, see k_attn.cu.
#include <cudaTypedefs.h>

#include "attn_work.cuh"

namespace ress {
using namespace ptx;
using namespace work;

namespace {

constexpr int kThreads = 640, kStages = 9, kSlots = 4, kItems = 4;
constexpr int kProducer = 16, kIssuer = 17;  // warps 0-15: softmax; issuers of slots 0, 1 and 2, 3: 17, 18
constexpr uint32_t kTileBytes = kTile * 128;
constexpr uint32_t kColSlot = 128, kColO = 64;  // TMEM: per slot S (and P), O
// flags of a tile: no more; (per slot) it has the tile; it is its first, its last of the item
// tiles go to the slots in turn
constexpr int kTerm = 1, kTurns = 1 << 16, kHas = 2, kBegin = kHas << kSlots, kEnd = kBegin << kSlots;
constexpr float kMost = 8192.0f;  // sum of 64 exponentials above which the reference is raised
// Lowest reference maximum: finite, so that rows that have seen no key yet give exponentials of 0.
constexpr float kMinRef = -2147483648.0f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRows = kSlots * 128;
constexpr int64_t kPartFloats = kRows * 66;  // a slot of partial results: rows of 64, maxima, sums

struct Item {
  int q0, nq, k0, nk, d, p, b;  // the sequence
  int h, tok;                   // head of K (-1: no more items), first token of the sequence
  int t0, t1, g0;            // tiles; number of the first among all of the CTA's
  int n[kSlots];             // tiles of each 128 rows' keys
  int parts;                 // 128 rows that the item has, 1..4: slot s takes part s mod `parts` (3: slot 3 idles) and,
  int ways;                  // of that, every `ways`th tile
  int part;                  // slot of partial results, or -1: whole
};

struct __align__(1024) Smem {
  uint8_t Q[kSlots][128 * 128];
  uint8_t K[kStages][kTileBytes];
  uint8_t V[kStages][kTileBytes];
  uint64_t kv_full[kStages], kv_empty[kStages];
  float other[kSlots][2][128];  // maxima and sums of slots that share rows
  uint64_t other_full[kSlots][4], other_empty[kSlots][4];  // (and their quarters)
  uint64_t q_full[kSlots], q_empty[kSlots], drain[2];
  uint64_t s_full[kSlots], p_full[kSlots], o_full[kSlots];
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

// Tokens of 128 rows of an item, and the tiles of the keys that any of them sees.
__device__ __forceinline__ int part_tokens(int nq, int tok, int s, int T) { return max(0, min(T, nq - tok - s * T)); }
__device__ __forceinline__ int part_tiles(const DenseArgs& a, const Seq& q, int tok, int s, int T) {
  const int n = part_tokens(q.nq, tok, s, T);
  if (n == 0) return 0;
  return (max(0, row_limit(a, q, q.d + tok + s * T + n - 1)) + kTile - 1) / kTile;
}
__device__ __forceinline__ int item_tiles(const DenseArgs& a, const Seq& q, int tok, int T) {
  int n = 0;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) n = max(n, part_tiles(a, q, tok, s, T));
  return n;
}
__device__ __forceinline__ int ways_of(int parts) { return parts == 1 ? 4 : parts == 2 ? 2 : 1; }

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
      mbar_init(&S.kv_empty[s], kSlots);
    }
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(&S.q_full[s], 1);
      mbar_init(&S.q_empty[s], 1);
      mbar_init(&S.s_full[s], 1);
      mbar_init(&S.p_full[s], 4);
      mbar_init(&S.o_full[s], 1);
      for (int q = 0; q < 4; ++q) {
        mbar_init(&S.other_full[s][q], 1);
        mbar_init(&S.other_empty[s][q], 1);
      }
    }
    for (int p = 0; p < 2; ++p) mbar_init(&S.drain[p], 1);
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&S.it_full[i], 1);
      mbar_init(&S.it_empty[i], 4 * kSlots);
    }
    S.abort = 0;
    fence_barrier_init();
    prefetch_tensormap(&tmQ);
    prefetch_tensormap(&tmK);
    prefetch_tensormap(&tmV);
  }
  if (warp == kIssuer) tmem_alloc(&S.tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = S.tmem_base;
  rows::stream_acquire();
  auto line_of = [&](const Seq& s) { return row_line(a, s, kSlots * T, [&](int n) { return n > 3 * T ? 8 : n > 2 * T ? 6 : n > T ? 5 : 3; }); };
  const Range range = find_range(a, line_of, gridDim.x, blockIdx.x, S.scratch, blockIdx.x == 0 ? a.status : nullptr);

  // 640 threads start with 96 registers each; the softmax warps, which hold a row's scores, get 104 of them
  // (512 x 104 + 128 x 64 <= 640 x 96).  A spilled register would go to L2: shared memory leaves next to no L1.
  if (warp >= kProducer) {
    regs_dec<64>();
    if (warp == kProducer) {
      // =============================== producer ====================================
      int g = 0, pub = 0;
      uint32_t loads = 0;  // times that each slot's Q was loaded, a byte per slot
      bool failed = false;
      const int box = a.table ? min(kTile, a.page & -a.page) : kTile;  // the page's power of two
      const int boxes = kTile / box;
        // The next item that this share has tiles of, to S.next (h -1: none left).  One lane looks for it, in shared
      // memory: the sequences' arithmetic in 64 bits would otherwise take the registers of the tile loop.
      auto advance = [&](bool first) {
        __syncwarp();
        if (lane == 0) {
          Cursor& c = S.cursor;
          Item& item = S.next;
          item.h = -1;
          if (first) seek(a, line_of, range.x0, range.b0, range.base, c);
          while (first || (next(a, line_of, c) && c.start < range.x1)) {
            first = false;
            const int tok = c.j * kSlots * T, n = item_tiles(a, c.s, tok, T);
            int t0, t1;
            tiles_of(c, range.x0, range.x1, n, t0, t1);
            if (t0 == t1 && (n > 0 || c.start < range.x0)) continue;
            item.q0 = c.s.q0, item.nq = c.s.nq, item.k0 = c.s.k0, item.nk = c.s.nk, item.d = c.s.d, item.p = c.s.p;
            item.h = c.h, item.b = c.b, item.tok = tok, item.t0 = t0, item.t1 = t1;
            for (int s = 0; s < kSlots; ++s) item.n[s] = part_tiles(a, c.s, tok, s, T);
            item.parts = min(kSlots, (c.s.nq - tok + T - 1) / T);
            item.ways = ways_of(item.parts);
            item.part = t0 == 0 && t1 == n ? -1 : 2 * (int)blockIdx.x + (c.start >= range.x0 ? 1 : 0);
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
          if (item.t0 == item.t1) continue;  // rows without keys
          const int h = item.h, nk = item.nk, t0 = item.t0, t1 = item.t1, k0 = item.k0;
          const int32_t* table = a.table ? a.table + item.b * a.table_stride : nullptr;
          // lanes 0..3: what slot `lane` takes of the item
          const int parts = item.parts, ways = item.ways, mine_part = lane % parts, way = lane / parts;
          const int last = lane < kSlots && way < ways ? min(t1, item.n[mine_part]) : 0;
          const uint32_t some = __ballot_sync(0xffffffffu, t0 + way < last);
          for (int s = 0; s < kSlots; ++s) {
            if (!(some >> s & 1)) continue;
            const uint32_t times = loads >> (8 * s) & 0xff;
            if (times > 0 && !wait(&S.q_empty[s], (times - 1) & 1, abort)) {
              failed = true;
              break;
            }
            if (lane == 0) {
              mbar_arrive_expect_tx(&S.q_full[s], T * G * 128);
              tma_load_4d(S.Q[s], &tmQ, &S.q_full[s], 0, 0, h, item.q0 + item.tok + s % parts * T);
            }
            __syncwarp();
            // counts to 255 and goes on at 128 + (same parity)
            loads = (loads & ~(0xffu << (8 * s))) | ((times == 255 ? 128 : times + 1) << (8 * s));
          }
          if (failed) break;
          // where this lane's box of a tile is: lanes 0..boxes-1 load K, the next ones V
          const bool mine = lane < 2 * boxes;
          const int at = (lane < boxes ? lane : lane - boxes) * box;  // its first key in the tile
          auto place = [&](int t, int& row, int& page) {
            const int key = t * kTile + at;
            row = k0 + key, page = 0;
            if (!table) return;
            row = key % a.page, page = (int)a.n_pages;  // no such page: TMA fills in zeros
            if (mine && key < nk) {
              const int id = table[key / a.page];
              if (id >= 0 && id < a.n_pages)
                page = id;
              else
                flag_status(a.status, kStatusBadIndex);
            }
          };
          int row, page;
          place(t0, row, page);
          for (int t = t0; t < t1; ++t) {
            const int s = g % kStages, u = g / kStages;
            int next_row = 0, next_page = 0;
            if (t + 1 < t1) place(t + 1, next_row, next_page);
            int flags = 0;
            if (t < last && (t - t0) % ways == way) {
              flags = kHas << lane | (ways > 1 ? kTurns : 0);
              if (t == t0 + way) flags |= kBegin << lane;
              if (t + ways >= last) flags |= kEnd << lane;
            }
            flags = __reduce_or_sync(0xffffffffu, flags);
            if (u > 0 && !wait(&S.kv_empty[s], (u - 1) & 1, abort)) {
              failed = true;
              break;
            }
            if (lane == 0) {
              S.flags[s] = flags;
              mbar_arrive_expect_tx(&S.kv_full[s], 2 * kTileBytes);
            }
            __syncwarp();
            if (mine)
              tma_load_4d((lane < boxes ? S.K[s] : S.V[s]) + at * 128, lane < boxes ? &tmK : &tmV, &S.kv_full[s], 0, h,
                          row, page);
            __syncwarp();
            row = next_row, page = next_page;
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
        if (!failed && !publish()) failed = true;
      }
      if (failed && lane == 0) {
        give_up(S, a.status);
        // let every copy already issued land before the CTA's shared memory goes away
        volatile int no_abort = 0;
        for (int back = 1; back <= kStages && g - back >= 0; ++back)
          mbar_wait(&S.kv_full[(g - back) % kStages], ((g - back) / kStages) & 1, &no_abort, kDrainNs);
        for (int s = 0; s < kSlots; ++s)
          if (loads >> (8 * s) & 0xff) mbar_wait(&S.q_full[s], ((loads >> (8 * s) & 0xff) - 1) & 1, &no_abort, kDrainNs);
      }
    } else if (warp < kIssuer + 2) {
      // ================================ MMA issuers ==================================
      const int pair = warp - kIssuer;
      const bool leader = elect_one();
      bool failed = false;
      constexpr uint32_t kQk = idesc16<kF16>(128, kTile, false), kPv = idesc16<kF16>(128, 64, true);
      constexpr uint64_t kStageUnits = kTileBytes >> 4, kQUnits = (128 * 128) >> 4;
      const uint64_t kd0 = sdesc_sw128(smem_u32(S.K[0])), vd0 = sdesc_sw128(smem_u32(S.V[0]));
      const uint64_t qd0 = sdesc_sw128(smem_u32(S.Q[2 * pair]));
      int st = 0;
      uint32_t phase = 0;
      // of each of the two slots: tiles' P and items' Q so far (parity); stage of the tile whose P V is to come (or -1);
      // whether that is its item's last, its item's first
      uint32_t p_phase[2] = {0, 0}, q_phase[2] = {0, 0};
      int held[2] = {-1, -1};
      bool ends[2] = {false, false}, begins[2] = {false, false};
      auto issue_pv = [&](int j) -> bool {
        const int slot = 2 * pair + j;
        if (!wait(&S.p_full[slot], p_phase[j], abort)) return false;
        tc_fence_after();
        if (leader) {
          const uint32_t tm = tmem + slot * kColSlot;
          const uint64_t vd = vd0 + (uint64_t)held[j] * kStageUnits;
#pragma unroll
          for (int k = 0; k < 4; ++k) mma_bf16_ts(tm + kColO, tm + 8 * k, vd + 128 * k, kPv, (k > 0 || !begins[j]) ? 1u : 0u);
          mma_commit(&S.kv_empty[held[j]]);
          if (ends[j]) mma_commit(&S.o_full[slot]);
        }
        __syncwarp();
        p_phase[j] ^= 1;
        held[j] = -1;
        return true;
      };
      // Per tile and slot: P V of the slot's tile before, then S.  The last P V of an item does not wait for a tile to
      // come: the producer may be waiting for the softmax warps to end the item.
      while (!failed) {
        if (!wait(&S.kv_full[st], phase, abort)) {
          failed = true;
          break;
        }
        const int flags = S.flags[st];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int slot = 2 * pair + j;
          const bool has = flags >> slot & kHas;
          if (failed) continue;
          if (has && (flags >> slot & kBegin)) {
            if (!wait(&S.q_full[slot], q_phase[j], abort)) failed = true;
            q_phase[j] ^= 1;
          }
          if (!failed && held[j] >= 0 && (has || ends[j] || (flags & kTerm) ||
                                           ((flags & kTurns) && mbar_ready(&S.p_full[slot], p_phase[j]))) &&
              !issue_pv(j))
            failed = true;
          if (failed || (flags & kTerm)) continue;
          if (has) {
            tc_fence_after();
            if (leader) {
              const uint64_t kd = kd0 + (uint64_t)st * kStageUnits, qd = qd0 + j * kQUnits;
#pragma unroll
              for (int k = 0; k < 4; ++k)
                mma_bf16_ss(tmem + slot * kColSlot, qd + 2 * k, kd + 2 * k, kQk, k > 0 ? 1u : 0u);
              mma_commit(&S.s_full[slot]);
              if (flags >> slot & kEnd) mma_commit(&S.q_empty[slot]);
            }
            held[j] = st, ends[j] = flags >> slot & kEnd, begins[j] = flags >> slot & kBegin;
          } else if (lane == 0) {
            mbar_arrive(&S.kv_empty[st]);
          }
          __syncwarp();
        }
        if (flags & kTerm) break;
        if (++st == kStages) st = 0, phase ^= 1;
        if (!failed && ((held[0] >= 0 && ends[0]) || (held[1] >= 0 && ends[1])) && !mbar_ready(&S.kv_full[st], phase)) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
            if (!failed && held[j] >= 0 && ends[j] && !issue_pv(j)) failed = true;
        }
      }
      if (failed && lane == 0) give_up(S, a.status);
      // wait for every MMA issued so far before TMEM is released
      if (leader) {
        mma_commit(&S.drain[pair]);
        volatile int no_abort = 0;
        mbar_wait(&S.drain[pair], 0, &no_abort, kDrainNs);
      }
      __syncwarp();
    }
  } else {
    regs_inc<104>();
    // ================================ softmax =====================================
    const int slot = warp >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;             // row within the slot
    const uint32_t tm = tmem + slot * kColSlot + ((uint32_t)(quarter * 32) << 16);
    const float kScale = kGen ? 1.0f : kLog2e * 0.125f;
    const float cap = a.cap, in = a.cap > 0.f ? 0.125f / a.cap : 0.125f * kLog2e, out = a.cap * kLog2e;
    uint32_t c = 0, ended = 0;        // tiles of this slot, and items with any, so far
    uint32_t turn1 = 0, turn23 = 0;   // items in which slot 1, slots 2 and 3 help another one, so far
    bool stop = false;
    for (int pub = 0; !stop; ++pub) {
      const int i = pub % kItems;
      if (!wait(&S.it_full[i], (pub / kItems) & 1, abort)) {
        give_up(S, a.status);
        break;
      }
      const Item& item = S.item[i];
      if (item.h < 0) break;
      const int parts = item.parts, ways = item.ways, part = slot % parts, way = slot / parts;
      const int ntok = way < ways ? part_tokens(item.nq, item.tok, part, T) : 0;
      const int from = item.t0 + way, tiles = way < ways ? max(0, min(item.t1, item.n[part]) - from + ways - 1) / ways : 0;
      const int tok = item.tok + part * T + r / G;  // of the sequence
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
        const int t = from + k * ways, key = t * kTile;
        if (!wait(&S.s_full[slot], c & 1, abort)) {
          give_up(S, a.status);
          stop = true;
          break;
        }
        tc_fence_after();
        if (any) {  // rows of a warp without any are garbage that nothing reads
          float alpha = 1.f, sum;
          uint32_t w[32];
          // Against the reference so far: a sum below kMost says that no exponential is above it, so the maximum is
          // looked for only in an item's first tile and where that fails.
          bool looked = k == 0;
#pragma unroll 1
          for (;;) {
            float x[64];
            {
              uint32_t v[64];
              RESS_TMEM_LD64(tm, v);
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
            if (looked) {
              float top = x[0];
#pragma unroll
              for (int e = 1; e < 63; e += 2) top = fmax3(top, x[e], x[e + 1]);
              top = fmaxf(top, x[63]) * kScale;
              if (k == 0) {
                m = fmaxf(top, kMinRef);
              } else if (top > m) {
                alpha = ex2(m - top);
                m = top;
              }
            }
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
            sum = (s0 + s2) + (s1 + s3);
            if (looked || !__any_sync(0xffffffffu, sum > kMost)) break;
            looked = true;
          }
          l = fmaf(l, alpha, sum);
          RESS_TMEM_ST32(tm, w);
          if (looked && k > 0) {  // the P V before this one is done: S of this tile was issued after it
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
          const int g = item.g0 + t - item.t0, st = g % kStages;
          if (!wait(&S.kv_full[st], (g / kStages) & 1, abort)) {
            give_up(S, a.status);
            stop = true;
            break;
          }
          zero_rows(S.V[st], item.nk - key, r);
          fence_proxy_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.p_full[slot]);
      }
      if (stop) break;
      if (tiles > 0) {
        if (!wait(&S.o_full[slot], ended & 1, abort)) {
          give_up(S, a.status);
          break;
        }
        ++ended;
        tc_fence_after();
      }
      // Slots with the same rows: the first of them adds the others' O, which it reads where they are, to its own:
      // O = sum_s 2^(m_s - m) O_s.
      const uint32_t turn = (slot == 1 ? turn1 : turn23) & 1;
      if (way > 0 && way < ways) {
        S.other[slot][0][r] = l == 0.f ? -INFINITY : m;
        S.other[slot][1][r] = l;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&S.other_full[slot][quarter]);
          mbar_arrive(&S.it_empty[i]);
        }
        if (!wait(&S.other_empty[slot][quarter], turn, abort)) {
          give_up(S, a.status);
          break;
        }
      } else {
        float by[kSlots] = {1.f, 0.f, 0.f, 0.f};  // weights of this slot and the others
        if (ways > 1) {
          float ms[kSlots];
          ms[0] = l == 0.f ? -INFINITY : m;
#pragma unroll
          for (int j = 1; j < kSlots; ++j) {
            ms[j] = -INFINITY;
            if (j < ways) {
              const int s = slot + j * parts;
              if (!wait(&S.other_full[s][quarter], (s == 1 ? turn1 : turn23) & 1, abort)) stop = true;
              ms[j] = S.other[s][0][r];
            }
          }
          if (stop) {
            give_up(S, a.status);
            break;
          }
          tc_fence_after();
          const float top = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
          by[0] = ms[0] == -INFINITY ? 0.f : ex2(ms[0] - top);
          l *= by[0];
#pragma unroll
          for (int j = 1; j < kSlots; ++j)
            if (ms[j] != -INFINITY) {
              by[j] = ex2(ms[j] - top);
              l = fmaf(by[j], S.other[slot + j * parts][1][r], l);
            }
          if (top != -INFINITY) m = top;
        }
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        const int64_t q = (int64_t)item.q0 + tok;
#pragma unroll 1
        for (int hc = 0; hc < 2 && any; ++hc) {
          uint32_t o[32];
          if (tiles > 0) {
            RESS_TMEM_LD32(tm + kColO + 32 * hc, o);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0u;
          }
          if (ways > 1) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by[0]);
#pragma unroll
            for (int j = 1; j < kSlots; ++j)
              if (j < ways && from + j < min(item.t1, item.n[part])) {
                uint32_t v[32];
                RESS_TMEM_LD32(tm + j * parts * kColSlot + kColO + 32 * hc, v);
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  o[e] = __float_as_uint(fmaf(__uint_as_float(v[e]), by[j], __uint_as_float(o[e])));
              }
          }
          if (!exists) continue;
          if (item.part >= 0) {
            float4* dst = reinterpret_cast<float4*>(a.part + item.part * kPartFloats + (part * 128 + r) * 64 + 32 * hc);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              dst[e] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]),
                                   __uint_as_float(o[4 * e + 3]));
          } else {
            uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.o.data) + q * a.o.token_stride +
                                                  head * a.o.head_stride + 32 * hc);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t w[4];
#pragma unroll
              for (int f = 0; f < 4; ++f)
                w[f] = pack2<kF16>(__uint_as_float(o[8 * e + 2 * f]) * inv, __uint_as_float(o[8 * e + 2 * f + 1]) * inv);
              dst[e] = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        }
        if (exists && item.part >= 0) {
          float* rest = a.part + item.part * kPartFloats + kRows * 64 + part * 128 + r;
          rest[0] = l == 0.f ? -INFINITY : m;
          rest[kRows] = l;
        } else if (exists && a.lse) {
          a.lse[head * a.rows + q] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          for (int j = 1; j < ways; ++j) mbar_arrive(&S.other_empty[slot + j * parts][quarter]);
          mbar_arrive(&S.it_empty[i]);
        }
      }
      turn1 += parts == 1;
      turn23 += parts <= 2;
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kIssuer) {
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
  auto line_of = [&](const Seq& s) { return row_line(a, s, kSlots * T, [&](int n) { return n > 3 * T ? 8 : n > 2 * T ? 6 : n > T ? 5 : 3; }); };
  const int first = blockIdx.x;
  const Range r = find_range(a, line_of, ctas, first + 1, scratch, nullptr);
  if (first + 1 >= r.active || r.total == 0) return;
  Cursor c;
  seek(a, line_of, r.x0, r.b0, r.base, c);
  const int64_t end = c.start + c.weight;
  if (c.start == r.x0 || (first > 0 && bound(r.total, r.active, first) > c.start)) return;
  const int tok0 = c.j * kSlots * T;
  const int n = item_tiles(a, c.s, tok0, T);
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
    if (rr / G >= part_tokens(c.s.nq, tok0, slot, T)) continue;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < parts; ++k) {
      int t0, t1;
      share(k, t0, t1);
      if (t0 == t1) continue;
      const float* p = slot_of(k);
      const float mk = p[kRows * 64 + row];
      if (mk == -INFINITY) continue;
      const float4 v = reinterpret_cast<const float4*>(p + row * 64)[sub];
      const float lk = p[kRows * 65 + row], top = fmaxf(m, mk);
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
  return launch_pdl(f16 ? k_flash_join<true> : k_flash_join<false>, dim3(ctas - 1, kRows / 32), 256, 0, st, true, a, ctas);
}

}  // namespace ress

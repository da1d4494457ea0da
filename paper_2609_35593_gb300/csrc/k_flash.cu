// Dense attention over packed sequences or a paged cache: O = softmax(s) V for the keys that each row sees,
// with s = cap tanh(q.k / 8 / cap) - slope |distance|, and log sum exp(s) of each row.
//
// One CTA per SM walks its share of the work (attn_work.cuh).  An item is 2 x 128 rows of one head of K and V:
// floor(128 / group) tokens, each with its `group` heads of Q, make 128 rows, so that heads which share K read it
// once and single tokens still fill rows.  Its halves ("slots") share the 128-key tiles that TMA brings in, half of
// what 128 rows at a time would take from L2.  An item with rows for one slot (single tokens) gives its tiles to the
// slots in turn, which join their sums on chip.  Warp roles (640 threads):
//   warps 4-19  16 rows of a slot each, a row on four lanes: online softmax in the exp2 domain.  The reference maximum is
//               that of an item's first columns, and only raised where a lane's 16 exponentials against it add up to more
//               than 2^13 (what P's 16 bits and O's 32 hold easily): O in TMEM is rescaled seldom, and no maximum is
//               formed otherwise.  Sums are float32, of the exponentials before they are rounded to 16 bits, one for
//               each lane until the item ends.
//   warp 0      item and tile producer: TMA of Q, K and V (128-byte swizzle), 5 stages of 32 KB, so that single
//               tokens, which only stream the cache, keep 100 KB per SM in flight
//   warp 1      issuer of S = Q K^T (M128 N128 K64, both from shared memory)
//   warps 2, 3  issuers of O += P V (M128 N64 K128, P from TMEM, V MN-major), a slot each.  S and P have columns of their
//               own: S of the next tile runs while the exponentials of this one are formed.
// What bounds it is the chain of a slot's tile: scores from TMEM, exponentials, P to TMEM and the hand-overs between
// warps, some 2,200 cycles of which the MMAs take 1,024, so the tiles are as large as TMEM allows, and the 16 warps of
// softmax (four to a sub-partition) work while others wait.  8 images at once (10,992 rows and keys, 16 heads) take 440 to 456 us,
// 1.1 PFLOP/s; other forms of the same results: a row per thread and 8 warps, S of 64 keys double-buffered under P 636,
// 128 keys with S and P apart 618; 12 warps, three slots of 64 keys 586; 16 warps, four slots of 64 keys and two issuers
// 553; this form at first 482 (its join looked for the shares itself, 25 us of that).
// Rows of V behind a sequence's last key are zeroed in shared memory (0 x NaN of a cache page never written
// would be NaN); keys there and masked ones are -inf by selection, whatever their scores are.
// Every mbarrier wait is bounded; one that gives up records RESS_ETIMEOUT and the CTA leaves, see k_attn.cu.
#include <cudaTypedefs.h>

#include "attn_work.cuh"

namespace ress {
using namespace ptx;
using namespace work;

namespace {

constexpr int kThreads = 640, kStages = 5, kSlots = 2, kItems = 4, kKeys = 128;
constexpr int kProducer = 0, kIssueS = 1, kIssuePv = 2, kSoftmax = 4;  // warps: producer, issuers, softmax
constexpr uint32_t kTileBytes = kKeys * 128;
constexpr uint32_t kColSlot = 256, kColP = 128, kColO = 192;  // TMEM: per slot S, P, O
// flags of a tile: no more; (per slot) it has the tile; it is its first, its last of the item
constexpr int kTerm = 1, kHas = 2, kBegin = kHas << kSlots, kEnd = kBegin << kSlots;
constexpr float kMost = 8192.0f;  // sum of 16 exponentials above which the reference is raised
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
  int ways;                  // 1: slot s takes 128 rows s; 2: there are only 128 rows, of which the slots take tiles in turn
  int part;                  // slot of partial results, or -1: whole
};

struct __align__(1024) Smem {
  uint8_t Q[kSlots][128 * 128];
  uint8_t K[kStages][kTileBytes];
  uint8_t V[kStages][kTileBytes];
  uint64_t kv_full[kStages], kv_empty[kStages];
  uint8_t row_token[128], row_head[128];   // of the 128 rows of a part
  float other[2][128];                     // items of one part: slot 1's maxima and sums
  uint64_t other_full[8], other_empty[8];  // (of each warp's rows)
  uint64_t q_full[kSlots], q_empty[kSlots], drain[1 + kSlots];
  uint64_t s_full[kSlots], s_free[kSlots], p_full[kSlots], o_full[kSlots];
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
  return (max(0, row_limit(a, q, q.d + tok + s * T + n - 1)) + kKeys - 1) / kKeys;
}
__device__ __forceinline__ int item_tiles(const DenseArgs& a, const Seq& q, int tok, int T) {
  int n = 0;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) n = max(n, part_tiles(a, q, tok, s, T));
  return n;
}

}  // namespace

// kGen: 1, capped scores; 2, scores with slopes; 3, both; 0, neither.  (One kernel for caps and slopes keeps slopes in registers and
// spills others: packed documents with a cap 218 us where 186; one for 2 and 3 takes 406 us where 346 on 10,992 causal rows.)
template <bool kF16, int kGen>
__global__ void __launch_bounds__(kThreads, 1)
    k_flash(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
            const __grid_constant__ CUtensorMap tmV, const __grid_constant__ DenseArgs a) {
  extern __shared__ uint8_t smem_raw[];
  Smem& S = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort = &S.abort;
  const int G = a.group, T = 128 / G;
  constexpr bool kSlopes = kGen >= 2, kCap = kGen & 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&S.kv_full[s], 1);
      mbar_init(&S.kv_empty[s], 1 + kSlots);
    }
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(&S.q_full[s], 1);
      mbar_init(&S.q_empty[s], 1);
      mbar_init(&S.s_full[s], 1);
      mbar_init(&S.s_free[s], 8);
      mbar_init(&S.p_full[s], 8);
      mbar_init(&S.o_full[s], 1);
    }
    for (int i = 0; i < 1 + kSlots; ++i) mbar_init(&S.drain[i], 1);
    for (int q = 0; q < 8; ++q) {
      mbar_init(&S.other_full[q], 1);
      mbar_init(&S.other_empty[q], 1);
    }
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&S.it_full[i], 1);
      mbar_init(&S.it_empty[i], 8 * kSlots);
    }
    S.abort = 0;
    fence_barrier_init();
    prefetch_tensormap(&tmQ);
    prefetch_tensormap(&tmK);
    prefetch_tensormap(&tmV);
  }
  if (const int r = (int)threadIdx.x - 512; r >= 0) {
    S.row_token[r] = r / G, S.row_head[r] = r % G;
    // rows that no token fills stay 0: what was there before might be scores too large for the short way to cap them
    if (r >= T * G) {
#pragma unroll 1
      for (int i = 0; i < kSlots * 8; ++i) reinterpret_cast<uint4*>(S.Q[i >> 3] + r * 128)[i & 7] = make_uint4(0u, 0u, 0u, 0u);
      fence_proxy_async_smem();
    }
  }
  if (warp == kIssueS) tmem_alloc(&S.tmem_base, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = S.tmem_base;
  rows::stream_acquire();
  auto line_of = [&](const Seq& s) { return row_line(a, s, kSlots * T, [&](int n) { return n > T ? 8 : 6; }); };
  Range range;  // (of the producer)
  if (a.n_seqs > 32) range = find_range(a, line_of, gridDim.x, blockIdx.x, S.scratch, blockIdx.x == 0 ? a.status : nullptr);

  // 640 threads start with 96 registers each; the softmax warps, which hold a row's scores, get 104 of them
  // (512 x 104 + 128 x 64 <= 640 x 96).  A spilled register goes to L2, as shared memory leaves next to no L1
  // (4 to 20 bytes are, see -Xptxas -v).
  if (warp < kSoftmax) {
    regs_dec<64>();
    if (warp == kProducer) {
      // =============================== producer ====================================
      int g = 0, pub = 0;
      if (a.n_seqs <= 32)
        range = find_range_warp(a, line_of, gridDim.x, blockIdx.x, blockIdx.x == 0 ? a.status : nullptr);
      uint32_t loads = 0;  // of each slot's Q so far, two bits a slot
      bool failed = false;
      const int box = a.table ? min(kKeys, a.page & -a.page) : kKeys;  // the page's power of two
      const int boxes = kKeys / box, page_shift = (a.page & (a.page - 1)) == 0 ? __ffs(a.page) - 1 : -1;
      if (lane == 0) a.share[2 * blockIdx.x].n = a.share[2 * blockIdx.x + 1].n = -1;
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
            item.ways = c.s.nq - tok > T ? 1 : kSlots;
            item.part = t0 == 0 && t1 == n ? -1 : share_slot(c, range.x0);
            if (item.part >= 0)
              a.share[item.part] = DenseShare{t0, t1, n, c.h, c.s.q0 + tok, min(c.s.nq - tok, kSlots * T), {}};
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
        advance(true);
        while (S.next.h >= 0 && !failed) {
          if (!publish()) {
            failed = true;
            break;
          }
          const Item& item = S.next;
          if (item.t0 == item.t1) {  // rows without keys
            advance(false);
            continue;
          }
          const int h = item.h, nk = item.nk, t0 = item.t0, t1 = item.t1, k0 = item.k0;
          const int32_t* table = a.table ? a.table + item.b * a.table_stride : nullptr;
          // the first lanes: what slot `lane` takes of the item
          const int ways = item.ways, mine_part = ways > 1 ? 0 : lane, way = ways > 1 ? lane : 0;
          const int last = lane < kSlots ? min(t1, item.n[mine_part]) : 0;
          const uint32_t some = __ballot_sync(0xffffffffu, t0 + way < last);
          // slopes: the nearest keys of a causal row first, or the reference would be raised from tile to tile
          const int step = kSlopes ? -1 : 1, begin = kSlopes ? t1 - 1 : t0;
          for (int s = 0; s < kSlots; ++s) {
            if (!(some >> s & 1)) continue;
            // phases of its barriers (2 bits: none yet, 1, 2, 1, ..)
            const uint32_t times = loads >> (2 * s) & 3;
            if (times > 0 && !wait(&S.q_empty[s], times - 1, abort)) {
              failed = true;
              break;
            }
            if (lane == 0) {
              mbar_arrive_expect_tx(&S.q_full[s], T * G * 128);
              tma_load_4d(S.Q[s], &tmQ, &S.q_full[s], 0, 0, h, item.q0 + item.tok + (ways > 1 ? 0 : s * T));
            }
            __syncwarp();
            loads = (loads & ~(3u << (2 * s))) | ((times == 1 ? 2 : 1) << (2 * s));
          }
          if (failed) break;
          // where this lane's box of a tile is: lanes 0..boxes-1 load K, the next ones V
          const bool mine = lane < 2 * boxes;
          const int at = (lane < boxes ? lane : lane - boxes) * box;  // its first key in the tile
          auto place = [&](int t, int& row, int& page) {
            const int key = t * kKeys + at;
            row = k0 + key, page = 0;
            if (!table) return;
            const int col = page_shift >= 0 ? key >> page_shift : key / a.page;
            row = key - col * a.page, page = (int)a.n_pages;  // no such page: TMA fills in zeros
            if (mine && key < nk) {
              const int id = table[col];
              if (id >= 0 && id < a.n_pages)
                page = id;
              else
                flag_status(a.status, kStatusBadIndex);
            }
          };
          int row, page;
          place(begin, row, page);
          for (int i = 0; i < t1 - t0; ++i) {
            const int s = g % kStages, u = g / kStages, t = begin + step * i;
            int next_row = 0, next_page = 0;
            if (i + 1 < t1 - t0) place(t + step, next_row, next_page);
            int flags = 0;
            if (ways > 1 ? lane < kSlots && i % kSlots == lane : t < last) {
              flags = kHas << lane;
              const bool is_low = t == t0, is_high = t == last - 1;
              if (ways > 1 ? i == lane : kSlopes ? is_high : is_low) flags |= kBegin << lane;
              if (ways > 1 ? i + kSlots >= t1 - t0 : kSlopes ? is_low : is_high) flags |= kEnd << lane;
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
            // the next item is looked for while the first tiles are worked on
            if (i == min(kStages, t1 - t0) - 1) advance(false);
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
        for (int s = 0; s < kSlots; ++s)
          if (loads >> (2 * s) & 3) mbar_wait(&S.q_full[s], (loads >> (2 * s) & 3) - 1, &no_abort, kDrainNs);
      }
    } else {
      // ================================ MMA issuers ==================================
      const bool leader = elect_one();
      bool failed = false;
      constexpr uint32_t kQk = idesc16<kF16>(128, kKeys, false), kPv = idesc16<kF16>(128, 64, true);
      constexpr uint64_t kStageUnits = kTileBytes >> 4, kQUnits = (128 * 128) >> 4;
      uint32_t phase = 0;
      if (warp == kIssueS) {
        const uint64_t kd0 = sdesc_sw128(smem_u32(S.K[0])), qd0 = sdesc_sw128(smem_u32(S.Q[0]));
        uint32_t s_phase[kSlots] = {1, 1}, q_phase[kSlots] = {0, 0};
        for (int st = 0; !failed;) {
          if (!wait(&S.kv_full[st], phase, abort)) {
            failed = true;
            break;
          }
          const int flags = S.flags[st];
          if (flags & kTerm) break;
          const uint64_t kd = kd0 + (uint64_t)st * kStageUnits;
#pragma unroll
          for (int s = 0; s < kSlots; ++s) {
            if (failed || !(flags & kHas << s)) continue;
            if (flags & kBegin << s) {
              failed = !wait(&S.q_full[s], q_phase[s], abort);
              q_phase[s] ^= 1;
            }
            // (the first time: at once)
            if (failed || !wait(&S.s_free[s], s_phase[s], abort)) {
              failed = true;
              continue;
            }
            s_phase[s] ^= 1;
            tc_fence_after();
            if (leader) {
              const uint64_t qd = qd0 + s * kQUnits;
#pragma unroll
              for (int k = 0; k < 4; ++k) mma_bf16_ss(tmem + s * kColSlot, qd + 2 * k, kd + 2 * k, kQk, k > 0 ? 1u : 0u);
              mma_commit(&S.s_full[s]);
              if (flags & kEnd << s) mma_commit(&S.q_empty[s]);
            }
            __syncwarp();
          }
          if (lane == 0) mbar_arrive(&S.kv_empty[st]);
          if (++st == kStages) st = 0, phase ^= 1;
        }
      } else {
        const int slot = warp - kIssuePv;
        const uint32_t tm = tmem + slot * kColSlot;
        const uint64_t vd0 = sdesc_sw128(smem_u32(S.V[0]));
        uint32_t p_phase = 0;
        for (int st = 0;;) {
          if (!wait(&S.kv_full[st], phase, abort)) {
            failed = true;
            break;
          }
          const int flags = S.flags[st];
          if (flags & kTerm) break;
          if (flags & kHas << slot) {
            if (!wait(&S.p_full[slot], p_phase, abort)) {
              failed = true;
              break;
            }
            p_phase ^= 1;
            tc_fence_after();
            if (leader) {
              const uint64_t vd = vd0 + (uint64_t)st * kStageUnits;
              mma_bf16_ts(tm + kColO, tm + kColP, vd, kPv, flags & kBegin << slot ? 0u : 1u);
#pragma unroll
              for (int k = 1; k < 8; ++k) mma_bf16_ts(tm + kColO, tm + kColP + 8 * k, vd + 128 * k, kPv, 1u);
              mma_commit(&S.o_full[slot]);
              mma_commit(&S.kv_empty[st]);
            }
            __syncwarp();
          } else if (lane == 0) {
            mbar_arrive(&S.kv_empty[st]);
          }
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
    // ================================ softmax =====================================
    const int idx = warp - kSoftmax, slot = idx >> 3, half = idx >> 2 & 1, quarter = warp & 3;
    const int r0 = quarter * 32 + half * 16 + (lane >> 2), two = 2 * (lane & 3);  // this lane's rows: r0, r0 + 8; columns
    const uint32_t tm = tmem + slot * kColSlot + ((uint32_t)(quarter * 32 + half * 16) << 16);
    const float kScale = kGen ? 1.0f : kLog2e * 0.125f;
    const float in = kCap ? 0.25f * kLog2e / a.cap : 0.125f * kLog2e, out = a.cap * kLog2e;
    // p = 2^(x kScale - m) of 64 columns, packed, and their sums
    auto exps = [&](const float (&x)[32], const float (&m)[2], uint32_t (&w)[16], float (&sum)[2]) {
      float s[2][2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float t0, t1;
        fma2(t0, t1, x[2 * e], x[2 * e + 1], kScale, kScale, -m[e & 1], -m[e & 1]);
        t0 = ex2(t0), t1 = ex2(t1);
        w[e] = pack2<kF16>(t0, t1);
        add2(s[e & 1][0], s[e & 1][1], s[e & 1][0], s[e & 1][1], t0, t1);
      }
      sum[0] = s[0][0] + s[0][1], sum[1] = s[1][0] + s[1][1];
    };
    // the largest score of 64 columns, of each row
    auto row_max = [&](const float (&x)[32], float (&top)[2]) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        top[i] = fmaxf(x[2 * i], x[2 * i + 1]);
#pragma unroll
        for (int j = 1; j < 8; ++j) top[i] = fmax3(top[i], x[4 * j + 2 * i], x[4 * j + 2 * i + 1]);
        top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
        top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2)) * kScale;
      }
    };
    // the reference maxima to those of these columns, where they are larger; what was summed up is to be scaled by alpha
    auto raise = [&](const float (&x)[32], float (&m)[2], float (&alpha)[2]) {
      float top[2];
      row_max(x, top);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        top[j] = fmaxf(top[j], m[j]);
        alpha[j] = ex2(m[j] - top[j]);
        m[j] = top[j];
      }
    };
    auto scale_o = [&](const float (&alpha)[2]) {
      uint32_t v[32];
      RESS_TMEM_LD16X64(tm + kColO, v);
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * alpha[e >> 1 & 1]);
      RESS_TMEM_ST16X64(tm + kColO, v);
    };
    uint32_t c = 0, turn = 0;  // tiles of this slot, and items of one part, so far
    bool stop = false;
    for (int pub = 0; !stop; ++pub) {
      const int i = pub % kItems;
      if (!wait(&S.it_full[i], (pub / kItems) & 1, abort)) {
        give_up(S, a.status);
        break;
      }
      // (Read again where it is needed after the tiles: what is kept over them in registers would be spilled, 447 us
      // where 438 on 8 images at once.)
      const Item& item = S.item[i];
      if (item.h < 0) break;
      auto part_of = [&]() { return item.ways > 1 ? 0 : slot; };
      int tiles, key, dkey;  // this slot's tiles, the first key of the first, from one to the next
      {
        const int ways = item.ways, way = ways > 1 ? slot : 0, last = min(item.t1, item.n[part_of()]);
        tiles = ways > 1 ? max(0, last - item.t0 - way + 1) >> 1 : max(0, last - item.t0);
        static_assert(kSlots == 2, "two slots take turns");
        key = (kSlopes ? (ways > 1 ? item.t1 - way : last) - 1 : item.t0 + way) * kKeys;
        dkey = kSlopes ? -ways * kKeys : ways * kKeys;
      }
      int pos[2], lim[2];
      float slope[2];
      int least = item.nk;
      bool any = false;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = r0 + 8 * j, t = S.row_token[r], part = part_of(), ntok = part_tokens(item.nq, item.tok, part, T);
        pos[j] = item.d + item.tok + part * T + t;
        lim[j] = t >= ntok ? 0 : a.causal ? max(0, min(item.nk, max(item.p, pos[j] + 1))) : item.nk;
        // rows that do not exist are masked for nobody's sake
        if (t < ntok) least = min(least, lim[j]), any = true;
        slope[j] = kSlopes && t < ntok ? a.slopes[item.h * G + S.row_head[r]] * kLog2e : 0.f;
      }
      least = __reduce_min_sync(0xffffffffu, least);
      any = __any_sync(0xffffffffu, any);
      // scores of the 64 keys from `first` on, as the exponentials take them
      auto scores = [&](const uint32_t (&v)[32], float (&x)[32], int first) {
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(v[e]);
        if (kGen) {
          if (kCap) {
            cap_scores(x, a, in, out);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] *= in;
          }
          if (kSlopes) {
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const int j = e >> 1 & 1;
              x[e] = fmaf(-slope[j], fabsf((float)(pos[j] - first - two) - (float)(8 * (e >> 2) + (e & 1))), x[e]);
            }
          }
        }
        if (__any_sync(0xffffffffu, first + 64 > least)) {  // (the vote keeps this a branch, not selects)
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = 8 * (e >> 2) + (e & 1) < lim[e >> 1 & 1] - first - two ? x[e] : -INFINITY;
        }
      };
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};  // reference maxima (log2 units), this lane's sums
      for (int k = 0; k < tiles; ++k, ++c, key += dkey) {
        if (!wait(&S.s_full[slot], c & 1, abort)) {
          give_up(S, a.status);
          stop = true;
          break;
        }
        tc_fence_after();
        if (any) {
          // Two halves of 64 columns.  Against the reference so far: sums below kMost say that no exponential is above
          // it, so the maximum is looked for only in an item's first columns and where that fails, which is found out
          // while the next load or the store is on its way.
          float x[32], sum[2], alpha[2];
          uint32_t v[32], w[16];
          RESS_TMEM_LD16X64(tm, v);
          scores(v, x, key);
          if (k == 0) {
            row_max(x, alpha);
            m[0] = fmaxf(alpha[0], kMinRef), m[1] = fmaxf(alpha[1], kMinRef);
          }
          exps(x, m, w, sum);
          // the P V before this one has read P and added to O
          if (c > 0 && !wait(&S.o_full[slot], (c - 1) & 1, abort)) {
            give_up(S, a.status);
            stop = true;
            break;
          }
          tc_fence_after();
          RESS_TMEM_ST16X32P_NOWAIT(tm + kColP, w);
          RESS_TMEM_LD16X64_NOWAIT(tm + 64, v);
          if (__any_sync(0xffffffffu, fmaxf(sum[0], sum[1]) > kMost)) {
            RESS_TMEM_WAIT_LD32(v);
            tmem_wait_st();
            RESS_TMEM_LD16X64(tm, v);
            scores(v, x, key);
            raise(x, m, alpha);
            l[0] *= alpha[0], l[1] *= alpha[1];
            exps(x, m, w, sum);
            RESS_TMEM_ST16X32P(tm + kColP, w);
            if (k > 0) scale_o(alpha);
            RESS_TMEM_LD16X64_NOWAIT(tm + 64, v);
          }
          l[0] += sum[0], l[1] += sum[1];
          RESS_TMEM_WAIT_LD32(v);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&S.s_free[slot]);  // S is in registers
          __syncwarp();
          scores(v, x, key + 64);
          exps(x, m, w, sum);
          RESS_TMEM_ST16X32P_NOWAIT(tm + kColP + 32, w);
          if (__any_sync(0xffffffffu, fmaxf(sum[0], sum[1]) > kMost)) {
            tmem_wait_st();
            raise(x, m, alpha);
            l[0] *= alpha[0], l[1] *= alpha[1];
            exps(x, m, w, sum);
            RESS_TMEM_ST16X32P(tm + kColP + 32, w);
            RESS_TMEM_LD16X32P(tm + kColP, w);  // the first half's P
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float2 y = unpack2<kF16>(w[e]);
              w[e] = pack2<kF16>(y.x * alpha[e & 1], y.y * alpha[e & 1]);
            }
            RESS_TMEM_ST16X32P(tm + kColP, w);
            if (k > 0) scale_o(alpha);
          }
          l[0] += sum[0], l[1] += sum[1];
          tmem_wait_st();
        } else {  // no rows in this warp: P is garbage that nothing reads
          __syncwarp();
          if (lane == 0) mbar_arrive(&S.s_free[slot]);
          __syncwarp();
          if (c > 0 && !wait(&S.o_full[slot], (c - 1) & 1, abort)) {
            give_up(S, a.status);
            stop = true;
            break;
          }
        }
        if (const int nk = key + kKeys > least ? item.nk : INT32_MAX; key + kKeys > nk) {  // V's rows behind the last key
          const int t = key / kKeys, g = item.g0 + (kSlopes ? item.t1 - 1 - t : t - item.t0), st = g % kStages;
          if (!wait(&S.kv_full[st], (g / kStages) & 1, abort)) {
            give_up(S, a.status);
            stop = true;
            break;
          }
          zero_rows(S.V[st], nk - key, (idx & 7) * 32 + lane);
          fence_proxy_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.p_full[slot]);
        __syncwarp();
      }
      if (stop) break;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        l[j] += __shfl_xor_sync(0xffffffffu, l[j], 1);
        l[j] += __shfl_xor_sync(0xffffffffu, l[j], 2);
        if (l[j] == 0.f) m[j] = -INFINITY;
      }
      // What does not take O is done before it is waited for: where the rows go (null: nowhere), and what is told of
      // their sums.
      const int ways = item.ways, way = ways > 1 ? slot : 0, whole = item.part < 0;
      char* dst[2];
      {
        const int part = part_of(), tok0 = item.tok + part * T, ntok = part_tokens(item.nq, item.tok, part, T);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = r0 + 8 * j, t = S.row_token[r], head = item.h * G + S.row_head[r];
          const int64_t q = (int64_t)item.q0 + tok0 + t;
          if (whole)
            dst[j] = reinterpret_cast<char*>(static_cast<uint16_t*>(a.o.data) + q * a.o.token_stride + head * a.o.head_stride) +
                     16 * (lane & 3);
          else
            dst[j] = reinterpret_cast<char*>(a.part + item.part * kPartFloats + (part * 128 + r) * 64) + 8 * (lane & 3);
          if (t >= ntok || way > 0) dst[j] = nullptr;
        }
      }
      auto tell = [&](int j) {
        if (!dst[j] || (lane & 3) != 0) return;
        const int r = r0 + 8 * j;
        if (!whole) {
          float* to = a.part + item.part * kPartFloats + part_of() * 128 + r;
          to[kRows * 64] = m[j], to[kRows * 65] = l[j];
        } else if (a.lse) {
          a.lse[(item.h * G + S.row_head[r]) * a.rows + item.q0 + item.tok + part_of() * T + S.row_token[r]] =
              l[j] == 0.f ? -INFINITY : (m[j] + lg2(l[j])) * 0.6931471805599453f;
        }
      };
      if (ways == 1) tell(0), tell(1);
      __syncwarp();
      if (tiles > 0) {
        if (!wait(&S.o_full[slot], (c - 1) & 1, abort)) {
          give_up(S, a.status);
          break;
        }
        tc_fence_after();
      }
      // Slots with the same rows: slot 0 adds the other's O, which it reads where it is, to its own,
      // O = sum_s 2^(m_s - m) O_s.
      if (way > 0) {
        if ((lane & 3) == 0) {
#pragma unroll
          for (int j = 0; j < 2; ++j) S.other[0][r0 + 8 * j] = m[j], S.other[1][r0 + 8 * j] = l[j];
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&S.other_full[idx & 7]);
          mbar_arrive(&S.it_empty[i]);
        }
        __syncwarp();
        if (!wait(&S.other_empty[idx & 7], turn & 1, abort)) {
          give_up(S, a.status);
          break;
        }
      } else {
        float by0[2], by1[2];
        if (ways > 1) {
          if (!wait(&S.other_full[idx & 7], turn & 1, abort)) {
            give_up(S, a.status);
            break;
          }
          tc_fence_after();
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float m1 = S.other[0][r0 + 8 * j], l1 = S.other[1][r0 + 8 * j], top = fmaxf(m[j], m1);
            by0[j] = m[j] == -INFINITY ? 0.f : ex2(m[j] - top);
            by1[j] = m1 == -INFINITY ? 0.f : ex2(m1 - top);
            m[j] = top;
            l[j] = fmaf(l[j], by0[j], l1 * by1[j]);
            tell(j);
          }
          __syncwarp();
        }
        if (any) {
          float o[32];
          {
            uint32_t v[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 0u;
            if (tiles > 0) RESS_TMEM_LD16X64(tm + kColO, v);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(v[e]);
          }
          if (ways > 1) {
            uint32_t v[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 0u;
            if (item.t0 + 1 < min(item.t1, item.n[0])) RESS_TMEM_LD16X64(tm + kColSlot + kColO, v);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              o[e] = fmaf(__uint_as_float(v[e]), by1[e >> 1 & 1], o[e] * by0[e >> 1 & 1]);
          }
          if (whole) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const float inv = l[j] == 0.f ? 0.f : __fdividef(1.0f, l[j]);
              uint32_t w[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                float y0, y1;
                mul2(y0, y1, o[4 * e + 2 * j], o[4 * e + 2 * j + 1], inv, inv);
                w[e] = pack2<kF16>(y0, y1);
              }
              // a row's four lanes: from two channels of every eight to eight of every 32
              transpose4(w[0], w[1], w[2], w[3], lane);
              transpose4(w[4], w[5], w[6], w[7], lane);
              if (dst[j]) {
                reinterpret_cast<uint4*>(dst[j])[0] = make_uint4(w[0], w[1], w[2], w[3]);
                reinterpret_cast<uint4*>(dst[j])[4] = make_uint4(w[4], w[5], w[6], w[7]);
              }
            }
          } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              if (!dst[j]) continue;
#pragma unroll
              for (int e = 0; e < 8; ++e)
                reinterpret_cast<float2*>(dst[j])[4 * e] = make_float2(o[4 * e + 2 * j], o[4 * e + 2 * j + 1]);
            }
          }
          __syncwarp();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (ways > 1) mbar_arrive(&S.other_empty[idx & 7]);
          mbar_arrive(&S.it_empty[i]);
        }
        __syncwarp();
      }
      turn += ways > 1;
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

// ------------------------------------------------------------------------------------
// Items that several CTAs had shares of: with m the largest of their maxima, O = sum_s 2^(m_s - m) O_s / l and
// l = sum_s 2^(m_s - m) l_s.  Block (s, y) takes the item that slot s has the first share of, if any: 32 of its rows,
// half a warp per row and step.
// ------------------------------------------------------------------------------------
template <bool kF16>
__global__ void __launch_bounds__(256) k_flash_join(const __grid_constant__ DenseArgs a, int ctas) {
  rows::stream_acquire();
  const DenseShare item = a.share[blockIdx.x];
  if (item.n < 0 || item.t0 != 0) return;
  const int G = a.group, T = 128 / G, sub = threadIdx.x & 15;
  for (int i = threadIdx.x >> 4; i < 32; i += 16) {
    const int row = blockIdx.y * 32 + i, tok = (row >> 7) * T + (row & 127) / G;
    if ((row & 127) >= T * G || tok >= item.count) continue;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = blockIdx.x, t1 = item.t1;;) {
      const float* p = a.part + s * kPartFloats;
      const float mk = p[kRows * 64 + row];
      if (mk != -INFINITY) {
        const float4 v = reinterpret_cast<const float4*>(p + row * 64)[sub];
        const float lk = p[kRows * 65 + row], top = fmaxf(m, mk);
        const float wa = m == -INFINITY ? 0.f : ex2(m - top), wb = ex2(mk - top);
        m = top;
        l = fmaf(l, wa, lk * wb);
        o.x = fmaf(o.x, wa, v.x * wb), o.y = fmaf(o.y, wa, v.y * wb);
        o.z = fmaf(o.z, wa, v.z * wb), o.w = fmaf(o.w, wa, v.w * wb);
      }
      if (t1 >= item.n || (s = next_share(a, s, ctas)) < 0) break;
      t1 = a.share[s].t1;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const int64_t q = (int64_t)item.first + tok;
    const int head = item.head * G + (row & 127) % G;
    uint2* dst = reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.o.data) + q * a.o.token_stride + head * a.o.head_stride);
    dst[sub] = make_uint2(pack2<kF16>(o.x * inv, o.y * inv), pack2<kF16>(o.z * inv, o.w * inv));
    if (a.lse && sub == 0) a.lse[head * a.rows + q] = l == 0.f ? -INFINITY : (m + lg2(l)) * 0.6931471805599453f;
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
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
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

cudaError_t launch_flash(const DenseArgs& args, cudaStream_t st) {
  DenseArgs a = args;
  if (a.cap > 0.f) set_cap(a);
  CUtensorMap tq, tk, tv;
  // a tensor without keys is not read, but needs a map
  const int64_t keys = a.table ? a.page : a.keys > 0 ? a.keys : 1, pages = a.table ? a.n_pages : 1;
  ress_heads k = a.k, v = a.v;
  if (!a.table && a.keys == 0) k = v = a.q, k.head_stride = v.head_stride = 64;
  const int box = a.table && (a.page & -a.page) < kKeys ? (a.page & -a.page) : kKeys;
  if (!make_row_map(&tq, a.q, a.type, a.rows, a.kv_heads, a.group, 128 / a.group) ||
      !make_key_map(&tk, k, a.type, keys, pages, a.k_page_stride, a.kv_heads, box) ||
      !make_key_map(&tv, v, a.type, keys, pages, a.v_page_stride, a.kv_heads, box))
    return cudaErrorInvalidValue;
  const bool f16 = a.type == RESS_F16;
  decltype(&k_flash<false, 0>) const kernels[4][2] = {{k_flash<false, 0>, k_flash<true, 0>}, {k_flash<false, 1>, k_flash<true, 1>},
                                                       {k_flash<false, 2>, k_flash<true, 2>}, {k_flash<false, 3>, k_flash<true, 3>}};
  const auto kern = kernels[dense_gen(a)][f16];
  const size_t smem = sizeof(Smem) + 1024;
  const int ctas = dense_ctas();
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  if ((e = launch_pdl(kern, ctas, kThreads, smem, st, true, tq, tk, tv, a)) != cudaSuccess) return e;
  if (ctas == 1) return e;
  return launch_pdl(f16 ? k_flash_join<true> : k_flash_join<false>, dim3(2 * ctas, kRows / 32), 256, 0, st, true, a, ctas);
}

}  // namespace ress

// What dense attention over packed or paged sequences (k_flash.cu) and its gradient (k_flash_bwd.cu) share:
// the sequences, the equal shares of their work that the CTAs take, and the rules of the masks.
//
// Work.  An item is what stays on chip while tiles stream past it: a range of query rows of one head of K
// (of all the heads of Q that share it), or in the gradient of K and V a range of keys.  Lengths are device
// data, so the host knows only the totals: every CTA adds up all sequences' work itself (a few hundred
// instructions, sequences over its threads) and takes share c of C of it, wherever that begins and ends.
// An item that several CTAs have shares of leaves partial results in the workspace, two slots per CTA, with a note
// of what they are of; a second kernel adds them up in the order of the shares: no atomics, the same bits for the
// same inputs.  (It looked for the shares itself at first, as the CTAs do, and took 20 to 40 us.)
// With whole items instead, 96 items of 344 tiles on 152 SMs (one image's rows over the keys of 32, 16 heads) would
// take one round of 344 tiles where 217 a CTA do.
//
// An item's work is kOver + mul x its length, a length being the keys (or rows) that it sees, in closed form
// over the items of a sequence: a constant up to some item, then linear (causal), the last one on its own.
#pragma once

#include <cfloat>

#include "row_ops.cuh"
#include "sm100_ptx.cuh"

namespace ress {
namespace work {
using namespace ptx;

constexpr int kMaxCtas = kDenseMaxCtas;
// An item's loads and epilogue, as work: three tiles of 128 keys (packed documents of 52 to 2531 rows 185 us; counted as
// two tiles 192, as four 198; long sequences the same).
constexpr int64_t kOver = 8 * 384;
constexpr int64_t kLeast = 8 * 256;  // least share of a CTA: two tiles
constexpr uint64_t kWaitNs = 2000000000ull;  // 2 s per wait
constexpr uint64_t kDrainNs = 200000000ull;  // 0.2 s to drain after an abort

// One sequence: rows [q0, q0 + nq) of Q, keys [k0, k0 + nk) (paged: positions 0..nk-1 of its table row).
// Row t stands at position d + t; with a causal mask it sees the keys below max(p, d + t + 1).
struct Seq {
  int q0, nq, k0, nk, d, p;
};

__device__ __forceinline__ Seq load_seq(const DenseArgs& a, int b, uint32_t* status) {
  Seq s;
  int64_t q0 = 0, q1 = a.rows, k0 = 0, k1 = a.keys;
  if (a.q_start) q0 = a.q_start[b], q1 = a.q_start[b + 1];
  if (a.table)
    k1 = a.lens[b];
  else if (a.k_start)
    k0 = a.k_start[b], k1 = a.k_start[b + 1];
  const int64_t most = a.table ? (int64_t)a.table_cols * a.page : a.keys;
  if (q0 < 0 || q1 < q0 || q1 > a.rows) {  // such a sequence has no rows
    if (status) flag_status(status, kStatusBadRow);
    q0 = q1 = 0;
  }
  if (k0 < 0 || k1 < k0 || k1 > most) {  // or no keys
    if (status) flag_status(status, kStatusBadRow);
    k0 = k1 = 0;
  }
  s.q0 = (int)q0, s.nq = (int)(q1 - q0), s.k0 = (int)k0, s.nk = (int)(k1 - k0);
  s.d = s.nk - s.nq;
  s.p = 0;
  if (a.causal && a.prefix) s.p = max(0, min(a.prefix[b], s.nk));
  return s;
}

// Keys that the row at position `pos` of a sequence sees: those below this.
__device__ __forceinline__ int row_limit(const DenseArgs& a, const Seq& s, int pos) {
  return a.causal ? min(s.nk, max(s.p, pos + 1)) : s.nk;
}

// Items 0..n-1 of one head of a sequence: lengths and work.
struct Line {
  int n, cnt;          // items; those of the constant length
  int64_t a, b, step;  // length of items below cnt; b + step j of the others
  int64_t last, last_mul;
  __device__ int64_t length(int j) const { return j == n - 1 ? last : j < cnt ? a : b + step * j; }
  __device__ int64_t before(int j) const {  // work of items 0..j-1
    if (n == 0) return 0;
    const int64_t m = min(j, n - 1), c = min((int64_t)cnt, m);
    int64_t w = m * kOver + 8 * (c * a + (m - c) * b + step * ((m * (m - 1) - c * (c - 1)) / 2));
    if (j == n) w += kOver + last_mul * last;
    return w;
  }
};

// Query rows as items of `per` tokens.  The last one's time per key: `eighths`(its tokens) / 8 of a full one's.
template <class F>
__device__ __forceinline__ Line row_line(const DenseArgs& a, const Seq& s, int per, F eighths) {
  Line l;
  l.n = (s.nq + per - 1) / per;
  l.cnt = l.n, l.a = s.nk, l.b = l.step = 0;
  if (a.causal && l.n > 0) {
    l.cnt = s.p - s.d >= per ? min(l.n, (s.p - s.d) / per) : 0;
    l.a = s.p, l.b = (int64_t)s.d + per, l.step = per;
  }
  l.last = s.nk;
  l.last_mul = eighths(s.nq - (l.n - 1) * per);
  return l;
}

// Keys as items of `per`; their lengths are the rows (tokens of all heads) that see any of them.
__device__ __forceinline__ int first_row(const DenseArgs& a, const Seq& s, int key) {
  return a.causal && key >= s.p ? max(0, min(s.nq, key - s.d)) : 0;
}
__device__ __forceinline__ Line key_line(const DenseArgs& a, const Seq& s, int per) {
  Line l;
  l.n = (s.nk + per - 1) / per;
  l.cnt = l.n, l.a = (int64_t)s.nq * a.group, l.b = l.step = 0;
  if (a.causal && l.n > 0) {
    const int top = max(s.d, s.p - 1);  // items that start here or before are seen by every row
    l.cnt = top >= 0 ? min(l.n, top / per + 1) : 0;
    l.b = (int64_t)s.nk * a.group, l.step = -per * a.group;
  }
  l.last = l.n > 0 ? (int64_t)(s.nq - first_row(a, s, (l.n - 1) * per)) * a.group : 0;
  l.last_mul = 8;
  return l;
}

// Share [x0, x1) of all work: sequence b0 holds x0 and begins at `base`.
struct Range {
  int64_t total, x0, x1, base;
  int b0, active;
};
// a / b of numbers that are mostly below 2^32 (a division of 64 bits takes some hundred instructions).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
__device__ __forceinline__ int active_ctas(int64_t total, int ctas) {
  return (int)max((int64_t)1, min((int64_t)ctas, quotient(total, kLeast)));
}
__device__ __forceinline__ int64_t bound(int64_t total, int active, int c) {
  const int64_t one = quotient(total, active);
  return one * c + quotient((total - one * active) * c, active);
}

// All threads of the CTA: share `cta` of `ctas`.  scratch: 34 words of shared memory; status: NULL, or where
// sequences outside their tensors are told.
template <class LineOf>
__device__ __forceinline__ Range find_range(const DenseArgs& a, LineOf line_of, int ctas, int cta, int64_t* scratch,
                                            uint32_t* status) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int per = (a.n_seqs + (int)blockDim.x - 1) / (int)blockDim.x;
  const int lo = min(a.n_seqs, tid * per), hi = min(a.n_seqs, lo + per);
  int64_t sum = 0;
  for (int b = lo; b < hi; ++b) {
    const Line l = line_of(load_seq(a, b, status));
    sum += a.kv_heads * l.before(l.n);
  }
  int64_t inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) scratch[warp] = inc;
  __syncthreads();
  int64_t before = inc - sum, total = 0;
  for (int w = 0; w < warps; ++w) {
    if (w < warp) before += scratch[w];
    total += scratch[w];
  }
  Range r;
  r.total = total;
  r.active = active_ctas(total, ctas);
  r.x0 = cta < r.active ? bound(total, r.active, cta) : total;
  r.x1 = cta < r.active ? bound(total, r.active, cta + 1) : total;
  if (r.x0 >= before && r.x0 < before + sum) {
    int64_t at = before;
    for (int b = lo; b < hi; ++b) {
      const Line l = line_of(load_seq(a, b, nullptr));
      const int64_t w = a.kv_heads * l.before(l.n);
      if (r.x0 < at + w) {
        scratch[32] = at;
        scratch[33] = b;
        break;
      }
      at += w;
    }
  }
  __syncthreads();
  r.base = scratch[32];
  r.b0 = (int)scratch[33];
  return r;
}

// The same by one warp, for up to 32 sequences.
template <class LineOf>
__device__ __forceinline__ Range find_range_warp(const DenseArgs& a, LineOf line_of, int ctas, int cta, uint32_t* status) {
  const int lane = threadIdx.x & 31;
  int64_t sum = 0;
  if (lane < a.n_seqs) {
    const Line l = line_of(load_seq(a, lane, status));
    sum = a.kv_heads * l.before(l.n);
  }
  int64_t inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  Range r;
  r.total = __shfl_sync(0xffffffffu, inc, 31);
  r.active = active_ctas(r.total, ctas);
  r.x0 = cta < r.active ? bound(r.total, r.active, cta) : r.total;
  r.x1 = cta < r.active ? bound(r.total, r.active, cta + 1) : r.total;
  const uint32_t here = __ballot_sync(0xffffffffu, r.x0 >= inc - sum && r.x0 < inc);
  r.b0 = here ? __ffs(here) - 1 : 0;
  r.base = __shfl_sync(0xffffffffu, inc - sum, r.b0);
  return r;
}

// The items that a share touches, one after another.
struct Cursor {
  Seq s;
  Line l;
  int b, h, j;
  int64_t start, weight;  // of the item, in all work
};
template <class LineOf>
__device__ __forceinline__ void seek(const DenseArgs& a, LineOf line_of, int64_t x, int b, int64_t base, Cursor& c) {
  c.b = b;
  c.s = load_seq(a, b, nullptr);
  c.l = line_of(c.s);
  const int64_t one = c.l.before(c.l.n), rem = x - base;
  c.h = (int)quotient(rem, one);
  const int64_t r = rem - c.h * one;
  // The item that holds r: by the line's formula in float, put right by the exact sums.
  int j;
  const float each = (float)(kOver + 8 * c.l.a);
  if ((float)r < each * (float)c.l.cnt || c.l.step == 0) {
    j = (int)((float)r / each);
  } else {  // each cnt + (m - cnt) (kOver + 8 b) + 4 step (m (m - 1) - cnt (cnt - 1)) = r
    const float n = (float)c.l.cnt, s4 = 4.f * (float)c.l.step, lin = (float)(kOver + 8 * c.l.b) - s4;
    const float rest = each * n - n * (float)(kOver + 8 * c.l.b) - s4 * n * (n - 1.f) - (float)r;
    j = (int)((-lin + sqrtf(fmaxf(lin * lin - 4.f * s4 * rest, 0.f))) / (2.f * s4));
  }
  j = max(0, min(j, c.l.n - 1));
  while (j > 0 && c.l.before(j) > r) --j;
  while (j < c.l.n - 1 && c.l.before(j + 1) <= r) ++j;
  c.j = j;
  c.start = base + c.h * one + c.l.before(j);
  c.weight = c.l.before(j + 1) - c.l.before(j);
}
// The next item (false: there is none).
template <class LineOf>
__device__ __forceinline__ bool next(const DenseArgs& a, LineOf line_of, Cursor& c) {
  c.start += c.weight;
  if (++c.j == c.l.n) {
    c.j = 0;
    if (++c.h == a.kv_heads) {
      c.h = 0;
      do {
        if (++c.b == a.n_seqs) return false;
        c.s = load_seq(a, c.b, nullptr);
        c.l = line_of(c.s);
      } while (c.l.n == 0);
    }
  }
  c.weight = c.l.before(c.j + 1) - c.l.before(c.j);
  return true;
}
// Tiles [t0, t1) of an item's n that share [x0, x1) has.
__device__ __forceinline__ void tiles_of(const Cursor& c, int64_t x0, int64_t x1, int n, int& t0, int& t1) {
  const int64_t lo = max(x0 - c.start, (int64_t)0), hi = min(x1 - c.start, c.weight);
  t0 = (int)quotient(lo * n, c.weight);
  t1 = (int)quotient(hi * n, c.weight);
}

// Slots of the workspace: a CTA's share of an item that began before its own shares, and of one that it is the first of.
__device__ __forceinline__ int share_slot(const Cursor& c, int64_t x0) { return 2 * (int)blockIdx.x + (c.start >= x0 ? 1 : 0); }
// The share after `slot` of the same item (shares without tiles have no note).
__device__ __forceinline__ int next_share(const DenseArgs& a, int slot, int ctas) {
  for (int c = slot / 2 + 1; c < ctas; ++c)
    if (a.share[2 * c].n >= 0) return 2 * c;
  return -1;  // (does not happen: the last share of an item ends it)
}

// Bounded wait for a whole warp: every lane tests the barrier, else lane 0 polls and tells the others, so that
// no lane leaves code its neighbours stay in.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  int ok = 1;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity, abort, kWaitNs) ? 1 : 0;
  ok = __shfl_sync(0xffffffffu, ok, 0);
  __syncwarp();
  return ok != 0;
}

// Registers of this warp's group of four (all four warps come here): fewer, or more of those that others gave up.
template <int N>
__device__ __forceinline__ void regs_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}

// 16 lanes of TMEM x 64 columns of 32 bits, or 32 columns of 16-bit pairs: lane t of the warp holds, of rows t / 4 and
// t / 4 + 8, of every 8 columns the (t mod 4)-th two next to each other (of every 4 pairs the (t mod 4)-th); register
// 4 j + 2 i + k (2 j + i) is row i's of the j-th 8 columns (4 pairs).
#define RESS_TMEM_LD16X64(taddr, r) \
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;" \
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), \
      "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), \
      "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), \
      "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), \
      "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), \
      "=r"(r[31]) \
      : "r"(taddr) \
      : "memory")
#define RESS_TMEM_ST16X64(taddr, r) \
  asm volatile("tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(taddr), \
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), \
      "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), \
      "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), \
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), \
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) \
      : "memory")
#define RESS_TMEM_LD16X32P(taddr, r) \
  asm volatile("tcgen05.ld.sync.aligned.16x128b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\ttcgen05.wait::ld.sync.aligned;" \
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), \
      "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), \
      "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) \
      : "r"(taddr) \
      : "memory")
#define RESS_TMEM_ST16X32P(taddr, r) \
  asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};\n\ttcgen05.wait::st.sync.aligned;" ::"r"(taddr), \
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), \
      "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), \
      "r"(r[14]), "r"(r[15]) \
      : "memory")

// The same loads and stores without their waits: the registers of a load are valid after RESS_TMEM_WAIT_LD32, through
// which they go.
#define RESS_TMEM_LD16X64_NOWAIT(taddr, r) \
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];" \
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), \
      "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), \
      "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), \
      "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), \
      "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), \
      "=r"(r[31]) \
      : "r"(taddr) \
      : "memory")
#define RESS_TMEM_WAIT_LD32(r) \
  asm volatile("tcgen05.wait::ld.sync.aligned;" \
      : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), \
      "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), \
      "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), \
      "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), \
      "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), \
      "+r"(r[31]) \
      : \
      : "memory")
#define RESS_TMEM_ST16X32P_NOWAIT(taddr, r) \
  asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), \
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), \
      "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), \
      "r"(r[14]), "r"(r[15]) \
      : "memory")
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Four lanes with four words each: lane i's word j becomes lane j's word i.
__device__ __forceinline__ void transpose4(uint32_t& w0, uint32_t& w1, uint32_t& w2, uint32_t& w3, int lane) {
  const bool odd = lane & 1, high = lane & 2;
  const uint32_t a = __shfl_xor_sync(0xffffffffu, odd ? w0 : w1, 1), b = __shfl_xor_sync(0xffffffffu, odd ? w2 : w3, 1);
  if (odd)
    w0 = a, w2 = b;
  else
    w1 = a, w3 = b;
  const uint32_t c = __shfl_xor_sync(0xffffffffu, high ? w0 : w2, 2), d = __shfl_xor_sync(0xffffffffu, high ? w1 : w3, 2);
  if (high)
    w0 = c, w1 = d;
  else
    w2 = c, w3 = d;
}

template <bool kF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (kF16)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool kF16>
__device__ __forceinline__ float2 unpack2(uint32_t v) {
  if (!kF16) return make_float2(bf16_lo(v), bf16_hi(v));
  float2 r;
  asm("{\n\t.reg .f16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}"
      : "=f"(r.x), "=f"(r.y)
      : "r"(v));
  return r;
}
template <bool kF16>
__host__ __device__ constexpr uint32_t idesc16(int M, int N, bool b_mn_major) {
  return kF16 ? idesc_bf16_f32(M, N, b_mn_major) & ~((1u << 7) | (1u << 10)) : idesc_bf16_f32(M, N, b_mn_major);
}

// The rows of a 128-row tile from `from` on become 0; thread i of 256 takes 64 of the 128 bytes of row i / 2.
__device__ __forceinline__ void zero_rows(uint8_t* tile, int from, int i) {
  if (i / 2 >= from) {
    uint4* p = reinterpret_cast<uint4*>(tile + (i / 2) * 128 + (i & 1) * 64);
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = make_uint4(0u, 0u, 0u, 0u);
  }
}

// (y0, y1) = top tanh(x / cap) of two scores, c = 2 log2(e) / cap: top (1 - 2 / (2^(c x) + 1)), off by 2^-21 top (the
// rounding near 1; relative to a score near 0 more, but it is an exponent).
__device__ __forceinline__ void capped2(float& x0, float& x1, float c, float top) {
  float e0, e1;
  fma2(e0, e1, x0, x1, c, c, 0.f, 0.f);
  e0 = ex2(e0), e1 = ex2(e1);
  add2(e0, e1, e0, e1, 1.f, 1.f);
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e0));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(e1));
  fma2(x0, x1, e0, e1, -2.f * top, -2.f * top, top, top);
}

__device__ __forceinline__ void mul2(float& d0, float& d1, float a0, float a1, float b0, float b1) {
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\t"
      "mul.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d0), "=f"(d1)
      : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

// Products q.k to capped scores in log2 units: up to half of the cap x times a polynomial in x^2 (set_cap), five packed
// instructions a pair on the FMA pipe, next to which the SFU forms the exponentials; above it capped2, whose four SFU operations a
// pair are twice what the exponentials take (with capped2 alone packed documents, cap 30, took 251 us where 239 with both).  A
// polynomial of one term less up to a quarter of the cap gains nothing.
__device__ __forceinline__ void cap_small2(float& x0, float& x1, const DenseArgs& a) {
  float z0, z1, p0, p1;
  mul2(z0, z1, x0, x1, x0, x1);
  fma2(p0, p1, z0, z1, a.cap_poly[3], a.cap_poly[3], a.cap_poly[2], a.cap_poly[2]);
  fma2(p0, p1, z0, z1, p0, p1, a.cap_poly[1], a.cap_poly[1]);
  fma2(p0, p1, z0, z1, p0, p1, a.cap_poly[0], a.cap_poly[0]);
  mul2(x0, x1, x0, x1, p0, p1);
}

// The same of a warp's 16 rows x 64 columns.  The two forms differ in their last bits, so each product's own size chooses
// between them: what is not seen (stale rows of a page, a batch's neighbours) changes no bit, and the warp only leaves capped2
// out where no product needs it.  Measured on f16 documents, cap 30 with no product above half of it, and cap 2 with most of them
// above: this 179 and 250 us; the warp's largest product choosing for all (what is not seen among them) 179 and 199; the same with zeros
// for what is not seen 208 and 223, of which most is the code (the loop of the softmax warps is near what the instruction
// cache holds); capped2 in all tiles with a mask 190 and 205.
__device__ __forceinline__ bool any_above_cap(const float (&x)[32], const DenseArgs& a) {
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < 32; e += 2) top = fmax3(top, fabsf(x[e]), fabsf(x[e + 1]));
  return __any_sync(0xffffffffu, !(top <= a.cap_small));
}
__device__ __forceinline__ void cap_scores(float (&x)[32], const DenseArgs& a, float in, float out) {
  if (!any_above_cap(x, a)) {
#pragma unroll
    for (int e = 0; e < 32; e += 2) cap_small2(x[e], x[e + 1], a);
  } else {
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      float y0 = x[e], y1 = x[e + 1];
      const bool s0 = fabsf(y0) <= a.cap_small, s1 = fabsf(y1) <= a.cap_small;
      cap_small2(y0, y1, a);
      capped2(x[e], x[e + 1], in, out);
      x[e] = s0 ? y0 : x[e], x[e + 1] = s1 ? y1 : x[e + 1];
    }
  }
}

// The same of two products, with the slope 1 - tanh^2 of the cap (back = 1 / out).  Above half of the cap 1 - t^2 would cancel
// (t is off by 2^-21, the slope at four caps 0.0013, at seven 3e-6): with e = 2^(2 log2(e) x / cap) and r = 1 / (1 + e) it is
// 4 e r^2, whose factors are off by 2^-22 of themselves on both sides of zero (e r is at most 1, and 1 where e is infinite).
// (Gradient of bf16 documents, cap 2 with most products above half of it: 340 us with 1 - t^2 alone, 390 with this; cap 30 with none
// above it 274 and 279.)
template <bool kLarge>
__device__ __forceinline__ void cap_slope2(float& x0, float& x1, float& c0, float& c1, const DenseArgs& a, float in, float out,
                                           float back) {
  float y0 = x0, y1 = x1, u0, u1;
  cap_small2(y0, y1, a);
  mul2(u0, u1, y0, y1, back, back);
  fma2(c0, c1, -u0, -u1, u0, u1, 1.f, 1.f);
  if (kLarge) {
    const bool s0 = fabsf(x0) <= a.cap_small, s1 = fabsf(x1) <= a.cap_small;
    float e0, e1, r0, r1, w0, w1;
    mul2(e0, e1, x0, x1, in, in);
    e0 = ex2(e0), e1 = ex2(e1);
    add2(r0, r1, e0, e1, 1.f, 1.f);
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r0));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(r1));
    fma2(x0, x1, r0, r1, -2.f * out, -2.f * out, out, out);
    mul2(w0, w1, e0, e1, r0, r1);
    w0 = fminf(w0, 1.f), w1 = fminf(w1, 1.f);
    mul2(r0, r1, r0, r1, 4.f, 4.f);
    mul2(w0, w1, w0, w1, r0, r1);
    x0 = s0 ? y0 : x0, x1 = s1 ? y1 : x1, c0 = s0 ? c0 : w0, c1 = s1 ? c1 : w1;
  } else {
    x0 = y0, x1 = y1;
  }
}

// Which kernel: 1, with a cap; 2, with slopes; 3, both.
inline int dense_gen(const DenseArgs& a) { return (a.cap > 0.f ? 1 : 0) + (a.slopes ? 2 : 0); }

// tanh(u) / u for u^2 = z up to 1/4: a polynomial fitted to it at Chebyshev points by reweighted least squares, off by
// 2^-20.8 of itself; its coefficients times what makes x = q.k out of u = x / (8 cap), and log2(e) cap u of tanh(u).
inline void set_cap(DenseArgs& a) {
  constexpr double kFit[4] = {0.999999463558197, -0.33326318860054016, 0.13190296292304993, -0.04440222308039665};
  const double u = 0.125 / a.cap;
  double scale = 0.125 * 1.4426950408889634;
  for (int k = 0; k < 4; ++k, scale *= u * u) a.cap_poly[k] = (float)(kFit[k] * scale);
  // (caps so small that the coefficients are beyond float32 have no such products)
  a.cap_small = a.cap > 1e-3f ? (float)fmin(0.5 / u, (double)FLT_MAX) : -1.f;
}

}  // namespace work
}  // namespace ress

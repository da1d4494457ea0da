// A paged cache's bookkeeping on the GPU: pages and slots for the next tokens of every sequence
// (k_cache_tables), and the keys and values written there (k_cache_write).  Both are bound by their launch
// for a few tokens, the second by HBM for many (each row read and written once, 16 bytes a lane).
#include "row_ops.cuh"
#include "sm100_ptx.cuh"

namespace ress {
using namespace ptx;

constexpr int kTablesThreads = 256, kTokensPerCta = 1024;

// Every CTA adds up all sequences' tokens and new pages (n_seqs numbers, mostly a handful; a second kernel
// for that would cost a launch), keeps the running totals in shared memory and finds its own tokens' sequences there
// by bisection.  A token that begins a page enters it into the table, so no CTA waits for another: pages that were
// held before are read from the table, new ones are computed.
__global__ void __launch_bounds__(kTablesThreads) k_cache_tables(const CacheTablesArgs a) {
  extern __shared__ int2 at[];  // per sequence: tokens before it, new pages before it; then the totals
  __shared__ int2 sums[kTablesThreads / 32];
  rows::stream_acquire();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool tells = blockIdx.x == 0;
  auto counts = [&](int b, int& have, int& add, int& held) -> int {
    have = a.have[b], add = a.add[b];
    if (have < 0 || add < 0 || add > INT32_MAX - a.page - have) {
      if (tells) flag_status(a.status, kStatusBadRow);
      have = max(have, 0), add = 0;
      if (have > INT32_MAX - a.page) have = INT32_MAX - a.page;
    }
    held = (have + a.page - 1) / a.page;
    return (have + add + a.page - 1) / a.page - held;
  };
  const int per = (a.n_seqs + kTablesThreads - 1) / kTablesThreads;
  const int lo = min(a.n_seqs, tid * per), hi = min(a.n_seqs, lo + per);
  // the totals saturate: what goes past 2^31 tokens or pages is past the slots and the free pages as well
  auto plus = [](int x, int y) { return (int)min((int64_t)x + y, (int64_t)INT32_MAX); };
  int2 sum = make_int2(0, 0);
  for (int b = lo; b < hi; ++b) {
    int have, add, held;
    const int fresh = counts(b, have, add, held);
    sum = make_int2(plus(sum.x, add), plus(sum.y, fresh));
  }
  int2 inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, inc.x, o), y = __shfl_up_sync(0xffffffffu, inc.y, o);
    if (lane >= o) inc = make_int2(plus(inc.x, x), plus(inc.y, y));
  }
  int2 before = make_int2(__shfl_up_sync(0xffffffffu, inc.x, 1), __shfl_up_sync(0xffffffffu, inc.y, 1));
  if (lane == 0) before = make_int2(0, 0);
  if (lane == 31) sums[warp] = inc;
  __syncthreads();
  for (int w = 0; w < warp; ++w) before = make_int2(plus(before.x, sums[w].x), plus(before.y, sums[w].y));
  for (int b = lo; b < hi; ++b) {
    int have, add, held;
    const int fresh = counts(b, have, add, held);
    at[b] = before;
    if (tells) {
      a.lens[b] = have + add;
      a.q_start[b] = before.x;
    }
    before = make_int2(plus(before.x, add), plus(before.y, fresh));
  }
  if (hi == a.n_seqs && (lo < hi || tid == 0)) at[a.n_seqs] = before;
  __syncthreads();
  const int total = at[a.n_seqs].x, taken = *a.taken;
  const int64_t first = max(taken, 0);
  if (tells && tid == 0) {
    a.q_start[a.n_seqs] = total;
    *a.taken_out = (int)min(first + at[a.n_seqs].y, (int64_t)INT32_MAX);
    if (taken < 0 || total > a.n_slots || first + at[a.n_seqs].y > a.n_free) flag_status(a.status, kStatusBadIndex);
  }
  const int64_t base = (int64_t)blockIdx.x * kTokensPerCta;
  for (int64_t i = base + tid; i < min(base + kTokensPerCta, a.n_slots); i += kTablesThreads) {
    int slot = -1, pos = -1;
    if (i < total) {
      int s0 = 0, s1 = a.n_seqs - 1;  // the last sequence that begins at or before i
      while (s0 < s1) {
        const int mid = (s0 + s1 + 1) / 2;
        if (at[mid].x <= i)
          s0 = mid;
        else
          s1 = mid - 1;
      }
      int have, add, held;
      counts(s0, have, add, held);
      pos = have + (int)(i - at[s0].x);
      const int col = pos / a.page;
      int id = -1;
      if (col < a.table_cols) {
        int32_t* entry = a.table + s0 * a.table_stride + col;
        if (col < held) {
          id = *entry;
        } else {
          const int64_t f = first + at[s0].y + col - held;
          if (f < a.n_free) {
            id = a.free[f];
            if (pos % a.page == 0) *entry = id;
          }
        }
      }
      const int64_t where = (int64_t)id * a.page + pos % a.page;
      if (id < 0 || where > INT32_MAX)
        flag_status(a.status, kStatusBadIndex);
      else
        slot = (int)where;
    }
    a.slots[i] = slot;
    a.pos[i] = pos;
  }
}

cudaError_t launch_cache_tables(const CacheTablesArgs& a, cudaStream_t st) {
  const size_t smem = ((size_t)a.n_seqs + 1) * sizeof(int2);
  cudaError_t e = cudaFuncSetAttribute(k_cache_tables, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (RESS_MAX_SEQS + 1) * (int)sizeof(int2));
  if (e != cudaSuccess) return e;
  const int64_t ctas = (a.n_slots + kTokensPerCta - 1) / kTokensPerCta;
  return launch_pdl(k_cache_tables, dim3((unsigned)(ctas < 1 ? 1 : ctas)), dim3(kTablesThreads), smem, st, true, a);
}

// `lanes` of a warp take one token (8 lanes per head, at most the whole warp): 16 bytes of K and of V each.
__global__ void __launch_bounds__(256) k_cache_write(const CacheWriteArgs a, int lanes) {
  rows::stream_acquire();
  const int per = 256 / lanes, sub = threadIdx.x % lanes;
  const int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / lanes;
  if (t >= a.tokens) return;
  const int slot = a.slots[t];
  if (slot == -1) return;  // no token
  if (slot < 0 || slot >= a.n_pages * a.page) {
    if (sub == 0) flag_status(a.status, kStatusBadIndex);
    return;
  }
  const int page = slot / a.page, row = slot % a.page;
  auto at = [](const ress_heads& h, int64_t token, int head, int chunk) -> uint4* {
    return reinterpret_cast<uint4*>(static_cast<uint16_t*>(h.data) + token * h.token_stride + head * h.head_stride) + chunk;
  };
#pragma unroll 4
  for (int j = sub; j < 8 * a.kv_heads; j += lanes) {
    const int head = j >> 3, chunk = j & 7;
    const uint4 k = ld_stream(at(a.k, t, head, chunk)), v = ld_stream(at(a.v, t, head, chunk));
    reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(at(a.kc, row, head, chunk)) + page * a.k_page_stride)[0] = k;
    reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(at(a.vc, row, head, chunk)) + page * a.v_page_stride)[0] = v;
  }
}

cudaError_t launch_cache_write(const CacheWriteArgs& a, cudaStream_t st) {
  const int lanes = a.kv_heads == 1 ? 8 : a.kv_heads == 2 ? 16 : 32;
  const int64_t ctas = (a.tokens + 256 / lanes - 1) / (256 / lanes);
  return launch_pdl(k_cache_write, dim3((unsigned)ctas), dim3(256), 0, st, true, a, lanes);
}

}  // namespace ress

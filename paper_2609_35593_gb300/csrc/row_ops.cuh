// What the row kernels share (layer norm, head norm with rotary positions, and their gradients):
// elements of the three types the rows come in, 16-byte vectors of them, sums over the threads of
// a row, and the rotary plan's phases.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "ress_internal.cuh"
#include "sm100_ptx.cuh"

namespace ress {
namespace rows {

// The kernels of this file's users start early (launch_pdl) and call this in every CTA before
// their first access to global memory; they call stream_release once their last loads are on the
// way.  See ptx::pdl_wait for what that asks of them: no __restrict__, no read-only loads.
__device__ __forceinline__ void stream_acquire() { ptx::pdl_wait(); }
__device__ __forceinline__ void stream_release() { ptx::pdl_trigger(); }

typedef __nv_bfloat16 bf16;
typedef __half f16;

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<bf16>(bf16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32<f16>(f16 v) { return __half2float(v); }

// one rounding, to nearest even
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ f16 from_f32<f16>(float v) { return __float2half_rn(v); }

// E consecutive elements as they lie in memory: 32-bit words (E = 1: one element's bits).
template <typename T, int E>
struct Vec {
  static constexpr int kWords = E * (int)sizeof(T) < 4 ? 1 : E * (int)sizeof(T) / 4;
  uint32_t w[kWords];
};

// Vectors are read once and bypass L1 where a lane's 16 bytes stand next to its neighbour's; a
// lane's second 16 bytes (E elements of more than 16 bytes) find the sector of the first in L1.
template <typename T, int E>
__device__ __forceinline__ Vec<T, E> load_vec(const T* p) {
  Vec<T, E> r;
  constexpr int kBytes = E * (int)sizeof(T);
  if constexpr (E == 1) {
    if constexpr (sizeof(T) == 4)
      r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    else
      r.w[0] = *reinterpret_cast<const uint16_t*>(p);
  } else if constexpr (kBytes == 8) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    r.w[0] = v.x, r.w[1] = v.y;
  } else if constexpr (kBytes == 16) {
    const uint4 v = ld_stream(reinterpret_cast<const uint4*>(p));
    r.w[0] = v.x, r.w[1] = v.y, r.w[2] = v.z, r.w[3] = v.w;
  } else {
    static_assert(kBytes % 16 == 0, "vectors of 8 bytes or whole 16");
#pragma unroll
    for (int k = 0; k < kBytes / 16; ++k) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[k];
      r.w[4 * k] = v.x, r.w[4 * k + 1] = v.y, r.w[4 * k + 2] = v.z, r.w[4 * k + 3] = v.w;
    }
  }
  return r;
}

template <typename T, int E>
__device__ __forceinline__ Vec<T, E> zero_vec() {
  Vec<T, E> r;
#pragma unroll
  for (int k = 0; k < Vec<T, E>::kWords; ++k) r.w[k] = 0u;
  return r;
}

template <typename T, int E>
__device__ __forceinline__ float elem(const Vec<T, E>& v, int j) {
  if constexpr (sizeof(T) == 4) {
    return __uint_as_float(v.w[j]);
  } else if constexpr (sizeof(T) == 2) {
    const uint16_t bits = (uint16_t)(v.w[j / 2] >> (16 * (j & 1)));
    if constexpr (__is_same(T, bf16))
      return __uint_as_float((uint32_t)bits << 16);
    else
      return __half2float(__ushort_as_half(bits));
  }
}

template <typename T, int E>
__device__ __forceinline__ void store_vec(T* p, const float (&v)[E]) {
  constexpr int kBytes = E * (int)sizeof(T);
  if constexpr (E == 1) {
    *p = from_f32<T>(v[0]);
  } else {
    uint32_t w[kBytes / 4];
#pragma unroll
    for (int k = 0; k < kBytes / 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        w[k] = __float_as_uint(v[k]);
      } else if constexpr (__is_same(T, bf16)) {
        w[k] = cvt_bf16x2(v[2 * k], v[2 * k + 1]);
      } else {
        const __half2 h = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
        w[k] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    if constexpr (kBytes == 8) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
      for (int k = 0; k < kBytes / 16; ++k)
        reinterpret_cast<uint4*>(p)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    }
  }
}

// A parameter (norm weight or bias) of either of the types parameters come in; NULL: `none`.
__device__ __forceinline__ float param_at(const void* p, int type, int64_t i, float none) {
  if (!p) return none;
  if (type == RESS_F32) return static_cast<const float*>(p)[i];
  if (type == RESS_BF16) return to_f32(static_cast<const bf16*>(p)[i]);
  return to_f32(static_cast<const f16*>(p)[i]);
}

// E consecutive parameters, col a multiple of E, aligned to 16 bytes (E = 4 of 16 bits: 8) where E > 1.
template <int E>
__device__ __forceinline__ void params_at(const void* p, int type, int64_t col, float none, float* out) {
  if constexpr (E == 1) {
    out[0] = param_at(p, type, col, none);
  } else if (!p) {
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = none;
  } else if (type == RESS_F32) {
#pragma unroll
    for (int k = 0; k < E / 4; ++k) {
      const float4 v = reinterpret_cast<const float4*>(static_cast<const float*>(p) + col)[k];
      out[4 * k] = v.x, out[4 * k + 1] = v.y, out[4 * k + 2] = v.z, out[4 * k + 3] = v.w;
    }
  } else {
    uint32_t w[E / 2];
    const uint16_t* at = static_cast<const uint16_t*>(p) + col;
    if constexpr (E == 8) {
      const uint4 v = *reinterpret_cast<const uint4*>(at);
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
      static_assert(E == 4, "1, 4 or 8 parameters");
      const uint2 v = *reinterpret_cast<const uint2*>(at);
      w[0] = v.x, w[1] = v.y;
    }
    if (type == RESS_BF16) {
#pragma unroll
      for (int k = 0; k < E / 2; ++k) out[2 * k] = bf16_lo(w[k]), out[2 * k + 1] = bf16_hi(w[k]);
    } else {
#pragma unroll
      for (int k = 0; k < E / 2; ++k) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
        out[2 * k] = f.x, out[2 * k + 1] = f.y;
      }
    }
  }
}

// Two floats for the packed float32 instructions, which do two operations per lane and issue: these
// kernels have enough arithmetic per byte for it to show (layer norm's gradient, 43,968 x 1024 bf16
// with a residual: 63 us packed, 80 one by one).
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 pack2(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ F2 both(float a) { return pack2(a, a); }
__device__ __forceinline__ void unpack2(F2 x, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v));
}
__device__ __forceinline__ float sum2(F2 x) {
  float a, b;
  unpack2(x, a, b);
  return a + b;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return d;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.v) : "l"(a.v), "l"(b.v));
  return d;
}

// Elements 2j and 2j + 1 of a thread's vectors.
template <typename T, int E, int V>
__device__ __forceinline__ F2 pair_of(const Vec<T, E> (&v)[V], int j) {
  if constexpr (E > 1 && __is_same(T, f16)) {
    const uint32_t w = v[2 * j / E].w[j % (E / 2)];
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return pack2(f.x, f.y);
  } else {
    return pack2(elem(v[2 * j / E], 2 * j % E), elem(v[(2 * j + 1) / E], (2 * j + 1) % E));
  }
}

// The sum of v over aligned segments of SEG lanes, in every lane of the segment.
template <int SEG>
__device__ __forceinline__ float segment_sum(float v) {
#pragma unroll
  for (int o = SEG / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Sums of N values over aligned segments of SEG lanes, N a power of two of at most SEG, by halves:
// each step sends one half of the values to the other half of the lanes, so that N values take
// N - 1 + log2(SEG / N) exchanges instead of N log2(SEG).  Lane l of a segment holds the sum of value
// l / (SEG / N).
template <int SEG, int N>
__device__ __forceinline__ float segment_sums(float (&v)[N]) {
  const int lane = (int)threadIdx.x & 31;
  int o = SEG / 2;
#pragma unroll
  for (int n = N; n > 1; n /= 2, o /= 2) {
    const bool up = (lane & o) != 0;
#pragma unroll
    for (int k = 0; k < n / 2; ++k) {
      const float send = up ? v[k] : v[k + n / 2], keep = up ? v[k + n / 2] : v[k];
      v[k] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
  }
  float r = v[0];
#pragma unroll
  for (int q = SEG / N / 2; q > 0; q /= 2) r += __shfl_xor_sync(0xffffffffu, r, q);
  return r;
}

// cos and sin of a position's angle.  The plan holds each frequency in turns per unit position as
// a 64-bit fixed-point fraction, so that the product with an integer position is taken modulo whole
// turns without a further error: the 64-bit product's wrap-around is the reduction.  Its upper 32 bits are the
// angle in units of 2^-31 half turns (what is dropped is less than 2^-32 turns), and float rounds that to 2^-24 of
// itself (a product in float is off by the position times 2^-24 turns).
__device__ __forceinline__ float2 rope_cos_sin(int32_t pos, uint64_t turns) {
  const uint64_t phase = (uint64_t)(int64_t)pos * turns;
  const float half_turns = (float)(int32_t)(phase >> 32) * 0x1p-31f;
  float2 r;
  sincospif(half_turns, &r.y, &r.x);
  return r;
}

// The axis of a pair.
__host__ __device__ inline int rope_axis(const ress_rope_plan& plan, int pair) {
  int a = 0, end = plan.axis_dims[0] / 2;
  while (pair >= end) end += plan.axis_dims[++a] / 2;
  return a;
}

// CTAs of a kernel that fit on an SM, for each number of warps.  Asked for once (the question takes about as long
// as a launch), and again after an answer that failed.
template <auto kKernel>
cudaError_t resident_ctas(int threads, size_t smem, int& ctas) {
  static std::atomic<int> known[1024 / 32 + 1];
  std::atomic<int>& at = known[threads / 32];
  ctas = at.load(std::memory_order_relaxed);
  if (ctas > 0) return cudaSuccess;
  const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, kKernel, threads, smem);
  if (e != cudaSuccess) return e;
  if (ctas < 1) return cudaErrorLaunchOutOfResources;
  at.store(ctas, std::memory_order_relaxed);
  return cudaSuccess;
}

inline int sm_count() {
  int dev = 0, n = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
  return n > 0 ? n : 1;
}

}  // namespace rows
}  // namespace ress

// Rows in registers as chunks of eight consecutive elements, shared by the
// row-wise kernels (rowwise.hip, layernorm.hip): loads and stores at any
// element address, and sums over a row's threads in a fixed order.
#pragma once

#include <type_traits>

#include "gemm_core.h"

namespace mdnn {
namespace {

// Eight consecutive elements at any element address.
typedef uint32_t u4v_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u4v_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u2v_a1 __attribute__((ext_vector_type(2), aligned(1)));
#define MDNN_GLOBAL __attribute__((address_space(1)))

template <class T>
struct Chunk {
  static constexpr bool H = sizeof(typename T::storage) == 2;
  typedef typename T::storage S;
  uint32_t w[H ? 4 : 8];
  __device__ __forceinline__ void load(const S* p) {
    if constexpr (H) {
      const u4v_a2 v = *(const MDNN_GLOBAL u4v_a2*)p;
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else {
      const u4v_a4 v = *(const MDNN_GLOBAL u4v_a4*)p, u = *(const MDNN_GLOBAL u4v_a4*)(p + 4);
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w, w[4] = u.x, w[5] = u.y, w[6] = u.z, w[7] = u.w;
    }
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (H)
      return to_f<T>((uint16_t)(w[e >> 1] >> ((e & 1) * 16)));
    else
      return __builtin_bit_cast(float, w[e]);
  }
  // clears elements 0 .. lo - 1
  __device__ __forceinline__ void clear(int lo) {
    asm("" : "+v"(lo));  // (the tests of lo stay here: hoisted out of a loop over rows they fill the scalar registers)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < lo) w[H ? e >> 1 : e] &= H && !(e & 1) ? 0xffff0000u : 0u;
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    if constexpr (H) {
      // (a vector conversion is one instruction for two elements)
      typedef float f2 __attribute__((ext_vector_type(2)));
      typedef std::conditional_t<T::id == MDNN_F16, _Float16, __bf16> E;
      typedef E e2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){v[2 * e], v[2 * e + 1]}, e2));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = __builtin_bit_cast(uint32_t, v[e]);
    }
  }
  // elements lo .. 7 (lo = 0: one vector store)
  __device__ __forceinline__ void store(S* p, int lo) const {
    if (lo == 0) {
      if constexpr (H) {
        *(MDNN_GLOBAL u4v_a2*)p = (u4v_a2){w[0], w[1], w[2], w[3]};
      } else {
        *(MDNN_GLOBAL u4v_a4*)p = (u4v_a4){w[0], w[1], w[2], w[3]};
        *(MDNN_GLOBAL u4v_a4*)(p + 4) = (u4v_a4){w[4], w[5], w[6], w[7]};
      }
    } else {
      asm("" : "+v"(lo));
#pragma unroll
      for (int e = 1; e < 8; ++e)
        if (e >= lo) {
          if constexpr (H)
            p[e] = (uint16_t)(w[e >> 1] >> ((e & 1) * 16));
          else
            p[e] = __builtin_bit_cast(float, w[e]);
        }
    }
  }
};

__device__ __forceinline__ float mul_rn(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
__device__ __forceinline__ float add_rn(float a, float b) {
#pragma clang fp contract(off)
  return a + b;
}
struct Sum2 {
  float a, b;
};
template <int TPR, int RPB>
__device__ __forceinline__ Sum2 row_reduce(Sum2 v, Sum2 (*buf)[RPB][TPR / 64 + 1], int flip) {
  constexpr int W = TPR < 64 ? TPR : 64;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) {
    v.a += __shfl_xor(v.a, o, W);
    v.b += __shfl_xor(v.b, o, W);
  }
  if constexpr (TPR > 64) {
    const int r = threadIdx.x / TPR;
    if ((threadIdx.x & 63) == 0) buf[flip][r][threadIdx.x % TPR >> 6] = v;
    __syncthreads();
    v = buf[flip][r][0];
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w) v.a += buf[flip][r][w].a, v.b += buf[flip][r][w].b;
  }
  return v;
}

// Where this thread's chunk c of a row lies: its first element, and how many
// of its leading elements are not its own (8: none is).
struct ChunkPos {
  int start, lo;
};
__device__ __forceinline__ ChunkPos chunk_pos(int c, int cols) {
  const int at = c * 8, last = cols - 8;
  return {at < last ? at : last, at <= last ? 0 : at < cols ? at - last : 8};
}

// One launch holds fewer than 2^32 threads: blocks beyond this many rows loop.
constexpr int64_t MAX_BLOCKS = 1 << 20;

}  // namespace
}  // namespace mdnn

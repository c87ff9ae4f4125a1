// How a tile of logits ends: in the softmax's statistics (forward) or in the
// logits' gradient (backward), from the accumulators.
#pragma once

#include <type_traits>

#include "xent.h"

namespace mdnn {
namespace {

// The bias of a tile's columns (-Inf past the piece: no probability), the labels
// and lse of its rows (+Inf where G is zero: ignored rows and those past M).
template <class TL, bool BWD>
struct XentNumbers {
  alignas(16) float bias[TL::BN];  // (read four at a time)
  int32_t label[TL::BM];
  float lse[BWD ? TL::BM : 1];
  __device__ __forceinline__ void load(const XentTile& x, int64_t M, int64_t N, int64_t m0, int64_t n0, int tid) {
    for (int i = tid; i < TL::BN; i += TL::NT) bias[i] = n0 + i >= N ? -INFINITY : x.bias ? x.bias[n0 + i] : 0.0f;
    for (int i = tid; i < TL::BM; i += TL::NT) {
      const int32_t c = m0 + i < M ? x.labels[m0 + i] : x.ignored;
      if constexpr (BWD) {
        const bool live = m0 + i < M && c != x.ignored;
        label[i] = live ? c : -1;
        const float l = live ? x.lse[m0 + i] : 0.0f;
        lse[i] = !live ? INFINITY : c >= 0 && c < x.classes ? (l == INFINITY ? 3.4e38f : l) : __builtin_nanf("");
      } else {
        label[i] = c;
      }
    }
  }
};

// room: LDS of the mainloop that no wave reads past the barrier in here.
template <class T, class TL, bool BWD>
__device__ __forceinline__ void xent_end(const XentTile& x, const XentNumbers<TL, BWD>& rn, int64_t M, int64_t N,
                                         int64_t m0, int64_t n0, int tm, int tn, int wm, int wn, int tid, char* room,
                                         float4_t (&acc)[TL::FM][TL::FN]) {
  constexpr int FM = TL::FM, FN = TL::FN;
  const int lane = tid & 63;
  // lane holds rows mw + 16 i, columns nw + 16 j + e of the tile
  const int mw = wm * TL::WTM + (lane & 15), nw = wn * TL::WTN + 4 * (lane >> 4);
  float4_t bq[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) bq[j] = *(const float4_t*)&rn.bias[nw + j * 16];
  if (n0 + TL::BN > N) {  // (columns past the piece: whatever they were multiplied from)
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = n0 + nw + j * 16 + e < N ? acc[i][j][e] : 0.0f;
  }
  __syncthreads();  // (the mainloop's last fragment reads are done)

  if constexpr (!BWD) {
    if (tm == 0 && tn == 0 && tid == 0) *x.done = 0;
    Pair* red = (Pair*)room;  // [WN][BM]
    static_assert(TL::WN * TL::BM * sizeof(Pair) <= TL::A_BYTES && TL::WM * TL::BN * 4 <= TL::A_BYTES, "room for the sums");
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      Pair v = {-INFINITY, 0.0f};
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[i][j][e] += bq[j][e];
          v.m = fmaxf(v.m, acc[i][j][e]);
        }
      v.m = fmaxf(v.m, __shfl_xor(v.m, 16, 64));
      v.m = fmaxf(v.m, __shfl_xor(v.m, 32, 64));
      const float ref = pair_ref(v.m);
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) v.s += __expf(acc[i][j][e] - ref);
      v.s += __shfl_xor(v.s, 16, 64);
      v.s += __shfl_xor(v.s, 32, 64);
      const int row = mw + i * 16;
      const int64_t at = (int64_t)rn.label[row] - x.n0 - n0 - nw;
      if (at >= 0 && at < TL::WTN && (at & 15) < 4 && m0 + row < M) {
        float z = 0.0f;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) z = at == j * 16 + e ? acc[i][j][e] : z;
        x.zlab[m0 + row] = z;
      }
      if (lane < 16) red[wn * TL::BM + row] = v;
    }
    __syncthreads();
    for (int r = tid; r < TL::BM; r += TL::NT) {
      if (m0 + r >= M) break;
      Pair v = red[r];
#pragma unroll
      for (int w = 1; w < TL::WN; ++w) v = join(v, red[w * TL::BM + r]);
      x.pairs[tn * M + m0 + r] = v;
    }
  } else {
    float sum[FN][4];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[j][e] = 0.0f;
    typedef typename T::storage S;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int row = mw + i * 16;
      const float l = rn.lse[row];
      const int64_t far = (int64_t)rn.label[row] - x.n0 - n0 - nw;
      const int at = far >= 0 && far < TL::WTN ? (int)far : -1;
      const bool dead = l == INFINITY, hit = __any(at >= 0), some = __any(dead);  // (few waves hold any)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int64_t n = n0 + nw + j * 16;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __expf(acc[i][j][e] + bq[j][e] - l);
        if (hit) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = at == j * 16 + e ? v[e] - 1.0f : v[e];
        }
        if (some) {
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = dead ? 0.0f : v[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[j][e] += v[e];
        if (m0 + row < x.rows && n < x.width) {
          S* d = (S*)x.g + (m0 + row) * x.ldg + n;
          if constexpr (sizeof(S) == 2) {
            // (a vector conversion is one instruction for two elements)
            typedef float f2 __attribute__((ext_vector_type(2)));
            typedef std::conditional_t<T::id == MDNN_F16, _Float16, __bf16> E;
            typedef E e2 __attribute__((ext_vector_type(2)));
            const float c = T::id == MDNN_F16 ? x.scale : 1.0f;
            uint2 q;
            q.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){v[0] * c, v[1] * c}, e2));
            q.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f2){v[2] * c, v[3] * c}, e2));
            *(uint2*)d = q;
          } else {
            *(float4_t*)d = (float4_t){v[0], v[1], v[2], v[3]};
          }
        }
      }
    }
    float alpha = 0.0f;
    if (x.alone) {
      const int n = __syncthreads_count(tid < TL::BM && rn.lse[tid < TL::BM ? tid : 0] != INFINITY);
      alpha = (x.loss_scale ? *x.loss_scale : 1.0f) / (float)(n > 0 ? n : 1) * (1.0f / x.scale);
      if (tn == 0 && tid == 0) *x.alpha = alpha;
    }
    if (x.part || x.db) {
      // over the 16 rows of the lanes, then the tile's wave rows in order
      float* red = (float*)room;  // [WM][BN]
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) sum[j][e] += __shfl_xor(sum[j][e], o, 64);
        }
      if ((lane & 15) == 0) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
          *(float4_t*)&red[wm * TL::BN + nw + j * 16] = (float4_t){sum[j][0], sum[j][1], sum[j][2], sum[j][3]};
      }
      __syncthreads();
      for (int c = tid; c < TL::BN; c += TL::NT) {
        if (n0 + c >= N) break;
        float s = red[c];
#pragma unroll
        for (int w = 1; w < TL::WM; ++w) s += red[w * TL::BN + c];
        if (x.db)
          x.db[x.n0 + n0 + c] = s * (alpha * x.scale);
        else
          x.part[tm * x.ldp + n0 + c] = s;
      }
    }
  }
}

}  // namespace
}  // namespace mdnn

// Logits of a piece of classes by the pipelined product (gemm_lds.h), each
// tile ending in the softmax's statistics (forward) or the logits' gradient
// (backward) from the accumulators: fp32 logits written and read again took 17
// us of each 124 us piece of 8192 x 2048 x 4096 forward (bf16), 150 of 640 us
// backward (4096 x 16384 x 4096).
//
// Bound by the product's matrix instructions.  A tile's end is one exponential
// per logit and does not run beside its own products; two workgroups to a CU
// (128 x 128) hide it behind each other's, one (256 x 256) spends about 4000
// cycles a wave on it against 2048 for each 64 of K.
#pragma once

#include "gemm_launch.h"
#include "xent.h"

namespace mdnn {
namespace {

template <class T, class TL, int NS, bool B_KC, bool BWD>
__global__ void __launch_bounds__(TL::NT, TL::OCC)
xent_tile_kernel(lds::MatArgs aa, lds::MatArgs ba, int64_t M, int64_t N, int64_t K, XentTile x) {
  typedef lds::MatLoader<true, TL::BM, TL::LA> LA;
  typedef lds::MatLoader<B_KC, TL::BN, TL::LB> LB;
  // (a stage an object: see gemm_lds_kernel)
  __shared__ __attribute__((aligned(1024))) char lds_a0[TL::A_BYTES];
  __shared__ __attribute__((aligned(1024))) char lds_b0[TL::B_BYTES];
  __shared__ __attribute__((aligned(1024))) char lds_a1[TL::A_BYTES];
  __shared__ __attribute__((aligned(1024))) char lds_b1[TL::B_BYTES];
  __shared__ __attribute__((aligned(NS > 2 ? 1024 : 1))) char lds_a2[NS > 2 ? TL::A_BYTES : 1];
  __shared__ __attribute__((aligned(NS > 2 ? 1024 : 1))) char lds_b2[NS > 2 ? TL::B_BYTES : 1];
  __shared__ __attribute__((aligned(NS > 3 ? 1024 : 1))) char lds_a3[NS > 3 ? TL::A_BYTES : 1];
  __shared__ __attribute__((aligned(NS > 3 ? 1024 : 1))) char lds_b3[NS > 3 ? TL::B_BYTES : 1];
  __shared__ float col_bias[TL::BN];
  __shared__ int32_t row_label[TL::BM];
  __shared__ float row_lse[BWD ? TL::BM : 1];
  char* const all_a[4] = {lds_a0, lds_a1, lds_a2, lds_a3};
  char* const all_b[4] = {lds_b0, lds_b1, lds_b2, lds_b3};
  lds::Stages<NS> st;
#pragma unroll
  for (int s = 0; s < NS; ++s) st.a[s] = all_a[s], st.b[s] = all_b[s];
  constexpr int FM = TL::FM, FN = TL::FN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / TL::WN, wn = wave % TL::WN;
  int tm, tn;
  tile_coords(ceil_div(M, TL::BM), ceil_div(N, TL::BN), tm, tn);
  const int64_t m0 = (int64_t)tm * TL::BM, n0 = (int64_t)tn * TL::BN;
  const int nk = (int)(K / lds::BK);

  LA la;
  LB lb;
  la.init(aa, m0, 0, wave, lane);
  lb.init(ba, n0, 0, wave, lane);
  const uint32_t wa = (uint32_t)(wave * TL::LA) * 1024u, wb = (uint32_t)(wave * TL::LB) * 1024u;
  // the rows' and columns' own numbers, for the tile's end (published by the mainloop's barriers)
  for (int i = tid; i < TL::BN; i += TL::NT) col_bias[i] = x.bias && n0 + i < N ? x.bias[n0 + i] : 0.0f;
  for (int i = tid; i < TL::BM; i += TL::NT) {
    row_label[i] = m0 + i < M ? x.labels[m0 + i] : x.ignored;
    if constexpr (BWD) row_lse[i] = m0 + i < M ? x.lse[m0 + i] : 0.0f;
  }

  float4_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = (float4_t){0.f, 0.f, 0.f, 0.f};
  lds::Frags<TL> f0, f1;
  const lds::LaneFrag fa_l = lds::lane_frag<true, TL::BM>(lane), fb_l = lds::lane_frag<B_KC, TL::BN>(lane);
#pragma unroll
  for (int s = 0; s < NS; ++s)
    if (s < nk) {
      la.issue(s, lds::lds_address(st.a[s]) + wa);
      lb.issue(s, lds::lds_address(st.b[s]) + wb);
    }
  lds::wait_tiles<NS - 1, TL::LA + TL::LB>((nk < NS ? nk : NS) - 1);  // tile 0 landed
  __syncthreads();
#pragma unroll
  for (int i = 0; i < FM; ++i) f0.a[i] = lds::fragment<true, TL::BM>(st.a[0], wm * TL::WTM + i * 16, 0, fa_l);
#pragma unroll
  for (int j = 0; j < FN; ++j) f0.b[j] = lds::fragment<B_KC, TL::BN>(st.b[0], wn * TL::WTN + j * 16, 0, fb_l);
  constexpr int U = NS % 2 == 0 ? NS : 2 * NS;
  int t = 0;
  for (; t + U - 1 + NS < nk; t += U)
    lds::pipeline_round<T, TL, NS, LA, LB, 0, U, false>(t, nk, st, wave, fa_l, fb_l, wm, wn, la, lb, f0, f1, acc);
  for (; t < nk; t += U)
    lds::pipeline_round<T, TL, NS, LA, LB, 0, U, true>(t, nk, st, wave, fa_l, fb_l, wm, wn, la, lb, f0, f1, acc);

  // lane holds rows mw + 16 i, columns nw + 16 j + e of the tile
  const int mw = wm * TL::WTM + (lane & 15), nw = wn * TL::WTN + 4 * (lane >> 4);
  float4_t bq[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) bq[j] = *(const float4_t*)&col_bias[nw + j * 16];
  const bool edge = n0 + TL::BN > N;  // columns past the piece: no logits
  __syncthreads();                    // (the mainloop's last fragment reads are done)

  if constexpr (!BWD) {
    Pair* red = (Pair*)lds_a0;  // [WN][BM]
    static_assert(TL::WN * TL::BM * sizeof(Pair) <= TL::A_BYTES, "room for the pairs");
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      Pair v = {-INFINITY, 0.0f};
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float z = acc[i][j][e] + bq[j][e];
          if (edge) z = n0 + nw + j * 16 + e < N ? z : -INFINITY;
          acc[i][j][e] = z;
          v.m = fmaxf(v.m, z);
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
      const int64_t at = (int64_t)row_label[row] - x.n0 - n0 - nw;
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
      const int32_t label = row_label[row];
      const bool live = label != x.ignored && m0 + row < M;
      const float l = label >= 0 && label < x.classes ? row_lse[row] : __builtin_nanf("");
      const int64_t far = (int64_t)label - x.n0 - n0 - nw;
      const int at = far >= 0 && far < TL::WTN ? (int)far : -1;
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int64_t n = n0 + nw + j * 16;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = __expf(acc[i][j][e] + bq[j][e] - l);
          v[e] = at == j * 16 + e ? v[e] - 1.0f : v[e];
          v[e] = live && (!edge || n + e < N) ? v[e] : 0.0f;
          sum[j][e] += v[e];
        }
        if (m0 + row < x.rows && n < x.ldg) {
          uint2 q;
          q.x = (uint32_t)from_f<T>(v[0] * x.scale) | ((uint32_t)from_f<T>(v[1] * x.scale) << 16);
          q.y = (uint32_t)from_f<T>(v[2] * x.scale) | ((uint32_t)from_f<T>(v[3] * x.scale) << 16);
          *(uint2*)((S*)x.g + (m0 + row) * x.ldg + n) = q;
        }
      }
    }
    if (x.part) {
      // over the 16 rows of the lanes, then the tile's wave rows in order
      float* red = (float*)lds_a0;  // [WM][BN]
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
        x.part[tm * x.classes + x.n0 + n0 + c] = s;
      }
    }
  }
}

template <class T, class TL, int NS, bool B_KC, bool BWD>
void launch_xent(const XentProduct& p, const XentTile& x, hipStream_t st) {
  const lds::MatArgs a{p.x, p.ldx, p.M}, b{p.w, p.ldw, p.w_kc ? p.N : p.ext};
  hipLaunchKernelGGL((xent_tile_kernel<T, TL, NS, B_KC, BWD>),
                     dim3((unsigned)(ceil_div(p.M, TL::BM) * ceil_div(p.N, TL::BN))), dim3(TL::NT), 0, st, a, b, p.M, p.N,
                     p.K, x);
}
template <class T, class TL, int NS>
void launch_xent_tile(const XentProduct& p, const XentTile& x, hipStream_t st) {
  if (p.backward)
    p.w_kc ? launch_xent<T, TL, NS, true, true>(p, x, st) : launch_xent<T, TL, NS, false, true>(p, x, st);
  else
    p.w_kc ? launch_xent<T, TL, NS, true, false>(p, x, st) : launch_xent<T, TL, NS, false, false>(p, x, st);
}

}  // namespace

template <class T>
mdnn_status_t xent_tiles(const XentProduct& p, const XentTile& x, hipStream_t st) {
  switch (xent_tile(p.M, p.N)) {
    case 256: launch_xent_tile<T, lds::Tile256, 2>(p, x, st); break;
    case 128: launch_xent_tile<T, lds::Tile128, 2>(p, x, st); break;
    default: launch_xent_tile<T, lds::Tile<64, 64, 2, 2, 2>, 4>(p, x, st); break;
  }
  return check_launch("xent_tile_kernel");
}

}  // namespace mdnn

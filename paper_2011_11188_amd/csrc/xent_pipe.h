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
#include "xent_end.h"

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
  __shared__ XentNumbers<TL, BWD> rn;
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
  rn.load(x, M, N, m0, n0, tid);  // (published by the mainloop's barriers)

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

  xent_end<T, TL, BWD>(x, rn, M, N, m0, n0, tm, tn, wm, wn, tid, lds_a0, acc);
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
  switch (xent_tile(p.M, p.N, p.K, p.backward)) {
    case 256: launch_xent_tile<T, lds::Tile256, 2>(p, x, st); break;
    case 128: launch_xent_tile<T, lds::Tile128, 2>(p, x, st); break;
    default: launch_xent_tile<T, lds::Tile<64, 64, 2, 2, 2>, 4>(p, x, st); break;
  }
  return check_launch("xent_tile_kernel");
}

}  // namespace mdnn

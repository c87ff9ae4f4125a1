// Logits of a piece of classes by the register-staged product (gemm_reg.h), for
// fp32 and for 16-bit rows on any element, each tile ending as the pipelined
// kernel's does (xent_end.h).
#include "gemm_launch.h"
#include "gemm_reg.h"
#include "xent_end.h"

namespace mdnn {
namespace {
using namespace reg;

template <class T, class TL, int NR, bool B_KC, bool BWD>
__global__ void __launch_bounds__(TL::NT, TL::OCC)
xent_reg_kernel(MatArgs aa, MatArgs ba, int64_t M, int64_t N, int64_t K, XentTile x) {
  typedef MatLoader<T, true, TL::BM, TL::LA> LA;
  typedef MatLoader<T, B_KC, TL::BN, TL::LB> LB;
  constexpr int FM = TL::FM, FN = TL::FN, ES = El<T>::ES, BK = El<T>::BK;
  __shared__ XentNumbers<TL, BWD> rn;
  __shared__ __attribute__((aligned(1024))) char a0[TL::A_BYTES];
  __shared__ __attribute__((aligned(1024))) char b0[TL::B_BYTES];
  __shared__ __attribute__((aligned(1024))) char a1[TL::A_BYTES];
  __shared__ __attribute__((aligned(1024))) char b1[TL::B_BYTES];
  char* const sa[2] = {a0, a1};
  char* const sb[2] = {b0, b1};
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / TL::WN, wn = wave % TL::WN;

  int tm, tn;
  tile_coords(ceil_div(M, TL::BM), ceil_div(N, TL::BN), tm, tn);
  const int64_t m0 = (int64_t)tm * TL::BM, n0 = (int64_t)tn * TL::BN;
  constexpr int64_t kbeg = 0;
  const int64_t kend = K;
  const int nk = (int)ceil_div(K, (int64_t)BK);

  LA la;
  LB lb;
  la.init(aa, m0, kbeg, kend, wave, lane);
  lb.init(ba, n0, kbeg, kend, wave, lane);
  const uint32_t wa = (uint32_t)(wave * TL::LA) * 1024u + (uint32_t)lane * 16u;
  const uint32_t wb = (uint32_t)(wave * TL::LB) * 1024u + (uint32_t)lane * 16u;
  const lds::LaneFrag fa = lane_frag<T, LA::KC, TL::BM>(lane), fb = lane_frag<T, LB::KC, TL::BN>(lane);

  // (chains, the last step and the wait: see gemm_reg_kernel)
  constexpr int NA = ES == 4 && FM * FN <= 4 ? 4 : 1;
  float4_t accs[NA][FM][FN];
#pragma unroll
  for (int q = 0; q < NA; ++q)
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) accs[q][i][j] = (float4_t){0.f, 0.f, 0.f, 0.f};

  constexpr bool LAST = !(LA::ANY_STEP && LB::ANY_STEP);
  const int n1 = LAST ? nk - 1 : nk;
  Sets<T, TL, NR> s;
#pragma unroll
  for (int r = 0; r < NR; ++r)
    if (r < n1) {
      la.load(r, s.a[r], s.fa[r]);
      lb.load(r, s.b[r], s.fb[r]);
    }
  rn.load(x, M, N, m0, n0, tid);  // (published by the mainloop's barriers)
  if (n1 > 0) {
    commit<ES>(sa[0] + wa, 0, s.a[0], s.fa[0], la);
    commit<ES>(sb[0] + wb, 0, s.b[0], s.fb[0], lb);
  }
  __syncthreads();
  constexpr int U = NR % 2 == 0 ? NR : 2 * NR;
  int t = 0;
  if (U + NR <= n1) __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  for (; t + U + NR <= n1; t += U)
    steps<T, TL, NR, LA, LB, 0, U, false, NA>(t, n1, sa, sb, wa, wb, wm, wn, fa, fb, la, lb, s, accs);
  uint4 za[TL::LA], zb[TL::LB];
  LastFix ga, gb;
  if (LAST && nk > 0) {
    const int64_t kz = kbeg + (int64_t)n1 * BK;
    LA qa;
    LB qb;
    qa.init(aa, m0, kz, kend, wave, lane);
    qb.init(ba, n0, kz, kend, wave, lane);
    qa.load_last(za, ga);
    qb.load_last(zb, gb);
  }
  for (; t < n1; t += U)
    steps<T, TL, NR, LA, LB, 0, U, true, NA>(t, n1, sa, sb, wa, wb, wm, wn, fa, fb, la, lb, s, accs);
  if (LAST && nk > 0) {
    char* const ta = n1 & 1 ? sa[1] : sa[0];
    char* const tb = n1 & 1 ? sb[1] : sb[0];
    commit_last<ES>(ta + wa, za, ga);
    commit_last<ES>(tb + wb, zb, gb);
    __syncthreads();
    tile_products<T, TL, LA, LB, NA>(ta, tb, wm, wn, fa, fb, accs);
  }
  float4_t(&acc)[FM][FN] = accs[0];
  if constexpr (NA == 4) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = (accs[0][i][j] + accs[1][i][j]) + (accs[2][i][j] + accs[3][i][j]);
  }

  xent_end<T, TL, BWD>(x, rn, M, N, m0, n0, tm, tn, wm, wn, tid, a0, acc);
}

template <class T, class TL, int NR, bool B_KC, bool BWD>
void launch(const XentProduct& p, const XentTile& x, hipStream_t st) {
  const MatArgs a{p.x, p.ldx, p.M, p.K}, b{p.w, p.ldw, p.N, p.K};
  hipLaunchKernelGGL((xent_reg_kernel<T, TL, NR, B_KC, BWD>),
                     dim3((unsigned)(ceil_div(p.M, TL::BM) * ceil_div(p.N, TL::BN))), dim3(TL::NT), 0, st, a, b, p.M, p.N,
                     p.K, x);
}
template <class T, class TL, int NR>
void launch_tile(const XentProduct& p, const XentTile& x, hipStream_t st) {
  if (p.backward)
    p.w_kc ? launch<T, TL, NR, true, true>(p, x, st) : launch<T, TL, NR, false, true>(p, x, st);
  else
    p.w_kc ? launch<T, TL, NR, true, false>(p, x, st) : launch<T, TL, NR, false, false>(p, x, st);
}

}  // namespace

// Tiles of 128 x 128 from 512 of them, two a compute unit: below, the last round of
// workgroups leaves most units idle (500 x 10007 x 777 fp32, 316 tiles: 114.5 us against
// 90 for 1256 of 64 x 64).
int xent_reg_tile(int64_t M, int64_t N) {
  return M > 64 && N > 64 && ceil_div(M, 128) * ceil_div(N, 128) >= 512 ? 128 : 64;
}

bool xent_reg_ok(mdnn_dtype_t t, const XentProduct& p) {
  return gemm_reg_ok(t, p.w_kc ? MDNN_NT : MDNN_NN, p.M, p.N, p.K, p.ldx, p.ldw, 1);
}

template <class T>
mdnn_status_t xent_reg(const XentProduct& p, const XentTile& x, hipStream_t st) {
  if (xent_reg_tile(p.M, p.N) == 128)
    launch_tile<T, TileR128, 2>(p, x, st);
  else
    launch_tile<T, TileR64, 4>(p, x, st);
  return check_launch("xent_reg_kernel");
}
template mdnn_status_t xent_reg<F32>(const XentProduct&, const XentTile&, hipStream_t);
template mdnn_status_t xent_reg<F16>(const XentProduct&, const XentTile&, hipStream_t);
template mdnn_status_t xent_reg<BF16>(const XentProduct&, const XentTile&, hipStream_t);

}  // namespace mdnn

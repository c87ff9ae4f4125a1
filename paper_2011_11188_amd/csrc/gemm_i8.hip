// 8-bit integer product with a scale for each row and each column:
//   D[m][n] = act(float(sum_k A[m][k] B[n][k]) * a_scale[m] * b_scale[n] + bias[n])
// on v_mfma_i32_16x16x64_i8.  Both operands are K-contiguous (the layout the
// quantisers write).  The int32 sums are exact (K <= 131071: 2^31 / 2^14), so
// the result depends on no order of summation.
//
// A 16-byte fragment of an operand is 16 consecutive k of one row, as one of
// 16-bit elements is 8: tiles of 128 bytes of k a row, their LDS layout and
// fragment reads are those of the 16-bit kernels (gemm_lds.h), with twice the
// k per byte.
#include "gemm_lds.h"
#include "gemm_reg.h"
#include "internal.h"

namespace mdnn {
namespace {

typedef int int4v __attribute__((ext_vector_type(4)));

constexpr int BKB = 128;           // bytes of k per step
constexpr int64_t I8_MAX_K = 131071;

__device__ __forceinline__ int4v mfma_i8(uint4 a, uint4 b, int4v c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(int4v, a), __builtin_bit_cast(int4v, b), c, 0, 0, 0);
}

struct I8Args {
  const int8_t *a, *b;
  const float *a_scale, *b_scale, *bias;  // bias: or null
  void* d;
  int64_t M, N, K, lda, ldb, ldd;
  int32_t act;
};

// ------------------------------------------------------------- epilogue

// Four consecutive floats from column n, columns past N read as the last.
__device__ __forceinline__ void load_cols(const float* p, int64_t n, int64_t N, float (&v)[4]) {
  if (n + 4 <= N) {
    Quad<F32> q;
    q.load(p + n);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = q.get(e);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = p[n + e < N ? n + e : N - 1];
  }
}

// One lane's four consecutive columns n .. n + 3 of row m.
template <class OutT>
__device__ __forceinline__ void store_i8(const I8Args& g, int64_t m, int64_t n, int4v acc, float sa,
                                         const float (&sb)[4], const float (&bias)[4]) {
  typedef typename OutT::storage S;
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = (float)acc[e] * sa * sb[e];
    if (g.bias) v[e] += bias[e];
    if (g.act == MDNN_ACT_RELU) v[e] = relu_f(v[e]);
  }
  S* d = (S*)g.d + m * g.ldd + n;
  if (n + 4 <= g.N) {
    Quad<OutT> q;
    if constexpr (Quad<OutT>::H) {
      q.q[0] = (uint32_t)from_f<OutT>(v[0]) | ((uint32_t)from_f<OutT>(v[1]) << 16);
      q.q[1] = (uint32_t)from_f<OutT>(v[2]) | ((uint32_t)from_f<OutT>(v[3]) << 16);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) q.q[e] = __float_as_uint(v[e]);
    }
    q.store(d);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < g.N) d[e] = from_f<OutT>(v[e]);
  }
}

// A wave's FM x FN fragments; mb, nb: this lane's first row and column.
template <class OutT, int FM, int FN>
__device__ __forceinline__ void epilogue_i8(const I8Args& g, int64_t mb, int64_t nb, const int4v (&acc)[FM][FN]) {
  float sa[FM], sb[FN][4], bias[FN][4];
#pragma unroll
  for (int i = 0; i < FM; ++i) sa[i] = g.a_scale[mb + i * 16 < g.M ? mb + i * 16 : g.M - 1];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    load_cols(g.b_scale, nb + j * 16, g.N, sb[j]);
    if (g.bias) load_cols(g.bias, nb + j * 16, g.N, bias[j]);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
      if (mb + i * 16 < g.M && nb + j * 16 < g.N) store_i8<OutT>(g, mb + i * 16, nb + j * 16, acc[i][j], sa[i], sb[j], bias[j]);
}

// ------------------------------------------------- register-staged kernel
// Rows that start on any byte, any K: chunks of 16 bytes are read at any
// address into registers and written to the swizzled LDS tiles (two stages,
// one barrier a step).  A chunk past the row's end is read from its last 16
// bytes and shifted; k past K is zero.

typedef uint32_t u4v_a1 __attribute__((ext_vector_type(4), aligned(1)));

__device__ __forceinline__ uint4 load_bytes(const int8_t* p) {
  const u4v_a1 v = *(const __attribute__((address_space(1))) u4v_a1*)p;
  return make_uint4(v.x, v.y, v.z, v.w);
}

// 16 bytes of a row from byte k, zero from K on.
__device__ __forceinline__ uint4 row_chunk(const int8_t* row, int64_t k, int64_t K) {
  if (k + 16 <= K) return load_bytes(row + k);
  if (k >= K) return make_uint4(0, 0, 0, 0);
  if (K >= 16) return reg::shift_chunk<1>(load_bytes(row + K - 16), (int)(k - (K - 16)));
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (e < K) w[e >> 2] |= (uint32_t)(uint8_t)row[e] << (8 * (e & 3));  // (k is 0 here)
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <class OutT, class TL>
__global__ void __launch_bounds__(TL::NT, TL::OCC) gemm_i8_any_kernel(I8Args g) {
  __shared__ __attribute__((aligned(1024))) char lds_a[2][TL::A_BYTES];
  __shared__ __attribute__((aligned(1024))) char lds_b[2][TL::B_BYTES];
  constexpr int FM = TL::FM, FN = TL::FN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / TL::WN, wn = wave % TL::WN;
  int tm, tn;
  tile_coords(ceil_div(g.M, TL::BM), ceil_div(g.N, TL::BN), tm, tn);
  const int64_t m0 = (int64_t)tm * TL::BM, n0 = (int64_t)tn * TL::BN;

  const int8_t *ra[TL::LA], *rb[TL::LB];
  int ka[TL::LA], kb[TL::LB];
#pragma unroll
  for (int i = 0; i < TL::LA; ++i) {
    const lds::LoadPos q = lds::load_pos<true, TL::BM, TL::LA>(wave, lane, i);
    ra[i] = g.a + (m0 + q.r < g.M ? m0 + q.r : g.M - 1) * g.lda;
    ka[i] = q.c * 2;
  }
#pragma unroll
  for (int i = 0; i < TL::LB; ++i) {
    const lds::LoadPos q = lds::load_pos<true, TL::BN, TL::LB>(wave, lane, i);
    rb[i] = g.b + (n0 + q.r < g.N ? n0 + q.r : g.N - 1) * g.ldb;
    kb[i] = q.c * 2;
  }
  uint4 va[TL::LA], vb[TL::LB];
  auto load = [&](int64_t k0) {
    if (k0 + BKB <= g.K) {
#pragma unroll
      for (int i = 0; i < TL::LA; ++i) va[i] = load_bytes(ra[i] + k0 + ka[i]);
#pragma unroll
      for (int i = 0; i < TL::LB; ++i) vb[i] = load_bytes(rb[i] + k0 + kb[i]);
    } else {
#pragma unroll
      for (int i = 0; i < TL::LA; ++i) va[i] = row_chunk(ra[i], k0 + ka[i], g.K);
#pragma unroll
      for (int i = 0; i < TL::LB; ++i) vb[i] = row_chunk(rb[i], k0 + kb[i], g.K);
    }
  };
  int4v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = (int4v){0, 0, 0, 0};
  const lds::LaneFrag fl = lds::lane_frag<true, TL::BM>(lane);
  const int nk = (int)ceil_div(g.K, BKB);
  if (nk > 0) load(0);
  for (int t = 0; t < nk; ++t) {
    char *sa = lds_a[t & 1], *sb = lds_b[t & 1];
#pragma unroll
    for (int i = 0; i < TL::LA; ++i) *(uint4*)(sa + (wave * TL::LA + i) * 1024 + lane * 16) = va[i];
#pragma unroll
    for (int i = 0; i < TL::LB; ++i) *(uint4*)(sb + (wave * TL::LB + i) * 1024 + lane * 16) = vb[i];
    if (t + 1 < nk) load((int64_t)(t + 1) * BKB);
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      uint4 fa[FM], fb[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[i] = lds::fragment<true, TL::BM>(sa, wm * TL::WTM + i * 16, kk, fl);
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[j] = lds::fragment<true, TL::BN>(sb, wn * TL::WTN + j * 16, kk, fl);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mfma_i8(fb[j], fa[i], acc[i][j]);
    }
  }
  epilogue_i8<OutT, FM, FN>(g, m0 + wm * TL::WTM + (lane & 15), n0 + wn * TL::WTN + 4 * (lane >> 4), acc);
}

typedef lds::Tile<64, 64, 2, 2, 4> TileI64;

template <class OutT>
mdnn_status_t run_i8(const I8Args& g, hipStream_t st) {
  const int64_t tiles = ceil_div(g.M, TileI64::BM) * ceil_div(g.N, TileI64::BN);
  hipLaunchKernelGGL((gemm_i8_any_kernel<OutT, TileI64>), dim3((unsigned)tiles), dim3(TileI64::NT), 0, st, g);
  return check_launch("gemm_i8_any_kernel");
}

}  // namespace
}  // namespace mdnn

using namespace mdnn;

extern "C" size_t mdnn_gemm_i8_workspace(int64_t M, int64_t N, int64_t K) {
  (void)M, (void)N, (void)K;
  return 0;
}

extern "C" mdnn_status_t mdnn_gemm_i8(int64_t M, int64_t N, int64_t K, const int8_t* A, int64_t lda,
                                      const float* a_scale, const int8_t* B, int64_t ldb, const float* b_scale,
                                      const float* bias, mdnn_act_t act, void* D, int64_t ldd, mdnn_dtype_t d_type,
                                      void* workspace, size_t ws_bytes, mdnn_stream_t stream) {
  if (M < 0 || N < 0 || K < 0) return fail(MDNN_ERR_SHAPE, "gemm_i8: negative size");
  if (K > I8_MAX_K) return fail(MDNN_ERR_SHAPE, "gemm_i8: K above %lld (32-bit sums)", (long long)I8_MAX_K);
  if (!dtype_ok(d_type)) return fail(MDNN_ERR_DTYPE, "gemm_i8: unknown d_type");
  if (act != MDNN_ACT_NONE && act != MDNN_ACT_RELU) return fail(MDNN_ERR_DTYPE, "gemm_i8: unknown act");
  if (M == 0 || N == 0) return MDNN_SUCCESS;
  if (!D || !a_scale || !b_scale || (K > 0 && (!A || !B))) return fail(MDNN_ERR_NULL, "gemm_i8: NULL buffer");
  if (lda < K || ldb < K || ldd < N) return fail(MDNN_ERR_LAYOUT, "gemm_i8: leading dimension below the width");
  if (!aligned(D, dtype_size(d_type)) || !aligned(a_scale, 4) || !aligned(b_scale, 4) || !aligned(bias, 4) ||
      !aligned(workspace, 16))
    return fail(MDNN_ERR_MISALIGNED, "gemm_i8: misaligned buffer");
  // (a launch holds fewer than 2^32 threads)
  if (M > INT64_MAX - 64 || N > INT64_MAX - 64 || ceil_div(M, 64) > (((int64_t)1 << 24) - 1) / ceil_div(N, 64))
    return fail(MDNN_ERR_SHAPE, "gemm_i8: problem too large for the launch grid");
  (void)ws_bytes;
  I8Args g = {};
  g.a = A, g.b = B, g.a_scale = a_scale, g.b_scale = b_scale, g.bias = bias, g.d = D;
  g.M = M, g.N = N, g.K = K, g.lda = lda, g.ldb = ldb, g.ldd = ldd, g.act = act;
  clear_error();
  const hipStream_t st = as_stream(stream);
  switch (d_type) {
    case MDNN_F32: return run_i8<F32>(g, st);
    case MDNN_F16: return run_i8<F16>(g, st);
    default: return run_i8<BF16>(g, st);
  }
}

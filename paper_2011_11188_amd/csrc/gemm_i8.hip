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

typedef int int4v __attribute__((ext_vector_type(4)));
typedef uint32_t u4v_a2 __attribute__((ext_vector_type(4), aligned(2)));
struct I8 {
  typedef int8_t storage;
};
template <> struct Mfma<I8> {
  typedef int4v Acc;
  static __device__ __forceinline__ int4v run(uint4 a, uint4 b, int4v c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(int4v, a), __builtin_bit_cast(int4v, b), c, 0, 0,
                                                 0);
  }
};

// The order of the tiles.  Where D is at least as wide as tall, groups of 8 tile
// columns: the 32 workgroups of an XCD then hold 8 x 4 tiles, the fewest panels in
// its L2 (16 columns x 2 rows: 1024 x 1024 x 4096 11.7 us against 9.5, 192 x 4096 x
// 4096 11.5 and 9.4, 1000 x 1001 x 4001 on any byte 18.7 and 16.0).  Which tiles
// run at once also decides which pieces of D are written together, and a D of
// hundreds of MB whose rows are whole multiples of 4 KB is slow to write down its
// columns: where the writes count, 16 tile columns, that is from 256 MB on (4096 x
// 65536 x 1024 fp32 451 us, groups of 8 485; 16384 x 16384 x 2048 fp16 565 and 571,
// groups of 8 tile rows 619; at 128 MB 8 columns still lead: 8192 x 8192 x 2048 fp16
// 130 us, 16 133; 4096 x 8192 x 1024 fp32 52 and 54) and up to four steps (8192 x 8192 x
// 128 bf16 48.7 and 50.7, 4096 x 8192 x 320 fp32 35.3 and 36.5).  Taller ones take
// groups of 4 tile rows on such rows (16384 x 8192 x 4096 420 us, 8 tile rows 476;
// 32768 x 8192 x 2048 523 and 569) and 8 on others (12000 x 5000 x 3200 176, 4 183) and
// far above N (65536 x 4096 x 1024 363, 4 379).
struct I8Order {
  bool by_cols;
  uint32_t group;
};
I8Order i8_tile_order(int64_t M, int64_t N, int64_t K, int64_t ldd, int64_t elem_bytes) {
  const bool by_cols = N >= M, pages = ldd * elem_bytes % 4096 == 0;
  const bool writes = K <= 512 || M >= ((int64_t)1 << 28) / elem_bytes / N;
  return {by_cols, by_cols ? (writes ? 16u : 8u) : pages && M / 8 < N ? 4u : 8u};
}

// The tile of rows on 16 bytes.
//   64 x 64 up to 128 tiles of 128 x 128 (1024 x 2048 x 4096 15.2 us, 128 x 128 18.6),
//     up to 160 with few steps (1500 x 1500 x 512 6.8 us, 128 x 128 7.2; x 2048 both
//     11.5).
//   256 x 256 from more than 256 tiles of 256 x 128 on (4096^3 57 us, 256 x 128 68),
//     unless their padding takes the gain.
//   128 x 128 of eight waves, two workgroups to a CU, store one tile while they
//     multiply the next.  They take the place of 256 x 256 where its last round leaves
//     many CUs idle: a round of 256 x 256 has the work of four of theirs and took the time of
//     2.6 to 3.2 above K = 1024 (five rounds for two: 4100 x 4100 x 4096 92 us, 256 x
//     256 96; six for two: 5184 x 4544 x 4096 106 and 100, x 1280 46.6 and 47.9; seven
//     for two: 5000 x 5500 x 2048 67 and 61), of 2.8 to 3.8 below (six for two: 5184 x
//     4544 x 640 30.5 and 34.6, x 1024 both 41.5; seven for two: 5000 x 5500 x 640 33.0
//     and 34.5, x 1024 42.3 and 41.9; eleven for three: 6500 x 6500 x 640 61 and 54),
//     and up to four steps of nearly all four (11 for 3 and less: 6144 x 4096 x 256 21
//     and 24, 9783 x 1984 x 256 18 and 26, 14000 x 5000 x 320 66 and 72; 41 for 11: 13000 x
//     13000 x 320 185 and 152; 4 for 1: 16384 x 16384 x 128 189 and 171, 8192 x 8192 x 512
//     65 and 62, 20000 x 4000 x 128 49 and 51), except where large tiles store slowly:
//     bf16, for its conversion (8192 x 8192 x 512 69 and 75, 32768 x 4096 x 128 97 and
//     106; but 13000 x 13000 x 320 195 and 183), and tall fp32 D in rows of whole pages
//     (32768 x 4096 x 128 117 and 148, 10240 x 8192 x 128 74 and 91; but x 512 110 and 105).
//   256 x 128 while they fill one workgroup per CU and above K = 1536 (2048 x 4096 x 4096
//     34.8 us, 128 x 128 of eight waves 36.8; at 1536 seven shapes of 160 to 470 tiles
//     were 1 to 14% slower, at 1800 7% faster to 4% slower but for 30000 x 300, 40.6
//     and 36.1).
//   128 x 128 of four waves with three stages, one workgroup to a CU, up to 256 tiles
//     above K = 1536 (2048 x 2048 x 4096 21.9 us, eight waves 24.3; at 1536 12.5 and
//     11.2, at 1800 16.7 and 16.0, 1100 x 3000 x 1800 15.6 and 16.4); more than one
//     tile to a CU goes to eight waves (1100 x 4096 x 4096 36.9 us, eight waves 28.2).
enum I8Tile { I8_64, I8_128, I8_128X8, I8_256X128, I8_256 };
I8Tile i8_tile_choice(int64_t M, int64_t N, int64_t K, int64_t ldd, mdnn_dtype_t d_type) {
  auto tiles = [&](int64_t bm, int64_t bn) { return ceil_div(M, bm) * ceil_div(N, bn); };
  auto rounds = [](int64_t n) { return ceil_div(n, (int64_t)256); };
  const int64_t t256 = tiles(256, 256), t = tiles(256, 128), t128 = tiles(128, 128);
  const bool padded = 5 * t256 > 3 * t, slow = d_type == MDNN_BF16 || (d_type == MDNN_F32 && N < M && ldd % 1024 == 0);
  const int line = K > 1024 ? 30 : K > 512 ? 33 : slow ? 99 : 37;  // tenths of a round of 128 x 128
  if (t128 <= (K <= 2048 ? 160 : 128)) return I8_64;
  if (t > 256 && !padded && 10 * rounds(t128) >= line * rounds(t256)) return I8_256;
  if (t > 160 && (t <= 256 || padded) && K > 1536) return I8_256X128;
  return t128 <= 256 && K > 1536 ? I8_128 : I8_128X8;
}

namespace {

constexpr int BKB = 128;           // bytes of k per step
constexpr int64_t I8_MAX_K = 131071;

struct I8Args {
  const int8_t *a, *b;
  const float *a_scale, *b_scale, *bias;  // bias: or null
  void* d;
  int64_t M, N, K, lda, ldb, ldd;
  int32_t act, d_type;
  uint32_t group;    // tile rows a group of workgroups walks together (tile columns with by_cols)
  bool by_cols;
  bool pairs;        // the tiled kernels' columns are ordered by pair_col
};

// ------------------------------------------------------------- epilogue

// The column that row r of a tile's B holds where D is of 16 bits: two
// neighbouring fragments' four columns of a lane are eight consecutive ones, 16
// bytes of D (8192 x 8192 x 128 fp16 40.7 us; in 8-byte stores, 16 rows by 32
// bytes each, 50.5, as long as fp32's with twice the bytes).
__device__ __forceinline__ int pair_col(int r) { return (r & ~31) | ((r & 12) << 1) | ((r & 16) >> 2) | (r & 3); }

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

template <class OutT>
__device__ __forceinline__ Quad<OutT> quad_of(const float (&v)[4]) {
  Quad<OutT> q;
  if constexpr (Quad<OutT>::H) {
    q.q[0] = (uint32_t)from_f<OutT>(v[0]) | ((uint32_t)from_f<OutT>(v[1]) << 16);
    q.q[1] = (uint32_t)from_f<OutT>(v[2]) | ((uint32_t)from_f<OutT>(v[3]) << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) q.q[e] = __float_as_uint(v[e]);
  }
  return q;
}

// One lane's four consecutive columns n .. n + 3 of row m.  The last product and
// the bias are one rounding by name, not by the compiler's choice, so that every
// kernel gives the same bits.
__device__ __forceinline__ void values_i8(const I8Args& g, int4v acc, float sa, const float (&sb)[4],
                                          const float (&bias)[4], float (&v)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float p = (float)acc[e] * sa;
    v[e] = p * sb[e];
    if (g.bias) v[e] = fmaf(p, sb[e], bias[e]);
    if (g.act == MDNN_ACT_RELU) v[e] = relu_f(v[e]);
  }
}
template <class OutT>
__device__ __forceinline__ void store_i8(const I8Args& g, int64_t m, int64_t n, const float (&v)[4]) {
  typedef typename OutT::storage S;
  S* d = (S*)g.d + m * g.ldd + n;
  if (n + 4 <= g.N) {
    quad_of<OutT>(v).store(d);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < g.N) d[e] = from_f<OutT>(v[e]);
  }
}

// A wave's FM x FN fragments; mb, nb: this lane's first row and the wave's
// first column.  PAIRS: the columns are in pair_col's order.
template <class OutT, int FM, int FN, bool PAIRS>
__device__ __forceinline__ void epilogue_i8_t(const I8Args& g, int64_t mb, int64_t nb, const int4v (&acc)[FM][FN]) {
  typedef typename OutT::storage S;
  const int q = (threadIdx.x & 63) >> 4;
  int64_t n[FN];
  float sa[FM], sb[FN][4], bias[FN][4];
#pragma unroll
  for (int i = 0; i < FM; ++i) sa[i] = g.a_scale[mb + i * 16 < g.M ? mb + i * 16 : g.M - 1];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    n[j] = nb + (PAIRS ? (j >> 1) * 32 + q * 8 + (j & 1) * 4 : j * 16 + q * 4);
    load_cols(g.b_scale, n[j], g.N, sb[j]);
    if (g.bias) load_cols(g.bias, n[j], g.N, bias[j]);
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int64_t m = mb + i * 16;
    if (m >= g.M) continue;
    if constexpr (PAIRS) {
#pragma unroll
      for (int j = 0; j < FN; j += 2) {
        float v[2][4];
        values_i8(g, acc[i][j], sa[i], sb[j], bias[j], v[0]);
        values_i8(g, acc[i][j + 1], sa[i], sb[j + 1], bias[j + 1], v[1]);
        if (n[j] + 8 <= g.N) {
          const Quad<OutT> a = quad_of<OutT>(v[0]), b = quad_of<OutT>(v[1]);
          *(__attribute__((address_space(1))) u4v_a2*)((S*)g.d + m * g.ldd + n[j]) = (u4v_a2){a.q[0], a.q[1], b.q[0], b.q[1]};
        } else {
          store_i8<OutT>(g, m, n[j], v[0]);
          store_i8<OutT>(g, m, n[j + 1], v[1]);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        if (n[j] >= g.N) continue;
        float v[4];
        values_i8(g, acc[i][j], sa[i], sb[j], bias[j], v);
        store_i8<OutT>(g, m, n[j], v);
      }
    }
  }
}

template <int FM, int FN, bool PAIRS>
__device__ __forceinline__ void epilogue_i8(const I8Args& g, int64_t mb, int64_t nb, const int4v (&acc)[FM][FN]) {
  switch (g.d_type) {
    case MDNN_F32: epilogue_i8_t<F32, FM, FN, false>(g, mb, nb, acc); break;
    case MDNN_F16: epilogue_i8_t<F16, FM, FN, PAIRS>(g, mb, nb, acc); break;
    default: epilogue_i8_t<BF16, FM, FN, PAIRS>(g, mb, nb, acc); break;
  }
}

// Tile of a workgroup: consecutive ids run on one XCD and walk groups of
// `group` tile rows column by column (by_cols: groups of tile columns row by
// row), so that the tiles at work on an XCD share its L2's panels of both
// operands.  In 32-bit arithmetic: the 64-bit divisions of tile_coords had
// taken a small product's prologue.
__device__ __forceinline__ void i8_tile(const I8Args& g, int bm, int bn, int& tm, int& tn) {
  const uint32_t tiles_m = (uint32_t)((g.M + bm - 1) / bm), tiles_n = (uint32_t)((g.N + bn - 1) / bn);
  const uint32_t major = g.by_cols ? tiles_n : tiles_m, minor = g.by_cols ? tiles_m : tiles_n;
  uint32_t id = blockIdx.x;
  if (gridDim.x % 8 == 0) id = (id % 8) * (gridDim.x / 8) + id / 8;
  const uint32_t whole = g.group * minor, gid = id / whole, in = id - gid * whole, first = gid * g.group;
  const uint32_t size = major - first < g.group ? major - first : g.group, b = in / size, a = first + in - b * size;
  tm = (int)(g.by_cols ? b : a);
  tn = (int)(g.by_cols ? a : b);
}

// ------------------------------------------------- register-staged kernel
// Rows that start on any byte, any K: chunks of 16 bytes are read at any
// address into one of NR register sets and written to the swizzled LDS tiles (two
// stages, one barrier a step).  A chunk past the row's end is read from its last
// 16 bytes and shifted; k past K is zero.  The last step's loads meet the whole
// steps' at a join past which the compiler does not count them: the first set's
// LDS writes wait for every load, the second set's too, so a round trip to memory
// is paid every NR steps and not hidden.  1000 x 777 x 1531 9.0 us (waves wait 68%
// of their cycles; matrix cores busy 6%, LDS 15%), 7 with rows on 16 bytes; 4095^3
// 109-114 us.

typedef uint32_t u4v_a1 __attribute__((ext_vector_type(4), aligned(1)));

__device__ __forceinline__ uint4 load_bytes(const int8_t* p) {
  const u4v_a1 v = *(const __attribute__((address_space(1))) u4v_a1*)p;
  return make_uint4(v.x, v.y, v.z, v.w);
}

// 16 bytes of a row from byte k, zero from K on, in two halves so that a
// thread's loads are all in flight before the first is waited for: the load,
// which stays inside the row, and the shift.  Rows of fewer than 16 bytes are
// read whole at once.
__device__ __forceinline__ uint4 load_row(const int8_t* row, int64_t k, int64_t K) {
  if (K >= 16) return load_bytes(row + (k + 16 <= K ? k : K - 16));  // (uniform)
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 15; ++e)
    if (e < K) w[e >> 2] |= (uint32_t)(uint8_t)row[e] << (8 * (e & 3));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 fix_row(uint4 v, int64_t k, int64_t K) {
  if (K >= 16) {
    const int64_t d = k + 16 - K;  // bytes past the row: how far back the chunk was read
    if (d > 0) v = reg::shift_chunk<1>(v, d < 16 ? (int)d : 0);
  }
  return k < K ? v : make_uint4(0, 0, 0, 0);
}

template <class TL, int NR>
__global__ void __launch_bounds__(TL::NT, TL::OCC) gemm_i8_any_kernel(I8Args g) {
  static_assert(NR % 2 == 0, "a set's steps have one LDS stage");
  __shared__ __attribute__((aligned(1024))) char lds_a[2][TL::A_BYTES];
  __shared__ __attribute__((aligned(1024))) char lds_b[2][TL::B_BYTES];
  constexpr int FM = TL::FM, FN = TL::FN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / TL::WN, wn = wave % TL::WN;
  int tm, tn;
  i8_tile(g, TL::BM, TL::BN, tm, tn);
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
    const int64_t n = n0 + (g.pairs ? pair_col(q.r) : q.r);
    rb[i] = g.b + (n < g.N ? n : g.N - 1) * g.ldb;
    kb[i] = q.c * 2;
  }
  struct Set {
    uint4 a[TL::LA], b[TL::LB];
  };
  auto load = [&](Set& v, int64_t k0) {
    if (k0 + BKB <= g.K) {
#pragma unroll
      for (int i = 0; i < TL::LA; ++i) v.a[i] = load_bytes(ra[i] + k0 + ka[i]);
#pragma unroll
      for (int i = 0; i < TL::LB; ++i) v.b[i] = load_bytes(rb[i] + k0 + kb[i]);
    } else {
#pragma unroll
      for (int i = 0; i < TL::LA; ++i) v.a[i] = load_row(ra[i], k0 + ka[i], g.K);
#pragma unroll
      for (int i = 0; i < TL::LB; ++i) v.b[i] = load_row(rb[i], k0 + kb[i], g.K);
#pragma unroll
      for (int i = 0; i < TL::LA; ++i) v.a[i] = fix_row(v.a[i], k0 + ka[i], g.K);
#pragma unroll
      for (int i = 0; i < TL::LB; ++i) v.b[i] = fix_row(v.b[i], k0 + kb[i], g.K);
    }
  };
  int4v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = (int4v){0, 0, 0, 0};
  const lds::LaneFrag fl = lds::lane_frag<true, TL::BM>(lane);
  const int nk = (int)ceil_div(g.K, BKB);
  Set set[NR];
#pragma unroll
  for (int u = 0; u < NR; ++u)
    if (u < nk) load(set[u], (int64_t)u * BKB);
  for (int t0 = 0; t0 < nk; t0 += NR) {
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      const int t = t0 + u;
      if (t >= nk) break;
      char *sa = lds_a[u & 1], *sb = lds_b[u & 1];
#pragma unroll
      for (int i = 0; i < TL::LA; ++i) *(uint4*)(sa + (wave * TL::LA + i) * 1024 + lane * 16) = set[u].a[i];
#pragma unroll
      for (int i = 0; i < TL::LB; ++i) *(uint4*)(sb + (wave * TL::LB + i) * 1024 + lane * 16) = set[u].b[i];
      if (t + NR < nk) load(set[u], (int64_t)(t + NR) * BKB);
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
          for (int j = 0; j < FN; ++j) acc[i][j] = Mfma<I8>::run(fb[j], fa[i], acc[i][j]);
      }
    }
  }
  epilogue_i8<FM, FN, true>(g, m0 + wm * TL::WTM + (lane & 15), n0 + wn * TL::WTN, acc);
}

// The last K % 16 bytes (K >= 16) of this lane's fragment rows mb + 16 i of A
// and of B's from nb on, as k 0 .. 15 of one more step in the first 16 lanes.
// Loaded a few steps before the end and added after it, so that nothing waits
// for them.
template <int FM, int FN>
struct LastBytes {
  uint4 a[FM], b[FN];
  __device__ __forceinline__ void load(const I8Args& g, int lane, int64_t mb, int64_t nb, bool pairs) {
#pragma unroll
    for (int j = 0; j < FN; ++j) b[j] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < FM; ++i) a[i] = make_uint4(0, 0, 0, 0);
    if (lane < 16) {  // (a request a row: the other lanes' copies would be three more)
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const int64_t n = nb + (pairs ? pair_col(j * 16 + lane) : j * 16 + lane);
        b[j] = load_bytes(g.b + (n < g.N ? n : g.N - 1) * g.ldb + g.K - 16);
      }
#pragma unroll
      for (int i = 0; i < FM; ++i) a[i] = load_bytes(g.a + (mb + i * 16 < g.M ? mb + i * 16 : g.M - 1) * g.lda + g.K - 16);
    }
  }
  __device__ __forceinline__ void add(const I8Args& g, int4v (&acc)[FM][FN]) {
    const int d = 16 - (int)(g.K & 15);
#pragma unroll
    for (int j = 0; j < FN; ++j) b[j] = reg::shift_chunk<1>(b[j], d);
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      a[i] = reg::shift_chunk<1>(a[i], d);
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = Mfma<I8>::run(b[j], a[i], acc[i][j]);
    }
  }
};

// Operands copied to rows of whole steps, zeros past K (grid y: A, B).
struct PackArgs {
  const int8_t* p[2];
  int8_t* to[2];
  int64_t ld[2];
  uint32_t chunks[2];  // rows x 16-byte chunks; 0: not copied
  int64_t K;
  uint32_t per;        // chunks a row
};
__global__ void __launch_bounds__(256) pack_rows_kernel(PackArgs a) {
  const int s = blockIdx.y;
  for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < a.chunks[s]; i += gridDim.x * 256u) {
    const uint32_t r = i / a.per;
    const int64_t k = (int64_t)(i - r * a.per) * 16;
    const uint4 v = fix_row(load_row(a.p[s] + r * a.ld[s], k < a.K ? k : 0, a.K), k, a.K);
    *(uint4*)(a.to[s] + (int64_t)i * 16) = v;
  }
}

// ------------------------------------------------- direct-to-LDS kernel
// 16-byte aligned rows (gemm_lds.h's pipeline): every lane's 16 bytes go
// straight from memory to LDS.  A K that is no multiple of the step reads
// through a range-checked buffer, whole 16-byte chunks past K as zeros; its
// last K % 16 bytes are one more fragment step from registers.  Large products
// keep the matrix cores busy in 56-72% of the cycles: 4096^3 55 us at the 2.1 GHz that
// half-zero codes leave under the power limit, 58 at the 1.7 of normal ones, so
// what fills the rest does not follow the clock (tiles on their way from beyond L2:
// waves are at waits 30% of their cycles); 16384 x 8192 x 8192 820-965 us at 1.5-1.7
// GHz, 2.3-2.7 POPS.  LDS reads take 26% of the cycles.  64 x 64 tiles wait for their
// loads: 256 x 4096 x 4096, one tile a CU, 10.1 us, 730 cycles a step against 128 of
// matrix work and as many of LDS reads; an L2 read takes 460.
struct I8Operand {
  const int8_t* p;
  int64_t ld, MN, K;
};
template <int W, int L, bool RAGGED>
struct I8Loader {
  static constexpr bool KC = true, SPLIT_ISSUE = true;
  static constexpr int P = L >= 2 ? 2 : 1;  // (a lane's k within a step depends on its load's parity)
  const char* base;
  lds::int4_t rsrc;
  int32_t left[P];
  uint32_t off[L];

  __device__ __forceinline__ void init(const I8Operand& a, int64_t mn0, int64_t kbeg, int wave, int lane,
                                       bool pairs = false) {
    base = (const char*)a.p + mn0 * a.ld + kbeg;
    const int32_t rows = a.MN - mn0 < W ? (int32_t)(a.MN - mn0) : W, ld = (int32_t)a.ld;
    if constexpr (RAGGED) {
      const int32_t bytes = (rows - 1) * ld + (int32_t)(a.K - kbeg);
      rsrc = lds::make_rsrc(base, bytes > 0 ? (uint32_t)bytes : 0u);
    }
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const lds::LoadPos q = lds::load_pos<true, W, L>(wave, lane, i);
      const int32_t c = pairs ? pair_col(q.r) : q.r, r = c < rows ? c : rows - 1;
      off[i] = (uint32_t)(r * ld + q.c * 2);
      if (i < P) left[i] = (int32_t)((a.K & ~(int64_t)15) - kbeg) - q.c * 2;
    }
  }
  // a whole step (any but a ragged last one)
  __device__ __forceinline__ void issue_one(int t, uint32_t dst, int i) {
    lds::dma_global(base + (int64_t)t * BKB, off[i], dst + (uint32_t)i * 1024u);
  }
  __device__ __forceinline__ void issue(int t, uint32_t dst) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if constexpr (RAGGED)
        lds::dma_buffer(rsrc, t * BKB < left[i % P] ? off[i] + (uint32_t)t * BKB : lds::OOB, dst + (uint32_t)i * 1024u);
      else
        issue_one(t, dst, i);
    }
  }
};
// A tile's rows reach below 2^31 bytes: offsets of every lane and load.
constexpr int64_t I8_MAX_LD = ((int64_t)1 << 31) / 256 - BKB;

template <class TL, int NS, bool RAGGED>
__global__ void __launch_bounds__(TL::NT, TL::OCC) gemm_i8_kernel(I8Args g) {
  typedef I8Loader<TL::BM, TL::LA, RAGGED> LA;
  typedef I8Loader<TL::BN, TL::LB, RAGGED> LB;
  static_assert(NS >= 2 && NS <= 4, "2 to 4 stages");
  static_assert(NS * (TL::A_BYTES + TL::B_BYTES) + 2 * (4 - NS) <= 160 * 1024, "LDS budget");
  // (a stage an object: see gemm_lds_kernel)
  __shared__ __attribute__((aligned(1024))) char lds_a0[TL::A_BYTES];
  __shared__ __attribute__((aligned(1024))) char lds_b0[TL::B_BYTES];
  __shared__ __attribute__((aligned(1024))) char lds_a1[TL::A_BYTES];
  __shared__ __attribute__((aligned(1024))) char lds_b1[TL::B_BYTES];
  __shared__ __attribute__((aligned(NS > 2 ? 1024 : 1))) char lds_a2[NS > 2 ? TL::A_BYTES : 1];
  __shared__ __attribute__((aligned(NS > 2 ? 1024 : 1))) char lds_b2[NS > 2 ? TL::B_BYTES : 1];
  __shared__ __attribute__((aligned(NS > 3 ? 1024 : 1))) char lds_a3[NS > 3 ? TL::A_BYTES : 1];
  __shared__ __attribute__((aligned(NS > 3 ? 1024 : 1))) char lds_b3[NS > 3 ? TL::B_BYTES : 1];
  char* const all_a[4] = {lds_a0, lds_a1, lds_a2, lds_a3};
  char* const all_b[4] = {lds_b0, lds_b1, lds_b2, lds_b3};
  constexpr int FM = TL::FM, FN = TL::FN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / TL::WN, wn = wave % TL::WN;
  lds::Stages<NS> st;
#pragma unroll
  for (int s = 0; s < NS; ++s) st.a[s] = all_a[s], st.b[s] = all_b[s];
  int tm, tn;
  i8_tile(g, TL::BM, TL::BN, tm, tn);
  const int64_t m0 = (int64_t)tm * TL::BM, n0 = (int64_t)tn * TL::BN;
  // steps that hold a whole 16-byte chunk
  const int nk = (int)ceil_div(g.K & ~(int64_t)15, (int64_t)BKB);

  LA la;
  LB lb;
  la.init(I8Operand{g.a, g.lda, g.M, g.K}, m0, 0, wave, lane);
  lb.init(I8Operand{g.b, g.ldb, g.N, g.K}, n0, 0, wave, lane, g.pairs);
  const uint32_t wa = (uint32_t)(wave * TL::LA) * 1024u, wb = (uint32_t)(wave * TL::LB) * 1024u;
  int4v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = (int4v){0, 0, 0, 0};
  // (256 x 256 tiles have no registers to keep them in over the loop)
  constexpr bool HOLD = FM + FN <= 8;
  const int64_t mb = m0 + wm * TL::WTM + (lane & 15), nw = n0 + wn * TL::WTN;
  const bool last = RAGGED && (g.K & 15) != 0;
  LastBytes<HOLD ? FM : 1, HOLD ? FN : 1> held;
  lds::Frags<TL> f0, f1;
  const lds::LaneFrag fa_l = lds::lane_frag<true, TL::BM>(lane), fb_l = lds::lane_frag<true, TL::BN>(lane);
  if (nk > 0) {
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (s < nk) {
        la.issue(s, lds::lds_address(st.a[s]) + wa);
        lb.issue(s, lds::lds_address(st.b[s]) + wb);
      }
  }
  if constexpr (RAGGED && !HOLD) {
    if (last) {
      LastBytes<FM, FN> v;
      v.load(g, lane, mb, nw, g.pairs);
      v.add(g, acc);
    }
  }
  if (nk > 0) {
    lds::wait_tiles<NS - 1, TL::LA + TL::LB>((nk < NS ? nk : NS) - 1);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FM; ++i) f0.a[i] = lds::fragment<true, TL::BM>(st.a[0], wm * TL::WTM + i * 16, 0, fa_l);
#pragma unroll
    for (int j = 0; j < FN; ++j) f0.b[j] = lds::fragment<true, TL::BN>(st.b[0], wn * TL::WTN + j * 16, 0, fb_l);
  }
  constexpr int U = NS % 2 == 0 ? NS : 2 * NS;
  int t = 0;
  for (; t + U - 1 + NS < nk - (RAGGED ? 1 : 0); t += U)  // (the last step is issued with its test)
    lds::pipeline_round<I8, TL, NS, LA, LB, 0, U, false>(t, nk, st, wave, fa_l, fb_l, wm, wn, la, lb, f0, f1, acc);
  if constexpr (RAGGED && HOLD)
    if (last) held.load(g, lane, mb, nw, g.pairs);
  for (; t < nk; t += U)
    lds::pipeline_round<I8, TL, NS, LA, LB, 0, U, true>(t, nk, st, wave, fa_l, fb_l, wm, wn, la, lb, f0, f1, acc);

  if constexpr (RAGGED && HOLD)
    if (last) held.add(g, acc);
  epilogue_i8<FM, FN, true>(g, mb, nw, acc);
}

// ------------------------------------------------------- few rows kernels
// At most 64 rows (one to a few samples): the time is B's read.  A block owns
// FN * 16 columns and its W waves share K; every wave has LDS of its own, so
// nothing waits for a barrier before the sums are added.  Eight lanes read 128
// bytes of one row: fragments read from memory directly would touch four rows
// in every four lanes, which the cache answers a line at a time (64 x 4096 x
// 4096: 12.1 us, 6.6 through LDS).

// The waves' sums, added in LDS, a fragment of the result a wave.
template <int FM, int FN, int W>
__device__ __forceinline__ void join_few(const I8Args& g, char* mem, int wave, int lane, int64_t m0, int64_t n0,
                                         const int4v (&acc)[FM][FN]) {
  __syncthreads();  // every wave is done with its stages
  int4v* part = (int4v*)mem;  // [W][FM * FN][64]
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) part[(wave * FM * FN + i * FN + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (int f = wave; f < FM * FN; f += W) {
    int4v sum[1][1] = {{part[f * 64 + lane]}};
#pragma unroll
    for (int w = 1; w < W; ++w) sum[0][0] += part[(w * FM * FN + f) * 64 + lane];
    epilogue_i8<1, 1, false>(g, m0 + f / FN * 16 + (lane & 15), n0 + f % FN * 16, sum);
  }
}

// Rows that start on any byte, any K: through two register sets.
template <int FM, int FN, int W>
__global__ void __launch_bounds__(W * 64) gemm_i8_few_any_kernel(I8Args g) {
  constexpr int A_BYTES = FM * 2048, STAGE = A_BYTES + FN * 2048;
  constexpr int ALL = W * STAGE, SUMS = W * FM * FN * 1024;
  __shared__ __attribute__((aligned(1024))) char mem[ALL > SUMS ? ALL : SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * (FN * 16), m0 = (int64_t)blockIdx.y * (FM * 16);
  const int steps = (int)ceil_div(g.K, (int64_t)BKB), per = (int)ceil_div(steps, W);
  const int s0 = wave * per, s1 = s0 + per < steps ? s0 + per : steps;
  const int8_t *ra[2 * FM], *rb[2 * FN];
  int kc[2];  // (a lane's k within a step depends on its load's parity)
#pragma unroll
  for (int i = 0; i < 2 * FM; ++i) {
    const lds::LoadPos q = lds::load_pos<true, FM * 16, 2 * FM>(0, lane, i);
    ra[i] = g.a + (m0 + q.r < g.M ? m0 + q.r : g.M - 1) * g.lda;
    if (i < 2) kc[i] = q.c * 2;
  }
#pragma unroll
  for (int i = 0; i < 2 * FN; ++i) {
    const lds::LoadPos q = lds::load_pos<true, FN * 16, 2 * FN>(0, lane, i);
    rb[i] = g.b + (n0 + q.r < g.N ? n0 + q.r : g.N - 1) * g.ldb;
  }
  struct Set {
    uint4 a[2 * FM], b[2 * FN];
  };
  auto load = [&](Set& v, int s) {
    const int64_t k0 = (int64_t)s * BKB;
    if (k0 + BKB <= g.K) {
#pragma unroll
      for (int i = 0; i < 2 * FN; ++i) v.b[i] = load_bytes(rb[i] + k0 + kc[i & 1]);
#pragma unroll
      for (int i = 0; i < 2 * FM; ++i) v.a[i] = load_bytes(ra[i] + k0 + kc[i & 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 2 * FN; ++i) v.b[i] = load_row(rb[i], k0 + kc[i & 1], g.K);
#pragma unroll
      for (int i = 0; i < 2 * FM; ++i) v.a[i] = load_row(ra[i], k0 + kc[i & 1], g.K);
#pragma unroll
      for (int i = 0; i < 2 * FN; ++i) v.b[i] = fix_row(v.b[i], k0 + kc[i & 1], g.K);
#pragma unroll
      for (int i = 0; i < 2 * FM; ++i) v.a[i] = fix_row(v.a[i], k0 + kc[i & 1], g.K);
    }
  };
  int4v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = (int4v){0, 0, 0, 0};
  const lds::LaneFrag fl = lds::lane_frag<true, 64>(lane);
  char* const own = mem + wave * STAGE;
  Set set[2];
  if (s0 < s1) load(set[0], s0);
  if (s0 + 1 < s1) load(set[1], s0 + 1);
  for (int t = s0; t < s1; t += 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (t + u >= s1) break;
      // (one wave's LDS accesses run in order: its writes, then its reads)
#pragma unroll
      for (int i = 0; i < 2 * FM; ++i) *(uint4*)(own + i * 1024 + lane * 16) = set[u].a[i];
#pragma unroll
      for (int i = 0; i < 2 * FN; ++i) *(uint4*)(own + A_BYTES + i * 1024 + lane * 16) = set[u].b[i];
      if (t + u + 2 < s1) load(set[u], t + u + 2);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        uint4 fa[FM], fb[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[j] = lds::fragment<true, FN * 16>(own + A_BYTES, j * 16, kk, fl);
#pragma unroll
        for (int i = 0; i < FM; ++i) fa[i] = lds::fragment<true, FM * 16>(own, i * 16, kk, fl);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j) acc[i][j] = Mfma<I8>::run(fb[j], fa[i], acc[i][j]);
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
  join_few<FM, FN, W>(g, mem, wave, lane, m0, n0, acc);
}

// 16-byte aligned rows: straight to LDS, NS steps of 128 k in flight.
template <int FM, int FN, int W, int NS>
__global__ void __launch_bounds__(W * 64) gemm_i8_few_lds_kernel(I8Args g) {
  constexpr int A_BYTES = FM * 2048, B_BYTES = FN * 2048, STAGE = A_BYTES + B_BYTES, LPT = 2 * (FM + FN);
  constexpr int ALL = W * NS * STAGE, SUMS = W * FM * FN * 1024;
  static_assert(ALL <= 160 * 1024 && SUMS <= 160 * 1024, "LDS budget");
  __shared__ __attribute__((aligned(1024))) char mem[ALL > SUMS ? ALL : SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * (FN * 16), m0 = (int64_t)blockIdx.y * (FM * 16);
  const int steps = (int)ceil_div(g.K & ~(int64_t)15, (int64_t)BKB), per = (int)ceil_div(steps, W);
  const int s0 = wave * per < steps ? wave * per : steps, nk = (s0 + per < steps ? s0 + per : steps) - s0;
  const int64_t kbeg = (int64_t)s0 * BKB;
  I8Loader<FM * 16, 2 * FM, true> la;
  I8Loader<FN * 16, 2 * FN, true> lb;
  la.init(I8Operand{g.a, g.lda, g.M, g.K}, m0, kbeg, 0, lane);
  lb.init(I8Operand{g.b, g.ldb, g.N, g.K}, n0, kbeg, 0, lane);
  const bool last = wave == W - 1 && (g.K & 15) != 0;
  LastBytes<FM, FN> held;
  if (last) held.load(g, lane, m0 + (lane & 15), n0, false);
  char* const own = mem + wave * (NS * STAGE);
  const uint32_t at = lds::lds_address(own);
#pragma unroll
  for (int s = 0; s < NS; ++s)
    if (s < nk) {
      lb.issue(s, at + s * STAGE + A_BYTES);
      la.issue(s, at + s * STAGE);
    }
  int4v acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = (int4v){0, 0, 0, 0};
  const lds::LaneFrag fl = lds::lane_frag<true, 64>(lane);
  for (int t = 0; t < nk; ++t) {
    lds::wait_tiles<NS - 1, LPT>(nk - 1 - t < NS - 1 ? nk - 1 - t : NS - 1);  // this wave's step t has landed
    asm volatile("" ::: "memory");
    const char* sa = own + (t % NS) * STAGE;
    uint4 fa[2][FM], fb[2][FN];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[kk][j] = lds::fragment<true, FN * 16>(sa + A_BYTES, j * 16, kk, fl);
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[kk][i] = lds::fragment<true, FM * 16>(sa, i * 16, kk, fl);
    }
    if (t + NS < nk) {
      // the fragments are in registers before their stage is filled again
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      lb.issue(t + NS, at + (t % NS) * STAGE + A_BYTES);
      la.issue(t + NS, at + (t % NS) * STAGE);
    }
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = Mfma<I8>::run(fb[kk][j], fa[kk][i], acc[i][j]);
  }
  if (last) held.add(g, acc);
  join_few<FM, FN, W>(g, mem, wave, lane, m0, n0, acc);
}

typedef lds::Tile<64, 64, 2, 2, 2> TileI64;
// rows on any byte: eight waves, half as many loads and their addresses a wave
// (1000 x 777 x 1531 9.0 us, four waves 9.8; 500 x 2000 x 1001 7.4 and 8.2)
typedef lds::Tile<64, 64, 4, 2, 4> TileI64x8;
// 128 x 128 with eight waves of 64 x 32 and two stages (64 KB): two workgroups
// per CU
typedef lds::Tile<128, 128, 2, 4, 4> TileI128x8;
// 128 x 128 with three stages (96 KB), 256 x 128 with eight waves of 64 x 64
// and three stages (144 KB): one workgroup per CU each
typedef lds::Tile<128, 128, 2, 2, 1> TileI128;
typedef lds::Tile<256, 128, 4, 2, 2> TileI256x128;

// 16-byte aligned rows, which the direct-to-LDS kernels take (K >= 16).
bool rows_aligned(const int8_t* p, int64_t ld) { return aligned(p, 16) && ld % 16 == 0 && ld <= I8_MAX_LD; }

// Unaligned operands of products of more than 256 tiles of 256 x 128 are
// worth a copy to aligned rows: 4095^3 109 us as they are, 81 with the copy;
// 4095 x 4095 x 513 39 and 35; 16383 x 4001 x 1001 161 and 117.
int64_t packed_ld(int64_t K) { return ceil_div(K, BKB) * BKB; }
bool pack_pays(int64_t M, int64_t N, int64_t K) {
  if (K % 16 == 0 || K < 16 || M <= 64 || N <= 32) return false;  // (few rows or columns: see run_i8)
  const int64_t tm = ceil_div(M, 256), tn = ceil_div(N, 128);
  // (a copy's chunks, and the stride over them, are counted in 32 bits)
  const int64_t rows = ((int64_t)1 << 31) / (packed_ld(K) / 16);
  return tm > 256 / tn && M <= rows && N <= rows;
}

template <class TL, int NS>
void launch_i8(const I8Args& g, hipStream_t st) {
  const dim3 grid((unsigned)(ceil_div(g.M, TL::BM) * ceil_div(g.N, TL::BN)));
  if (g.K % BKB != 0)
    hipLaunchKernelGGL((gemm_i8_kernel<TL, NS, true>), grid, dim3(TL::NT), 0, st, g);
  else
    hipLaunchKernelGGL((gemm_i8_kernel<TL, NS, false>), grid, dim3(TL::NT), 0, st, g);
}

template <class TL, int NR>
void launch_any(const I8Args& g, hipStream_t st) {
  const int64_t tiles = ceil_div(g.M, TL::BM) * ceil_div(g.N, TL::BN);
  hipLaunchKernelGGL((gemm_i8_any_kernel<TL, NR>), dim3((unsigned)tiles), dim3(TL::NT), 0, st, g);
}

// W, NS: waves and stages for rows on 16 bytes; WANY: waves for others.
template <int FM, int FN, int W, int NS, int WANY = W>
mdnn_status_t launch_few(const I8Args& g, bool rows16, hipStream_t st) {
  const dim3 grid((unsigned)ceil_div(g.N, FN * 16), (unsigned)ceil_div(g.M, FM * 16));
  if (rows16)
    hipLaunchKernelGGL((gemm_i8_few_lds_kernel<FM, FN, W, NS>), grid, dim3(W * 64), 0, st, g);
  else
    hipLaunchKernelGGL((gemm_i8_few_any_kernel<FM, FN, WANY>), grid, dim3(WANY * 64), 0, st, g);
  return check_launch("gemm_i8_few_kernel");
}

// Few rows: FM fragments of rows; FN columns of 16 as the caller chose.  FM is
// the least that needs no more than one block per CU (64 x 1024 x 4096 with 1
// 4.2 us, 4 5.7; 64 x 2048 x 8192 with 2 7.2, 4 9.4; 40 x 201 x 7085 on any
// byte 8.6 and 14.5), and otherwise what holds the rows, which reads B once (40
// x 4096 x 1024 with 3 3.8 us, 1 4.6).  Up to 16 rows four waves of four stages
// read weights from memory fastest (1 x 4096 x 4096 5.7 us cold, 1 x 8192 x 8192
// 14.2; eight of two 6.1 and 15.6, where the weights are in the cache 4.3 and
// 4.2).
template <int FN>
mdnn_status_t run_few(const I8Args& g, bool rows16, hipStream_t st) {
  auto enough = [&](int fm) {
    return g.M <= fm * 16 || ceil_div(g.M, (int64_t)fm * 16) * ceil_div(g.N, (int64_t)FN * 16) <= 256;
  };
  if (enough(1)) return launch_few<1, FN, 4, 4, 8>(g, rows16, st);
  if (enough(2)) return launch_few<2, FN, 4, 3>(g, rows16, st);
  if (g.M <= 48) return launch_few<3, FN, 4, FN == 1 ? 3 : 2>(g, rows16, st);
  return launch_few<4, FN, 4, FN == 1 ? 3 : 2>(g, rows16, st);
}

mdnn_status_t run_i8(I8Args g, void* ws, size_t ws_bytes, hipStream_t st) {
  bool a16 = rows_aligned(g.a, g.lda), b16 = rows_aligned(g.b, g.ldb);
  if ((!a16 || !b16) && ws && pack_pays(g.M, g.N, g.K) && ws_bytes >= mdnn_gemm_i8_workspace(g.M, g.N, g.K)) {
    const int64_t ld = packed_ld(g.K);
    PackArgs p = {};
    p.K = g.K, p.per = (uint32_t)(ld / 16);
    p.p[0] = g.a, p.ld[0] = g.lda, p.to[0] = (int8_t*)ws, p.chunks[0] = a16 ? 0 : (uint32_t)g.M * p.per;
    p.p[1] = g.b, p.ld[1] = g.ldb, p.to[1] = (int8_t*)ws + g.M * ld, p.chunks[1] = b16 ? 0 : (uint32_t)g.N * p.per;
    const uint32_t most = p.chunks[0] > p.chunks[1] ? p.chunks[0] : p.chunks[1];
    const uint32_t blocks = most / 256 + 1;
    hipLaunchKernelGGL(pack_rows_kernel, dim3(blocks < 65536 ? blocks : 65536, 2), dim3(256), 0, st, p);
    MDNN_TRY(check_launch("pack_rows_kernel"));
    if (!a16 && !b16) g.K = ld;  // (zeros past K in both)
    if (!a16) g.a = p.to[0], g.lda = ld;
    if (!b16) g.b = p.to[1], g.ldb = ld;
    a16 = b16 = true;
  }
  const bool rows16 = a16 && b16 && g.K >= 16;
  auto tiles = [&](int64_t bm, int64_t bn) { return ceil_div(g.M, bm) * ceil_div(g.N, bn); };
  // (K == 0 and other K < 16: the kernels for rows on any byte.)
  // Up to one workgroup per CU, the few-rows kernel's waves that share K beat
  // a 64 x 64 tile's serial loop over it: 64 x 16 tiles (64 x 4096 x 4096 6.6
  // us, 64 x 32 tiles 7.7, 64 x 64 tiles 9.5), then 64 x 32 (128 x 4096 x
  // 4096: 11.6, 7.3 and 9.6 us); from two workgroups per CU on it is behind
  // (192 x 4096 x 4096: 16.9, 14.4, 9.9 us).  Rows of at most 64 and columns
  // of at most 32 stay on it, their tiles being mostly padding elsewhere
  // (64 x 8192 x 8192 14.8 us, 64 x 64 tiles 16.3; 16384 x 32 x 4096 13.4,
  // 18.6).  64 x 16 tiles read A once per 16 columns: not where A is the
  // larger operand (4096 x 64 x 4096: 12.2 us, 64 x 32 tiles 8.0).
  // (Their grid: fewer than 2^32 threads by column tiles, row tiles in y.)
  const bool fits = g.N < (int64_t)1 << 26 && g.M <= (int64_t)65535 * 64;
  if (fits && (g.M <= 16 || g.N <= 16 || (tiles(g.M <= 32 ? 32 : 64, 16) <= 256 && g.M <= g.N)))
    return run_few<1>(g, rows16, st);
  if (fits && (g.M <= 64 || g.N <= 32 || tiles(64, 32) <= 256)) return run_few<2>(g, rows16, st);
  if (!rows16) {
    // 256 x 128 tiles from more than 256 of them on (4095^3 108 us, 128 x 128
    // tiles 120, 64 x 64 206) unless steps are few (9783 x 1984 x 129 30.2 us, 128
    // x 128 23.7; 4095 x 4095 x 513 40 and 39), 128 x 128 from more than 128 (2000
    // x 2000 x 3001 28 us, 256 x 128 41, 64 x 64 43; 1000 x 2000 x 3001 27, 64 x
    // 64 25)
    if (tiles(256, 128) > 256 && g.K > 512)
      launch_any<lds::Tile<256, 128, 4, 2, 2>, 2>(g, st);
    else if (tiles(128, 128) > 128)
      launch_any<TileI128x8, 2>(g, st);
    else
      launch_any<TileI64x8, 2>(g, st);
    return check_launch("gemm_i8_any_kernel");
  }
  switch (i8_tile_choice(g.M, g.N, g.K, g.ldd, (mdnn_dtype_t)g.d_type)) {
    case I8_64: launch_i8<TileI64, 3>(g, st); break;
    case I8_128: launch_i8<TileI128, 3>(g, st); break;
    case I8_128X8: launch_i8<TileI128x8, 2>(g, st); break;
    case I8_256X128: launch_i8<TileI256x128, 3>(g, st); break;
    case I8_256: launch_i8<lds::Tile256, 2>(g, st); break;
  }
  return check_launch("gemm_i8_kernel");
}

}  // namespace
}  // namespace mdnn

using namespace mdnn;

extern "C" size_t mdnn_gemm_i8_workspace(int64_t M, int64_t N, int64_t K) {
  if (M < 0 || N < 0 || K < 0 || K > I8_MAX_K || M == 0 || N == 0 || !pack_pays(M, N, K)) return 0;
  return (size_t)(M + N) * (size_t)packed_ld(K);
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
  // (a launch holds fewer than 2^32 threads: 64 x 64 tiles of 256, and half as many tiles of 512 where a side is one tile)
  if (M > INT64_MAX - 64 || N > INT64_MAX - 64 || ceil_div(M, 64) > (((int64_t)1 << 24) - 2) / ceil_div(N, 64))
    return fail(MDNN_ERR_SHAPE, "gemm_i8: problem too large for the launch grid");
  I8Args g = {};
  g.a = A, g.b = B, g.a_scale = a_scale, g.b_scale = b_scale, g.bias = bias, g.d = D;
  g.M = M, g.N = N, g.K = K, g.lda = lda, g.ldb = ldb, g.ldd = ldd, g.act = act;
  g.d_type = d_type, g.pairs = d_type != MDNN_F32;
  const I8Order order = i8_tile_order(M, N, K, ldd, (int64_t)dtype_size(d_type));
  g.by_cols = order.by_cols, g.group = order.group;
  clear_error();
  return run_i8(g, workspace, ws_bytes, as_stream(stream));
}

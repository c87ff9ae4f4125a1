// dW of up to 1024 rows of 16-bit operands: D[r][c] = a * sum over m of P[m][r] Q[m][c],
// P and Q rows on 16 bytes in the workspace (x's copy and G).
//
// Bound: D's writes.  The product is few 64-deep steps; the GEMM's tiles store it as
// the matrix instruction leaves it, 16 rows by 8 bytes of every lane, at 3.3
// TB/s on 16-byte rows and 1.1 on others (6912 x 27552 fp16 117-133 us, x 27551 358).
// Here a tile turns in LDS and leaves in whole rows, 16 bytes a lane, at any
// element address: a call's time, 64 x 32768 x 4096 bf16 by feature 475 -> 240 us, by
// class fp16 257 -> 212, 32 x 27551 x 6912 fp16 397 -> 300, 256 x 32768 x 4096 bf16 443 ->
// 381, 1000 x 5003 x 1000 fp16 67.5 -> 64.5.
#include "gemm_lds.h"
#include "internal.h"
#include "row_chunk.h"
#include "xent.h"

namespace mdnn {
namespace {

// Up to four steps 64 rows of 256, one step in LDS and three workgroups a CU beside each
// other (64 x 32768 x 4096 bf16 233 us, two steps 251; tiles of 128 x 128 251).  Then
// 128 x 128, which read less for a tile (1000 x 60001 x 577 bf16 383 us, 64 x 256 443),
// and where they are three a CU at most with two steps in LDS (1000 x 5003 x 1000
// fp16 65.0 us, one 68.8; 1000 x 32768 x 4096 bf16 868 and 828).
typedef lds::Tile<64, 256, 1, 4, 3> TileWide;
typedef lds::Tile<128, 128, 2, 2, 3> TileSquare;
typedef lds::Tile<128, 128, 2, 2, 2> TileSquare2;

// NS: steps in LDS
template <class T, class OutT, class TL, int NS>
__global__ void __launch_bounds__(TL::NT, TL::OCC)
xent_outer_kernel(lds::MatArgs pa, lds::MatArgs qa, int64_t R, int64_t C, int steps, const float* alpha, void* d,
                  int64_t ldd) {
  typedef lds::MatLoader<false, TL::BM, TL::LA> LA;
  typedef lds::MatLoader<false, TL::BN, TL::LB> LB;
  typedef typename OutT::storage DS;
  constexpr int ES = (int)sizeof(DS), E = 16 / ES;        // elements of a 16-byte store
  constexpr int ROWS = ES == 2 ? 64 : 32;                 // rows in LDS at a time
  constexpr int STRIDE = TL::BN * ES + 16;                // bytes (rows 4 banks on: the fragments' 16 rows differ)
  constexpr int STEP = TL::A_BYTES + TL::B_BYTES, ROOM = NS * STEP;
  static_assert(ROWS * STRIDE <= ROOM && TL::WTM % ROWS == 0, "room for the rows");
  __shared__ __attribute__((aligned(1024))) char room[ROOM];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / TL::WN, wn = wave % TL::WN;
  int tm, tn;
  tile_coords(ceil_div(R, TL::BM), ceil_div(C, TL::BN), tm, tn);
  const int64_t r0 = (int64_t)tm * TL::BM, c0 = (int64_t)tn * TL::BN;
  LA la;
  LB lb;
  la.init(pa, r0, 0, wave, lane);
  lb.init(qa, c0, 0, wave, lane);
  const float a = *alpha;
  const lds::LaneFrag fa = lds::lane_frag<false, TL::BM>(lane), fb = lds::lane_frag<false, TL::BN>(lane);
  float4_t acc[TL::FM][TL::FN];
#pragma unroll
  for (int i = 0; i < TL::FM; ++i)
#pragma unroll
    for (int j = 0; j < TL::FN; ++j) acc[i][j] = (float4_t){0.f, 0.f, 0.f, 0.f};
  auto issue = [&](int s) {
    const uint32_t to = lds::lds_address(room) + (uint32_t)(s % NS * STEP);
    la.issue(s, to + (uint32_t)(wave * TL::LA) * 1024u);
    lb.issue(s, to + (uint32_t)TL::A_BYTES + (uint32_t)(wave * TL::LB) * 1024u);
  };
  if (NS > 1) issue(0);
  for (int s = 0; s < steps; ++s) {
    if (NS == 1) {
      if (s > 0) __syncthreads();  // (the last step's reads are done)
      issue(s);
    }
    lds::wait_vm_lgkm0<0>();
    __syncthreads();
    if (NS > 1 && s + 1 < steps) issue(s + 1);
    const char *sa = room + s % NS * STEP, *sb = sa + TL::A_BYTES;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      uint4 fragA[TL::FM], fragB[TL::FN];
#pragma unroll
      for (int i = 0; i < TL::FM; ++i) fragA[i] = lds::fragment<false, TL::BM>(sa, wm * TL::WTM + i * 16, kk, fa);
#pragma unroll
      for (int j = 0; j < TL::FN; ++j) fragB[j] = lds::fragment<false, TL::BN>(sb, wn * TL::WTN + j * 16, kk, fb);
#pragma unroll
      for (int i = 0; i < TL::FM; ++i)
#pragma unroll
        for (int j = 0; j < TL::FN; ++j) acc[i][j] = Mfma<T>::run(fragB[j], fragA[i], acc[i][j]);
    }
  }
  constexpr int PER = TL::BN / E;  // threads of a row
#pragma unroll
  for (int h = 0; h < TL::BM / ROWS; ++h) {
    __syncthreads();  // (the fragments', or the rows' before, last reads are done)
#pragma unroll
    for (int i = 0; i < ROWS / 16; ++i)
#pragma unroll
      for (int j = 0; j < TL::FN; ++j) {
        if (h * ROWS / TL::WTM != wm) continue;  // (another wave's rows)
        const float4_t v = acc[h * ROWS % TL::WTM / 16 + i][j] * a;
        char* p = room + (i * 16 + (lane & 15)) * STRIDE + (wn * TL::WTN + j * 16 + 4 * (lane >> 4)) * ES;
        if constexpr (ES == 2)
          *(uint2*)p = make_uint2((uint32_t)from_f<OutT>(v[0]) | ((uint32_t)from_f<OutT>(v[1]) << 16),
                                  (uint32_t)from_f<OutT>(v[2]) | ((uint32_t)from_f<OutT>(v[3]) << 16));
        else
          *(float4_t*)p = v;
      }
    __syncthreads();
    const int64_t c = c0 + (tid % PER) * E;
    if (c < C) {
#pragma unroll
      for (int k = 0; k < ROWS * PER / TL::NT; ++k) {
        const int r = tid / PER + k * (TL::NT / PER);
        const int64_t row = r0 + h * ROWS + r;
        if (row >= R) break;
        const uint4 v = *(const uint4*)(room + r * STRIDE + (tid % PER) * 16);
        DS* o = (DS*)d + row * ldd + c;
        if (c + E <= C) {
          typedef std::conditional_t<ES == 2, u4v_a2, u4v_a4> V;
          *(MDNN_GLOBAL V*)o = (V){v.x, v.y, v.z, v.w};
        } else {
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (c + e < C) {
              if constexpr (ES == 2)
                o[e] = (uint16_t)(w[e >> 1] >> ((e & 1) * 16));
              else
                o[e] = __builtin_bit_cast(float, w[e]);
            }
        }
      }
    }
  }
}

template <class T, class OutT, class TL, int NS>
void launch_tile(const lds::MatArgs& a, const lds::MatArgs& b, int64_t R, int64_t C, int steps, const float* alpha, void* d,
                 int64_t ldd, hipStream_t st) {
  hipLaunchKernelGGL((xent_outer_kernel<T, OutT, TL, NS>), dim3((unsigned)(ceil_div(R, TL::BM) * ceil_div(C, TL::BN))),
                     dim3(TL::NT), 0, st, a, b, R, C, steps, alpha, d, ldd);
}

template <class T, class OutT>
void launch_outer(const lds::MatArgs& a, const lds::MatArgs& b, int64_t R, int64_t C, int steps, const float* alpha, void* d,
                  int64_t ldd, hipStream_t st) {
  if (steps <= 4)
    launch_tile<T, OutT, TileWide, 1>(a, b, R, C, steps, alpha, d, ldd, st);
  else if (ceil_div(R, 128) * ceil_div(C, 128) < 768)
    launch_tile<T, OutT, TileSquare2, 2>(a, b, R, C, steps, alpha, d, ldd, st);
  else
    launch_tile<T, OutT, TileSquare, 1>(a, b, R, C, steps, alpha, d, ldd, st);
}

}  // namespace

// Up to 1024 rows (1000 x 60001 x 577 bf16 383 us against the GEMM's 387, 2000 697 and 664;
// 4000 x 32768 x 4096 2697 and 2622), more tiles than 64 (64 x 1000 x 777 bf16, 64 either
// way round: 30.0 against 29.4; 9 x 5003 x 1000 fp16, 320: 32.5 against 36.0), and the
// loaders' 32-bit offsets reach a step's 64 rows.
bool xent_outer_ok(int64_t R, int64_t C, int64_t rows) {
  const int64_t tiles = ceil_div(R, TileWide::BM) * ceil_div(C, TileWide::BN);
  return rows <= 1024 && R < (int64_t)1 << 24 && C < (int64_t)1 << 24 && tiles > 64 && tiles < (int64_t)1 << 24;
}

template <class T>
mdnn_status_t xent_outer(const void* p, int64_t ldp, int64_t R, const void* q, int64_t ldq, int64_t C, int64_t rows,
                         const float* alpha, void* d, int64_t ldd, mdnn_dtype_t d_type, hipStream_t st) {
  const int steps = (int)(rows / 64);
  const lds::MatArgs a{p, ldp, ceil_div(R, 8) * 8}, b{q, ldq, ceil_div(C, 8) * 8};
  if (d_type == MDNN_F32)
    launch_outer<T, F32>(a, b, R, C, steps, alpha, d, ldd, st);
  else
    launch_outer<T, T>(a, b, R, C, steps, alpha, d, ldd, st);
  return check_launch("xent_outer_kernel");
}
template mdnn_status_t xent_outer<F16>(const void*, int64_t, int64_t, const void*, int64_t, int64_t, int64_t, const float*,
                                       void*, int64_t, mdnn_dtype_t, hipStream_t);
template mdnn_status_t xent_outer<BF16>(const void*, int64_t, int64_t, const void*, int64_t, int64_t, int64_t, const float*,
                                        void*, int64_t, mdnn_dtype_t, hipStream_t);

}  // namespace mdnn

// dW of up to 512 rows of 16-bit operands: D[r][c] = a * sum over m of P[m][r] Q[m][c],
// P and Q rows on 16 bytes in the workspace (x's copy and G).
//
// Bound: D's writes.  The product is few 64-deep steps; the GEMM's tiles store it as
// the matrix instruction leaves it, 16 rows by 8 bytes of every lane, at 3.3
// TB/s on 16-byte rows and 1.1 on others (6912 x 27552 fp16 117-133 us, x 27551 358).
// Here a tile turns in LDS and leaves in whole rows, 16 bytes a lane, at any
// element address: a call's time, 64 x 32768 x 4096 bf16 by feature 475 -> 240 us, by
// class fp16 257 -> 212, 32 x 27551 x 6912 fp16 397 -> 300, 16 x 32768 x 1024 bf16 74 -> 56.
// A step's loads are waited for at once: three workgroups a CU run beside each
// other (256 x 32768 x 4096 bf16 443 -> 382 us, 512 x 20000 x 2048 245 -> 222).
#include "gemm_lds.h"
#include "internal.h"
#include "row_chunk.h"
#include "xent.h"

namespace mdnn {
namespace {

typedef lds::Tile<64, 256, 1, 4, 3> TileOuter;

template <class T, class OutT>
__global__ void __launch_bounds__(TileOuter::NT, TileOuter::OCC)
xent_outer_kernel(lds::MatArgs pa, lds::MatArgs qa, int64_t R, int64_t C, int steps, const float* alpha, void* d,
                  int64_t ldd) {
  typedef TileOuter TL;
  typedef lds::MatLoader<false, TL::BM, TL::LA> LA;
  typedef lds::MatLoader<false, TL::BN, TL::LB> LB;
  typedef typename OutT::storage DS;
  constexpr int ES = (int)sizeof(DS), E = 16 / ES;        // elements of a 16-byte store
  constexpr int ROWS = ES == 2 ? 64 : 32;                 // rows in LDS at a time
  constexpr int STRIDE = TL::BN * ES + 16;                // bytes (rows 4 banks on: the fragments' 16 rows differ)
  constexpr int ROOM = TL::A_BYTES + TL::B_BYTES;
  static_assert(ROWS * STRIDE <= ROOM, "room for the rows");
  __shared__ __attribute__((aligned(1024))) char room[ROOM];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int tm, tn;
  tile_coords(ceil_div(R, TL::BM), ceil_div(C, TL::BN), tm, tn);
  const int64_t r0 = (int64_t)tm * TL::BM, c0 = (int64_t)tn * TL::BN;
  char *const sa = room, *const sb = room + TL::A_BYTES;
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
  for (int s = 0; s < steps; ++s) {
    if (s > 0) __syncthreads();  // (the last step's reads are done)
    la.issue(s, lds::lds_address(sa) + (uint32_t)(wave * TL::LA) * 1024u);
    lb.issue(s, lds::lds_address(sb) + (uint32_t)(wave * TL::LB) * 1024u);
    lds::wait_vm_lgkm0<0>();
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      uint4 fragA[TL::FM], fragB[TL::FN];
#pragma unroll
      for (int i = 0; i < TL::FM; ++i) fragA[i] = lds::fragment<false, TL::BM>(sa, i * 16, kk, fa);
#pragma unroll
      for (int j = 0; j < TL::FN; ++j) fragB[j] = lds::fragment<false, TL::BN>(sb, wave * TL::WTN + j * 16, kk, fb);
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
        const float4_t v = acc[h * (ROWS / 16) + i][j] * a;
        char* p = room + (i * 16 + (lane & 15)) * STRIDE + (wave * TL::WTN + j * 16 + 4 * (lane >> 4)) * ES;
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

}  // namespace

// Up to 512 rows (512 x 60001 x 577 bf16 256 us against the GEMM's 245, 384 237 and 237,
// 1000 443 and 384; 1000 x 32768 x 4096 831 and 847), more tiles than 64 (64 x 1000 x 777
// bf16, 64 either way round: 30.0 against 29.4; 9 x 5003 x 1000 fp16, 320: 32.5 against
// 36.0), and the loaders' 32-bit offsets reach a step's 64 rows.
bool xent_outer_ok(int64_t R, int64_t C, int64_t rows) {
  const int64_t tiles = ceil_div(R, TileOuter::BM) * ceil_div(C, TileOuter::BN);
  return rows <= 512 && R < (int64_t)1 << 24 && C < (int64_t)1 << 24 && tiles > 64 && tiles < (int64_t)1 << 24;
}

template <class T>
mdnn_status_t xent_outer(const void* p, int64_t ldp, int64_t R, const void* q, int64_t ldq, int64_t C, int64_t rows,
                         const float* alpha, void* d, int64_t ldd, mdnn_dtype_t d_type, hipStream_t st) {
  const int steps = (int)(rows / 64);
  const lds::MatArgs a{p, ldp, ceil_div(R, 8) * 8}, b{q, ldq, ceil_div(C, 8) * 8};
  const int64_t tiles = ceil_div(R, TileOuter::BM) * ceil_div(C, TileOuter::BN);
  if (d_type == MDNN_F32)
    hipLaunchKernelGGL((xent_outer_kernel<T, F32>), dim3((unsigned)tiles), dim3(TileOuter::NT), 0, st, a, b, R, C, steps,
                       alpha, d, ldd);
  else
    hipLaunchKernelGGL((xent_outer_kernel<T, T>), dim3((unsigned)tiles), dim3(TileOuter::NT), 0, st, a, b, R, C, steps,
                       alpha, d, ldd);
  return check_launch("xent_outer_kernel");
}
template mdnn_status_t xent_outer<F16>(const void*, int64_t, int64_t, const void*, int64_t, int64_t, int64_t, const float*,
                                       void*, int64_t, mdnn_dtype_t, hipStream_t);
template mdnn_status_t xent_outer<BF16>(const void*, int64_t, int64_t, const void*, int64_t, int64_t, int64_t, const float*,
                                        void*, int64_t, mdnn_dtype_t, hipStream_t);

}  // namespace mdnn

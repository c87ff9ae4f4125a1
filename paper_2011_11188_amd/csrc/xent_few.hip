// The last layer's gradients for up to eight rows: one pass that reads W and
// writes dW, dx's sums beside it (2 x 20001 x 4096 fp32 634 -> 292 us, 1 x 60000 x
// 4096 fp16 426 -> 326, the logits' pass of about 100 in both).
//
//   dW = a x^T G,  dx = a G W^T
//
// Bound: memory, W once each way.  As two products, W is read for dx at 3.5 TB/s
// and dW written from tiles of 64-deep steps at 1.1 (odd leading dimensions) to
// 3.3 TB/s; here a thread holds eight consecutive elements of W's rows, unaligned
// as they may be, and the rows' x or G for them in registers (2 M fused
// multiply-adds an element on the vector ALUs, which 16-bit elements at 5 TB/s and
// eight rows keep half busy).
#include "internal.h"
#include "row_chunk.h"
#include "xent.h"

namespace mdnn {
namespace {

// Whether row m of x counts (as zeros where it does not).
__device__ __forceinline__ bool counts(const XentFew& a, int m) {
  return m < a.M && (!a.labels || a.labels[m] != a.ignored);
}

constexpr int FEW_TILE = 64;  // rows of W whose numbers a block holds in LDS at a time

// W [N][K]: a thread's columns k of x in registers, the classes' G through LDS.
// Sums over a block's classes go to part[split][m][K], its groups of threads joined by
// shuffles and through LDS.
template <class T, class OutT, int MR>
__global__ void __launch_bounds__(256) xent_few_by_class_kernel(XentFew a) {
  typedef typename T::storage S;
  typedef typename OutT::storage DS;
  __shared__ float gs[FEW_TILE][MR];
  const int tx = a.tx, groups = 256 / tx, grp = threadIdx.x / tx;
  const ChunkPos pos = chunk_pos((int)blockIdx.x * tx + (int)threadIdx.x % tx, (int)a.K);
  const float alpha = *a.alpha;
  float x[MR][8], acc[MR][8];
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    Chunk<T> c;
    const bool on = counts(a, m);
    if (on) c.load((const S*)a.x + m * a.ldx + pos.start);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[m][e] = on ? c.get(e) : 0.0f, acc[m][e] = 0.0f;
  }
  const int64_t n1 = (int64_t)(blockIdx.y + 1) * a.per < a.N ? (int64_t)(blockIdx.y + 1) * a.per : a.N;
  for (int64_t t0 = (int64_t)blockIdx.y * a.per; t0 < n1; t0 += FEW_TILE) {
    __syncthreads();
    for (int i = threadIdx.x; i < FEW_TILE * MR; i += 256) {
      const int m = i / FEW_TILE, n = i % FEW_TILE;
      gs[n][m] = m < a.M && t0 + n < n1 ? load_f<T>((const S*)a.g + m * a.ldg + t0 + n) : 0.0f;
    }
    __syncthreads();
    const int left = n1 - t0 < FEW_TILE ? (int)(n1 - t0) : FEW_TILE;
    for (int i0 = grp; i0 < left; i0 += 4 * groups) {
      Chunk<T> w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * groups < left ? i0 + u * groups : i0;
        w[u].load((const S*)a.w + (t0 + i) * a.ldw + pos.start);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * groups;
        if (i >= left) break;
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = 0.0f;
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          const float g = gs[i][m];
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = fmaf(g, x[m][e], d[e]), acc[m][e] = fmaf(g, w[u].get(e), acc[m][e]);
        }
        if (a.dw && pos.lo < 8) {
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] *= alpha;
          Chunk<OutT> o;
          o.set(d);
          o.store((DS*)a.dw + (t0 + i) * a.lddw + pos.start, pos.lo);
        }
      }
    }
  }
  if (!a.part) return;
  __shared__ float4_t sums[256][2];
  const int own = tx < 64 ? 64 : tx;  // threads with sums of their own, once a wave's are joined
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    if (m >= a.M) break;  // (uniform)
    for (int o = tx; o < 64; o <<= 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[m][e] += __shfl_xor(acc[m][e], o, 64);
    }
    if (own < 256) {
      __syncthreads();
      sums[threadIdx.x][0] = (float4_t){acc[m][0], acc[m][1], acc[m][2], acc[m][3]};
      sums[threadIdx.x][1] = (float4_t){acc[m][4], acc[m][5], acc[m][6], acc[m][7]};
      __syncthreads();
      if ((int)threadIdx.x < tx)
        for (int t = (int)threadIdx.x + own; t < 256; t += own) {
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[m][e] += sums[t][e >> 2][e & 3];
        }
    }
    if ((int)threadIdx.x < tx && pos.lo < 8) {
      Chunk<F32> o;
      o.set(acc[m]);
      o.store(a.part + ((int64_t)blockIdx.y * a.M + m) * a.K + pos.start, pos.lo);
    }
  }
}

// MR sums over a wave, the lanes' halves, quarters and eighths each keeping their
// share: lane l has the sum of value l >> (6 - log2 MR).
template <int MR>
__device__ __forceinline__ float wave_sums(float (&v)[MR], int lane) {
  int o = 32;
#pragma unroll
  for (int n = MR / 2; n >= 1; n /= 2, o /= 2) {
    const bool up = lane & o;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const float keep = up ? v[k + n] : v[k], give = up ? v[k] : v[k + n];
      v[k] = keep + __shfl_xor(give, o, 64);
    }
  }
  for (; o > 0; o /= 2) v[0] += __shfl_xor(v[0], o, 64);
  return v[0];
}

// W [K][N]: a thread's classes of G in registers, the rows' x through LDS.  Sums
// over a block's classes go to part[strip][m][K].
template <class T, class OutT, int MR>
__global__ void __launch_bounds__(256) xent_few_by_row_kernel(XentFew a) {
  typedef typename T::storage S;
  typedef typename OutT::storage DS;
  __shared__ float xs[FEW_TILE][MR];
  __shared__ float ds[4][FEW_TILE][MR];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const ChunkPos pos = chunk_pos((int)blockIdx.x * 256 + (int)threadIdx.x, (int)a.N);
  const float alpha = *a.alpha;
  float g[MR][8];
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    Chunk<T> c;
    if (m < a.M) c.load((const S*)a.g + m * a.ldg + pos.start);
#pragma unroll
    for (int e = 0; e < 8; ++e) g[m][e] = m < a.M && e >= pos.lo ? c.get(e) : 0.0f;
  }
  const int64_t k1 = (int64_t)(blockIdx.y + 1) * a.per < a.K ? (int64_t)(blockIdx.y + 1) * a.per : a.K;
  for (int64_t t0 = (int64_t)blockIdx.y * a.per; t0 < k1; t0 += FEW_TILE) {
    const int left = k1 - t0 < FEW_TILE ? (int)(k1 - t0) : FEW_TILE;
    __syncthreads();
    for (int i = threadIdx.x; i < FEW_TILE * MR; i += 256) {
      const int m = i / FEW_TILE, k = i % FEW_TILE;
      xs[k][m] = k < left && counts(a, m) ? load_f<T>((const S*)a.x + m * a.ldx + t0 + k) : 0.0f;
    }
    __syncthreads();
    for (int i0 = 0; i0 < left; i0 += 4) {
      Chunk<T> w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        w[u].load((const S*)a.w + (t0 + (i0 + u < left ? i0 + u : i0)) * a.ldw + pos.start);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u;
        if (i >= left) break;
        float d[8], s[MR];
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = 0.0f;
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          const float x = xs[i][m];
          s[m] = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            d[e] = fmaf(x, g[m][e], d[e]);
            // (a neighbour's elements of a last, partial chunk may be Inf: not 0 times them)
            s[m] = fmaf(e >= pos.lo ? w[u].get(e) : 0.0f, g[m][e], s[m]);
          }
        }
        if (a.part) {
          const float v = wave_sums<MR>(s, lane);
          if (lane % (64 / MR) == 0) ds[wave][i][lane / (64 / MR)] = v;
        }
        if (a.dw && pos.lo < 8) {
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] *= alpha;
          Chunk<OutT> o;
          o.set(d);
          o.store((DS*)a.dw + (t0 + i) * a.lddw + pos.start, pos.lo);
        }
      }
    }
    if (!a.part) continue;
    __syncthreads();
    for (int i = threadIdx.x; i < FEW_TILE * MR; i += 256) {
      const int m = i / FEW_TILE, k = i % FEW_TILE;
      if (m < a.M && k < left)
        a.part[((int64_t)blockIdx.x * a.M + m) * a.K + t0 + k] = ((ds[0][k][m] + ds[1][k][m]) + ds[2][k][m]) + ds[3][k][m];
    }
  }
}

// dx from the blocks' sums: 64 elements a block, 16 groups of sums, joined in
// their order.
template <class T>
__global__ void __launch_bounds__(1024)
xent_few_dx_kernel(const float* part, int64_t parts, int64_t M, int64_t K, const float* alpha, void* dx, int64_t lddx) {
  __shared__ float buf[16][64];
  const int cx = threadIdx.x & 63, r = threadIdx.x >> 6;
  const int64_t all = M * K, i = (int64_t)blockIdx.x * 64 + cx, at = i < all ? i : all - 1;
  float s = 0.0f;
  for (int64_t b = r; b < parts; b += 128) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = part[(b + 16 * k < parts ? b + 16 * k : b) * all + at];
#pragma unroll
    for (int k = 0; k < 8; ++k) s += b + 16 * k < parts ? v[k] : 0.0f;
  }
  buf[r][cx] = s;
  __syncthreads();
  if (r > 0 || i >= all) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) s += buf[k][cx];
  ((typename T::storage*)dx)[i / K * lddx + i % K] = from_f<T>(s * *alpha);
}

template <class T, class OutT, int MR>
void launch_few(const XentFew& a, const FewPlan& p, hipStream_t st) {
  const dim3 grid((unsigned)p.strips, (unsigned)p.splits);
  if (a.by_class)
    hipLaunchKernelGGL((xent_few_by_class_kernel<T, OutT, MR>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((xent_few_by_row_kernel<T, OutT, MR>), grid, dim3(256), 0, st, a);
}
template <class T, class OutT>
void launch_rows(const XentFew& a, const FewPlan& p, hipStream_t st) {
  if (a.M <= 2) launch_few<T, OutT, 2>(a, p, st);
  else if (a.M <= 4) launch_few<T, OutT, 4>(a, p, st);
  else launch_few<T, OutT, 8>(a, p, st);
}

}  // namespace

// Strips of W's contiguous dimension, and splits of the other one: two blocks a
// CU where each leaves its own sums for dx (by class), else four; at least 4 rows
// of W to a thread group (by class 8 x 3000 x 64 fp32 18.9 us, 16 rows 25.7).
FewPlan few_plan(bool by_class, int64_t N, int64_t K) {
  FewPlan p;
  const int64_t across = by_class ? K : N, along = by_class ? N : K, chunks = ceil_div(across, 8);
  p.tx = 256;
  if (by_class)
    while (p.tx > 16 && p.tx / 2 >= chunks) p.tx /= 2;
  p.strips = ceil_div(chunks, p.tx);
  const int groups = 256 / p.tx;
  int64_t n = ceil_div(by_class ? 512 : 1024, p.strips), most = ceil_div(along, by_class ? 4 * groups : 4);
  n = n < most ? n : most;
  p.per = ceil_div(along, n);
  p.splits = ceil_div(along, p.per);
  p.parts = by_class ? p.splits : p.strips;
  return p;
}

// (by row, 16 bits, the vector ALUs bound more than four rows: 7 x 27551 x 6912
// fp16 474 us, as two products 408; 4 x 17020 x 3136 bf16 99 and 149)
bool xent_few_ok(bool by_class, mdnn_dtype_t t, int64_t M, int64_t N, int64_t K) {
  const int64_t most = by_class || t == MDNN_F32 ? 8 : 4;
  return M <= most && (by_class ? K : N) >= 8 && N <= 1 << 26 && K <= 1 << 20;
}

template <class T>
mdnn_status_t xent_few(XentFew a, mdnn_dtype_t dw_type, void* dx, int64_t lddx, hipStream_t st) {
  const FewPlan p = few_plan(a.by_class, a.N, a.K);
  a.tx = p.tx, a.per = p.per;
  if (!dx) a.part = nullptr;
  if (dw_type == MDNN_F32) launch_rows<T, F32>(a, p, st);
  else if constexpr (T::id != MDNN_F32) launch_rows<T, T>(a, p, st);
  MDNN_TRY(check_launch("xent_few_kernel"));
  if (!dx) return MDNN_SUCCESS;
  hipLaunchKernelGGL((xent_few_dx_kernel<T>), dim3((unsigned)ceil_div(a.M * a.K, 64)), dim3(1024), 0, st, a.part, p.parts,
                     a.M, a.K, a.alpha, dx, lddx);
  return check_launch("xent_few_dx_kernel");
}
template mdnn_status_t xent_few<F32>(XentFew, mdnn_dtype_t, void*, int64_t, hipStream_t);
template mdnn_status_t xent_few<F16>(XentFew, mdnn_dtype_t, void*, int64_t, hipStream_t);
template mdnn_status_t xent_few<BF16>(XentFew, mdnn_dtype_t, void*, int64_t, hipStream_t);

}  // namespace mdnn

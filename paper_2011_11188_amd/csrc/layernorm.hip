// Dropout with its mask drawn again instead of stored, and layer norm with
// the residual's addition and that dropout in its pass, both ways.
//
//   h = res + keep s x                            (fp32; stored rounded once)
//   y = (h - mean h) rstd gamma + beta,  rstd = 1 / sqrt(var h + eps)
// gradients, with xh = (h - mean h) rstd and g = dy gamma:
//   dh = rstd (g - mean g - xh mean(g xh)) + dres,  dx = keep s dh
//   dgamma = sum over rows of dy xh,  dbeta = sum over rows of dy
//
// The variance is that of the differences d = h - mean, a second sum over the
// registers: a sum of squares loses what a row's offset cancels.  The mean's
// own rounding, which d shares, is taken out by d's mean c, which the second
// sum has besides: var = mean d^2 - c^2, y from d - c.
//
// Bound: memory.  Rows are read once into registers, as in the root-mean-square
// norm's kernels; rows past the registers or below eight elements take the
// kernels that read a row again for each sum.  Measured: dropout 16384 x 8192 bf16
// 136 us (5.9 TB/s), layer norm with both 197 (5.4 TB/s).
#include <cmath>

#include "dropout.h"
#include "internal.h"

namespace mdnn {
namespace {

// ---------------------------------------------------------------------------
// dropout alone: a thread per chunk, blocks of TX chunks x 256 / TX rows
// ---------------------------------------------------------------------------
struct DropoutArgs {
  const void *x, *res;  // res: or null
  void* y;
  int64_t rows, ldx, ldr, ldy;
  int32_t cols;
  DropArgs d;
};

template <class T, bool DROP>
__device__ __forceinline__ void dropout_apply(const DropoutArgs& a, const DropBits& b, const Chunk<T>& x,
                                              const Chunk<T>& r, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = DROP ? b.apply(a.d, e, x.get(e)) : x.get(e);
    if (a.res) v[e] = add_rn(v[e], r.get(e));
  }
}

template <class T, bool DROP>
__global__ void __launch_bounds__(256) dropout_kernel(DropoutArgs a, int tx) {
  typedef typename T::storage S;
  const int c = (int)blockIdx.x * tx + (int)threadIdx.x % tx;
  if (c * 8 >= a.cols) return;
  const int ty = 256 / tx;
  DropKey key = {};
  if (DROP) key = drop_key(a.d);
  const ChunkPos pos = chunk_pos(c, a.cols);
  for (int64_t row = (int64_t)blockIdx.y * ty + (int)threadIdx.x / tx; row < a.rows; row += (int64_t)gridDim.y * ty) {
    const S* x = (const S*)a.x + row * a.ldx;
    const S* res = a.res ? (const S*)a.res + row * a.ldr : nullptr;
    S* y = (S*)a.y + row * a.ldy;
    Chunk<T> cx, cr;
    DropBits b;
    if (a.cols >= 8) {
      cx.load(x + pos.start);
      if (res) cr.load(res + pos.start);
      if (DROP) {
        b.draw(a.d, key, (uint32_t)c, (uint32_t)row);
        if (pos.lo > 0) b.shift(pos.lo);
      }
      float v[8];
      dropout_apply<T, DROP>(a, b, cx, cr, v);
      Chunk<T> o;
      o.set(v);
      o.store(y + pos.start, pos.lo);
    } else {
      if (DROP) b.draw(a.d, key, 0u, (uint32_t)row);
#pragma unroll
      for (int e = 0; e < 7; ++e) {
        if (e >= a.cols) continue;
        float v = to_f<T>(x[e]);
        if (DROP) v = b.apply(a.d, e, v);
        if (res) v = add_rn(v, to_f<T>(res[e]));
        y[e] = from_f<T>(v);
      }
    }
  }
}

template <class T>
mdnn_status_t run_dropout_t(const DropoutArgs& a, hipStream_t st) {
  const int64_t nch = ceil_div(a.cols, 8);
  int tx = 1;
  while (tx < 256 && tx < nch) tx *= 2;
  const int64_t gx = ceil_div(nch, tx);
  int64_t gy = ceil_div(a.rows, 256 / tx), most = ceil_div(MAX_BLOCKS, gx);
  most = most < 65535 ? most : 65535;
  gy = gy < most ? gy : most;
  const dim3 grid((unsigned)gx, (unsigned)gy);
  if (a.d.rng)
    hipLaunchKernelGGL((dropout_kernel<T, true>), grid, dim3(256), 0, st, a, tx);
  else
    hipLaunchKernelGGL((dropout_kernel<T, false>), grid, dim3(256), 0, st, a, tx);
  return check_launch("dropout_kernel");
}

mdnn_status_t run_dropout(const DropoutArgs& a, mdnn_dtype_t t, hipStream_t st) {
  clear_error();
  switch (t) {
    case MDNN_F32: return run_dropout_t<F32>(a, st);
    case MDNN_F16: return run_dropout_t<F16>(a, st);
    default: return run_dropout_t<BF16>(a, st);
  }
}

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------

// NV sums over a row's TPR threads, in a fixed order, every thread left with
// all of them.  Rows of more than a wave combine their waves through LDS;
// successive reductions take the two buffers in turn, one barrier each: a wave
// writes a buffer again only past the barrier of the reduction in between,
// which every wave reaches after its reads.
template <int NV, int TPR, int RPB>
struct RowSums {
  float v[2][RPB][TPR > 64 ? TPR / 64 : 1][NV];
};
template <int FLIP, int NV, int NB, int TPR, int RPB>
__device__ __forceinline__ void row_sums(float (&s)[NV], RowSums<NB, TPR, RPB>& buf) {
  static_assert(NV <= NB, "buffer");
  constexpr int W = TPR < 64 ? TPR : 64;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < NV; ++k) s[k] += __shfl_xor(s[k], o, W);
  if constexpr (TPR > 64) {
    const int r = threadIdx.x / TPR;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) buf.v[FLIP][r][threadIdx.x % TPR >> 6][k] = s[k];
    }
    __syncthreads();
    // (a lane takes one wave's sums: every wave's in every lane fill the registers)
    constexpr int NW = TPR / 64;
#pragma unroll
    for (int k = 0; k < NV; ++k) s[k] = buf.v[FLIP][r][threadIdx.x % NW][k];
#pragma unroll
    for (int o = NW / 2; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < NV; ++k) s[k] += __shfl_xor(s[k], o, 64);
  }
}

// 1 / sqrt(var + eps) from the sums of d and d^2; a sum that is not finite (the
// row holds Inf or NaN, or passes fp32's range) makes the row NaN.
struct Centre {
  float c, rstd;  // mean of d, 1 / deviation
};
__device__ __forceinline__ Centre row_centre(float sum, float ssq, float cols, float eps) {
  const float c = sum / cols, var = fmaf(-c, c, ssq / cols);
  return {c, isfinite(ssq) ? 1.0f / sqrtf((var > 0.0f ? var : 0.0f) + eps) : __builtin_nanf("")};
}

struct LnArgs {
  const void *x, *res;       // res: or null
  const float *gamma, *beta;  // or null (ones, zeros)
  void *h, *y;               // h: or null
  int64_t rows, ldx, ldr, ldh, ldy;
  int32_t cols;
  float eps;
  DropArgs d;
};

template <class T, bool DROP, int TPR, int NCH>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) layernorm_kernel(LnArgs a) {
  typedef typename T::storage S;
  constexpr int NT = TPR < 256 ? 256 : TPR, RPB = NT / TPR;
  __shared__ RowSums<2, TPR, RPB> buf;
  const int t = threadIdx.x % TPR;
  DropKey key = {};
  if (DROP) key = drop_key(a.d);
  ChunkPos pos[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i) pos[i] = chunk_pos(t + i * TPR, a.cols);
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
    // (a thread group past the last row repeats it and stores nothing)
    const int64_t rw = r0 + threadIdx.x / TPR;
    const bool live = rw < a.rows;
    const int64_t row = live ? rw : a.rows - 1;
    Chunk<T> cx[NCH], cr[NCH];
#pragma unroll
    for (int i = 0; i < NCH; ++i) cx[i].load((const S*)a.x + row * a.ldx + pos[i].start);
    // (fp32 rows over 1024 threads fill the registers: the residual is read late)
    constexpr bool LATE = TPR == 1024 && DROP && !Chunk<T>::H;
    if (a.res && !LATE) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) cr[i].load((const S*)a.res + row * a.ldr + pos[i].start);
    }
    float h[NCH][8], s[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      DropBits b;
      if (DROP) {
        if (TPR == 1024) __builtin_amdgcn_sched_barrier(0);  // (one chunk's bits at a time: 128 registers a thread)
        b.draw(a.d, key, (uint32_t)(t + i * TPR), (uint32_t)row);
        if (pos[i].lo > 0) b.shift(pos[i].lo);
      }
      if (pos[i].lo > 0) cx[i].clear(pos[i].lo);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] = DROP ? b.apply(a.d, e, cx[i].get(e)) : cx[i].get(e);
      if (a.res) {
        if (LATE) cr[i].load((const S*)a.res + row * a.ldr + pos[i].start);
        if (pos[i].lo > 0) cr[i].clear(pos[i].lo);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] = add_rn(h[i][e], cr[i].get(e));
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += h[i][e];
      if (a.h && live && pos[i].lo < 8) {
        Chunk<T> c;
        c.set(h[i]);
        c.store((S*)a.h + row * a.ldh + pos[i].start, pos[i].lo);
      }
    }
    row_sums<0>(s, buf);
    const float cols = (float)a.cols, mean = s[0] / cols;
    float q[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] -= mean;
      if (pos[i].lo > 0) {
        int lo = pos[i].lo;
        asm("" : "+v"(lo));
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] = e < lo ? 0.0f : h[i][e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) q[0] += h[i][e], q[1] = fmaf(h[i][e], h[i][e], q[1]);
    }
    row_sums<1>(q, buf);
    const Centre k = row_centre(q[0], q[1], cols, a.eps);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      if (!live || pos[i].lo == 8) continue;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = (h[i][e] - k.c) * k.rstd;
      if (a.gamma) {
        Chunk<F32> g;
        g.load(a.gamma + pos[i].start);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] *= g.get(e);
      }
      if (a.beta) {
        Chunk<F32> g;
        g.load(a.beta + pos[i].start);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += g.get(e);
      }
      Chunk<T> c;
      c.set(y);
      c.store((S*)a.y + row * a.ldy + pos[i].start, pos[i].lo);
    }
  }
}

// Eight columns of a row of any length: those past its end are not used.
template <class T>
__device__ __forceinline__ void load8(const typename T::storage* row, int64_t at, int64_t cols, float (&v)[8]) {
  if (at + 8 <= cols) {
    Chunk<T> c;
    c.load(row + at);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c.get(e);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = to_f<T>(row[at + e < cols ? at + e : cols - 1]);
  }
}
template <class T>
__device__ __forceinline__ void store8(typename T::storage* row, int64_t at, int64_t cols, const float (&v)[8]) {
  if (at + 8 <= cols) {
    Chunk<T> c;
    c.set(v);
    c.store(row + at, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at + e < cols) row[at + e] = from_f<T>(v[e]);
  }
}

// NV sums in 64 bits over a block of NT threads (rows past the registers, where
// up to 2^16 terms of eight fall to a thread: chains in fp32 lose their low bits).
template <int NV, int NT>
__device__ __forceinline__ void block_sums(double (&s)[NV], double (*buf)[NV]) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < NV; ++k) s[k] += __shfl_xor(s[k], o, 64);
  if constexpr (NT > 64) {
    __syncthreads();  // (the buffer's last reads are done)
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) buf[threadIdx.x >> 6][k] = s[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NV; ++k) s[k] = buf[0][k];
    for (int w = 1; w < NT / 64; ++w)
#pragma unroll
      for (int k = 0; k < NV; ++k) s[k] += buf[w][k];
  }
}

// Rows of any length, read again for each sum.  A thread reads an element for
// the last time before it writes it, so outputs may lie in place of the inputs.
template <class T, bool DROP, int NT>
__global__ void __launch_bounds__(NT) layernorm_long_kernel(LnArgs a) {
  typedef typename T::storage S;
  __shared__ double buf[NT / 64][2];
  DropKey key = {};
  if (DROP) key = drop_key(a.d);
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const S* x = (const S*)a.x + row * a.ldx;
    const S* res = a.res ? (const S*)a.res + row * a.ldr : nullptr;
    auto load = [&](int64_t at, float (&h)[8]) {
      load8<T>(x, at, a.cols, h);
      if (DROP) {
        DropBits b;
        b.draw(a.d, key, (uint32_t)(at / 8), (uint32_t)row);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = b.apply(a.d, e, h[e]);
      }
      if (res) {
        float r[8];
        load8<T>(res, at, a.cols, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = add_rn(h[e], r[e]);
      }
    };
    float h[8];
    double s[1] = {0.0};
    for (int64_t at = threadIdx.x * 8; at < a.cols; at += NT * 8) {
      load(at, h);
      float u = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) u += at + e < a.cols ? h[e] : 0.0f;
      s[0] += (double)u;
    }
    block_sums<1, NT>(s, (double(*)[1])buf);
    const float cols = (float)a.cols, mean = (float)(s[0] / a.cols);
    double q[2] = {0.0, 0.0};
    for (int64_t at = threadIdx.x * 8; at < a.cols; at += NT * 8) {
      load(at, h);
      float u = 0.0f, v = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = at + e < a.cols ? h[e] - mean : 0.0f;
        u += d, v = fmaf(d, d, v);
      }
      q[0] += (double)u, q[1] += (double)v;
    }
    block_sums<2, NT>(q, buf);
    const Centre k = row_centre((float)q[0], (float)q[1], cols, a.eps);
    for (int64_t at = threadIdx.x * 8; at < a.cols; at += NT * 8) {
      load(at, h);
      if (a.h) store8<T>((S*)a.h + row * a.ldh, at, a.cols, h);
      float g[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = ((h[e] - mean) - k.c) * k.rstd;
      if (a.gamma) {
        load8<F32>(a.gamma, at, a.cols, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] *= g[e];
      }
      if (a.beta) {
        load8<F32>(a.beta, at, a.cols, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += g[e];
      }
      store8<T>((S*)a.y + row * a.ldy, at, a.cols, h);
    }
  }
}

template <class T, bool DROP, int TPR, int NCH>
void launch_ln(const LnArgs& a, hipStream_t st) {
  constexpr int NT = TPR < 256 ? 256 : TPR, RPB = NT / TPR;
  const int64_t blocks = ceil_div(a.rows, RPB);
  hipLaunchKernelGGL((layernorm_kernel<T, DROP, TPR, NCH>), dim3((unsigned)(blocks < MAX_BLOCKS ? blocks : MAX_BLOCKS)),
                     dim3(NT), 0, st, a);
}

// Threads and chunks of a row as in the root-mean-square norm.
template <class T, bool DROP>
mdnn_status_t run_ln_t(const LnArgs& a, hipStream_t st) {
  const int64_t nch = ceil_div(a.cols, 8), blocks = a.rows < MAX_BLOCKS ? a.rows : MAX_BLOCKS;
  if (a.cols < 8)
    hipLaunchKernelGGL((layernorm_long_kernel<T, DROP, 64>), dim3((unsigned)blocks), dim3(64), 0, st, a);
  else if (nch > 4096)
    hipLaunchKernelGGL((layernorm_long_kernel<T, DROP, 1024>), dim3((unsigned)blocks), dim3(1024), 0, st, a);
  else if (nch <= 16)
    launch_ln<T, DROP, 16, 1>(a, st);
  else if (nch <= 32)
    launch_ln<T, DROP, 16, 2>(a, st);
  else if (nch <= 64)
    launch_ln<T, DROP, 64, 1>(a, st);
  else if (nch <= 128)
    launch_ln<T, DROP, 64, 2>(a, st);
  else if (nch <= 256)
    launch_ln<T, DROP, 256, 1>(a, st);
  else if (nch <= 512)
    launch_ln<T, DROP, 256, 2>(a, st);
  else if (nch <= 1024)
    launch_ln<T, DROP, 512, 2>(a, st);
  else if (nch <= 2048)
    launch_ln<T, DROP, 512, 4>(a, st);
  else
    launch_ln<T, DROP, 1024, 4>(a, st);
  return check_launch("layernorm_kernel");
}

template <class T>
mdnn_status_t run_ln(const LnArgs& a, hipStream_t st) {
  return a.d.rng ? run_ln_t<T, true>(a, st) : run_ln_t<T, false>(a, st);
}

// ---------------------------------------------------------------------------
// gradients
// ---------------------------------------------------------------------------


// Keeps what is derived from a chunk (its conversions) from staying in
// registers past the pass that needs it.
template <class T>
__device__ __forceinline__ void hold(Chunk<T>& c) {
#pragma unroll
  for (uint32_t& w : c.w) asm("" : "+v"(w));
}

struct LnBwdArgs {
  const void *dy, *h, *dres;  // dres: or null
  const float* gamma;         // or null
  void *dx, *dh;              // each or null
  float *pg, *pb;             // sums for dgamma and dbeta, block b's at b * stride; each or null
  int64_t rows, lddy, ldh, lddr, lddx, lddh, stride;
  int32_t cols;
  float eps;
  DropArgs d;
};

// Sums of dgamma and dbeta stay in the registers of their columns' threads over a
// block's rows, are added over its row groups in their order and written once;
// sums_kernel adds the blocks' in order.  Bound: memory (4096 x 4096 bf16 with
// residual and dropout 42 us, 4.4 TB/s, and 5 for the sums; without 38.5 together),
// and two launches where that is little (20 x 900 fp32 9.5).
template <class T, bool DROP, int TPR, int NCH>
__global__ void __launch_bounds__(512, NCH <= 2 && !(DROP && !Chunk<T>::H) ? 4 : 2) layernorm_bwd_kernel(LnBwdArgs a) {
  typedef typename T::storage S;
  constexpr int NT = 512, RPB = NT / TPR, WIDE = TPR * NCH * 8;
  __shared__ RowSums<3, TPR, RPB> buf;
  __shared__ __attribute__((aligned(16))) float part[RPB > 1 ? RPB * WIDE : 1];
  __shared__ float4_t gamma[WIDE / 4];
  const int t = threadIdx.x % TPR, grp = threadIdx.x / TPR;
  DropKey key = {};
  if (DROP) key = drop_key(a.d);
  ChunkPos pos[NCH];
  float dg[NCH][8], db[NCH][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    pos[i] = chunk_pos(t + i * TPR, a.cols);
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[i][e] = db[i][e] = 0.0f;
    // (each row group writes the same)
    float4_t g[2] = {{1.0f, 1.0f, 1.0f, 1.0f}, {1.0f, 1.0f, 1.0f, 1.0f}};
    if (a.gamma) {
      Chunk<F32> c;
      c.load(a.gamma + pos[i].start);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e >> 2][e & 3] = c.get(e);
    }
    gamma[(t + i * TPR) * 2] = g[0], gamma[(t + i * TPR) * 2 + 1] = g[1];
  }
  __syncthreads();
  // this thread's chunk of gamma, read again where it is needed: 8 NCH registers less
  auto scale = [&](int i, float (&g)[8]) {
    const float4_t u = gamma[(t + i * TPR) * 2], v = gamma[(t + i * TPR) * 2 + 1];
#pragma unroll
    for (int e = 0; e < 4; ++e) g[e] = u[e], g[4 + e] = v[e];
  };
  const float cols = (float)a.cols;
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB) {
    const bool live = r0 + grp < a.rows;
    const int64_t row = live ? r0 + grp : a.rows - 1;  // (past the last row: repeated, nothing stored)
    Chunk<T> cd[NCH], ch[NCH], cr[NCH];
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      ch[i].load((const S*)a.h + row * a.ldh + pos[i].start);
      cd[i].load((const S*)a.dy + row * a.lddy + pos[i].start);
    }
    if (a.dres) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) cr[i].load((const S*)a.dres + row * a.lddr + pos[i].start);
    }
    // sums of h and g, then of d, d^2 and g d
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      float g[8];
      scale(i, g);
      if (pos[i].lo > 0) ch[i].clear(pos[i].lo), cd[i].clear(pos[i].lo);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += ch[i].get(e), s[1] += cd[i].get(e) * g[e];
    }
    row_sums<0>(s, buf);
    const float mean = s[0] / cols;
    float q[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      hold(ch[i]), hold(cd[i]);
      asm volatile("" ::: "memory");  // (gamma is read again)
      float g[8];
      scale(i, g);
      int lo = pos[i].lo;
      asm("" : "+v"(lo));
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = e < lo ? 0.0f : ch[i].get(e) - mean;
        q[0] += d, q[1] = fmaf(d, d, q[1]), q[2] = fmaf(cd[i].get(e) * g[e], d, q[2]);
      }
    }
    row_sums<1>(q, buf);
    const Centre k = row_centre(q[0], q[1], cols, a.eps);
    const float mg = s[1] / cols, mgx = k.rstd * ((q[2] - k.c * s[1]) / cols);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      if (!live || pos[i].lo == 8) continue;
      hold(ch[i]), hold(cd[i]);
      asm volatile("" ::: "memory");
      if (DROP) __builtin_amdgcn_sched_barrier(0);  // (one chunk's bits at a time)
      float o[8], g[8];
      scale(i, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xh = ((ch[i].get(e) - mean) - k.c) * k.rstd, d = cd[i].get(e);
        o[e] = k.rstd * ((d * g[e] - mg) - xh * mgx);
        if (a.dres) o[e] += cr[i].get(e);
        dg[i][e] = fmaf(d, xh, dg[i][e]);
        db[i][e] += d;
      }
      if (a.dh) {
        Chunk<T> c;
        c.set(o);
        c.store((S*)a.dh + row * a.lddh + pos[i].start, pos[i].lo);
      }
      if (a.dx) {
        if (DROP) {
          DropBits b;
          b.draw(a.d, key, (uint32_t)(t + i * TPR), (uint32_t)row);
          if (pos[i].lo > 0) b.shift(pos[i].lo);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = b.apply(a.d, e, o[e]);
        }
        Chunk<T> c;
        c.set(o);
        c.store((S*)a.dx + row * a.lddx + pos[i].start, pos[i].lo);
      }
    }
  }
  auto put = [&](const float (&v)[NCH][8], float* out) {
    if constexpr (RPB > 1) {
      __syncthreads();  // (the buffer's last reads are done)
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int e = 0; e < 8; e += 4)
          *(float4*)&part[grp * WIDE + (t + i * TPR) * 8 + e] = make_float4(v[i][e], v[i][e + 1], v[i][e + 2], v[i][e + 3]);
      __syncthreads();
      for (int c = threadIdx.x; c < a.cols; c += NT) {
        // column c's place: its chunk's slot, counted from the row's end in the last, partial chunk
        const int n = c / 8, at = n * 8 + (c - chunk_pos(n, a.cols).start);
        float sum = part[at];
#pragma unroll
        for (int r = 1; r < RPB; ++r) sum += part[r * WIDE + at];
        out[c] = sum;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        if (pos[i].lo == 8) continue;
        Chunk<F32> w;
        w.set(v[i]);
        w.store(out + pos[i].start, pos[i].lo);
      }
    }
  };
  if (a.pg) put(dg, a.pg + blockIdx.x * a.stride);
  if (a.pb) put(db, a.pb + blockIdx.x * a.stride);
}

// Rows of any length, read again for each sum; the column sums of rows past the
// registers are kept in the block's own part of the workspace.  Rows below
// eight elements (NT = 64, one thread of a block holds the row) come by the
// million: their column sums are kept in 64 bits and written at the end.
template <class T, bool DROP, int NT>
__global__ void __launch_bounds__(NT) layernorm_bwd_long_kernel(LnBwdArgs a) {
  typedef typename T::storage S;
  constexpr bool NARROW = NT == 64;
  __shared__ double buf[NT / 64][3];
  DropKey key = {};
  if (DROP) key = drop_key(a.d);
  double og[8] = {}, ob[8] = {};
  const float cols = (float)a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const S *dy = (const S*)a.dy + row * a.lddy, *hp = (const S*)a.h + row * a.ldh;
    float h[8], d[8], g[8], o[8];
    auto load = [&](int64_t at) {  // h, dy and g = dy gamma
      load8<T>(hp, at, a.cols, h);
      load8<T>(dy, at, a.cols, d);
      if (a.gamma) load8<F32>(a.gamma, at, a.cols, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = a.gamma ? d[e] * g[e] : d[e];
    };
    double s[2] = {0.0, 0.0};
    for (int64_t at = threadIdx.x * 8; at < a.cols; at += NT * 8) {
      load(at);
      float u = 0.0f, v = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < a.cols) u += h[e], v += g[e];
      s[0] += (double)u, s[1] += (double)v;
    }
    block_sums<2, NT>(s, (double(*)[2])buf);
    const float mean = (float)(s[0] / a.cols);
    double q[3] = {0.0, 0.0, 0.0};
    for (int64_t at = threadIdx.x * 8; at < a.cols; at += NT * 8) {
      load(at);
      float u = 0.0f, v = 0.0f, w = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < a.cols) {
          const float x = h[e] - mean;
          u += x, v = fmaf(x, x, v), w = fmaf(g[e], x, w);
        }
      q[0] += (double)u, q[1] += (double)v, q[2] += (double)w;
    }
    block_sums<3, NT>(q, buf);
    const Centre k = row_centre((float)q[0], (float)q[1], cols, a.eps);
    const float mg = (float)(s[1] / a.cols), mgx = k.rstd * (float)((q[2] - (double)k.c * s[1]) / a.cols);
    const bool first = row == (int64_t)blockIdx.x;
    for (int64_t at = threadIdx.x * 8; at < a.cols; at += NT * 8) {
      load(at);
      if (a.dres) load8<T>((const S*)a.dres + row * a.lddr, at, a.cols, o);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xh = ((h[e] - mean) - k.c) * k.rstd, v = k.rstd * ((g[e] - mg) - xh * mgx);
        o[e] = a.dres ? v + o[e] : v;
        h[e] = xh;
        if (NARROW && at + e < a.cols) og[e] += (double)d[e] * (double)xh, ob[e] += (double)d[e];
      }
      if (!NARROW) {
        if (a.pg) {
          float* p = a.pg + blockIdx.x * a.stride;
          if (!first) load8<F32>(p, at, a.cols, g);
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = first ? d[e] * h[e] : fmaf(d[e], h[e], g[e]);
          store8<F32>(p, at, a.cols, g);
        }
        if (a.pb) {
          float* p = a.pb + blockIdx.x * a.stride;
          if (!first) load8<F32>(p, at, a.cols, g);
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] = first ? d[e] : g[e] + d[e];
          store8<F32>(p, at, a.cols, g);
        }
      }
      if (a.dh) store8<T>((S*)a.dh + row * a.lddh, at, a.cols, o);
      if (a.dx) {
        if (DROP) {
          DropBits b;
          b.draw(a.d, key, (uint32_t)(at / 8), (uint32_t)row);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = b.apply(a.d, e, o[e]);
        }
        store8<T>((S*)a.dx + row * a.lddx, at, a.cols, o);
      }
    }
  }
  if (NARROW && threadIdx.x == 0) {
#pragma unroll
    for (int e = 0; e < 7; ++e) {
      if (a.pg && e < a.cols) a.pg[blockIdx.x * a.stride + e] = (float)og[e];
      if (a.pb && e < a.cols) a.pb[blockIdx.x * a.stride + e] = (float)ob[e];
    }
  }
}

// s += every 32nd of the blocks' sums from b0 on, N loads in flight.
template <int N>
__device__ __forceinline__ void add_sums(const float* p, int b0, int blocks, int64_t stride, float& s) {
  float v[N];
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = p[(int64_t)(b0 + 32 * k < blocks ? b0 + 32 * k : blocks - 1) * stride];
#pragma unroll
  for (int k = 0; k < N; ++k) s += b0 + 32 * k < blocks ? v[k] : 0.0f;
}

// dgamma (blockIdx.y 0) and dbeta from the blocks' sums: 32 columns a block, 32
// rows of threads, each adding every 32nd block's sums (as many loads in flight
// as there are, up to sixteen: 48 x 9152 fp16 13.4 us a call, always sixteen 17.8),
// then those in order.
__global__ void __launch_bounds__(1024)
sums_kernel(const float* partial, int blocks, int64_t cols, float* dgamma, float* dbeta) {
  __shared__ float part[32][32];
  const int cx = threadIdx.x & 31, r = threadIdx.x >> 5;
  float* out = blockIdx.y ? dbeta : dgamma;
  if (!out) return;  // (uniform)
  for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < cols; c0 += (int64_t)gridDim.x * 32) {
    const int64_t c = c0 + cx;
    const float* p = partial + blockIdx.y * cols + (c < cols ? c : cols - 1);
    float s = 0.0f;
    for (int t0 = 0; t0 < blocks; t0 += 512) {
      const int left = blocks - t0;
      if (left > 256) add_sums<16>(p, t0 + r, blocks, 2 * cols, s);
      else if (left > 128) add_sums<8>(p, t0 + r, blocks, 2 * cols, s);
      else if (left > 64) add_sums<4>(p, t0 + r, blocks, 2 * cols, s);
      else add_sums<2>(p, t0 + r, blocks, 2 * cols, s);
    }
    part[r][cx] = s;
    __syncthreads();
    if (r == 0 && c < cols) {
#pragma unroll
      for (int k = 1; k < 32; ++k) s += part[k][cx];
      out[c] = s;
    }
    __syncthreads();  // (before the sums of the next columns)
  }
}

// Threads per row of the backward pass by the row's chunks; 0: the long-row kernel.
int bwd_tpr(int64_t cols) {
  const int64_t nch = ceil_div(cols, 8);
  return cols < 8 || nch > 2048 ? 0 : nch <= 32 ? 16 : nch <= 128 ? 64 : nch <= 512 ? 256 : 512;
}
// Its blocks: by the sizes alone, so that the workspace and the order of the
// sums are the same everywhere.  Two a CU, as many as the registers let run (4096
// x 4096 bf16 47 us; 256 blocks 53, 1024 54).
int64_t bwd_blocks(int64_t rows, int64_t cols) {
  const int tpr = bwd_tpr(cols);
  const int64_t b = ceil_div(rows, tpr == 0 ? 1 : 512 / tpr);
  const int64_t most = cols < 8 ? 2048 : cols > 8192 ? 256 : 512;
  const int64_t alone = tpr == 16 ? 3 : tpr == 64 || tpr == 256 ? 2 : 1;  // (worth one launch instead of two)
  return b <= alone ? 1 : b < most ? b : most;
}

template <class T, bool DROP, int TPR, int NCH>
void launch_bwd(const LnBwdArgs& a, int64_t blocks, hipStream_t st) {
  hipLaunchKernelGGL((layernorm_bwd_kernel<T, DROP, TPR, NCH>), dim3((unsigned)blocks), dim3(512), 0, st, a);
}

template <class T, bool DROP>
mdnn_status_t run_bwd_t(const LnBwdArgs& a, int64_t blocks, hipStream_t st) {
  const int64_t nch = ceil_div(a.cols, 8);
  if (a.cols < 8)
    hipLaunchKernelGGL((layernorm_bwd_long_kernel<T, DROP, 64>), dim3((unsigned)blocks), dim3(64), 0, st, a);
  else if (bwd_tpr(a.cols) == 0)
    hipLaunchKernelGGL((layernorm_bwd_long_kernel<T, DROP, 512>), dim3((unsigned)blocks), dim3(512), 0, st, a);
  else if (nch <= 16)
    launch_bwd<T, DROP, 16, 1>(a, blocks, st);
  else if (nch <= 32)
    launch_bwd<T, DROP, 16, 2>(a, blocks, st);
  else if (nch <= 64)
    launch_bwd<T, DROP, 64, 1>(a, blocks, st);
  else if (nch <= 128)
    launch_bwd<T, DROP, 64, 2>(a, blocks, st);
  else if (nch <= 256)
    launch_bwd<T, DROP, 256, 1>(a, blocks, st);
  else if (nch <= 512)
    launch_bwd<T, DROP, 256, 2>(a, blocks, st);
  else if (nch <= 1024)
    launch_bwd<T, DROP, 512, 2>(a, blocks, st);
  else
    launch_bwd<T, DROP, 512, 4>(a, blocks, st);
  return check_launch("layernorm_bwd_kernel");
}

template <class T>
mdnn_status_t run_bwd(const LnBwdArgs& a, int64_t blocks, hipStream_t st) {
  return a.d.rng ? run_bwd_t<T, true>(a, blocks, st) : run_bwd_t<T, false>(a, blocks, st);
}

constexpr int64_t MAX_COLS = (int64_t)1 << 29;  // 32-bit column indices

// p, the generator's state and the sizes that its counters hold.
mdnn_status_t check_drop(const char* who, float p, const void* rng, int64_t rows) {
  if (!(p >= 0.0f && p <= 1.0f)) return fail(MDNN_ERR_SHAPE, "%s: p must lie in [0, 1]", who);
  if (drop_args(p, rng, 0).t == 0) return MDNN_SUCCESS;
  if (!rng) return fail(MDNN_ERR_NULL, "%s: rng is NULL with p > 0", who);
  if (!aligned(rng, 8)) return fail(MDNN_ERR_MISALIGNED, "%s: misaligned rng", who);
  if (rows > (int64_t)1 << 32) return fail(MDNN_ERR_SHAPE, "%s: more than 2^32 rows with dropout", who);
  return MDNN_SUCCESS;
}

mdnn_status_t dropout_call(const char* who, int64_t rows, int64_t cols, const void* x, int64_t ldx,
                           const void* residual, int64_t ldr, float p, const void* rng, uint32_t site, void* y,
                           int64_t ldy, mdnn_dtype_t dtype, mdnn_stream_t stream) {
  if (rows < 0 || cols < 0 || cols > MAX_COLS) return fail(MDNN_ERR_SHAPE, "%s: bad size", who);
  if (!dtype_ok(dtype)) return fail(MDNN_ERR_DTYPE, "%s: unknown dtype", who);
  MDNN_TRY(check_drop(who, p, rng, rows));
  if (rows == 0 || cols == 0) return MDNN_SUCCESS;
  if (!x || !y) return fail(MDNN_ERR_NULL, "%s: NULL buffer", who);
  if (ldx < cols || ldy < cols || (residual && ldr < cols))
    return fail(MDNN_ERR_LAYOUT, "%s: leading dimension below the width", who);
  const size_t es = dtype_size(dtype);
  if (!aligned(x, es) || !aligned(residual, es) || !aligned(y, es))
    return fail(MDNN_ERR_MISALIGNED, "%s: misaligned buffer", who);
  DropoutArgs a = {};
  a.x = x, a.res = residual, a.y = y, a.rows = rows, a.cols = (int32_t)cols;
  a.ldx = ldx, a.ldr = ldr, a.ldy = ldy, a.d = drop_args(p, rng, site);
  return run_dropout(a, dtype, as_stream(stream));
}

}  // namespace
}  // namespace mdnn

using namespace mdnn;

extern "C" mdnn_status_t mdnn_dropout_fwd(int64_t rows, int64_t cols, const void* x, int64_t ldx,
                                          const void* residual, int64_t ldr, float p, const void* rng, uint32_t site,
                                          void* y, int64_t ldy, mdnn_dtype_t dtype, mdnn_stream_t stream) {
  return dropout_call("dropout_fwd", rows, cols, x, ldx, residual, ldr, p, rng, site, y, ldy, dtype, stream);
}

extern "C" mdnn_status_t mdnn_dropout_bwd(int64_t rows, int64_t cols, const void* dy, int64_t lddy, float p,
                                          const void* rng, uint32_t site, void* dx, int64_t lddx, mdnn_dtype_t dtype,
                                          mdnn_stream_t stream) {
  return dropout_call("dropout_bwd", rows, cols, dy, lddy, nullptr, 0, p, rng, site, dx, lddx, dtype, stream);
}

extern "C" mdnn_status_t mdnn_layernorm_fwd(int64_t rows, int64_t cols, const void* x, int64_t ldx,
                                            const void* residual, int64_t ldr, float p, const void* rng, uint32_t site,
                                            const float* gamma, const float* beta, float eps, void* h, int64_t ldh,
                                            void* y, int64_t ldy, mdnn_dtype_t dtype, mdnn_stream_t stream) {
  const char* who = "layernorm_fwd";
  if (rows < 0 || cols < 1 || cols > MAX_COLS) return fail(MDNN_ERR_SHAPE, "%s: bad size", who);
  if (!(eps > 0.0f && std::isfinite(eps))) return fail(MDNN_ERR_SHAPE, "%s: eps must be positive and finite", who);
  if (!dtype_ok(dtype)) return fail(MDNN_ERR_DTYPE, "%s: unknown dtype", who);
  MDNN_TRY(check_drop(who, p, rng, rows));
  if (rows == 0) return MDNN_SUCCESS;
  if (!x || !y) return fail(MDNN_ERR_NULL, "%s: x or y is NULL", who);
  if (ldx < cols || ldy < cols || (residual && ldr < cols) || (h && ldh < cols))
    return fail(MDNN_ERR_LAYOUT, "%s: leading dimension below the width", who);
  const size_t es = dtype_size(dtype);
  if (!aligned(x, es) || !aligned(residual, es) || !aligned(h, es) || !aligned(y, es) || !aligned(gamma, 4) ||
      !aligned(beta, 4))
    return fail(MDNN_ERR_MISALIGNED, "%s: misaligned buffer", who);
  clear_error();
  LnArgs a = {};
  a.x = x, a.res = residual, a.gamma = gamma, a.beta = beta, a.h = h, a.y = y, a.rows = rows, a.cols = (int32_t)cols;
  a.ldx = ldx, a.ldr = ldr, a.ldh = ldh, a.ldy = ldy, a.eps = eps, a.d = drop_args(p, rng, site);
  const hipStream_t st = as_stream(stream);
  switch (dtype) {
    case MDNN_F32: return run_ln<F32>(a, st);
    case MDNN_F16: return run_ln<F16>(a, st);
    default: return run_ln<BF16>(a, st);
  }
}

extern "C" size_t mdnn_layernorm_bwd_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols < 1 || cols > MAX_COLS) return 0;
  const int64_t blocks = bwd_blocks(rows, cols);
  return blocks == 1 ? 0 : (size_t)blocks * 2 * (size_t)cols * 4;  // the blocks' sums
}

extern "C" mdnn_status_t mdnn_layernorm_bwd(int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* h,
                                            int64_t ldh, const float* gamma, float eps, const void* dres, int64_t lddr,
                                            float p, const void* rng, uint32_t site, void* dx, int64_t lddx, void* dh,
                                            int64_t lddh, float* dgamma, float* dbeta, mdnn_dtype_t dtype,
                                            void* workspace, size_t ws_bytes, mdnn_stream_t stream) {
  const char* who = "layernorm_bwd";
  if (rows < 0 || cols < 1 || cols > MAX_COLS) return fail(MDNN_ERR_SHAPE, "%s: bad size", who);
  if (!(eps > 0.0f && std::isfinite(eps))) return fail(MDNN_ERR_SHAPE, "%s: eps must be positive and finite", who);
  if (!dtype_ok(dtype)) return fail(MDNN_ERR_DTYPE, "%s: unknown dtype", who);
  MDNN_TRY(check_drop(who, p, rng, rows));
  if (!aligned(dgamma, 4) || !aligned(dbeta, 4)) return fail(MDNN_ERR_MISALIGNED, "%s: misaligned buffer", who);
  const hipStream_t st = as_stream(stream);
  if (rows == 0) {
    clear_error();
    if (dgamma) MDNN_TRY(fill_zero(dgamma, (size_t)cols * 4, st));
    return dbeta ? fill_zero(dbeta, (size_t)cols * 4, st) : MDNN_SUCCESS;
  }
  if (!dx && !dh && !dgamma && !dbeta) return MDNN_SUCCESS;
  if (!dy || !h) return fail(MDNN_ERR_NULL, "%s: dy or h is NULL", who);
  if (lddy < cols || ldh < cols || (dres && lddr < cols) || (dx && lddx < cols) || (dh && lddh < cols))
    return fail(MDNN_ERR_LAYOUT, "%s: leading dimension below the width", who);
  const size_t es = dtype_size(dtype);
  if (!aligned(dy, es) || !aligned(h, es) || !aligned(dres, es) || !aligned(dx, es) || !aligned(dh, es) ||
      !aligned(gamma, 4))
    return fail(MDNN_ERR_MISALIGNED, "%s: misaligned buffer", who);
  const bool sums = dgamma || dbeta;
  const size_t need = sums ? mdnn_layernorm_bwd_workspace(rows, cols) : 0;
  if (need > 0 && (!workspace || ws_bytes < need || !aligned(workspace, 256)))
    return fail(MDNN_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) required", who, need);
  clear_error();
  const int64_t blocks = bwd_blocks(rows, cols);
  LnBwdArgs a = {};
  a.dy = dy, a.h = h, a.dres = dres, a.gamma = gamma, a.dx = dx, a.dh = dh;
  // (a single block's sums are the gradients)
  a.pg = !dgamma || blocks == 1 ? dgamma : (float*)workspace;
  a.pb = !dbeta || blocks == 1 ? dbeta : (float*)workspace + cols;
  a.stride = 2 * cols;
  a.rows = rows, a.lddy = lddy, a.ldh = ldh, a.lddr = lddr, a.lddx = lddx, a.lddh = lddh, a.cols = (int32_t)cols;
  a.eps = eps, a.d = drop_args(p, rng, site);
  switch (dtype) {
    case MDNN_F32: MDNN_TRY(run_bwd<F32>(a, blocks, st)); break;
    case MDNN_F16: MDNN_TRY(run_bwd<F16>(a, blocks, st)); break;
    default: MDNN_TRY(run_bwd<BF16>(a, blocks, st)); break;
  }
  if (!sums || blocks == 1) return MDNN_SUCCESS;
  const int64_t tiles = ceil_div(cols, 32);
  hipLaunchKernelGGL(sums_kernel, dim3((unsigned)(tiles < MAX_BLOCKS / 2 ? tiles : MAX_BLOCKS / 2), 2), dim3(1024), 0, st,
                     (const float*)workspace, (int)blocks, cols, dgamma, dbeta);
  return check_launch("layernorm sums_kernel");
}

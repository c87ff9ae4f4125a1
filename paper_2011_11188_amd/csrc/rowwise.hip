// Row-wise operators around the 8-bit product: root-mean-square norm with the
// residual's addition (16-bit / fp32 or 8-bit output), its gradients, and the
// quantisers of rows and of columns.
//
//   h = x + res                                  (fp32; stored rounded once)
//   y = h * rstd * gamma,  rstd = 1 / sqrt(mean(h^2) + eps)
//   codes of a row t: a = max(max|t|, 2^-100), q = rint(fl(t * fl(127 / a))),
//   scale = fl(a / 127); for the norm t = fl(h * gamma) and the scale is
//   multiplied by rstd: rstd is common to the row, so it cancels from the
//   codes, and the sum of squares and the maximum need one pass over the row
//   and one reduction together.
//
// Bound: memory.  A row is read once, kept in registers (chunks of eight
// consecutive elements, TPR threads per row, NCH chunks per thread), reduced
// and written once.  Chunks are read and written at element alignment (one
// unaligned access each); a row's last, partial chunk is read from the row's
// last eight elements and the ones that belong to its neighbour are cleared,
// so every load is unconditional and lies inside the row.  Rows longer than
// the registers hold, or below eight elements, take the two-pass kernels.
#include <cmath>

#include "internal.h"
#include "row_chunk.h"

namespace mdnn {
namespace {

constexpr float A_MIN = 0x1p-100f;  // smallest row maximum the codes resolve (127 / a stays finite)

// Codes of four values: fl(t * inv) rounded to the nearest even integer (by
// adding 1.5 * 2^23, whose last place is 1), the low bytes packed.  The
// product is rounded before the addition: no contraction.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
#pragma clang fp contract(off)
  constexpr float MAGIC = 12582912.0f;
  const float pa = a * inv, pb = b * inv, pc = c * inv, pd = d * inv;
  const uint32_t ua = __float_as_uint(pa + MAGIC), ub = __float_as_uint(pb + MAGIC);
  const uint32_t uc = __float_as_uint(pc + MAGIC), ud = __float_as_uint(pd + MAGIC);
  const uint32_t lo = __builtin_amdgcn_perm(ub, ua, 0x0c0c0400u), hi = __builtin_amdgcn_perm(ud, uc, 0x0c0c0400u);
  return lo | (hi << 16);
}
__device__ __forceinline__ void store_codes(int8_t* p, uint32_t lo4, uint32_t hi4, int lo) {
  if (lo == 0) {
    *(MDNN_GLOBAL u2v_a1*)p = (u2v_a1){lo4, hi4};
  } else {
    asm("" : "+v"(lo));
#pragma unroll
    for (int e = 1; e < 8; ++e)
      if (e >= lo) p[e] = (int8_t)((e < 4 ? lo4 : hi4) >> (8 * (e & 3)));
  }
}

// From a row's largest magnitude (as bits: NaN above Inf above the rest) the
// factor of the codes and the scale; not finite: scale NaN, all codes 0.
struct RowScale {
  float inv, scale;
  uint32_t mask;  // 0: the codes are 0
};
__device__ __forceinline__ RowScale row_scale(uint32_t bits, bool bad) {
  RowScale r;
  if (bad || bits >= 0x7f800000u) {
    r.inv = 0.0f, r.scale = __builtin_nanf(""), r.mask = 0u;
  } else {
    const float f = __uint_as_float(bits), a = f > A_MIN ? f : A_MIN;
    r.inv = 127.0f / a, r.scale = a / 127.0f, r.mask = 0xffffffffu;
  }
  return r;
}

// 1 / sqrt(mean + eps); a sum that is not finite (the row holds Inf or NaN,
// or its squares pass fp32's range) makes the whole row NaN.
__device__ __forceinline__ float row_rstd(float ssq, float cols, float eps) {
  return isfinite(ssq) ? 1.0f / sqrtf(ssq / cols + eps) : __builtin_nanf("");
}

// Two sums, or a sum and a maximum of bit patterns, over a row's TPR threads,
// in a fixed order.  Rows of more than a wave combine their waves through one
// of two LDS buffers in turn (`flip`), so a loop over rows has one barrier.
struct SumMax {
  float s;
  uint32_t m;
};
template <int TPR>
__device__ __forceinline__ SumMax row_reduce(SumMax v, SumMax (*buf)[TPR / 64 + 1], int flip) {
  constexpr int W = TPR < 64 ? TPR : 64;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) {
    v.s += __shfl_xor(v.s, o, W);
    const uint32_t u = (uint32_t)__shfl_xor((int)v.m, o, W);
    v.m = u > v.m ? u : v.m;
  }
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) buf[flip][threadIdx.x >> 6] = v;
    __syncthreads();
    v = buf[flip][0];
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w) {
      const SumMax u = buf[flip][w];
      v.s += u.s;
      v.m = u.m > v.m ? u.m : v.m;
    }
  }
  return v;
}
enum RowMode { QUANT = 0, NORM = 1, NORM_I8 = 2 };

struct RowArgs {
  const void *x, *res;  // res: or null
  const float* gamma;   // or null (ones)
  void *h, *y;          // h: or null
  int8_t* q;
  float* scale;
  int64_t rows, ldx, ldr, ldh, ldy, ldq;
  int32_t cols;
  float eps;
};

template <class T, int MODE, int TPR, int NCH>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) row_kernel(RowArgs a) {
  typedef typename T::storage S;
  constexpr int NT = TPR < 256 ? 256 : TPR, RPB = NT / TPR;
  __shared__ SumMax buf[2][TPR / 64 + 1];
  const int t = threadIdx.x % TPR;
  ChunkPos pos[NCH];
#pragma unroll
  for (int i = 0; i < NCH; ++i) pos[i] = chunk_pos(t + i * TPR, a.cols);
  int flip = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB, flip ^= 1) {
    // (a thread group past the last row repeats it and stores nothing)
    const int64_t rw = r0 + threadIdx.x / TPR;
    const bool live = rw < a.rows;
    const int64_t row = live ? rw : a.rows - 1;
    Chunk<T> cx[NCH], cr[NCH];
#pragma unroll
    for (int i = 0; i < NCH; ++i) cx[i].load((const S*)a.x + row * a.ldx + pos[i].start);
    if (MODE != QUANT && a.res) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) cr[i].load((const S*)a.res + row * a.ldr + pos[i].start);
    }
    float h[NCH][8];
    SumMax v = {0.0f, 0u};
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      if (pos[i].lo > 0) cx[i].clear(pos[i].lo);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] = cx[i].get(e);
      if (MODE != QUANT && a.res) {
        if (pos[i].lo > 0) cr[i].clear(pos[i].lo);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] = add_rn(h[i][e], cr[i].get(e));
      }
      if (MODE != QUANT) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v.s = fmaf(h[i][e], h[i][e], v.s);
        if (a.h && live && pos[i].lo < 8) {
          Chunk<T> c;
          c.set(h[i]);
          c.store((S*)a.h + row * a.ldh + pos[i].start, pos[i].lo);
        }
        if (MODE == NORM_I8 && a.gamma) {
          Chunk<F32> g;
          g.load(a.gamma + pos[i].start);
#pragma unroll
          for (int e = 0; e < 8; ++e) h[i][e] = mul_rn(h[i][e], g.get(e));
        }
      }
      if (MODE != NORM) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t u = __float_as_uint(h[i][e]) & 0x7fffffffu;
          v.m = u > v.m ? u : v.m;
        }
      }
    }
    v = row_reduce<TPR>(v, buf, flip);
    const float rstd = MODE == QUANT ? 1.0f : row_rstd(v.s, (float)a.cols, a.eps);
    if (MODE == NORM) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        if (!live || pos[i].lo == 8) continue;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = h[i][e] * rstd;
        if (a.gamma) {
          Chunk<F32> g;
          g.load(a.gamma + pos[i].start);
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] *= g.get(e);
        }
        Chunk<T> c;
        c.set(y);
        c.store((S*)a.y + row * a.ldy + pos[i].start, pos[i].lo);
      }
    } else {
      const RowScale k = row_scale(v.m, MODE == NORM_I8 && !isfinite(v.s));
      if (live && t == 0) a.scale[row] = MODE == QUANT ? k.scale : k.scale * rstd;
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        if (!live || pos[i].lo == 8) continue;
        const uint32_t q0 = codes4(h[i][0], h[i][1], h[i][2], h[i][3], k.inv) & k.mask;
        const uint32_t q1 = codes4(h[i][4], h[i][5], h[i][6], h[i][7], k.inv) & k.mask;
        store_codes(a.q + row * a.ldq + pos[i].start, q0, q1, pos[i].lo);
      }
    }
  }
}

// Rows of any length, element by element, read again for each use, LONG_U
// elements of a thread in flight (past the row's end: its last element again,
// not used; one in flight: 4096 x 40000 bf16 725 us, eight 370).  A thread adds
// the elements in flight in fp32 and those sums in 64 bits: up to 2^19 elements
// fall to one, and in a chain of fp32 additions terms of one size lose their low
// bits on one side (2^26 columns of 0.1: the norm off by 2.7e-4).  A thread
// reads an element for the last time before it writes that element, so
// outputs may lie in place of the inputs as in the kernel above.
constexpr int LONG_U = 8;
template <class T>
struct LongRow {
  typedef typename T::storage S;
  float v[LONG_U];
  __device__ __forceinline__ void load(const S* p, int c0, int cols) {
#pragma unroll
    for (int u = 0; u < LONG_U; ++u) v[u] = to_f<T>(p[c0 + u * 1024 < cols ? c0 + u * 1024 : cols - 1]);
  }
};

template <class T, int MODE>
__global__ void __launch_bounds__(1024) row_long_kernel(RowArgs a) {
  typedef typename T::storage S;
  __shared__ SumMax buf[2][17];
  int flip = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, flip ^= 1) {
    const S* x = (const S*)a.x + row * a.ldx;
    const S* res = MODE != QUANT && a.res ? (const S*)a.res + row * a.ldr : nullptr;
    auto load = [&](int c0, LongRow<T>& h, LongRow<F32>& g) {
      LongRow<T> r;
      h.load(x, c0, a.cols);
      if (res) r.load(res, c0, a.cols);
      if (MODE != QUANT && a.gamma) g.load(a.gamma, c0, a.cols);
      if (res) {
#pragma unroll
        for (int u = 0; u < LONG_U; ++u) h.v[u] = add_rn(h.v[u], r.v[u]);
      }
    };
    LongRow<T> h;
    LongRow<F32> g;
    SumMax v = {0.0f, 0u};
    double sum = 0.0;
    for (int c0 = threadIdx.x; c0 < a.cols; c0 += LONG_U * 1024) {
      load(c0, h, g);
      float s = 0.0f;
#pragma unroll
      for (int u = 0; u < LONG_U; ++u) {
        if (c0 + u * 1024 >= a.cols) continue;
        float t = h.v[u];
        if (MODE != QUANT) s = fmaf(t, t, s);
        if (MODE == NORM_I8 && a.gamma) t = mul_rn(t, g.v[u]);
        const uint32_t b = __float_as_uint(t) & 0x7fffffffu;
        v.m = b > v.m ? b : v.m;
      }
      if (MODE != QUANT) sum += (double)s;
    }
    v.s = (float)sum;
    v = row_reduce<1024>(v, buf, flip);
    const float rstd = MODE == QUANT ? 1.0f : row_rstd(v.s, (float)a.cols, a.eps);
    const RowScale k = row_scale(v.m, MODE == NORM_I8 && !isfinite(v.s));
    if (MODE != NORM && threadIdx.x == 0) a.scale[row] = MODE == QUANT ? k.scale : k.scale * rstd;
    for (int c0 = threadIdx.x; c0 < a.cols; c0 += LONG_U * 1024) {
      load(c0, h, g);
#pragma unroll
      for (int u = 0; u < LONG_U; ++u) {
        const int c = c0 + u * 1024;
        if (c >= a.cols) continue;
        if (MODE != QUANT && a.h) ((S*)a.h + row * a.ldh)[c] = from_f<T>(h.v[u]);
        if (MODE == NORM) {
          float y = h.v[u] * rstd;
          if (a.gamma) y *= g.v[u];
          ((S*)a.y + row * a.ldy)[c] = from_f<T>(y);
        } else {
          const float t = MODE == NORM_I8 && a.gamma ? mul_rn(h.v[u], g.v[u]) : h.v[u];
          a.q[row * a.ldq + c] = (int8_t)(codes4(t, 0.0f, 0.0f, 0.0f, k.inv) & k.mask);
        }
      }
    }
  }
}

template <class T, int MODE, int TPR, int NCH>
void launch_rows(const RowArgs& a, hipStream_t st) {
  constexpr int NT = TPR < 256 ? 256 : TPR, RPB = NT / TPR;
  const int64_t blocks = ceil_div(a.rows, RPB);
  hipLaunchKernelGGL((row_kernel<T, MODE, TPR, NCH>), dim3((unsigned)(blocks < MAX_BLOCKS ? blocks : MAX_BLOCKS)),
                     dim3(NT), 0, st, a);
}

// One or two chunks a thread, as few threads of a row idle as that allows
// (8192 x 1024 bf16, 128 chunks, with codes: 64 threads x 2 chunks 11.4 us,
// 256 x 1 15.5; 4096 x 4096: 256 x 2 19.4 us, 512 x 1 21.6, 64 x 8 25.0;
// 8192 x 8192: 512 x 2 83.9 us, 256 x 4 90.6): the chunks' conversions, not the
// loads in flight, tell the shapes apart.
template <class T, int MODE>
mdnn_status_t run_rows_t(const RowArgs& a, hipStream_t st) {
  const int64_t nch = ceil_div(a.cols, 8);
  if (a.cols < 8 || nch > 4096) {
    const int64_t blocks = a.rows < MAX_BLOCKS ? a.rows : MAX_BLOCKS;
    hipLaunchKernelGGL((row_long_kernel<T, MODE>), dim3((unsigned)blocks), dim3(1024), 0, st, a);
  } else if (nch <= 16) {
    launch_rows<T, MODE, 16, 1>(a, st);
  } else if (nch <= 32) {
    launch_rows<T, MODE, 16, 2>(a, st);
  } else if (nch <= 64) {
    launch_rows<T, MODE, 64, 1>(a, st);
  } else if (nch <= 128) {
    launch_rows<T, MODE, 64, 2>(a, st);
  } else if (nch <= 256) {
    launch_rows<T, MODE, 256, 1>(a, st);
  } else if (nch <= 512) {
    launch_rows<T, MODE, 256, 2>(a, st);
  } else if (nch <= 1024) {
    launch_rows<T, MODE, 512, 2>(a, st);
  } else if (nch <= 2048) {
    launch_rows<T, MODE, 512, 4>(a, st);
  } else {
    launch_rows<T, MODE, 1024, 4>(a, st);
  }
  return check_launch("row_kernel");
}

template <int MODE>
mdnn_status_t run_rows(const RowArgs& a, mdnn_dtype_t t, hipStream_t st) {
  clear_error();
  switch (t) {
    case MDNN_F32: return run_rows_t<F32, MODE>(a, st);
    case MDNN_F16: return run_rows_t<F16, MODE>(a, st);
    default: return run_rows_t<BF16, MODE>(a, st);
  }
}

// ---------------------------------------------------------------------------
// gradients of the norm
//   g = dy * gamma, xh = h * rstd, c = mean(g * xh)
//   dx = rstd * (g - xh * c) + dres,  dgamma = sum over rows of dy * xh
// One reduction per row for sum h^2 and sum g * h together.  Blocks of 512
// threads, two to a CU, walk their rows and keep the dgamma sums of their
// threads' columns in registers; a block writes them once, and the blocks'
// sums are added in a fixed order.  Loading the next row ahead gained nothing
// (4096 x 4096 bf16: 28.4 us against 28.1: the other block's loads fill the gap),
// blocks of 1024 threads wait for each other (28.6; 8192 x 8192 114 against 109).
// Bound by HBM: 4096 x 4096 fp16 32 us from memory with the blocks' sums (4.4 TB/s).
// ---------------------------------------------------------------------------
constexpr int BWD_NT(int tpr) { return tpr <= 512 ? 512 : 1024; }
struct BwdArgs {
  const void *dy, *h, *dres;  // dres: or null
  const float* gamma;         // or null
  void* dx;                   // or null
  float* partial;             // [blocks][cols], or null
  int64_t rows, lddy, ldh, lddr, lddx;
  int32_t cols;
  float eps;
};

template <class T, int TPR, int NCH>
__global__ void __launch_bounds__(BWD_NT(TPR)) norm_bwd_kernel(BwdArgs a) {
  typedef typename T::storage S;
  constexpr int NT = BWD_NT(TPR), RPB = NT / TPR, WIDE = TPR * NCH * 8;
  __shared__ Sum2 buf[2][RPB][TPR / 64 + 1];
  __shared__ __attribute__((aligned(16))) float part[RPB > 1 ? RPB * WIDE : 1];
  const int t = threadIdx.x % TPR, grp = threadIdx.x / TPR;
  ChunkPos pos[NCH];
  float dg[NCH][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    pos[i] = chunk_pos(t + i * TPR, a.cols);
#pragma unroll
    for (int e = 0; e < 8; ++e) dg[i][e] = 0.0f;
  }
  // (fp32 rows over 1024 threads fill the registers: gamma and the residual's gradient are read late)
  constexpr bool LATE = TPR == 1024 && !Chunk<T>::H;
  int flip = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < a.rows; r0 += (int64_t)gridDim.x * RPB, flip ^= 1) {
    const float* gamma = a.gamma;
    if (LATE) asm("" : "+s"(gamma));  // (read again for every row)
    const bool live = r0 + grp < a.rows;
    const int64_t row = live ? r0 + grp : a.rows - 1;  // (past the last row: repeated, nothing stored)
    Chunk<T> cd[NCH], ch[NCH], cr[NCH];
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      cd[i].load((const S*)a.dy + row * a.lddy + pos[i].start);
      ch[i].load((const S*)a.h + row * a.ldh + pos[i].start);
    }
    if (a.dres && !LATE) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) cr[i].load((const S*)a.dres + row * a.lddr + pos[i].start);
    }
    Sum2 v = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      Chunk<F32> g;
      if (gamma) g.load(gamma + pos[i].start);
      if (pos[i].lo > 0) ch[i].clear(pos[i].lo), cd[i].clear(pos[i].lo);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float h = ch[i].get(e), d = cd[i].get(e);
        v.a = fmaf(h, h, v.a);
        v.b = fmaf(gamma ? d * g.get(e) : d, h, v.b);
      }
    }
    v = row_reduce<TPR, RPB>(v, buf, flip);
    const float rstd = row_rstd(v.a, (float)a.cols, a.eps), c = rstd * v.b / (float)a.cols;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      if (!live || pos[i].lo == 8) continue;
      Chunk<F32> g;
      if (gamma) g.load(gamma + pos[i].start);
      if (a.dres && LATE) cr[i].load((const S*)a.dres + row * a.lddr + pos[i].start);
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xh = ch[i].get(e) * rstd, d = cd[i].get(e);
        o[e] = rstd * ((gamma ? d * g.get(e) : d) - xh * c);
        if (a.dres) o[e] += cr[i].get(e);
        dg[i][e] = fmaf(d, xh, dg[i][e]);
      }
      if (a.dx) {
        Chunk<T> w;
        w.set(o);
        w.store((S*)a.dx + row * a.lddx + pos[i].start, pos[i].lo);
      }
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (int64_t)blockIdx.x * a.cols;
  if constexpr (RPB > 1) {
    // the block's row groups, added in their order
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int e = 0; e < 8; e += 4)
        *(float4*)&part[grp * WIDE + (t + i * TPR) * 8 + e] = make_float4(dg[i][e], dg[i][e + 1], dg[i][e + 2], dg[i][e + 3]);
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += NT) {
      // column c's place: its chunk's slot, counted from the row's end in the last, partial chunk
      const int k = c / 8, at = k * 8 + (c - chunk_pos(k, a.cols).start);
      float s = part[at];
#pragma unroll
      for (int r = 1; r < RPB; ++r) s += part[r * WIDE + at];
      out[c] = s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      if (pos[i].lo == 8) continue;
      Chunk<F32> w;
      w.set(dg[i]);
      w.store(out + pos[i].start, pos[i].lo);
    }
  }
}

// dgamma from the blocks' sums: 32 columns a block, 32 rows of threads, each
// adding every 32nd block's sums (sixteen loads in flight), then those in
// order.  4.8 us for 512 blocks of 4096 columns: a launch and one round trip.
__global__ void __launch_bounds__(1024) dgamma_kernel(const float* partial, int blocks, int64_t cols, float* dgamma) {
  __shared__ float part[32][32];
  const int cx = threadIdx.x & 31, r = threadIdx.x >> 5;
  for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < cols; c0 += (int64_t)gridDim.x * 32) {
    const int64_t c = c0 + cx;
    const float* p = partial + (c < cols ? c : cols - 1);
    float s = 0.0f;
    for (int b0 = r; b0 < blocks; b0 += 512) {
      float v[16];
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = p[(int64_t)(b0 + 32 * k < blocks ? b0 + 32 * k : r) * cols];
#pragma unroll
      for (int k = 0; k < 16; ++k) s += b0 + 32 * k < blocks ? v[k] : 0.0f;
    }
    part[r][cx] = s;
    __syncthreads();
    if (r == 0 && c < cols) {
#pragma unroll
      for (int k = 1; k < 32; ++k) s += part[k][cx];
      dgamma[c] = s;
    }
    __syncthreads();  // (before the sums of the next columns)
  }
}

// Rows of any length: read twice, dgamma's sums kept in the block's own row
// of the partials.  Rows below eight elements (NARROW) come by the million: a
// thread keeps its one column's sum in 64 bits and writes it at the end (as a
// chain in fp32 it was 1.7e-4 off over 2^22 rows of one value).
template <class T, bool NARROW>
__global__ void __launch_bounds__(1024) norm_bwd_long_kernel(BwdArgs a) {
  typedef typename T::storage S;
  __shared__ Sum2 buf[2][1][17];
  double own = 0.0;
  int flip = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, flip ^= 1) {
    const S *dy = (const S*)a.dy + row * a.lddy, *hp = (const S*)a.h + row * a.ldh;
    LongRow<T> h, d, r;
    LongRow<F32> g, p;
    double sum_a = 0.0, sum_b = 0.0;
    for (int c0 = threadIdx.x; c0 < a.cols; c0 += LONG_U * 1024) {
      h.load(hp, c0, a.cols);
      d.load(dy, c0, a.cols);
      if (a.gamma) g.load(a.gamma, c0, a.cols);
      Sum2 s = {0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < LONG_U; ++u) {
        if (c0 + u * 1024 >= a.cols) continue;
        s.a = fmaf(h.v[u], h.v[u], s.a);
        s.b = fmaf(a.gamma ? d.v[u] * g.v[u] : d.v[u], h.v[u], s.b);
      }
      sum_a += (double)s.a, sum_b += (double)s.b;
    }
    const Sum2 v = row_reduce<1024, 1>(Sum2{(float)sum_a, (float)sum_b}, buf, flip);
    const float rstd = row_rstd(v.a, (float)a.cols, a.eps), k = rstd * v.b / (float)a.cols;
    float* sums = a.partial && !NARROW ? a.partial + (int64_t)blockIdx.x * a.cols : nullptr;
    const bool first = row == (int64_t)blockIdx.x;
    for (int c0 = threadIdx.x; c0 < a.cols; c0 += LONG_U * 1024) {
      h.load(hp, c0, a.cols);
      d.load(dy, c0, a.cols);
      if (a.gamma) g.load(a.gamma, c0, a.cols);
      if (a.dres) r.load((const S*)a.dres + row * a.lddr, c0, a.cols);
      if (sums && !first) p.load(sums, c0, a.cols);
#pragma unroll
      for (int u = 0; u < LONG_U; ++u) {
        const int c = c0 + u * 1024;
        if (c >= a.cols) continue;
        const float xh = h.v[u] * rstd;
        float o = rstd * ((a.gamma ? d.v[u] * g.v[u] : d.v[u]) - xh * k);
        if (a.dres) o += r.v[u];
        if (sums) sums[c] = first ? d.v[u] * xh : fmaf(d.v[u], xh, p.v[u]);
        if (NARROW) own += (double)d.v[u] * (double)xh;  // (one column a thread)
        if (a.dx) ((S*)a.dx + row * a.lddx)[c] = from_f<T>(o);
      }
    }
  }
  if (NARROW && a.partial && (int)threadIdx.x < a.cols) a.partial[(int64_t)blockIdx.x * a.cols + threadIdx.x] = (float)own;
}

// Threads per row of the backward pass by the row's chunks; 0: the long-row kernel.
int bwd_tpr(int64_t cols) {
  const int64_t nch = ceil_div(cols, 8);
  return cols < 8 || nch > 2048 ? 0 : nch <= 32 ? 16 : nch <= 128 ? 64 : nch <= 512 ? 256 : nch <= 1024 ? 512 : 1024;
}
// Its blocks (as many as the chip runs at once): by the sizes alone, so that
// the workspace and the order of dgamma's sums are the same everywhere.
int64_t bwd_blocks(int64_t rows, int64_t cols) {
  const int tpr = bwd_tpr(cols);
  const int64_t b = ceil_div(rows, tpr == 0 ? 1 : BWD_NT(tpr) / tpr), most = tpr == 0 || tpr == 1024 ? 256 : 512;
  // A single block needs no second launch: worth up to three rows a thread
  // group of 16 (96 x 112 bf16 5.3 us, over two launches 5.7), two of 64 or 256
  // (16 x 1000 5.7 and 6.5, 4 x 4096 6.3 and 6.9; 24 x 1000 7.5 and 6.5).
  const int64_t alone = tpr == 16 ? 3 : tpr == 64 || tpr == 256 ? 2 : 1;
  return b <= alone ? 1 : b < most ? b : most;
}

template <class T, int TPR, int NCH>
void launch_bwd(const BwdArgs& a, int64_t blocks, hipStream_t st) {
  hipLaunchKernelGGL((norm_bwd_kernel<T, TPR, NCH>), dim3((unsigned)blocks), dim3(BWD_NT(TPR)), 0, st, a);
}

template <class T>
mdnn_status_t run_bwd(const BwdArgs& a, hipStream_t st) {
  const int64_t nch = ceil_div(a.cols, 8), blocks = bwd_blocks(a.rows, a.cols);
  if (a.cols < 8)
    hipLaunchKernelGGL((norm_bwd_long_kernel<T, true>), dim3((unsigned)blocks), dim3(1024), 0, st, a);
  else if (bwd_tpr(a.cols) == 0)
    hipLaunchKernelGGL((norm_bwd_long_kernel<T, false>), dim3((unsigned)blocks), dim3(1024), 0, st, a);
  else if (nch <= 16)
    launch_bwd<T, 16, 1>(a, blocks, st);
  else if (nch <= 32)
    launch_bwd<T, 16, 2>(a, blocks, st);
  else if (nch <= 64)
    launch_bwd<T, 64, 1>(a, blocks, st);
  else if (nch <= 128)
    launch_bwd<T, 64, 2>(a, blocks, st);
  else if (nch <= 256)
    launch_bwd<T, 256, 1>(a, blocks, st);
  else if (nch <= 512)
    launch_bwd<T, 256, 2>(a, blocks, st);
  else if (nch <= 1024)
    launch_bwd<T, 512, 2>(a, blocks, st);
  else
    launch_bwd<T, 1024, 2>(a, blocks, st);
  return check_launch("norm_bwd_kernel");
}

// ---------------------------------------------------------------------------
// columns: codes of x[rows][cols] with a scale for each column, stored
// transposed, q[cols][rows].  Pass 1: column maxima of row slabs; pass 2:
// every tile takes its columns' maxima over the slabs, quantises and turns
// the tile round in LDS.  Bound by x's two reads, the second from the
// last-level cache where it fits: 4096 x 4096 fp32 25 us, 11.0 (6.1 TB/s) and
// 14.4 us (5.8 TB/s).
// ---------------------------------------------------------------------------
// Rows of a slab: about a thousand blocks of 256 columns in pass 1, at most
// 256 slabs (every tile of pass 2 reads its columns' maxima of each).
int64_t slab_rows(int64_t rows, int64_t cols) {
  int64_t most = ceil_div(1024, ceil_div(cols, 256));
  most = most > 256 ? 256 : most;
  const int64_t per = ceil_div(ceil_div(rows, most), 16) * 16;
  return per < 32 ? 32 : per;
}
// (none where one tile holds all rows: it takes its own maxima, in one launch;
// 128 x 4096 bf16 6.7 -> 3.7 us)
constexpr int QT_C = 64, QT_R = 128;  // tile of pass 2: columns, rows
int64_t slab_count(int64_t rows, int64_t cols) { return rows > QT_R && cols > 0 ? ceil_div(rows, slab_rows(rows, cols)) : 0; }

// Four consecutive elements of a row: those from `start` (a quad past the
// row's end starts at its last four and overlaps its neighbour), or, in rows
// below four columns (NARROW), its elements with the last repeated.
template <class T, bool NARROW>
__device__ __forceinline__ Quad<T> load_quad(const typename T::storage* row, int64_t start, int64_t cols) {
  Quad<T> q;
  if constexpr (!NARROW) {
    q.load(row + start);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const typename T::storage v = row[e < cols ? e : cols - 1];
      if constexpr (!Quad<T>::H)
        q.q[e] = __float_as_uint(v);
      else if (e & 1)
        q.q[e >> 1] |= (uint32_t)v << 16;
      else
        q.q[e >> 1] = v;
    }
  }
  return q;
}
template <bool NARROW>
__device__ __forceinline__ int64_t quad_start(int64_t c, int64_t cols) {
  return NARROW ? 0 : c + 4 <= cols ? c : cols - 4;
}

template <class T, bool NARROW>
__global__ void __launch_bounds__(256)
colmax_kernel(const typename T::storage* x, int64_t ldx, int64_t rows, int64_t cols, int64_t per, uint32_t* partial) {
  __shared__ uint32_t red[4][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c0 = (int64_t)blockIdx.x * 256, start = quad_start<NARROW>(c0 + lane * 4, cols);
  const int64_t r0 = (int64_t)blockIdx.y * per, r1 = r0 + per < rows ? r0 + per : rows;
  uint32_t m[4] = {0u, 0u, 0u, 0u};
  for (int64_t r = r0 + wave; r < r1; r += 32) {
    Quad<T> v[8];  // eight rows in flight (past the slab: the first again)
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = load_quad<T, NARROW>(x + (r + 4 * k < r1 ? r + 4 * k : r) * ldx, start, cols);
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t u = __float_as_uint(v[k].get(e)) & 0x7fffffffu;
        m[e] = u > m[e] ? u : m[e];
      }
  }
  // (lanes whose quads overlap write the same values)
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (start + e >= c0) red[wave][start + e - c0] = m[e];
  __syncthreads();
  if (c0 + threadIdx.x >= cols) return;
  uint32_t v = red[0][threadIdx.x];
#pragma unroll
  for (int w = 1; w < 4; ++w) v = red[w][threadIdx.x] > v ? red[w][threadIdx.x] : v;
  partial[(int64_t)blockIdx.y * cols + c0 + threadIdx.x] = v;
}

template <class T, bool NARROW>
__global__ void __launch_bounds__(256)
quant_t_kernel(const typename T::storage* x, int64_t ldx, int64_t rows, int64_t cols, const uint32_t* partial,
               int slabs, int8_t* q, int64_t ldq, float* scale) {
  // (three columns of room before the tile's: a last tile of fewer than four columns starts its quads before it)
  __shared__ uint32_t top[16][QT_C + 4];
  __shared__ float inv[QT_C + 3];
  __shared__ uint32_t mask[QT_C + 3];
  __shared__ uint32_t tile[QT_C + 3][QT_R / 4 + 1];
  const int tid = threadIdx.x, part = tid >> 4;
  const int64_t c0 = (int64_t)blockIdx.x * QT_C, start = quad_start<NARROW>(c0 + (tid & 15) * 4, cols);
  const int cq = (int)(start - c0) + 3;
  // the columns' maxima over the slabs: a quad of columns and every 16th slab
  // a thread; 4 x 4 blocks of the tile, four rows' quads, are read meanwhile
  Quad<F32> u[4];
  auto load_top = [&](int s0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int s = s0 + 16 * k < slabs ? s0 + 16 * k : slabs - 1;
      u[k] = load_quad<F32, NARROW>((const float*)partial + (int64_t)s * cols, start, cols);
    }
  };
  uint32_t m[4] = {0u, 0u, 0u, 0u};
  auto take_top = [&] {
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) m[e] = u[k].q[e] > m[e] ? u[k].q[e] : m[e];
  };
  Quad<T> v[QT_R / 64][4];
  auto load = [&](int64_t r0) {
#pragma unroll
    for (int p = 0; p < QT_R / 64; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t r = r0 + (part + p * 16) * 4 + e;  // (past the last row: the last again, never stored)
        v[p][e] = load_quad<T, NARROW>(x + (r < rows ? r : rows - 1) * ldx, start, cols);
      }
  };
  int64_t r0 = (int64_t)blockIdx.y * QT_R;
  if (slabs == 0 && rows > 0) {
    load(r0);
#pragma unroll
    for (int p = 0; p < QT_R / 64; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t b = __float_as_uint(v[p][e].get(j)) & 0x7fffffffu;
          m[j] = b > m[j] ? b : m[j];
        }
  } else if (slabs > 0) {
    load_top(part);
    load(r0);
    take_top();
    for (int s = part + 64; s < slabs; s += 64) {
      load_top(s);
      take_top();
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (cq + e >= 3) top[part][cq + e - 3] = m[e];
  __syncthreads();
  if (tid < QT_C) {
    uint32_t b = top[0][tid];
#pragma unroll
    for (int p = 1; p < 16; ++p) b = top[p][tid] > b ? top[p][tid] : b;
    const RowScale k = row_scale(b, false);
    inv[tid + 3] = k.inv;
    mask[tid + 3] = k.mask;
    if (blockIdx.y == 0 && c0 + tid < cols) scale[c0 + tid] = k.scale;
  }
  __syncthreads();
  typedef uint32_t u1_a1 __attribute__((aligned(1)));
  while (r0 < rows) {
    // one word of four rows per column
#pragma unroll
    for (int p = 0; p < QT_R / 64; ++p)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        tile[cq + j][part + p * 16] =
            codes4(v[p][0].get(j), v[p][1].get(j), v[p][2].get(j), v[p][3].get(j), inv[cq + j]) & mask[cq + j];
    const int64_t next = r0 + (int64_t)gridDim.y * QT_R;
    if (next < rows) load(next);
    __syncthreads();
    const int w = tid % (QT_R / 4), cc = tid / (QT_R / 4);
    int8_t* o = q + (c0 + cc) * ldq + r0 + w * 4;
    if (r0 + QT_R <= rows && c0 + QT_C <= cols) {
#pragma unroll
      for (int p = 0; p < QT_C / 8; ++p) *(MDNN_GLOBAL u1_a1*)(o + p * 8 * ldq) = tile[cc + p * 8 + 3][w];
    } else {
      const int64_t left = rows - r0 - w * 4;
      for (int p = 0; p < QT_C / 8; ++p) {
        if (c0 + cc + p * 8 >= cols) break;
        const uint32_t w4 = tile[cc + p * 8 + 3][w];
        if (left >= 4) {
          *(MDNN_GLOBAL u1_a1*)(o + p * 8 * ldq) = w4;
        } else {
          for (int e = 0; e < left; ++e) o[p * 8 * ldq + e] = (int8_t)(w4 >> (8 * e));
        }
      }
    }
    __syncthreads();
    r0 = next;
  }
}

template <class T, bool NARROW>
mdnn_status_t launch_quant_t(int64_t rows, int64_t cols, const void* x, int64_t ldx, int8_t* q, int64_t ldq,
                             float* scale, uint32_t* partial, hipStream_t st) {
  typedef typename T::storage S;
  const int64_t slabs = slab_count(rows, cols);
  if (slabs > 0) {
    hipLaunchKernelGGL((colmax_kernel<T, NARROW>), dim3((unsigned)ceil_div(cols, 256), (unsigned)slabs), dim3(256), 0,
                       st, (const S*)x, ldx, rows, cols, slab_rows(rows, cols), partial);
    MDNN_TRY(check_launch("colmax_kernel"));
  }
  int64_t gy = ceil_div(rows, QT_R);
  gy = gy < 1 ? 1 : gy > 65535 ? 65535 : gy;
  hipLaunchKernelGGL((quant_t_kernel<T, NARROW>), dim3((unsigned)ceil_div(cols, QT_C), (unsigned)gy), dim3(256), 0, st,
                     (const S*)x, ldx, rows, cols, partial, (int)slabs, q, ldq, scale);
  return check_launch("quant_t_kernel");
}

template <class T>
mdnn_status_t run_quant_t(int64_t rows, int64_t cols, const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale,
                          uint32_t* partial, hipStream_t st) {
  return cols < 4 ? launch_quant_t<T, true>(rows, cols, x, ldx, q, ldq, scale, partial, st)
                  : launch_quant_t<T, false>(rows, cols, x, ldx, q, ldq, scale, partial, st);
}

constexpr int64_t MAX_COLS = (int64_t)1 << 29;  // 32-bit column indices; a launch holds fewer than 2^32 threads a dimension

bool eps_ok(float eps) { return eps > 0.0f && std::isfinite(eps); }

}  // namespace
}  // namespace mdnn

using namespace mdnn;

extern "C" mdnn_status_t mdnn_quantize_i8(int64_t rows, int64_t cols, const void* x, int64_t ldx, mdnn_dtype_t x_type,
                                          int8_t* q, int64_t ldq, float* scale, mdnn_stream_t stream) {
  if (rows < 0 || cols < 0 || cols > MAX_COLS) return fail(MDNN_ERR_SHAPE, "quantize_i8: bad size");
  if (!dtype_ok(x_type)) return fail(MDNN_ERR_DTYPE, "quantize_i8: unknown dtype");
  if (rows == 0) return MDNN_SUCCESS;
  if (!scale || (cols > 0 && (!x || !q))) return fail(MDNN_ERR_NULL, "quantize_i8: NULL buffer");
  if (ldx < cols || ldq < cols) return fail(MDNN_ERR_LAYOUT, "quantize_i8: leading dimension below the width");
  if (!aligned(x, dtype_size(x_type)) || !aligned(scale, 4))
    return fail(MDNN_ERR_MISALIGNED, "quantize_i8: misaligned buffer");
  RowArgs a = {};
  a.x = x, a.q = q, a.scale = scale, a.rows = rows, a.cols = (int32_t)cols, a.ldx = ldx, a.ldq = ldq;
  return run_rows<QUANT>(a, x_type, as_stream(stream));
}

extern "C" size_t mdnn_quantize_i8_t_workspace(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || cols > MAX_COLS) return 0;
  return (size_t)slab_count(rows, cols) * (size_t)cols * 4;
}

extern "C" mdnn_status_t mdnn_quantize_i8_t(int64_t rows, int64_t cols, const void* x, int64_t ldx,
                                            mdnn_dtype_t x_type, int8_t* q, int64_t ldq, float* scale, void* workspace,
                                            size_t ws_bytes, mdnn_stream_t stream) {
  if (rows < 0 || cols < 0 || cols > MAX_COLS) return fail(MDNN_ERR_SHAPE, "quantize_i8_t: bad size");
  if (!dtype_ok(x_type)) return fail(MDNN_ERR_DTYPE, "quantize_i8_t: unknown dtype");
  if (cols == 0) return MDNN_SUCCESS;
  if (!scale || (rows > 0 && (!x || !q))) return fail(MDNN_ERR_NULL, "quantize_i8_t: NULL buffer");
  if (ldx < cols || ldq < rows) return fail(MDNN_ERR_LAYOUT, "quantize_i8_t: leading dimension below the width");
  if (!aligned(x, dtype_size(x_type)) || !aligned(scale, 4))
    return fail(MDNN_ERR_MISALIGNED, "quantize_i8_t: misaligned buffer");
  const size_t need = mdnn_quantize_i8_t_workspace(rows, cols);
  if (need > 0 && (!workspace || ws_bytes < need || !aligned(workspace, 16)))
    return fail(MDNN_ERR_WORKSPACE, "quantize_i8_t: workspace of %zu bytes (16-byte aligned) required", need);
  clear_error();
  const hipStream_t st = as_stream(stream);
  switch (x_type) {
    case MDNN_F32: return run_quant_t<F32>(rows, cols, x, ldx, q, ldq, scale, (uint32_t*)workspace, st);
    case MDNN_F16: return run_quant_t<F16>(rows, cols, x, ldx, q, ldq, scale, (uint32_t*)workspace, st);
    default: return run_quant_t<BF16>(rows, cols, x, ldx, q, ldq, scale, (uint32_t*)workspace, st);
  }
}

// Checks and arguments that both forward norms share.
static mdnn_status_t norm_args(const char* who, RowArgs& a, int64_t rows, int64_t cols, const void* x, int64_t ldx,
                               const void* residual, int64_t ldr, const float* gamma, float eps, void* h, int64_t ldh,
                               mdnn_dtype_t dtype) {
  if (rows < 0 || cols < 1 || cols > MAX_COLS) return fail(MDNN_ERR_SHAPE, "%s: bad size", who);
  if (!eps_ok(eps)) return fail(MDNN_ERR_SHAPE, "%s: eps must be positive and finite", who);
  if (!dtype_ok(dtype)) return fail(MDNN_ERR_DTYPE, "%s: unknown dtype", who);
  if (rows == 0) return MDNN_SUCCESS;
  if (!x) return fail(MDNN_ERR_NULL, "%s: x is NULL", who);
  if (ldx < cols || (residual && ldr < cols) || (h && ldh < cols))
    return fail(MDNN_ERR_LAYOUT, "%s: leading dimension below the width", who);
  const size_t es = dtype_size(dtype);
  if (!aligned(x, es) || !aligned(residual, es) || !aligned(h, es) || !aligned(gamma, 4))
    return fail(MDNN_ERR_MISALIGNED, "%s: misaligned buffer", who);
  a = {};
  a.x = x, a.res = residual, a.gamma = gamma, a.h = h, a.rows = rows, a.cols = (int32_t)cols;
  a.ldx = ldx, a.ldr = ldr, a.ldh = ldh, a.eps = eps;
  return MDNN_SUCCESS;
}

extern "C" mdnn_status_t mdnn_rmsnorm_fwd(int64_t rows, int64_t cols, const void* x, int64_t ldx,
                                          const void* residual, int64_t ldr, const float* gamma, float eps, void* h,
                                          int64_t ldh, void* y, int64_t ldy, mdnn_dtype_t dtype,
                                          mdnn_stream_t stream) {
  RowArgs a;
  MDNN_TRY(norm_args("rmsnorm_fwd", a, rows, cols, x, ldx, residual, ldr, gamma, eps, h, ldh, dtype));
  if (rows == 0) return MDNN_SUCCESS;
  if (!y) return fail(MDNN_ERR_NULL, "rmsnorm_fwd: y is NULL");
  if (ldy < cols) return fail(MDNN_ERR_LAYOUT, "rmsnorm_fwd: leading dimension below the width");
  if (!aligned(y, dtype_size(dtype))) return fail(MDNN_ERR_MISALIGNED, "rmsnorm_fwd: misaligned buffer");
  a.y = y, a.ldy = ldy;
  return run_rows<NORM>(a, dtype, as_stream(stream));
}

extern "C" mdnn_status_t mdnn_rmsnorm_i8_fwd(int64_t rows, int64_t cols, const void* x, int64_t ldx,
                                             const void* residual, int64_t ldr, const float* gamma, float eps, void* h,
                                             int64_t ldh, int8_t* q, int64_t ldq, float* scale, mdnn_dtype_t dtype,
                                             mdnn_stream_t stream) {
  RowArgs a;
  MDNN_TRY(norm_args("rmsnorm_i8_fwd", a, rows, cols, x, ldx, residual, ldr, gamma, eps, h, ldh, dtype));
  if (rows == 0) return MDNN_SUCCESS;
  if (!q || !scale) return fail(MDNN_ERR_NULL, "rmsnorm_i8_fwd: q or scale is NULL");
  if (ldq < cols) return fail(MDNN_ERR_LAYOUT, "rmsnorm_i8_fwd: leading dimension below the width");
  if (!aligned(scale, 4)) return fail(MDNN_ERR_MISALIGNED, "rmsnorm_i8_fwd: misaligned buffer");
  a.q = q, a.ldq = ldq, a.scale = scale;
  return run_rows<NORM_I8>(a, dtype, as_stream(stream));
}

extern "C" size_t mdnn_rmsnorm_bwd_workspace(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols < 1 || cols > MAX_COLS) return 0;
  return (size_t)bwd_blocks(rows, cols) * (size_t)cols * 4;  // the blocks' sums
}

extern "C" mdnn_status_t mdnn_rmsnorm_bwd(int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* h,
                                          int64_t ldh, const float* gamma, float eps, const void* dres, int64_t lddr,
                                          void* dx, int64_t lddx, float* dgamma, mdnn_dtype_t dtype, void* workspace,
                                          size_t ws_bytes, mdnn_stream_t stream) {
  if (rows < 0 || cols < 1 || cols > MAX_COLS) return fail(MDNN_ERR_SHAPE, "rmsnorm_bwd: bad size");
  if (!eps_ok(eps)) return fail(MDNN_ERR_SHAPE, "rmsnorm_bwd: eps must be positive and finite");
  if (!dtype_ok(dtype)) return fail(MDNN_ERR_DTYPE, "rmsnorm_bwd: unknown dtype");
  if (dgamma && !aligned(dgamma, 4)) return fail(MDNN_ERR_MISALIGNED, "rmsnorm_bwd: misaligned buffer");
  const hipStream_t st = as_stream(stream);
  if (rows == 0) {
    clear_error();
    return dgamma ? fill_zero(dgamma, (size_t)cols * 4, st) : MDNN_SUCCESS;
  }
  if (!dx && !dgamma) return MDNN_SUCCESS;
  if (!dy || !h) return fail(MDNN_ERR_NULL, "rmsnorm_bwd: dy or h is NULL");
  if (lddy < cols || ldh < cols || (dres && lddr < cols) || (dx && lddx < cols))
    return fail(MDNN_ERR_LAYOUT, "rmsnorm_bwd: leading dimension below the width");
  const size_t es = dtype_size(dtype);
  if (!aligned(dy, es) || !aligned(h, es) || !aligned(dres, es) || !aligned(dx, es) || !aligned(gamma, 4))
    return fail(MDNN_ERR_MISALIGNED, "rmsnorm_bwd: misaligned buffer");
  const size_t need = dgamma ? mdnn_rmsnorm_bwd_workspace(rows, cols) : 0;
  if (need > 0 && (!workspace || ws_bytes < need || !aligned(workspace, 256)))
    return fail(MDNN_ERR_WORKSPACE, "rmsnorm_bwd: workspace of %zu bytes (256-byte aligned) required", need);
  clear_error();
  BwdArgs a = {};
  // (a single block's sums are the gradient)
  const int64_t blocks = bwd_blocks(rows, cols);
  a.dy = dy, a.h = h, a.dres = dres, a.gamma = gamma, a.dx = dx;
  a.partial = !dgamma || blocks == 1 ? dgamma : (float*)workspace;
  a.rows = rows, a.lddy = lddy, a.ldh = ldh, a.lddr = lddr, a.lddx = lddx, a.cols = (int32_t)cols, a.eps = eps;
  switch (dtype) {
    case MDNN_F32: MDNN_TRY(run_bwd<F32>(a, st)); break;
    case MDNN_F16: MDNN_TRY(run_bwd<F16>(a, st)); break;
    default: MDNN_TRY(run_bwd<BF16>(a, st)); break;
  }
  if (!dgamma || blocks == 1) return MDNN_SUCCESS;
  const int64_t tiles = ceil_div(cols, 32);
  hipLaunchKernelGGL(dgamma_kernel, dim3((unsigned)(tiles < MAX_BLOCKS ? tiles : MAX_BLOCKS)), dim3(1024), 0, st, (const float*)workspace,
                     (int)blocks, cols, dgamma);
  return check_launch("dgamma_kernel");
}

// A last layer z = x W + bias of many classes with its softmax cross entropy,
// both ways, without the logits of all classes at once.
//
//   lse_i = log sum_j exp(z_ij),  loss_i = lse_i - z_i,label(i)
//   G_ij = exp(z_ij - lse_i) - [j = label(i)]      (0 in ignored rows)
//   dx = a G W^T,  dW = a x^T G,  db = a sum_i G_i,  a = S / counted rows
//
// The classes are taken in pieces.  Forward, a piece leaves each row's maximum
// m and the sum of exp(z - m); the pairs of all pieces are joined at the end.
// Backward, lse is known, so a piece's G follows from its logits alone and goes
// into the two products at once.
//
// In 16 bits G is stored as 2^15 G for fp16 (probabilities of 1e-5 are subnormal
// there, those of 1e-8 nothing; times 2^15 the least normal one is 1.9e-9) and
// G for bf16: one rounding of the same size as a result's own.  The factor a
// comes after the products, in fp32, so the loss scale does not move G.
#include <cmath>

#include "gemm_core.h"
#include "internal.h"
#include "xent.h"

namespace mdnn {
namespace {

// ---------------------------------------------------------------- forward

// A row's piece of logits to its pair (m, sum exp(z - m)); the label's logit.
__global__ void __launch_bounds__(256)
xent_stats_kernel(const float* z, int64_t ldz, int64_t M, int64_t nc, int64_t n0, const int32_t* labels, Pair* pairs,
                  float* zlab) {
  __shared__ Pair buf[4];
  for (int64_t row = blockIdx.x; row < M; row += gridDim.x) {
    const float* p = z + row * ldz;
    const int64_t at = (int64_t)labels[row] - n0;
    Pair v = {-INFINITY, 0.0f};
    for (int64_t c = threadIdx.x * 4; c < nc; c += 1024) {
      float e[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = c + k < nc ? p[c + k] : -INFINITY;
      float m = fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3]));
      m = fmaxf(m, v.m);
      const float ref = pair_ref(m);
      v.s = v.s * __expf(v.m - ref) + ((__expf(e[0] - ref) + __expf(e[1] - ref)) + (__expf(e[2] - ref) + __expf(e[3] - ref)));
      v.m = m;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = join(v, Pair{__shfl_xor(v.m, o, 64), __shfl_xor(v.s, o, 64)});
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
      pairs[row] = join(join(buf[0], buf[1]), join(buf[2], buf[3]));
      if (at >= 0 && at < nc) zlab[row] = p[at];
    }
    __syncthreads();
  }
}

struct Tally {
  double sum;
  int64_t count;
};

// Pairs of all pieces to lse and the rows' losses: 64 rows a block, 16 groups
// of pieces, joined in their order.  A block leaves its losses' sum and the
// number of its rows that count; a single block writes the mean.
__global__ void __launch_bounds__(1024)
xent_rows_kernel(const Pair* pairs, int64_t pieces, int64_t M, int64_t N, const float* zlab, const int32_t* labels,
                 int32_t ignored, float* lse, float* row_loss, float* loss, Tally* tally) {
  __shared__ Pair buf[16][64];
  const int r = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * 64 + r, at = row < M ? row : M - 1;
  const int64_t per = ceil_div(pieces, 16), p0 = g * per, p1 = p0 + per < pieces ? p0 + per : pieces;
  Pair v = {-INFINITY, 0.0f};
  for (int64_t p = p0; p < p1; p += 8) {
    Pair u[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) u[k] = pairs[(p + k < p1 ? p + k : p) * M + at];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (p + k < p1) v = join(v, u[k]);
  }
  buf[g][r] = v;
  __syncthreads();
  if (g > 0) return;
#pragma unroll
  for (int k = 1; k < 16; ++k) v = join(v, buf[k][r]);
  Tally t = {0.0, 0};
  if (row < M) {
    const float l = v.m + logf(v.s);
    const int32_t label = labels[row];
    const bool counts = label != ignored;
    const float one = !counts ? 0.0f : label >= 0 && label < N ? l - zlab[row] : __builtin_nanf("");
    if (lse) lse[row] = l;
    if (row_loss) row_loss[row] = one;
    t = {(double)one, counts ? 1 : 0};
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    t.sum += __shfl_xor(t.sum, o, 64);
    t.count += __shfl_xor((long long)t.count, o, 64);
  }
  if (r > 0) return;
  if (gridDim.x > 1)
    tally[blockIdx.x] = t;
  else if (loss)
    *loss = (float)(t.sum / (double)(t.count > 0 ? t.count : 1));
}

__global__ void __launch_bounds__(1024) xent_mean_kernel(const Tally* tally, int64_t n, float* loss) {
  __shared__ Tally buf[16];
  Tally t = {0.0, 0};
  for (int64_t i = threadIdx.x; i < n; i += 1024) t.sum += tally[i].sum, t.count += tally[i].count;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    t.sum += __shfl_xor(t.sum, o, 64);
    t.count += __shfl_xor((long long)t.count, o, 64);
  }
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = t;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int w = 1; w < 16; ++w) t.sum += buf[w].sum, t.count += buf[w].count;
  *loss = (float)(t.sum / (double)(t.count > 0 ? t.count : 1));
}

// --------------------------------------------------------------- backward

// Block 0 counts the rows with a label that is not ignored and leaves
// a = S / count, times `scale`; the others copy x to rows of ldc elements,
// ignored rows, rows past M and columns past K as zeros (what an ignored row
// holds, Inf and NaN among it, must not reach dW as 0 * Inf).
template <class T>
__global__ void __launch_bounds__(256)
xent_prepare_kernel(const typename T::storage* x, int64_t ldx, int64_t M, int64_t K, const int32_t* labels,
                    int32_t ignored, const float* loss_scale, float scale, float* alpha, typename T::storage* copy,
                    int64_t rows, int64_t ldc) {
  if (blockIdx.x == 0) {
    __shared__ int64_t buf[4];
    int64_t n = 0;
    for (int64_t i0 = threadIdx.x; i0 < M; i0 += 2048) {
      int32_t v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = i0 + 256 * k < M ? labels[i0 + 256 * k] : ignored;
#pragma unroll
      for (int k = 0; k < 8; ++k) n += v[k] != ignored;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor((long long)n, o, 64);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
      n = buf[0] + buf[1] + buf[2] + buf[3];
      *alpha = (loss_scale ? *loss_scale : 1.0f) / (float)(n > 0 ? n : 1) * scale;
    }
    return;
  }
  constexpr int E = 16 / sizeof(typename T::storage);  // elements of a 16-byte chunk
  const int64_t per = ldc / E;
  for (int64_t row = blockIdx.x - 1; row < rows; row += gridDim.x - 1) {
    const bool live = row < M && labels[row < M ? row : 0] != ignored;
    const typename T::storage* p = x + row * ldx;
    for (int64_t c = threadIdx.x; c < per; c += 256) {
      typename T::storage v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = live && c * E + e < K ? p[c * E + e] : (typename T::storage)0;
      *(uint4*)(copy + row * ldc + c * E) = __builtin_bit_cast(uint4, v);
    }
  }
}

// Logits of a piece to G (type T, rows of ldg elements; z and G may be the
// same memory in fp32): 32 rows a block, four columns a thread.  Rows past M and
// columns past nc become zeros.  part: the block's column sums, or null.
template <class T>
__global__ void __launch_bounds__(256)
xent_grad_kernel(const float* z, int64_t ldz, int64_t M, int64_t rows, int64_t nc, int64_t n0, const int32_t* labels,
                 int32_t ignored, int64_t N, const float* lse, float scale, typename T::storage* g, int64_t ldg,
                 float* part) {
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= ldg) return;
  for (int64_t b = blockIdx.y; b * 32 < rows; b += gridDim.y) {
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t r1 = b * 32 + 32 < rows ? b * 32 + 32 : rows;
    for (int64_t r = b * 32; r < r1; ++r) {
      float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      const int32_t label = r < M ? labels[r] : ignored;
      if (r < M && label != ignored) {
        const float l = label >= 0 && label < N ? lse[r] : __builtin_nanf("");
        const int64_t at = (int64_t)label - n0 - c;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < nc) v[e] = __expf(z[r * ldz + c + e] - l) - (e == at ? 1.0f : 0.0f);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sum[e] += v[e];
        if (c + e < ldg) g[r * ldg + c + e] = from_f<T>(v[e] * scale);
      }
    }
    if (part) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < nc) part[b * N + n0 + c + e] = sum[e];
    }
  }
}

// db from the row blocks' column sums, in their order.
__global__ void __launch_bounds__(256)
xent_db_kernel(const float* part, int64_t blocks, int64_t N, const float* alpha, float scale, float* db) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= N) return;
  double s = 0.0;
  for (int64_t b = 0; b < blocks; b += 8) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = b + k < blocks ? part[(b + k) * N + c] : 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) s += (double)v[k];
  }
  db[c] = (float)s * (*alpha * scale);
}

template <class T>
__global__ void __launch_bounds__(256)
xent_round_kernel(const float* src, int64_t rows, int64_t cols, typename T::storage* dst, int64_t ld) {
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < cols; c += (int64_t)gridDim.x * 256)
      dst[r * ld + c] = from_f<T>(src[r * cols + c]);
}

// ------------------------------------------------------------------- plans

size_t pad256(size_t n) { return (n + 255) / 256 * 256; }

// Classes of a piece: as many as `bytes` of M rows hold, in whole multiples of
// 256, at least one.
int64_t piece_classes(int64_t M, int64_t N, size_t elem, size_t bytes) {
  int64_t nc = (int64_t)(bytes / elem) / M / 256 * 256;
  nc = nc < 256 ? 256 : nc;
  return nc < N ? nc : N;
}

struct FwdPlan {
  int64_t nc, pieces, blocks;
  size_t pairs, zlab, tally, z, gemm, gemm_bytes, bytes;
};
FwdPlan fwd_plan(int64_t M, int64_t N, int64_t K, mdnn_dtype_t t) {
  FwdPlan p;
  p.nc = piece_classes(M, N, 4, (size_t)64 << 20);
  p.pieces = ceil_div(N, p.nc);
  p.blocks = ceil_div(M, 64);
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at += pad256(n); return o; };
  p.pairs = take((size_t)p.pieces * M * sizeof(Pair));
  p.zlab = take((size_t)M * 4);
  p.tally = take((size_t)p.blocks * sizeof(Tally));
  p.z = take((size_t)M * p.nc * 4);
  const size_t a = gemm_ws_bytes(t, M, p.nc, K), b = gemm_ws_bytes(t, M, N - (p.pieces - 1) * p.nc, K);
  p.gemm_bytes = a > b ? a : b;
  p.gemm = take(p.gemm_bytes);
  p.bytes = at;
  return p;
}

struct BwdPlan {
  int64_t nc, pieces, rows, kc, ldg, blocks;
  size_t alpha, copy, z, g, part, acc, gemm, gemm_bytes, bytes;
};
BwdPlan bwd_plan(int64_t M, int64_t N, int64_t K, mdnn_dtype_t t) {
  BwdPlan p;
  const bool h = t != MDNN_F32;
  const size_t es = dtype_size(t);
  p.nc = piece_classes(M, N, 4, (size_t)256 << 20);
  p.pieces = ceil_div(N, p.nc);
  p.rows = h ? ceil_div(M, 64) * 64 : M;
  p.kc = h ? ceil_div(K, 8) * 8 : ceil_div(K, 4) * 4;
  p.ldg = h ? ceil_div(p.nc, 64) * 64 : ceil_div(p.nc, 4) * 4;
  p.blocks = ceil_div(p.rows, 32);  // (of xent_grad_kernel, padding rows too)
  size_t at = 0;
  auto take = [&](size_t n) { const size_t o = at; at += pad256(n); return o; };
  p.alpha = take(4);
  p.copy = take((size_t)p.rows * p.kc * es);
  p.z = take((size_t)M * p.ldg * 4);
  p.g = h ? take((size_t)p.rows * p.ldg * 2) : p.z;
  p.part = take((size_t)p.blocks * N * 4);
  p.acc = take(h && p.pieces > 1 ? (size_t)M * K * 4 : 0);
  const int64_t last = N - (p.pieces - 1) * p.nc;
  p.gemm_bytes = 0;
  for (int64_t n : {p.nc, last})
    for (size_t b : {gemm_ws_bytes(t, M, n, K), gemm_ws_bytes(t, M, K, n), gemm_ws_bytes(t, n, K, p.rows),
                     gemm_ws_bytes(t, K, n, p.rows)})
      p.gemm_bytes = b > p.gemm_bytes ? b : p.gemm_bytes;
  p.gemm = take(p.gemm_bytes);
  p.bytes = at;
  return p;
}

constexpr int64_t MAX_ROWS = (int64_t)1 << 24, MAX_N = 0x7fffffff;

bool sizes_ok(int64_t M, int64_t N, int64_t K) {
  return M >= 0 && M <= MAX_ROWS && N >= 1 && N <= MAX_N && K >= 1 && K <= MAX_N;
}

// Checks that both directions share.
mdnn_status_t check_common(const char* who, mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, const void* x,
                           int64_t ldx, const void* w, int64_t ldw, mdnn_dtype_t t, const float* bias,
                           const int32_t* labels) {
  if (layout != MDNN_NN && layout != MDNN_NT) return fail(MDNN_ERR_LAYOUT, "%s: layout must be NN or NT", who);
  if (!sizes_ok(M, N, K)) return fail(MDNN_ERR_SHAPE, "%s: bad size", who);
  if (!dtype_ok(t)) return fail(MDNN_ERR_DTYPE, "%s: unknown dtype", who);
  if (M == 0) return MDNN_SUCCESS;
  if (!x || !w || !labels) return fail(MDNN_ERR_NULL, "%s: NULL buffer", who);
  if (ldx < K || ldw < (layout == MDNN_NN ? N : K))
    return fail(MDNN_ERR_LAYOUT, "%s: leading dimension below the width", who);
  const size_t es = dtype_size(t);
  if (!aligned(x, es) || !aligned(w, es) || !aligned(bias, 4) || !aligned(labels, 4))
    return fail(MDNN_ERR_MISALIGNED, "%s: misaligned buffer", who);
  return MDNN_SUCCESS;
}

// W's piece from class n0 on.
const void* w_piece(mdnn_layout_t layout, const void* w, int64_t ldw, int64_t n0, size_t es) {
  return (const char*)w + (layout == MDNN_NN ? n0 : n0 * ldw) * es;
}

unsigned capped(int64_t n, int64_t most) { return (unsigned)(n < most ? n : most); }

template <class T>
mdnn_status_t run_bwd(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx, const void* w,
                      int64_t ldw, const float* bias, const int32_t* labels, int32_t ignored, const float* lse,
                      const float* loss_scale, void* dx, int64_t lddx, void* dw, int64_t lddw, mdnn_dtype_t dw_type,
                      float* db, char* ws, hipStream_t st) {
  typedef typename T::storage S;
  constexpr bool H = sizeof(S) == 2;
  const mdnn_dtype_t t = T::id;
  const BwdPlan p = bwd_plan(M, N, K, t);
  const float scale = t == MDNN_F16 ? 32768.0f : 1.0f;
  float* alpha = (float*)(ws + p.alpha);
  S* copy = (S*)(ws + p.copy);
  float* z = (float*)(ws + p.z);
  S* g = (S*)(ws + p.g);
  float* part = db ? (float*)(ws + p.part) : nullptr;
  void* gw = ws + p.gemm;
  const bool joined = H && p.pieces > 1;
  float* acc = joined ? (float*)(ws + p.acc) : nullptr;
  hipLaunchKernelGGL((xent_prepare_kernel<T>), dim3(capped(p.rows, 1 << 16) + 1), dim3(256), 0, st, (const S*)x, ldx, M,
                     K, labels, ignored, loss_scale, 1.0f / scale, alpha, copy, p.rows, p.kc);
  MDNN_TRY(check_launch("xent_prepare_kernel"));
  for (int64_t n0 = 0; n0 < N; n0 += p.nc) {
    const int64_t nc = n0 + p.nc < N ? p.nc : N - n0;
    const void* wp = w_piece(layout, w, ldw, n0, sizeof(S));
    MDNN_TRY(gemm_mixed_ws(layout, M, nc, K, 1.0f, copy, p.kc, wp, ldw, t, 0.0f, nullptr, 0, z, p.ldg, MDNN_F32,
                           bias ? bias + n0 : nullptr, MDNN_ACT_NONE, nullptr, 0, gw, p.gemm_bytes, st));
    hipLaunchKernelGGL((xent_grad_kernel<T>), dim3((unsigned)ceil_div(p.ldg, 1024), capped(ceil_div(p.rows, 32), 65535)),
                       dim3(256), 0, st, z, p.ldg, M, p.rows, nc, n0, labels, ignored, N, lse, scale, g, p.ldg, part);
    MDNN_TRY(check_launch("xent_grad_kernel"));
    if (dx) {
      const mdnn_layout_t back = layout == MDNN_NN ? MDNN_NT : MDNN_NN;
      void* d = joined ? (void*)acc : dx;
      const int64_t ldd = joined ? K : lddx;
      MDNN_TRY(gemm_mixed_ws(back, M, K, nc, 1.0f, g, p.ldg, wp, ldw, t, n0 > 0 ? 1.0f : 0.0f, d, ldd, d, ldd,
                             joined ? MDNN_F32 : t, nullptr, MDNN_ACT_NONE, nullptr, 0, gw, p.gemm_bytes, st, nullptr,
                             alpha));
    }
    if (dw) {
      const size_t ds = dtype_size(dw_type);
      if (layout == MDNN_NN)
        MDNN_TRY(gemm_mixed_ws(MDNN_TN, K, nc, p.rows, 1.0f, copy, p.kc, g, p.ldg, t, 0.0f, nullptr, 0,
                               (char*)dw + n0 * ds, lddw, dw_type, nullptr, MDNN_ACT_NONE, nullptr, 0, gw, p.gemm_bytes,
                               st, nullptr, alpha));
      else
        MDNN_TRY(gemm_mixed_ws(MDNN_TN, nc, K, p.rows, 1.0f, g, p.ldg, copy, p.kc, t, 0.0f, nullptr, 0,
                               (char*)dw + n0 * lddw * ds, lddw, dw_type, nullptr, MDNN_ACT_NONE, nullptr, 0, gw,
                               p.gemm_bytes, st, nullptr, alpha));
    }
  }
  if (dx && joined) {
    hipLaunchKernelGGL((xent_round_kernel<T>), dim3(capped(ceil_div(K, 256), 1024), capped(M, 65535)), dim3(256), 0, st,
                       acc, M, K, (S*)dx, lddx);
    MDNN_TRY(check_launch("xent_round_kernel"));
  }
  if (db) {
    hipLaunchKernelGGL(xent_db_kernel, dim3((unsigned)ceil_div(N, 256)), dim3(256), 0, st, part, p.blocks, N, alpha,
                       scale, db);
    MDNN_TRY(check_launch("xent_db_kernel"));
  }
  return MDNN_SUCCESS;
}

}  // namespace
}  // namespace mdnn

using namespace mdnn;

extern "C" size_t mdnn_linear_xent_fwd_workspace(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K,
                                                 mdnn_dtype_t dtype) {
  if ((layout != MDNN_NN && layout != MDNN_NT) || !sizes_ok(M, N, K) || !dtype_ok(dtype) || M == 0) return 0;
  return fwd_plan(M, N, K, dtype).bytes;
}

extern "C" mdnn_status_t mdnn_linear_xent_fwd(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, const void* x,
                                              int64_t ldx, const void* w, int64_t ldw, mdnn_dtype_t dtype,
                                              const float* bias, const int32_t* labels, int32_t ignored, float* loss,
                                              float* row_loss, float* lse, void* workspace, size_t ws_bytes,
                                              mdnn_stream_t stream) {
  const char* who = "linear_xent_fwd";
  MDNN_TRY(check_common(who, layout, M, N, K, x, ldx, w, ldw, dtype, bias, labels));
  if (!aligned(loss, 4) || !aligned(row_loss, 4) || !aligned(lse, 4))
    return fail(MDNN_ERR_MISALIGNED, "%s: misaligned buffer", who);
  const hipStream_t st = as_stream(stream);
  clear_error();
  if (M == 0) return loss ? fill_zero(loss, 4, st) : MDNN_SUCCESS;
  if (!loss && !row_loss && !lse) return MDNN_SUCCESS;
  const FwdPlan p = fwd_plan(M, N, K, dtype);
  if (!workspace || ws_bytes < p.bytes || !aligned(workspace, 256))
    return fail(MDNN_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) required", who, p.bytes);
  char* ws = (char*)workspace;
  Pair* pairs = (Pair*)(ws + p.pairs);
  float *zlab = (float*)(ws + p.zlab), *z = (float*)(ws + p.z);
  Tally* tally = (Tally*)(ws + p.tally);
  for (int64_t i = 0; i < p.pieces; ++i) {
    const int64_t n0 = i * p.nc, nc = n0 + p.nc < N ? p.nc : N - n0;
    MDNN_TRY(gemm_mixed_ws(layout, M, nc, K, 1.0f, x, ldx, w_piece(layout, w, ldw, n0, dtype_size(dtype)), ldw, dtype,
                           0.0f, nullptr, 0, z, p.nc, MDNN_F32, bias ? bias + n0 : nullptr, MDNN_ACT_NONE, nullptr, 0,
                           ws + p.gemm, p.gemm_bytes, stream));
    hipLaunchKernelGGL(xent_stats_kernel, dim3(capped(M, 1 << 20)), dim3(256), 0, st, z, p.nc, M, nc, n0, labels,
                       pairs + i * M, zlab);
    MDNN_TRY(check_launch("xent_stats_kernel"));
  }
  hipLaunchKernelGGL(xent_rows_kernel, dim3((unsigned)p.blocks), dim3(1024), 0, st, pairs, p.pieces, M, N, zlab, labels,
                     ignored, lse, row_loss, loss, tally);
  MDNN_TRY(check_launch("xent_rows_kernel"));
  if (loss && p.blocks > 1) {
    hipLaunchKernelGGL(xent_mean_kernel, dim3(1), dim3(1024), 0, st, tally, p.blocks, loss);
    MDNN_TRY(check_launch("xent_mean_kernel"));
  }
  return MDNN_SUCCESS;
}

extern "C" size_t mdnn_linear_xent_bwd_workspace(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K,
                                                 mdnn_dtype_t dtype) {
  if ((layout != MDNN_NN && layout != MDNN_NT) || !sizes_ok(M, N, K) || !dtype_ok(dtype) || M == 0) return 0;
  return bwd_plan(M, N, K, dtype).bytes;
}

extern "C" mdnn_status_t mdnn_linear_xent_bwd(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, const void* x,
                                              int64_t ldx, const void* w, int64_t ldw, mdnn_dtype_t dtype,
                                              const float* bias, const int32_t* labels, int32_t ignored,
                                              const float* lse, const float* loss_scale, void* dx, int64_t lddx,
                                              void* dw, int64_t lddw, mdnn_dtype_t dw_type, float* db, void* workspace,
                                              size_t ws_bytes, mdnn_stream_t stream) {
  const char* who = "linear_xent_bwd";
  MDNN_TRY(check_common(who, layout, M, N, K, x, ldx, w, ldw, dtype, bias, labels));
  if (dw && (!dtype_ok(dw_type) || (dw_type != MDNN_F32 && dw_type != dtype)))
    return fail(MDNN_ERR_DTYPE, "%s: dw_type must be fp32 or dtype", who);
  if (dw && lddw < (layout == MDNN_NN ? N : K))
    return fail(MDNN_ERR_LAYOUT, "%s: leading dimension below the width", who);
  if ((dw && !aligned(dw, dtype_size(dw_type))) || !aligned(db, 4))
    return fail(MDNN_ERR_MISALIGNED, "%s: misaligned buffer", who);
  const hipStream_t st = as_stream(stream);
  if (M == 0) {  // no row: the sums over rows are zeros (products of no depth)
    clear_error();
    if (dw)
      MDNN_TRY(gemm_mixed_ws(MDNN_TN, layout == MDNN_NN ? K : N, layout == MDNN_NN ? N : K, 0, 1.0f, nullptr, 0, nullptr,
                             0, dtype, 0.0f, nullptr, 0, dw, lddw, dw_type, nullptr, MDNN_ACT_NONE, nullptr, 0, nullptr,
                             0, stream));
    return db ? fill_zero(db, (size_t)N * 4, st) : MDNN_SUCCESS;
  }
  if (!dx && !dw && !db) return MDNN_SUCCESS;
  if (!lse) return fail(MDNN_ERR_NULL, "%s: lse is NULL", who);
  if (dx && lddx < K) return fail(MDNN_ERR_LAYOUT, "%s: leading dimension below the width", who);
  if (!aligned(lse, 4) || !aligned(loss_scale, 4) || (dx && !aligned(dx, dtype_size(dtype))))
    return fail(MDNN_ERR_MISALIGNED, "%s: misaligned buffer", who);
  const size_t need = bwd_plan(M, N, K, dtype).bytes;
  if (!workspace || ws_bytes < need || !aligned(workspace, 256))
    return fail(MDNN_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) required", who, need);
  clear_error();
  char* ws = (char*)workspace;
  switch (dtype) {
    case MDNN_F32:
      return run_bwd<F32>(layout, M, N, K, x, ldx, w, ldw, bias, labels, ignored, lse, loss_scale, dx, lddx, dw, lddw,
                          dw_type, db, ws, st);
    case MDNN_F16:
      return run_bwd<F16>(layout, M, N, K, x, ldx, w, ldw, bias, labels, ignored, lse, loss_scale, dx, lddx, dw, lddw,
                          dw_type, db, ws, st);
    default:
      return run_bwd<BF16>(layout, M, N, K, x, ldx, w, ldw, bias, labels, ignored, lse, loss_scale, dx, lddx, dw, lddw,
                           dw_type, db, ws, st);
  }
}

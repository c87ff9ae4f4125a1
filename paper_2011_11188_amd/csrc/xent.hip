// A last layer z = x W + bias of many classes with its softmax cross entropy,
// both ways, without the logits of all classes at once.
//
//   lse_i = log sum_j exp(z_ij),  loss_i = lse_i - z_i,label(i)
//   G_ij = exp(z_ij - lse_i) - [j = label(i)]      (0 in ignored rows)
//   dx = a G W^T,  dW = a x^T G,  db = a sum_i G_i,  a = S / counted rows
//
// The classes are taken in pieces.  Forward, tiles of a piece leave each row's
// maximum m and the sum of exp(z - m); the pairs of all tiles are joined.
// Backward, lse is known, so a piece's G follows from its logits alone and goes
// into the two products at once.
//
// The logits never leave a tile's registers: tiled (16 bits), all products run on
// the pipelined kernel (xent_pipe.h).  Operands that it cannot read (sizes that
// are no multiples of 64, rows off 16 bytes) are copied to padded rows, W by
// pieces, where there are rows enough to pay for that; otherwise, and in fp32, the
// register-staged kernel takes them as they are (xent_reg.hip).  Where neither
// can (contiguous extents below 16 bytes, a table's rows further apart than 32-bit
// offsets reach over 256 classes), or so few tiles over a long K that K has to be
// split, a piece's fp32 logits go through the workspace.
//
// In 16 bits G is stored as 2^15 G for fp16 (probabilities of 1e-5 are subnormal
// there, those of 1e-8 nothing; times 2^15 the least normal one is 1.9e-9) and
// G for bf16: one rounding of the same size as a result's own.  The factor a
// comes after the products, in fp32, so the loss scale does not move G.
#include <cmath>
#include <type_traits>

#include "gemm_launch.h"
#include "internal.h"
#include "xent.h"

namespace mdnn {

// 256 from one tile a CU on, but for so few steps that a tile is mostly its end,
// which two workgroups a CU of 128 run beside each other's (backward 8192 x 16384 x
// 128 bf16 312 us, 256 325; 4096 x 32768 x 256 440 and 430; forward 9024 x 4416 x 64
// 32.0 and 33.1, 8192 x 16384 x 128 87 and 81).  Then 128 from one a CU on (64: 2000 x
// 3008 x 512 fp16 23.6 us, 128 17.8; 300 x 20032 x 640 bf16 31.5 and 22.9; 100 x 32768
// x 4096 fp16 89 and 76), for rows that fill them.
int xent_tile(int64_t M, int64_t N, int64_t K, bool backward) {
  auto tiles = [&](int64_t side) { return ceil_div(M, side) * ceil_div(N, side); };
  if (M > 128 && tiles(256) >= 256 && K > (backward ? 128 : 64)) return 256;
  return M > 64 && tiles(128) >= 256 ? 128 : 64;
}

namespace {

constexpr int64_t MAX_ROWS = (int64_t)1 << 24, MAX_N = 0x7fffffff;

// ---------------------------------------------------------------- forward

// A row's piece of logits in the workspace: rows of ldz, or the parts of a split
// product, `splits` of them one after another without their bias.
struct Logits {
  const float* z;
  int64_t ldz, part;  // part: elements between parts
  int32_t splits;
  const float* bias;  // with parts: the piece's, or null
  // four elements of a row from c on, the parts added in their order, four of
  // them in flight (past the piece: its last element again)
  __device__ __forceinline__ void quad(int64_t row, int64_t c, int64_t nc, float (&e)[4]) const {
    if (splits == 1) {
      const float4_t q = *(const float4_t*)(z + row * ldz + c);  // (rows of whole quads)
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = q[k];
      return;
    }
    const float* p = z + row * ldz;
    int64_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k] = c + k < nc ? c + k : nc - 1, e[k] = 0.0f;
    for (int s = 0; s < splits; s += 4) {
      float v[4][4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k) v[u][k] = p[(s + u < splits ? s + u : s) * part + at[k]];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] += s + u < splits ? v[u][k] : 0.0f;
    }
    if (bias) {
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] += bias[at[k]];
    }
  }
};

// A row's piece of logits to its pair (m, sum exp(z - m)); the label's logit.
__global__ void __launch_bounds__(256)
xent_stats_kernel(Logits z, int64_t M, int64_t nc, int64_t n0, const int32_t* labels, Pair* pairs, float* zlab,
                  uint32_t* done) {
  __shared__ Pair buf[4];
  if (blockIdx.x == 0 && threadIdx.x == 0) *done = 0;
  for (int64_t row = blockIdx.x; row < M; row += gridDim.x) {
    const int64_t at = (int64_t)labels[row] - n0;
    Pair v = {-INFINITY, 0.0f};
    for (int64_t c = threadIdx.x * 4; c < nc; c += 1024) {
      float e[4];
      z.quad(row, c, nc, e);
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = c + k < nc ? e[k] : -INFINITY;
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
      if (at >= 0 && at < nc) {
        float e[4];
        z.quad(row, at & ~(int64_t)3, nc, e);
        zlab[row] = at & 2 ? (at & 1 ? e[3] : e[2]) : (at & 1 ? e[1] : e[0]);
      }
    }
    __syncthreads();
  }
}

struct Tally {
  double sum;
  int64_t count;
};

// The pairs of a piece's tiles, and those of the pieces before it (`before`, or
// null), joined: RPB rows a block, 1024 / RPB groups that take the tiles in turn,
// eight in flight, joined in a fixed order.  To `after` (which may be `before`)
// where more pieces follow, else to lse and the rows' losses: a block leaves its
// losses' sum and the number of its rows that count, and the last one to do so
// (counted in `done`, which a kernel before this one has cleared) adds all blocks'
// in their order for the mean.  Up to 1024 rows, 16 a block: one row of 512 tiles
// takes one round of loads (5.3 us, 64 rows a block 9.0).
int rows_per_block(int64_t M) { return M <= 1024 ? 16 : 64; }

template <int RPB>
__global__ void __launch_bounds__(1024)
xent_rows_kernel(const Pair* pairs, int64_t pieces, const Pair* before, Pair* after, int64_t M, int64_t N,
                 const float* zlab, const int32_t* labels, int32_t ignored, float* lse, float* row_loss, float* loss,
                 Tally* tally, uint32_t* done) {
  constexpr int G = 1024 / RPB;
  __shared__ Pair buf[G][RPB + (RPB < 64)];  // (odd rows where columns are read)
  __shared__ Pair rows[RPB];
  const int g = threadIdx.x / RPB;
  int r = threadIdx.x % RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + r;
  const int64_t at = row < M ? row : M - 1;
  Pair v = {-INFINITY, 0.0f};
  if (before && g == 0) v = before[at];
  for (int64_t p = g; p < pieces; p += 8 * G) {
    Pair u[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) u[k] = pairs[(p + k * G < pieces ? p + k * G : p) * M + at];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (p + k * G < pieces) v = join(v, u[k]);
  }
  buf[g][r] = v;
  __syncthreads();
  if constexpr (RPB == 64) {
    if (g > 0) return;
#pragma unroll
    for (int k = 1; k < G; ++k) v = join(v, buf[k][r]);
  } else {
    // a wave joins one row's groups, then wave 0 goes on with the rows
    static_assert(RPB == 16, "a wave a row");
    v = buf[threadIdx.x & 63][threadIdx.x >> 6];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = join(v, Pair{__shfl_xor(v.m, o, 64), __shfl_xor(v.s, o, 64)});
    if ((threadIdx.x & 63) == 0) rows[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    r = threadIdx.x;
    row = r < RPB ? (int64_t)blockIdx.x * RPB + r : M;
    if (r < RPB) v = rows[r];
  }
  if (after) {
    if (row < M) after[row] = v;
    return;
  }
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
  if (!loss) return;
  if (gridDim.x > 1) {
    // (tallies cross the XCDs' caches: stores and loads at device scope)
    uint32_t last = 0;
    if (r == 0) {
      __hip_atomic_store(&tally[blockIdx.x].sum, t.sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&tally[blockIdx.x].count, t.count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __hip_atomic_fetch_add(done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    if (!__shfl((int)last, 0, 64)) return;
    t = {0.0, 0};
    for (uint32_t b = r; b < gridDim.x; b += 64) {
      t.sum += __hip_atomic_load(&tally[b].sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      t.count += __hip_atomic_load(&tally[b].count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      t.sum += __shfl_xor(t.sum, o, 64);
      t.count += __shfl_xor((long long)t.count, o, 64);
    }
  }
  if (r == 0) *loss = (float)(t.sum / (double)(t.count > 0 ? t.count : 1));
}

// --------------------------------------------------------------- backward

typedef uint32_t chunk_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t chunk_a4 __attribute__((ext_vector_type(4), aligned(4)));

// 16 bytes of a row from element c on, at any element address; zeros from
// element `cols` on.
template <class S>
__device__ __forceinline__ uint4 chunk16(const S* row, int64_t c, int64_t cols) {
  typedef std::conditional_t<sizeof(S) == 2, chunk_a2, chunk_a4> V;
  constexpr int E = 16 / sizeof(S);
  if (c + E <= cols) {
    const V v = *(const __attribute__((address_space(1))) V*)(row + c);
    return make_uint4(v.x, v.y, v.z, v.w);
  }
  struct {
    S e[E];
  } v;
#pragma unroll
  for (int k = 0; k < E; ++k) v.e[k] = c + k < cols ? row[c + k] : (S)0;
  return __builtin_bit_cast(uint4, v);
}

// [rows][cols] of 16-bit elements at any address to rows of ldc (a multiple of
// 8), zeros past cols and in rows .. all - 1; gx by gy blocks.
struct Pack {
  const uint16_t* src;
  int64_t ld, rows, cols;
  uint16_t* dst;
  int64_t all, ldc;
  uint32_t gx, gy;
};

__device__ __forceinline__ void pack_block(const Pack& p, uint32_t block) {
  const int64_t c = ((int64_t)(block % p.gx) * 64 + (threadIdx.x & 63)) * 8;
  if (c >= p.ldc) return;
  for (int64_t r0 = ((int64_t)(block / p.gx) * 4 + (threadIdx.x >> 6)) * 4; r0 < p.all; r0 += (int64_t)p.gy * 16) {
    uint4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      v[k] = r0 + k < p.rows ? chunk16(p.src + (r0 + k) * p.ld, c, p.cols) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (r0 + k < p.all) *(uint4*)(p.dst + (r0 + k) * p.ldc + c) = v[k];
  }
}

// One copy, or two beside each other.
__global__ void __launch_bounds__(256) xent_pack_kernel(Pack a, Pack b) {
  const uint32_t first = a.gx * a.gy;
  if (blockIdx.x < first)
    pack_block(a, blockIdx.x);
  else
    pack_block(b, blockIdx.x - first);
}

// Block 0 counts the rows with a label that is not ignored and leaves
// a = S / count, times `scale`; the others copy x to rows of ldc elements,
// ignored rows, rows past M and columns past K as zeros (what an ignored row
// holds, Inf and NaN among it, must not reach dW as 0 * Inf).  Blocks from `own` on
// copy W's first piece, where that is packed.
template <class T>
__global__ void __launch_bounds__(256)
xent_prepare_kernel(const typename T::storage* x, int64_t ldx, int64_t M, int64_t K, const int32_t* labels,
                    int32_t ignored, const float* loss_scale, float scale, float* alpha, typename T::storage* copy,
                    int64_t rows, int64_t ldc, uint32_t own, Pack w) {
  if (blockIdx.x >= own) {
    pack_block(w, blockIdx.x - own);
    return;
  }
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
  for (int64_t row = blockIdx.x - 1; row < rows; row += own - 1) {
    const bool live = row < M && labels[row < M ? row : 0] != ignored;
    const typename T::storage* p = x + row * ldx;
    for (int64_t c = threadIdx.x; c < per; c += 256) {
      *(uint4*)(copy + row * ldc + c * E) = live ? chunk16(p, c * E, K) : make_uint4(0, 0, 0, 0);
    }
  }
}

// Logits of a piece to G (type T, rows of ldg elements): GRAD_ROWS rows a block, both in flight, four columns
// a thread.  Rows past M and columns past nc become zeros.  part: the block's
// column sums, or null.
constexpr int GRAD_ROWS = 2;
template <class T>
__global__ void __launch_bounds__(256)
xent_grad_kernel(Logits z, int64_t M, int64_t rows, int64_t nc, int64_t n0, const int32_t* labels, int32_t ignored,
                 int64_t N, const float* lse, float scale, typename T::storage* g, int64_t ldg, float* part,
                 int64_t ldp, const float* loss_scale, float* alpha) {
  typedef typename T::storage S;
  if (alpha && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {  // (few rows)
    int n = 0;
    for (int64_t r = 0; r < M; ++r) n += labels[r] != ignored;
    *alpha = (loss_scale ? *loss_scale : 1.0f) / (float)(n > 0 ? n : 1) * (1.0f / scale);
  }
  const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= ldg) return;
  for (int64_t b = blockIdx.y; b * GRAD_ROWS < rows; b += gridDim.y) {
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t r1 = b * GRAD_ROWS + GRAD_ROWS < rows ? b * GRAD_ROWS + GRAD_ROWS : rows;
    for (int64_t r0 = b * GRAD_ROWS; r0 < r1; r0 += GRAD_ROWS) {
      float q[GRAD_ROWS][4];
      int32_t label[GRAD_ROWS];
      float l[GRAD_ROWS];
#pragma unroll
      for (int k = 0; k < GRAD_ROWS; ++k) {
        const int64_t r = r0 + k < M ? r0 + k : M - 1;
        z.quad(r, c, nc, q[k]);
        label[k] = labels[r], l[k] = lse[r];
      }
#pragma unroll
      for (int k = 0; k < GRAD_ROWS; ++k) {
        if (r0 + k >= r1) break;
        const bool live = r0 + k < M && label[k] != ignored;
        const float at_l = label[k] >= 0 && label[k] < N ? l[k] : __builtin_nanf("");
        const int64_t at = (int64_t)label[k] - n0 - c;
        S o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = __expf(q[k][e] - at_l) - (e == at ? 1.0f : 0.0f);
          v = live && c + e < nc ? v : 0.0f;
          sum[e] += v;
          o[e] = from_f<T>(v * scale);
        }
        S* d = g + (r0 + k) * ldg + c;
        if constexpr (sizeof(S) == 2)
          *(uint2*)d = make_uint2((uint32_t)o[0] | ((uint32_t)o[1] << 16), (uint32_t)o[2] | ((uint32_t)o[3] << 16));
        else
          *(float4_t*)d = (float4_t){o[0], o[1], o[2], o[3]};
      }
    }
    if (part) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < nc) part[b * ldp + c + e] = sum[e];
    }
  }
}

// db from the row blocks' column sums: 64 columns a block, four groups of row
// blocks (eight loads in flight), joined in their order.
__global__ void __launch_bounds__(256)
xent_db_kernel(const float* part, int64_t blocks, int64_t ldp, int64_t cols, const float* alpha, float scale, float* db) {
  __shared__ double buf[4][64];
  const int cx = threadIdx.x & 63, r = threadIdx.x >> 6;
  const int64_t c = (int64_t)blockIdx.x * 64 + cx, at = c < cols ? c : cols - 1;
  const int64_t per = ceil_div(blocks, 4), b1 = (r + 1) * per < blocks ? (r + 1) * per : blocks;
  double s = 0.0;
  for (int64_t b = r * per; b < b1; b += 8) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = part[(b + k < b1 ? b + k : b) * ldp + at];
#pragma unroll
    for (int k = 0; k < 8; ++k) s += b + k < b1 ? (double)v[k] : 0.0;
  }
  buf[r][cx] = s;
  __syncthreads();
  if (r == 0 && c < cols) db[c] = (float)(((buf[0][cx] + buf[1][cx]) + buf[2][cx]) + buf[3][cx]) * (*alpha * scale);
}

template <class T>
__global__ void __launch_bounds__(256)
xent_round_kernel(const float* src, int64_t rows, int64_t cols, typename T::storage* dst, int64_t ld) {
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < cols; c += (int64_t)gridDim.x * 256)
      dst[r * ld + c] = from_f<T>(src[r * cols + c]);
}

// dx from the parts of its product, in their order, times the factor.
template <class T>
__global__ void __launch_bounds__(256)
xent_parts_kernel(const float* part, int parts, int64_t rows, int64_t cols, const float* alpha, typename T::storage* dst,
                  int64_t ld) {
  const float a = *alpha;
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < cols; c += (int64_t)gridDim.x * 256) {
      const float* p = part + r * cols + c;
      float s = 0.0f;
      for (int k0 = 0; k0 < parts; k0 += 8) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = p[(k0 + k < parts ? k0 + k : k0) * rows * cols];
#pragma unroll
        for (int k = 0; k < 8; ++k) s += k0 + k < parts ? v[k] : 0.0f;
      }
      dst[r * ld + c] = from_f<T>(s * a);
    }
}

// ------------------------------------------------------------------- plans

int64_t up(int64_t n, int64_t to) { return ceil_div(n, to) * to; }

// Classes of a piece: as many as `elems` elements of `rows` a class hold, in
// whole multiples of 256, at least one, at most 2^26 (a launch holds fewer than
// 2^32 threads).
int64_t piece_classes(int64_t N, int64_t rows, int64_t elems) {
  int64_t nc = elems / rows / 256 * 256;
  nc = nc < 256 ? 256 : nc < (1 << 26) ? nc : 1 << 26;
  return nc < N ? nc : N;
}

// How a call runs: the tiles read the operands as they are (TILED) or copies in
// the workspace (PACKED), or the register-staged tiles do (STAGED), or a piece's
// logits go through the workspace (GENERAL).  The sizes alone name the way; rows
// that it cannot read (addresses, leading dimensions) fall back to the next, and
// the caller's workspace holds every way that its sizes allow.
enum Way { TILED, PACKED, STAGED, GENERAL };

// Where copying W pays (two passes over it at memory speed and a launch, against
// products at about twice the register-staged kernel's rate): by the rows and by the
// whole product.  Forward, copied and not: 1000 x 5003 x 1000 fp16 30.5 and 36.9 us,
// 400 x 14787 x 6490 bf16 190 and 238, but 320 x 40805 x 955 94 and 64, 1000 x 3001 x
// 301 22.6 and 17.5; backward: 320 x 14787 x 6490 439 and 510, 1000 x 2049 x 650 40 and
// 49, but 192 x 40805 x 955 173 and 161, 1000 x 3001 x 301 46.4 and 39.6.
bool pack_pays(int64_t M, int64_t N, int64_t K, bool backward) {
  return M >= (backward ? 256 : 384) && (double)M * N * K >= (backward ? 0x1p30 : 0x1p32);
}

Way way_by_size(int64_t M, int64_t N, int64_t K, mdnn_dtype_t t, bool backward) {
  // (a grid of less than half the chip's CUs over a long K: split in the general product)
  if (ceil_div(M, 64) * ceil_div(N, 64) < 128 && K > 512) return GENERAL;
  if (t != MDNN_F32 && M * up(K, 64) < (int64_t)1 << 31) {  // (32-bit offsets reach every row of x)
    if ((N % 64 == 0 || (!backward && N % 8 == 0)) && K % 64 == 0) return TILED;
    if (pack_pays(M, N, K, backward)) return PACKED;
  }
  const int64_t e = 16 / (int64_t)dtype_size(t);
  return K >= e && N >= e ? STAGED : GENERAL;
}
Way way_below(Way w) { return w == TILED ? STAGED : GENERAL; }

// Classes of a table [N][K] that one tile product takes: as many, in whole
// multiples of 256, as 32-bit offsets reach in rows up to a sixteenth (64 elements)
// wider than K; wider ones go through stored logits, as all such tables did (64 x
// 250880 x 14336 bf16 forward 1739 us, in four products 1412; 512 rows 3423 and 3471;
// 2 x 4300000 x 256 fp32 4300 and 1891).  Class-contiguous rows are addressed step by
// step, all their classes at once.
int64_t reach_classes(mdnn_layout_t layout, int64_t K, mdnn_dtype_t t) {
  if (layout == MDNN_NN) return MAX_N;
  const int64_t wide = K + (K > 1024 ? K / 16 : 64), most = (int64_t)1 << (t == MDNN_F32 ? 30 : 31);
  const int64_t n = most / wide / 256 * 256 - 256;
  return n < 256 ? 256 : n;
}

// Rows of class-contiguous W [K][ldw], of nc classes each, that one product over the
// classes takes: all, or as many, in whole multiples of 256, as 32-bit offsets reach
// (dx of 64 x 250880 x 14336 bf16: the gradients 8871 us, in two products 5917).
int64_t reach_rows(int64_t K, int64_t nc, int64_t ldw, mdnn_dtype_t t) {
  const int64_t most = (int64_t)1 << (t == MDNN_F32 ? 30 : 31), n = (most - 1) / ldw / 256 * 256;
  return n < 256 || (K - 1) * ldw + nc < most ? K : n;
}

// Pieces of nc classes, or a few fewer so that the last, too, holds a 16-byte chunk,
// as the register-staged tiles need of class-contiguous rows: a last piece of one to
// three classes sent all pieces through stored logits (gradients, fp32: 16384 x 8193
// x 512 3.90 ms, two pieces of at least nine 3.39; 2^20 x 2305 x 64 19.6 and 15.0).
int64_t whole_chunks(int64_t N, int64_t nc, mdnn_dtype_t t) {
  while (N % nc > 0 && N % nc < 16 / (int64_t)dtype_size(t)) nc -= 8;
  return nc;
}

// The tile that a way's products take.
int way_tile(Way w, int64_t M, int64_t N, int64_t K, bool backward) {
  return w == STAGED ? xent_reg_tile(M, N) : xent_tile(M, N, up(K, 64), backward);
}

struct Space {
  size_t at = 0;
  size_t take(size_t n) {
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  }
};

// K split of a general piece's logits where their tiles are few (1: the
// product's own ways), at least 256 deep (8 x 3619 over 1216 fp32 23 us a call, 128
// deep 27), parts of at most 32 MB.
SplitPlan logit_splits(int64_t M, int64_t nc, int64_t K) {
  SplitPlan p{1, K};
  const int64_t tiles = ceil_div(M, 64) * ceil_div(nc, 64);
  int64_t n = tiles < 128 ? ceil_div((int64_t)512, tiles) : 1;
  n = n < K / 256 ? n : K / 256;
  const int64_t most = ((int64_t)8 << 20) / (M * nc);
  n = n < most ? n : most;
  if (n < 2) return p;
  p.k_per_split = up(ceil_div(K, n), 64);
  p.splits = (int)ceil_div(K, p.k_per_split);
  return p;
}

// A general piece's logits.
mdnn_status_t general_logits(mdnn_layout_t layout, int64_t M, int64_t nc, int64_t K, const void* x, int64_t ldx,
                             const void* w, int64_t ldw, mdnn_dtype_t t, const float* bias, float* z, int64_t ldz,
                             void* gw, size_t gw_bytes, Logits& out, hipStream_t st) {
  const SplitPlan s = logit_splits(M, nc, K);
  if (s.splits > 1 && gemm_reg_ok(t, layout, M, nc, K, ldx, ldw, s.splits)) {
    Epilogue ep{};
    ep.alpha = 1.0f, ep.partial = z, ep.k_per_split = s.k_per_split;
    out = {z, nc, M * nc, s.splits, bias};
    return gemm_reg(t, MDNN_F32, layout, M, nc, K, x, ldx, w, ldw, ep, s.splits, st);
  }
  out = {z, ldz, 0, 1, nullptr};
  return gemm_mixed_ws(layout, M, nc, K, 1.0f, x, ldx, w, ldw, t, 0.0f, nullptr, 0, z, ldz, MDNN_F32, bias, MDNN_ACT_NONE,
                       nullptr, 0, gw, gw_bytes, st);
}
size_t logit_bytes(int64_t M, int64_t nc, int64_t K, int64_t ldz) {
  const size_t a = (size_t)logit_splits(M, nc, K).splits * M * nc * 4, b = (size_t)M * ldz * 4;
  return a > b ? a : b;
}

struct FwdPlan {
  int64_t nc, pieces, blocks, kc, ldw;
  size_t pairs, run, zlab, tally, done, z, copy, pack, gemm, gemm_bytes, bytes;
};
FwdPlan fwd_plan(Way way, mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, mdnn_dtype_t t) {
  FwdPlan p = {};
  Space s;
  p.blocks = ceil_div(M, rows_per_block(M));
  p.kc = up(K, 64);
  if (way == GENERAL) {
    p.nc = piece_classes(N, M, (int64_t)16 << 20);
  } else {
    p.nc = piece_classes(N, ceil_div(M, 64), (int64_t)32 << 20);  // pairs of 64 columns at least
    const int64_t most = way == PACKED ? piece_classes(N, p.kc, (int64_t)128 << 20) : reach_classes(layout, K, t);
    p.nc = p.nc < most ? p.nc : most;
    if (way == STAGED && layout == MDNN_NN) p.nc = whole_chunks(N, p.nc, t);
  }
  p.pieces = ceil_div(N, p.nc);
  const int64_t last = N - (p.pieces - 1) * p.nc;
  int64_t tiles = 1;
  if (way != GENERAL)
    for (int64_t n : {p.nc, last}) {
      const int64_t k = ceil_div(n, way_tile(way, M, n, K, false));
      tiles = k > tiles ? k : tiles;
    }
  p.pairs = s.take((size_t)tiles * M * sizeof(Pair));
  p.run = s.take(p.pieces > 1 ? (size_t)M * sizeof(Pair) : 0);
  p.zlab = s.take((size_t)M * 4);
  p.tally = s.take((size_t)p.blocks * sizeof(Tally));
  p.done = s.take(4);
  if (way == GENERAL) {
    const size_t za = logit_bytes(M, p.nc, K, up(p.nc, 4)), zb = logit_bytes(M, last, K, up(p.nc, 4));
    p.z = s.take(za > zb ? za : zb);
    const size_t a = gemm_ws_bytes(t, M, p.nc, K), b = gemm_ws_bytes(t, M, last, K);
    p.gemm_bytes = a > b ? a : b;
    p.gemm = s.take(p.gemm_bytes);
  } else if (way != STAGED) {
    p.copy = s.take((size_t)M * p.kc * 2);  // x, where its rows are not as the tiles read them
    p.ldw = layout == MDNN_NN ? up(p.nc, 64) : p.kc;
    p.pack = s.take(way == PACKED ? (size_t)(layout == MDNN_NN ? p.kc : up(p.nc, 64)) * p.ldw * 2 : 0);
  }
  p.bytes = s.at;
  return p;
}

// Depth split of dx on the register-staged kernel, whose classes are the depth:
// two rounds of two workgroups a CU (500 x 777 over 10007 fp32 198 us on its 104
// tiles), parts of at most 64 MB and, as a step of fp32 takes several times one of
// 16 bits, at least 128 deep (14 x 514 over 1392 33.5 us a call, 512 deep 43.2) or
// 512 (128 x 1664 over 2176 fp16 39.3, 128 deep 43.0).
SplitPlan dx_splits(int64_t M, int64_t K, int64_t depth, mdnn_dtype_t t) {
  const int64_t least = t == MDNN_F32 ? 128 : 512;
  SplitPlan p{1, depth};
  int64_t n = 1024 / (ceil_div(M, 64) * ceil_div(K, 64));
  n = n < depth / least ? n : depth / least;
  const int64_t most = ((int64_t)16 << 20) / (M * K);
  n = n < most ? n : most;
  if (n < 2) return p;
  p.k_per_split = up(ceil_div(depth, n), 64);
  p.splits = (int)ceil_div(depth, p.k_per_split);
  return p;
}

struct BwdPlan {
  int64_t nc, pieces, rows, kc, ldg, blocks, ldw;
  int64_t span;  // classes of a tile product: the piece's, or as many as its loaders reach
  size_t alpha, copy, z, g, part, acc, pack, few, parts, gemm, gemm_bytes, bytes;
  bool is_few;
};
BwdPlan bwd_plan(Way way, mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, mdnn_dtype_t t) {
  BwdPlan p = {};
  Space s;
  const bool h = t != MDNN_F32;
  const size_t es = dtype_size(t);
  // (fp32: a depth below 8 of dW's product would take a kernel for narrow operands: 4 rows, 30912 x 134, 35 us)
  p.rows = h ? up(M, 64) : M < 8 ? 8 : M;
  p.kc = h ? up(K, 64) : up(K, 4);
  p.nc = piece_classes(N, p.rows, (int64_t)128 << 20);
  if (way == GENERAL || way == PACKED) {  // (stored logits; W's copy)
    const int64_t most = way == GENERAL ? piece_classes(N, M, (int64_t)32 << 20) : piece_classes(N, p.kc, (int64_t)128 << 20);
    p.nc = p.nc < most ? p.nc : most;
  }
  if (way == STAGED && layout == MDNN_NN) p.nc = whole_chunks(N, p.nc, t);
  p.span = p.nc;
  if (way == TILED || way == STAGED) {
    const int64_t most = reach_classes(layout, K, t);
    p.span = p.nc < most ? p.nc : most;
  }
  p.pieces = ceil_div(N, p.nc);
  p.ldg = up(p.nc, h ? 64 : 4);
  const int64_t last = N - (p.pieces - 1) * p.nc;
  // row blocks that leave column sums
  p.blocks = ceil_div(p.rows, GRAD_ROWS);
  if (way != GENERAL) {
    p.blocks = 1;
    for (int64_t n : {p.nc, last})
      for (int64_t s : {n < p.span ? n : p.span, n - (n - 1) / p.span * p.span}) {  // (the widths of its tile products)
        const int64_t b = ceil_div(M, way_tile(way, M, s, K, true));
        p.blocks = b > p.blocks ? b : p.blocks;
      }
  }
  p.alpha = s.take(4);
  p.copy = s.take((size_t)p.rows * p.kc * es);
  if (way == GENERAL) {
    const size_t za = logit_bytes(M, p.nc, K, p.ldg), zb = logit_bytes(M, last, K, p.ldg);
    p.z = s.take(za > zb ? za : zb);
  }
  p.g = s.take((size_t)p.rows * p.ldg * es);
  p.part = s.take((size_t)p.blocks * p.nc * 4);
  p.acc = s.take(h && p.pieces > 1 ? (size_t)M * K * 4 : 0);
  p.ldw = layout == MDNN_NN ? p.ldg : p.kc;
  p.pack = s.take(way == PACKED ? (size_t)(layout == MDNN_NN ? p.kc : p.ldg) * p.ldw * 2 : 0);
  for (int64_t n : {p.nc, last})
    for (size_t b : {gemm_ws_bytes(t, M, n, K), gemm_ws_bytes(t, M, K, n), gemm_ws_bytes(t, M, K, up(n, 64)),
                     gemm_ws_bytes(t, n, K, p.rows), gemm_ws_bytes(t, K, n, p.rows)})
      p.gemm_bytes = b > p.gemm_bytes ? b : p.gemm_bytes;
  p.is_few = p.pieces == 1 && xent_few_ok(layout == MDNN_NT, t, M, N, K);
  p.few = s.take(p.is_few ? (size_t)few_plan(layout == MDNN_NT, N, K).parts * M * K * 4 : 0);
  const int splits = dx_splits(M, K, N, t).splits;
  p.parts = s.take((way == STAGED || way == GENERAL) && p.pieces == 1 && splits > 1 ? (size_t)splits * M * K * 4 : 0);
  p.gemm = s.take(p.gemm_bytes);
  p.bytes = s.at;
  return p;
}

// Whether W's rows are as the tiles read them: on 16 bytes, 32-bit offsets over
// a tile product's rows; or as the register-staged tiles do.
bool w_fits(Way way, mdnn_layout_t layout, int64_t M, int64_t K, int64_t ldx, const void* w, int64_t ldw, int64_t N,
            int64_t nc, mdnn_dtype_t t) {
  if (way == TILED)
    return aligned(w, 16) && ldw % 8 == 0 && (layout == MDNN_NN ? 64 * ldw + nc : (nc + 255) * ldw) < (int64_t)1 << 31;
  if (way == STAGED) {
    const int64_t last = N - (N - 1) / nc * nc;
    return xent_reg_ok(t, XentProduct{nullptr, w, ldx, ldw, M, nc, K, nc, layout == MDNN_NT, false}) &&
           xent_reg_ok(t, XentProduct{nullptr, w, ldx, ldw, M, last, K, last, layout == MDNN_NT, false});
  }
  return true;
}

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

Pack pack_of(const void* src, int64_t ld, int64_t rows, int64_t cols, void* dst, int64_t all, int64_t ldc) {
  const int64_t gx = ceil_div(ldc, 512), most = ((int64_t)1 << 22) / gx;
  return {(const uint16_t*)src, ld, rows, cols, (uint16_t*)dst, all, ldc, (uint32_t)gx,
          capped(ceil_div(all, 16), most < 1 ? 1 : most)};
}
// (either may be empty)
mdnn_status_t pack(const Pack& a, const Pack& b, hipStream_t st) {
  const uint32_t blocks = a.gx * a.gy + b.gx * b.gy;
  if (blocks == 0) return MDNN_SUCCESS;
  hipLaunchKernelGGL(xent_pack_kernel, dim3(blocks), dim3(256), 0, st, a, b);
  return check_launch("xent_pack_kernel");
}

// Classes n0 .. n0 + nc - 1 of W as the tiles read them: in place, or copied to
// rows of ldc by `copy`, zeros past the sizes (the depth to kc, classes to a multiple of 64).
struct Piece {
  const void* w;
  int64_t ldw, ext;  // ext: classes that class-contiguous rows have memory for
};
Piece take_piece(Way way, mdnn_layout_t layout, const void* w, int64_t ldw, size_t es, int64_t n0, int64_t nc, int64_t K,
                 int64_t kc, void* room, int64_t ldc, Pack& copy) {
  const void* p = w_piece(layout, w, ldw, n0, es);
  copy = {};
  if (way != PACKED) return {p, ldw, nc};
  const int64_t all = up(nc, 64);
  copy = layout == MDNN_NN ? pack_of(p, ldw, K, nc, room, kc, ldc) : pack_of(p, ldw, nc, K, room, all, ldc);
  return {room, ldc, all};
}

template <class T>
mdnn_status_t tiles(Way way, const XentProduct& p, const XentTile& x, hipStream_t st) {
  if constexpr (T::id != MDNN_F32) {
    if (way != STAGED) return xent_tiles<T>(p, x, st);
  }
  return xent_reg<T>(p, x, st);
}

template <class T>
mdnn_status_t run_fwd(Way way, mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx,
                      const void* w, int64_t ldw, const float* bias, const int32_t* labels, int32_t ignored, float* loss,
                      float* row_loss, float* lse, char* ws, hipStream_t st) {
  const mdnn_dtype_t t = T::id;
  const FwdPlan p = fwd_plan(way, layout, M, N, K, t);
  Pair *pairs = (Pair*)(ws + p.pairs), *run = (Pair*)(ws + p.run);
  float *zlab = (float*)(ws + p.zlab), *z = (float*)(ws + p.z);
  Tally* tally = (Tally*)(ws + p.tally);
  uint32_t* done = (uint32_t*)(ws + p.done);
  Pack x_copy = {};
  if (way < STAGED && !(aligned(x, 16) && ldx % 8 == 0 && K % 64 == 0 && (M + 255) * ldx < (int64_t)1 << 31)) {
    x_copy = pack_of(x, ldx, M, K, ws + p.copy, M, p.kc);
    x = ws + p.copy, ldx = p.kc;
  }
  for (int64_t i = 0; i < p.pieces; ++i) {
    const int64_t n0 = i * p.nc, nc = n0 + p.nc < N ? p.nc : N - n0;
    const float* b = bias ? bias + n0 : nullptr;
    int64_t n = 1;
    if (way == GENERAL) {
      const int64_t ldz = up(p.nc, 4);
      Logits q;
      MDNN_TRY(general_logits(layout, M, nc, K, x, ldx, w_piece(layout, w, ldw, n0, dtype_size(t)), ldw, t, b, z, ldz,
                              ws + p.gemm, p.gemm_bytes, q, st));
      hipLaunchKernelGGL(xent_stats_kernel, dim3(capped(M, 1 << 20)), dim3(256), 0, st, q, M, nc, n0, labels, pairs, zlab,
                         done);
      MDNN_TRY(check_launch("xent_stats_kernel"));
    } else {
      Pack copy;
      const Piece q = take_piece(way, layout, w, ldw, dtype_size(t), n0, nc, K, p.kc, ws + p.pack, p.ldw, copy);
      MDNN_TRY(pack(x_copy, copy, st));
      x_copy = {};
      XentProduct a = {x, q.w, ldx, q.ldw, M, nc, way == STAGED ? K : p.kc, q.ext, layout == MDNN_NT, false};
      XentTile e = {};
      e.bias = b, e.labels = labels, e.ignored = ignored, e.n0 = n0, e.classes = N, e.pairs = pairs, e.zlab = zlab, e.done = done;
      MDNN_TRY(tiles<T>(way, a, e, st));
      n = ceil_div(nc, way_tile(way, M, nc, K, false));
    }
    const Pair* before = i > 0 ? run : nullptr;
    Pair* after = i + 1 < p.pieces ? run : nullptr;
    if (rows_per_block(M) == 16)
      hipLaunchKernelGGL(xent_rows_kernel<16>, dim3((unsigned)p.blocks), dim3(1024), 0, st, pairs, n, before, after, M, N,
                         zlab, labels, ignored, lse, row_loss, loss, tally, done);
    else
      hipLaunchKernelGGL(xent_rows_kernel<64>, dim3((unsigned)p.blocks), dim3(1024), 0, st, pairs, n, before, after, M, N,
                         zlab, labels, ignored, lse, row_loss, loss, tally, done);
    MDNN_TRY(check_launch("xent_rows_kernel"));
  }
  return MDNN_SUCCESS;
}

// Whether a gradient's product of 16-bit operands may split its depth, where its
// 128 x 128 tiles are below 128 (else none is split).  From 128 tiles of 64 x 64 on,
// whole depths run on those.  Up to 256 they are one round of workgroups, and parts and
// their sum win the sooner the fewer they are (bf16, whole and split: 512 x 1024 over
// 3968 15.4 and 16.3 us, over 6976 23.0 and 21.3; 512 x 1536 over 7040 23.6 and 24.6,
// over 9984 31.2 and 29.5; 1000 x 1000 NN over 9984 40.2 and 38.1, but NT 32.2 and 36.6);
// above they are two, and parts win from about 3000 on (448 x 2368 over 2560 26.2 and
// 19.5; 1408 x 1408 over 2560 22.3 and 23.6, over 4032 31.6 and 29.0; 640 x 3200 over
// 2944 29.8 and 29.4, over 6016 55 and 46).
bool product_splits(int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = ceil_div(M, 64) * ceil_div(N, 64);
  return tiles < 128 || K > (tiles > 256 ? 3000 : 40 * tiles);
}

template <class T>
mdnn_status_t run_bwd(Way way, mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, const void* x, int64_t ldx,
                      const void* w, int64_t ldw, const float* bias, const int32_t* labels, int32_t ignored,
                      const float* lse, const float* loss_scale, void* dx, int64_t lddx, void* dw, int64_t lddw,
                      mdnn_dtype_t dw_type, float* db, char* ws, hipStream_t st) {
  typedef typename T::storage S;
  constexpr bool H = sizeof(S) == 2;
  const mdnn_dtype_t t = T::id;
  const BwdPlan p = bwd_plan(way, layout, M, N, K, t);
  const float scale = t == MDNN_F16 ? 32768.0f : 1.0f;
  float* alpha = (float*)(ws + p.alpha);
  S* copy = (S*)(ws + p.copy);
  float* z = (float*)(ws + p.z);
  S* g = (S*)(ws + p.g);
  float* part = db ? (float*)(ws + p.part) : nullptr;
  void* gw = ws + p.gemm;
  const bool joined = H && p.pieces > 1;
  float* acc = joined ? (float*)(ws + p.acc) : nullptr;
  // Few rows are read where they are: their kernels leave out the ignored ones.
  const bool few = p.is_few && (dx || dw);
  const XentProduct in_place = {x, w, ldx, ldw, M, p.span, K, p.span, layout == MDNN_NT, true};
  const bool here = few && (way == GENERAL || (way == STAGED && xent_reg_ok(t, in_place)) ||
                            (way == TILED && aligned(x, 16) && ldx % 8 == 0 && (M + 255) * ldx < (int64_t)1 << 31));
  if (here) {
    copy = (S*)x;
  } else {
    const uint32_t own = capped(p.rows, 1 << 16) + 1;
    Pack first;
    take_piece(way, layout, w, ldw, dtype_size(t), 0, p.nc < N ? p.nc : N, K, p.kc, ws + p.pack, p.ldw, first);
    hipLaunchKernelGGL((xent_prepare_kernel<T>), dim3(own + first.gx * first.gy), dim3(256), 0, st, (const S*)x, ldx, M, K,
                       labels, ignored, loss_scale, 1.0f / scale, alpha, copy, p.rows, p.kc, own, first);
    MDNN_TRY(check_launch("xent_prepare_kernel"));
  }
  const int64_t ldc = here ? ldx : p.kc;
  for (int64_t n0 = 0; n0 < N; n0 += p.nc) {
    const int64_t nc = n0 + p.nc < N ? p.nc : N - n0;
    const float* b = bias ? bias + n0 : nullptr;
    Piece q = {w_piece(layout, w, ldw, n0, sizeof(S)), ldw, nc};
    // db of `n` classes from class s of the piece on, from the column sums that `blocks` row blocks left
    auto sums = [&](int64_t s, int64_t n, int64_t blocks) {
      hipLaunchKernelGGL(xent_db_kernel, dim3((unsigned)ceil_div(n, 64)), dim3(256), 0, st, part + s, blocks, p.nc, n,
                         alpha, scale, db + n0 + s);
      return check_launch("xent_db_kernel");
    };
    if (way == GENERAL) {
      Logits l;
      MDNN_TRY(general_logits(layout, M, nc, K, copy, ldc, q.w, ldw, t, b, z, p.ldg, gw, p.gemm_bytes, l, st));
      hipLaunchKernelGGL((xent_grad_kernel<T>),
                         dim3((unsigned)ceil_div(p.ldg, 1024), capped(ceil_div(p.rows, GRAD_ROWS), 65535)), dim3(256), 0, st, l, M,
                         p.rows, nc, n0, labels, ignored, N, lse, scale, g, p.ldg, part, p.nc, loss_scale,
                         here ? alpha : nullptr);
      MDNN_TRY(check_launch("xent_grad_kernel"));
      if (db) MDNN_TRY(sums(0, nc, p.blocks));
    } else {
      Pack next;
      q = take_piece(way, layout, w, ldw, dtype_size(t), n0, nc, K, p.kc, ws + p.pack, p.ldw, next);
      if (n0 > 0) MDNN_TRY(pack(next, {}, st));  // (the first is copied beside x)
      for (int64_t s = 0; s < nc; s += p.span) {
        const int64_t n = s + p.span < nc ? p.span : nc - s;
        XentProduct a = {copy, w_piece(layout, q.w, q.ldw, s, sizeof(S)), ldc, q.ldw, M, n, way == STAGED ? K : p.kc,
                         q.ext - s, layout == MDNN_NT, true};
        XentTile e = {};
        e.bias = b ? b + s : nullptr, e.labels = labels, e.ignored = ignored, e.n0 = n0 + s, e.classes = N, e.lse = lse;
        const int64_t blocks = ceil_div(M, way_tile(way, M, n, K, true));
        e.alone = blocks == 1, e.loss_scale = loss_scale, e.alpha = alpha, e.db = e.alone ? db : nullptr;
        e.scale = scale, e.g = g + s, e.ldg = p.ldg, e.width = p.ldg - s, e.rows = p.rows, e.ldp = p.nc;
        e.part = e.alone || !part ? nullptr : part + s;
        MDNN_TRY(tiles<T>(way, a, e, st));
        if (db && blocks > 1) MDNN_TRY(sums(s, n, blocks));
      }
    }
    if (few) {
      XentFew a = {};
      a.x = copy, a.g = g, a.w = q.w, a.dw = dw, a.part = (float*)(ws + p.few), a.alpha = alpha;
      a.labels = here ? labels : nullptr, a.ignored = ignored;
      a.M = M, a.N = N, a.K = K, a.ldx = ldc, a.ldg = p.ldg, a.ldw = q.ldw, a.lddw = lddw, a.by_class = layout == MDNN_NT;
      return xent_few<T>(a, dw ? dw_type : MDNN_F32, dx, lddx, st);
    }
    const mdnn_layout_t back = layout == MDNN_NN ? MDNN_NT : MDNN_NN;
    const SplitPlan sp = dx_splits(M, K, nc, t);
    if (dx && (way == STAGED || way == GENERAL) && p.pieces == 1 && sp.splits > 1 &&
        gemm_reg_ok(t, back, M, K, nc, p.ldg, q.ldw, sp.splits)) {
      Epilogue ep{};
      ep.alpha = 1.0f, ep.partial = (float*)(ws + p.parts), ep.k_per_split = sp.k_per_split;
      MDNN_TRY(gemm_reg(t, MDNN_F32, back, M, K, nc, g, p.ldg, q.w, q.ldw, ep, sp.splits, st));
      hipLaunchKernelGGL((xent_parts_kernel<T>), dim3(capped(ceil_div(K, 256), 1024), capped(M, 4096)), dim3(256), 0, st,
                         ep.partial, sp.splits, M, K, alpha, (S*)dx, lddx);
      MDNN_TRY(check_launch("xent_parts_kernel"));
    } else if (dx) {
      char* d = joined ? (char*)acc : (char*)dx;
      const int64_t ldd = joined ? K : lddx;
      const size_t gb = product_splits(M, K, nc) ? p.gemm_bytes : 0, dd = joined ? 4 : sizeof(S);
      // (class-contiguous W: dx's columns in as many products as 32-bit offsets reach of W's rows)
      const int64_t per = layout == MDNN_NN ? reach_rows(K, nc, q.ldw, t) : K;
      for (int64_t f = 0; f < K; f += per)
        // (a copied piece's padding is zeros on both sides: whole steps)
        MDNN_TRY(gemm_mixed_ws(back, M, f + per < K ? per : K - f, way == PACKED ? up(nc, 64) : nc, 1.0f, g, p.ldg,
                               (const S*)q.w + f * q.ldw, q.ldw, t, n0 > 0 ? 1.0f : 0.0f, d + f * dd, ldd, d + f * dd, ldd,
                               joined ? MDNN_F32 : t, nullptr, MDNN_ACT_NONE, nullptr, 0, gb ? gw : nullptr, gb, st, nullptr,
                               alpha, 0, way == PACKED ? p.kc : 0));
    }
    if (dw) {
      const size_t ds = dtype_size(dw_type), gb = product_splits(nc, K, p.rows) ? p.gemm_bytes : 0;
      void* gv = gb ? gw : nullptr;
      if constexpr (H) {
        if (layout == MDNN_NN ? xent_outer_ok(K, nc, p.rows) : xent_outer_ok(nc, K, p.rows)) {
          if (layout == MDNN_NN)
            MDNN_TRY(xent_outer<T>(copy, p.kc, K, g, p.ldg, nc, p.rows, alpha, (char*)dw + n0 * ds, lddw, dw_type, st));
          else
            MDNN_TRY(xent_outer<T>(g, p.ldg, nc, copy, p.kc, K, p.rows, alpha, (char*)dw + n0 * lddw * ds, lddw, dw_type, st));
          continue;
        }
      }
      if (layout == MDNN_NN)
        MDNN_TRY(gemm_mixed_ws(MDNN_TN, K, nc, p.rows, 1.0f, copy, p.kc, g, p.ldg, t, 0.0f, nullptr, 0,
                               (char*)dw + n0 * ds, lddw, dw_type, nullptr, MDNN_ACT_NONE, nullptr, 0, gv, gb, st,
                               nullptr, alpha, p.kc, up(nc, 8)));
      else
        MDNN_TRY(gemm_mixed_ws(MDNN_TN, nc, K, p.rows, 1.0f, g, p.ldg, copy, p.kc, t, 0.0f, nullptr, 0,
                               (char*)dw + n0 * lddw * ds, lddw, dw_type, nullptr, MDNN_ACT_NONE, nullptr, 0, gv,
                               gb, st, nullptr, alpha, up(nc, 8), p.kc));
    }
  }
  if (dx && joined) {
    hipLaunchKernelGGL((xent_round_kernel<T>), dim3(capped(ceil_div(K, 256), 1024), capped(M, 4096)), dim3(256), 0, st,
                       acc, M, K, (S*)dx, lddx);
    MDNN_TRY(check_launch("xent_round_kernel"));
  }
  return MDNN_SUCCESS;
}

}  // namespace

XentWay xent_way(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, int64_t ldx, const void* w, int64_t ldw,
                 mdnn_dtype_t t, bool backward) {
  for (Way way = way_by_size(M, N, K, t, backward);; way = way_below(way)) {
    int64_t nc, ld = ldx;
    if (backward) {
      const BwdPlan p = bwd_plan(way, layout, M, N, K, t);
      nc = p.span, ld = p.kc;  // (x's copy)
    } else {
      nc = fwd_plan(way, layout, M, N, K, t).nc;
    }
    if (w_fits(way, layout, M, K, ld, w, ldw, N, nc, t)) return {(int32_t)way, nc};
  }
}

}  // namespace mdnn

using namespace mdnn;

// Bytes of a call's workspace: the most that a way open to its sizes takes.
static size_t fwd_bytes(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, mdnn_dtype_t t) {
  size_t most = 0;
  for (Way w = way_by_size(M, N, K, t, false);; w = way_below(w)) {
    const size_t b = fwd_plan(w, layout, M, N, K, t).bytes;
    most = b > most ? b : most;
    if (w == GENERAL || w == PACKED) return most;
  }
}
static size_t bwd_bytes(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, mdnn_dtype_t t) {
  size_t most = 0;
  for (Way w = way_by_size(M, N, K, t, true);; w = way_below(w)) {
    const size_t b = bwd_plan(w, layout, M, N, K, t).bytes;
    most = b > most ? b : most;
    if (w == GENERAL || w == PACKED) return most;
  }
}

extern "C" size_t mdnn_linear_xent_fwd_workspace(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K,
                                                 mdnn_dtype_t dtype) {
  if ((layout != MDNN_NN && layout != MDNN_NT) || !sizes_ok(M, N, K) || !dtype_ok(dtype) || M == 0) return 0;
  return fwd_bytes(layout, M, N, K, dtype);
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
  const size_t need = fwd_bytes(layout, M, N, K, dtype);
  if (!workspace || ws_bytes < need || !aligned(workspace, 256))
    return fail(MDNN_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) required", who, need);
  const Way way = (Way)xent_way(layout, M, N, K, ldx, w, ldw, dtype, false).way;
  char* ws = (char*)workspace;
  switch (dtype) {
    case MDNN_F32:
      return run_fwd<F32>(way, layout, M, N, K, x, ldx, w, ldw, bias, labels, ignored, loss, row_loss, lse, ws, st);
    case MDNN_F16:
      return run_fwd<F16>(way, layout, M, N, K, x, ldx, w, ldw, bias, labels, ignored, loss, row_loss, lse, ws, st);
    default:
      return run_fwd<BF16>(way, layout, M, N, K, x, ldx, w, ldw, bias, labels, ignored, loss, row_loss, lse, ws, st);
  }
}

extern "C" size_t mdnn_linear_xent_bwd_workspace(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K,
                                                 mdnn_dtype_t dtype) {
  if ((layout != MDNN_NN && layout != MDNN_NT) || !sizes_ok(M, N, K) || !dtype_ok(dtype) || M == 0) return 0;
  return bwd_bytes(layout, M, N, K, dtype);
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
  const size_t need = bwd_bytes(layout, M, N, K, dtype);
  if (!workspace || ws_bytes < need || !aligned(workspace, 256))
    return fail(MDNN_ERR_WORKSPACE, "%s: workspace of %zu bytes (256-byte aligned) required", who, need);
  clear_error();
  const Way way = (Way)xent_way(layout, M, N, K, ldx, w, ldw, dtype, true).way;
  char* ws = (char*)workspace;
  switch (dtype) {
    case MDNN_F32:
      return run_bwd<F32>(way, layout, M, N, K, x, ldx, w, ldw, bias, labels, ignored, lse, loss_scale, dx, lddx, dw, lddw,
                          dw_type, db, ws, st);
    case MDNN_F16:
      return run_bwd<F16>(way, layout, M, N, K, x, ldx, w, ldw, bias, labels, ignored, lse, loss_scale, dx, lddx, dw, lddw,
                          dw_type, db, ws, st);
    default:
      return run_bwd<BF16>(way, layout, M, N, K, x, ldx, w, ldw, bias, labels, ignored, lse, loss_scale, dx, lddx, dw, lddw,
                           dw_type, db, ws, st);
  }
}

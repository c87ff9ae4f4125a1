// Pieces of the last layer's cross entropy shared by its kernels.
#pragma once

#include "common.h"
#include "internal.h"

namespace mdnn {

// A maximum m and the sum of exp(z - m) over some logits z of a row.  m is
// -Inf where there is no logit above it (none at all, or classes masked by a
// bias of -Inf): such a pair adds nothing, and differences are then taken from
// 0 so that they are no NaN.
struct Pair {
  float m, s;
};
__device__ __forceinline__ float pair_ref(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ Pair join(Pair a, Pair b) {
  const float m = fmaxf(a.m, b.m), ref = pair_ref(m);
  return {m, a.s * __expf(a.m - ref) + b.s * __expf(b.m - ref)};
}

// What a tile of a piece's logits turns into in place of being stored.
struct XentTile {
  const float* bias;  // the piece's, or null
  const int32_t* labels;
  int32_t ignored;
  int64_t n0, classes;  // the piece's first class; all classes
  // forward: tile column t leaves a pair for each row at pairs[t * M + row], the label's column its logit
  Pair* pairs;
  float* zlab;
  uint32_t* done;  // cleared
  // backward: G times `scale` in the operands' type, rows of ldg elements (a multiple of 64), zeros in rows M .. rows - 1
  // and columns past the product's up to `width` (memory of a row from g on); part: column sums of tile row t at
  // part[t * ldp + column], or null
  const float* lse;
  float scale;
  void* g;
  int64_t ldg, width, rows, ldp;
  float* part;
  // where one tile row holds all rows: db itself in place of part (or null), and a = S / counted rows over `scale` to alpha
  bool alone;
  const float* loss_scale;
  float *alpha, *db;
};

// The products whose tiles end so (16-bit operands, x K-contiguous, W
// K-contiguous or, w_kc false, class-contiguous), with the preconditions of the
// pipelined kernel: K a multiple of 64, 16-byte aligned rows, an extent of
// class-contiguous rows (ext, >= N) that is a multiple of 8.
struct XentProduct {
  const void *x, *w;
  int64_t ldx, ldw, M, N, K, ext;
  bool w_kc, backward;
};
// 256, 128 or 64: the side of the tiles, by the sizes.
int xent_tile(int64_t M, int64_t N, int64_t K, bool backward);
template <class T>
mdnn_status_t xent_tiles(const XentProduct& p, const XentTile& x, hipStream_t st);

// How a call runs (host code, for the calls and their tests): 0 tiles read W as it is, 1 copied, 2 the register-staged
// tiles do, 3 logits through the workspace; the classes of one tile product.
struct XentWay {
  int32_t way;
  int64_t classes;
};
XentWay xent_way(mdnn_layout_t layout, int64_t M, int64_t N, int64_t K, int64_t ldx, const void* w, int64_t ldw,
                 mdnn_dtype_t t, bool backward);

// The same by the register-staged kernel: any type, element address and
// leading dimension that xent_reg_ok takes (ext is not used); tiles of 128 or 64.
int xent_reg_tile(int64_t M, int64_t N);
bool xent_reg_ok(mdnn_dtype_t t, const XentProduct& p);
template <class T>
mdnn_status_t xent_reg(const XentProduct& p, const XentTile& x, hipStream_t st);

// dW and dx of up to eight rows in one pass over W (xent_few.hip).
struct XentFew {
  const void *x, *g, *w;
  const int32_t* labels;  // rows of x whose label is ignored count as zeros; null: they are
  int32_t ignored;
  void* dw;               // or null
  float* part;            // few_plan's parts [parts][M][K], or null
  const float* alpha;
  int64_t M, N, K, ldx, ldg, ldw, lddw;
  bool by_class;
  int tx;       // set by xent_few
  int64_t per;
};
struct FewPlan {
  int tx;                              // threads across a row of W
  int64_t strips, splits, per, parts;  // per: rows of W in a split
};
FewPlan few_plan(bool by_class, int64_t N, int64_t K);
bool xent_few_ok(bool by_class, mdnn_dtype_t t, int64_t M, int64_t N, int64_t K);
template <class T>
mdnn_status_t xent_few(XentFew a, mdnn_dtype_t dw_type, void* dx, int64_t lddx, hipStream_t st);

// D [R][ldd] of d_type = *alpha * P^T Q for `rows` rows, a multiple of 64, of 16-bit P [rows][ldp >= R] and Q [rows][ldq
// >= C] on 16 bytes, leading dimensions up(R, 64) and up(C, 64) (xent_outer.hip).
bool xent_outer_ok(int64_t R, int64_t C, int64_t rows);
template <class T>
mdnn_status_t xent_outer(const void* p, int64_t ldp, int64_t R, const void* q, int64_t ldq, int64_t C, int64_t rows,
                         const float* alpha, void* d, int64_t ldd, mdnn_dtype_t d_type, hipStream_t st);

}  // namespace mdnn

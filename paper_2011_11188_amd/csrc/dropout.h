// Dropout's decisions, drawn where they are needed and never stored: element
// (r, c) of a tensor takes 16 bits of Philox 4x32 with ten rounds (Salmon,
// Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011)
// under the 64-bit key `seed` at the counter (c / 8, r, step, site): 128 bits
// for eight columns, the lowest 16 bits of the first word first.  It is
// dropped where they are below t = floor(p 2^16 + 1/2); what is kept is
// multiplied by 2^16 / (2^16 - t), the inverse of the exact chance to be kept.
//
// A block of eight costs twenty 32 x 32 -> 64-bit products and is drawn while
// the rows' loads are on their way.
#pragma once

#include <math.h>

#include "row_chunk.h"

namespace mdnn {
namespace {

struct DropArgs {
  const uint64_t* rng;  // device: {seed, step}; null without dropout
  uint32_t t, site;
  float s;
};

// Host: t and s of a chance p in [0, 1] (t = 2^16 drops everything).
inline DropArgs drop_args(float p, const void* rng, uint32_t site) {
  DropArgs d;
  d.t = (uint32_t)floor((double)p * 65536.0 + 0.5);
  d.s = d.t < 65536 ? 65536.0f / (float)(65536 - d.t) : 0.0f;
  d.rng = d.t ? (const uint64_t*)rng : nullptr;
  d.site = site;
  return d;
}

struct DropKey {
  uint32_t k0, k1, step;
};
__device__ __forceinline__ DropKey drop_key(const DropArgs& d) {
  const uint64_t seed = d.rng[0];
  return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)d.rng[1]};
}

// The 16 bits of eight consecutive columns of a row, in order.
struct DropBits {
  uint32_t w[4];
  __device__ __forceinline__ void draw(const DropArgs& d, DropKey k, uint32_t block, uint32_t row) {
    uint32_t a = block, b = row, c = k.step, e = d.site;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
      const uint64_t u = (uint64_t)a * 0xD2511F53u, v = (uint64_t)c * 0xCD9E8D57u;
      a = (uint32_t)(v >> 32) ^ b ^ k.k0;
      b = (uint32_t)v;
      c = (uint32_t)(u >> 32) ^ e ^ k.k1;
      e = (uint32_t)u;
      k.k0 += 0x9E3779B9u;
      k.k1 += 0xBB67AE85u;
    }
    w[0] = a, w[1] = b, w[2] = c, w[3] = e;
  }
  // For a chunk whose first `lo` elements are not its own: the bits move up to
  // the elements that are (those below lo are not used).
  __device__ __forceinline__ void shift(int lo) {
    if (lo & 4) w[3] = w[1], w[2] = w[0];
    if (lo & 2) w[3] = w[2], w[2] = w[1], w[1] = w[0];
    if (lo & 1) {
      w[3] = (w[3] << 16) | (w[2] >> 16);
      w[2] = (w[2] << 16) | (w[1] >> 16);
      w[1] = (w[1] << 16) | (w[0] >> 16);
      w[0] = w[0] << 16;
    }
  }
  // keep ? s * x : 0 (a selection: what is dropped may be Inf or NaN)
  __device__ __forceinline__ float apply(const DropArgs& d, int e, float x) const {
    const uint32_t half = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
    return half >= d.t ? mul_rn(x, d.s) : 0.0f;
  }
};

}  // namespace
}  // namespace mdnn

// Host build of the shared-memory layout of a logits tile's numbers: where the
// bias lies that the tile's end reads four at a time.
#include <stddef.h>

#include "../paper_2011_11188_amd/csrc/gemm_lds.h"
#include "../paper_2011_11188_amd/csrc/xent_end.h"

using namespace mdnn;

extern "C" int host_xent_numbers_alignment() {
  typedef XentNumbers<lds::Tile256, false> F;
  typedef XentNumbers<lds::Tile<64, 64, 2, 2, 2>, true> B;
  const size_t a = alignof(F) < alignof(B) ? alignof(F) : alignof(B);
  return offsetof(F, bias) % 16 == 0 && offsetof(B, bias) % 16 == 0 ? (int)a : 0;
}

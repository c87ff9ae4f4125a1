// The last layer's products with BF16 operands (xent_tiles), a translation unit
// of their own.
#include "xent_pipe.h"

namespace mdnn {
template mdnn_status_t xent_tiles<BF16>(const XentProduct&, const XentTile&, hipStream_t);
}  // namespace mdnn

// Products with 4-bit weights, many rows, bfloat16 activations.
#include "int4_tiles.h"

namespace wq {

hipError_t launch_int4_tiles_bfloat(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, hipStream_t s) {
    return launch_tiles_of<WQ_BF16>(x, x_stride, w, o, s);
}

}  // namespace wq

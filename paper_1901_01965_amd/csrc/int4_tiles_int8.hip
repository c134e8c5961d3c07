// Products with 4-bit weights, many rows, int8 activations.
#include "int4_tiles.h"

namespace wq {

hipError_t launch_int4_tiles_int8(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, int parts, hipStream_t s) {
    return launch_tiles_of<WQ_I8>(x, x_stride, w, o, parts, s);
}

}  // namespace wq

// Products with 4-bit weights, few rows, bfloat16 activations.
#include "int4_rows.h"

namespace wq {

hipError_t launch_int4_rows_bfloat(const void* x, long long x_stride, const Int4Weights& w, const Int4Output& o, hipStream_t s) {
    return launch_rows_of<WQ_BF16>(x, x_stride, w, o, s);
}

}  // namespace wq

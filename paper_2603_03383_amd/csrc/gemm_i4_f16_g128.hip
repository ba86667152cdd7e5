// Products with 4-bit weights: f16 rows, groups of 128 features.
#include "gemm_i4.h"

namespace mdz {
template int launch_i4<f16_t, 1>(const I4Product&, bool, bool, const I4Plan&, hipStream_t);
}

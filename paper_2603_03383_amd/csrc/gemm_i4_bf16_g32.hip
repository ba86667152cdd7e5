// Products with 4-bit weights: bf16 rows, groups of 32 features.
#include "gemm_i4.h"

namespace mdz {
template int launch_i4<bf16_t, 4>(const I4Product&, bool, bool, const I4Plan&, hipStream_t);
}

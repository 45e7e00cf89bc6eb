// Attention over the 4-bit cache, heads of 128 elements.
#include "bnn_cache4_attend.h"

namespace bnn {
int launch_cache4_attend128(const Attend4& a, int dtype, int rows, hipStream_t s) { return launch_attend_type<128>(a, dtype, rows, s); }
}  // namespace bnn

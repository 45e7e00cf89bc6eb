// Attention over the 4-bit cache, heads of 96 elements.
#include "bnn_cache4_attend.h"

namespace bnn {
int launch_cache4_attend96(const Attend4& a, int dtype, int rows, hipStream_t s) { return launch_attend_type<96>(a, dtype, rows, s); }
}  // namespace bnn

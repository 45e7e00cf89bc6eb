// Attention over the 4-bit cache, heads of 64 elements.
#include "bnn_cache4_attend.h"

namespace bnn {
int launch_cache4_attend64(const Attend4& a, int dtype, int rows, hipStream_t s) { return launch_attend_type<64>(a, dtype, rows, s); }
}  // namespace bnn

// Attention over a cache of codes: keys in 4 bits, values in 4.
#include "jq_codes.h"

namespace jq {
template hipError_t launch_sweeps<RowsCoded<4, 4>>(const AttendArgs&, int, int, bool, dim3, hipStream_t);
}  // namespace jq

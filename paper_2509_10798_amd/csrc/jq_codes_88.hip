// Attention over a cache of codes: keys in 8 bits, values in 8.
#include "jq_codes.h"

namespace jq {
template hipError_t launch_sweeps<RowsCoded<8, 8>>(const AttendArgs&, int, int, bool, dim3, hipStream_t);
}  // namespace jq

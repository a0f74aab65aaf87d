// The kernels of decoding on a pruned cache in bf16.  A code object of its own, so that the
// kernels of an eviction step keep the places in theirs that jq_lib.hip chooses for them.
#include "jq_attend.hip"
#include "jq_weight.hip"

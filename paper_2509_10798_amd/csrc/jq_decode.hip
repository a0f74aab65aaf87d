// The second translation unit of libjq.so: the kernels of decoding on a pruned cache.  A code object of its own, so that the
// kernels of an eviction step keep the places in theirs that jq_lib.hip chooses for them.
#include "jq_attend.hip"
#include "jq_weight.hip"

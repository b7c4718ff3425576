// Attention over the paged cache for heads of 96 coordinates.
#include "kv_many.h"

namespace ivftq {
template hipError_t kv_attend_d<96>(const KvAttend&, const KvWork&, int, hipStream_t);
}

// Attention over the paged cache for heads of 256 coordinates.
#include "kv_many.h"

namespace ivftq {
template hipError_t kv_attend_d<256>(const KvAttend&, const KvWork&, int, hipStream_t);
}

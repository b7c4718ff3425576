// Scores of pages and attention over chosen pages for heads of 256 coordinates.
#include "kv_pick.h"

namespace ivftq {
template hipError_t kv_score_d<256>(const KvAttend&, const void*, float*, int, hipStream_t);
template hipError_t kv_picked_d<256>(const KvAttend&, const PickWork&, const int32_t*, int, int, hipStream_t);
}

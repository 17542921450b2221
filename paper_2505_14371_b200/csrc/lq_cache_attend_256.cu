// Attention over the quantised cache, rows of 256 coordinates.
#include "lq_cache_attend.cuh"

namespace lq {
cudaError_t launch_cache_attend_256(const CacheAttendArgs& a, cudaStream_t s) { return attend::launch<256>(a, s); }
}  // namespace lq

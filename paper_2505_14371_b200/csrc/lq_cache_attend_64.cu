// Attention over the quantised cache, rows of 64 coordinates.
#include "lq_cache_attend.cuh"

namespace lq {
cudaError_t launch_cache_attend_64(const CacheAttendArgs& a, cudaStream_t s) { return attend::launch<64>(a, s); }
}  // namespace lq

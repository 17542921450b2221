// Attention over the quantised cache, rows of 128 coordinates.
#include "lq_cache_attend.cuh"

namespace lq {
cudaError_t launch_cache_attend_128(const CacheAttendArgs& a, cudaStream_t s) { return attend::launch<128>(a, s); }
}  // namespace lq

// The row kernel of attention over f16 caches.
#include "kvr_attend_rows.cuh"

namespace kvr {
cudaError_t launch_attend_f16(const AttendArgs &a, int tiles, int slices, cudaStream_t s) { return launch_rows<KVR_CACHE_F16>(a, tiles, slices, s); }
}  // namespace kvr

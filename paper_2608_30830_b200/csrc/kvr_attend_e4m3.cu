// The row kernel of attention over e4m3 caches.
#include "kvr_attend_rows.cuh"

namespace kvr {
cudaError_t launch_attend_e4m3(const AttendArgs &a, int tiles, int slices, cudaStream_t s) { return launch_rows<KVR_CACHE_E4M3>(a, tiles, slices, s); }
}  // namespace kvr

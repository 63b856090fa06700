// The row kernel of attention over int8 caches.
#include "kvr_attend_rows.cuh"

namespace kvr {
cudaError_t launch_attend_int8(const AttendArgs &a, int tiles, int slices, cudaStream_t s) { return launch_rows<KVR_CACHE_INT8>(a, tiles, slices, s); }
}  // namespace kvr

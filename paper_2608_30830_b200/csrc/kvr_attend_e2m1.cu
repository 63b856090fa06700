// Attention over e2m1 caches: the row kernel.
#include "kvr_attend_rows.cuh"

namespace kvr {
cudaError_t launch_attend_e2m1(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s) {
  return launch_rows<KVR_CACHE_E2M1>(a, tiles, slices, s);
}
}  // namespace kvr

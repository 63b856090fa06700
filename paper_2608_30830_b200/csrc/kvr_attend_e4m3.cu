// Attention over e4m3 caches: both kernels.
#include "kvr_attend_rows.cuh"
#include "kvr_attend_tiles.cuh"

namespace kvr {
cudaError_t launch_attend_e4m3(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s) {
  return tiles ? launch_rows<KVR_CACHE_E4M3>(a, tiles, slices, s) : launch_tiles<KVR_CACHE_E4M3>(a, map, s);
}
}  // namespace kvr

// Attention over bf16 caches: both kernels.
#include "kvr_attend_rows.cuh"
#include "kvr_attend_tiles.cuh"

namespace kvr {
cudaError_t launch_attend_bf16(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s) {
  return tiles ? launch_rows<KVR_CACHE_BF16>(a, tiles, slices, s) : launch_tiles<KVR_CACHE_BF16>(a, map, s);
}
}  // namespace kvr

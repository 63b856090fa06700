// Attention over e2m1 caches: both kernels.
#include "kvr_attend_rows4.cuh"
#include "kvr_attend_tiles.cuh"

namespace kvr {
cudaError_t launch_attend_e2m1(const AttendArgs &a, int tiles, const Rows4 &r4, const CUtensorMap &map, cudaStream_t s) {
  if (!tiles) return launch_tiles<KVR_CACHE_E2M1>(a, map, s);
  if (a.c.head_dim <= 64) return launch_rows4<64>(a, tiles, r4, map, s);
  if (a.c.head_dim <= 128) return launch_rows4<128>(a, tiles, r4, map, s);
  return launch_rows4<256>(a, tiles, r4, map, s);
}
}  // namespace kvr

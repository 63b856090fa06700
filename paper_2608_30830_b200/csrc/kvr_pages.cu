// kvr_cache_copy, and the copies behind kvr_request_fork, kvr_request_resize and kvr_pool_compact.
//
// A pair's rows are contiguous in each plane (a tile).  A warp takes up to 4 KiB of a tile at a time, 8 loads of 16 bytes a lane under way:
// 32 warps an SM keep 128 KiB in flight, which is what the memory's latency asks for, and tiles of any size (1 to 32 KiB in use) leave few
// lanes idle.  Bytes are read once and written once: bound by memory.  3,000 blocks of 64 planes (tiles of 4,352 bytes; 1.67 GB
// read and written) 289 us, 5.8 TB/s, 0.89 of a plain copy; the last blocks of 8 requests, 32 layers, 7 us with the call.
#include "kvr_pages.cuh"

#include <type_traits>

#include "kvr_cache.cuh"

namespace kvr {
namespace {

constexpr int kCopyThreads = 256, kCopyAhead = 8, kCopyPiece = 32 * 16 * kCopyAhead;

struct CopyArgs {
  PoolView v;
  FastDiv per_pair, per_plane;         // pieces of a pair, of a tile
  const int2 *pairs;
  const int32_t *rows;                 // or NULL: all_rows of each
  int32_t *status;
  int all_rows;
  unsigned pieces;
};

struct DevicePairs {};

template <class List>
__global__ void __launch_bounds__(kCopyThreads, 4) copy_kernel(const __grid_constant__ CopyArgs a, const __grid_constant__ List list) {
  constexpr bool kInline = std::is_same<List, InlinePairs>::value;
  const int lane = threadIdx.x & 31;
  const unsigned warps = gridDim.x * (kCopyThreads / 32);
  for (unsigned piece = blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); piece < a.pieces; piece += warps) {
    const unsigned i = a.per_pair.div(piece), rest = piece - i * a.per_pair.d, plane = a.per_plane.div(rest);
    const int from = (int)(rest - plane * a.per_plane.d) * kCopyPiece;
    int2 pair;
    if constexpr (kInline) pair = list.pair[i]; else pair = __ldg(a.pairs + i);
    int rows = a.all_rows;
    if constexpr (!kInline) {
      if (a.rows) rows = __ldg(a.rows + i);
      if (pair.x == -1) continue;      // a place that is not in use
      const bool block = (unsigned)pair.x < (unsigned)a.v.num_blocks && (unsigned)pair.y < (unsigned)a.v.num_blocks;
      if (!block || (unsigned)rows > (unsigned)a.v.block_size) {
        if (rest == 0 && lane == 0) report(a.status, block ? KVR_DEV_BAD_LENGTH : KVR_DEV_BAD_BLOCK);
        continue;
      }
    }
    const int bytes = rows * a.v.row_bytes;          // of a tile: at most 1 GiB
    const char *src = a.v.base + plane * a.v.plane_stride + pair.x * a.v.block_stride + from + lane * 16;
    char *dst = a.v.base + plane * a.v.plane_stride + pair.y * a.v.block_stride + from + lane * 16;
    const int left = bytes - from - lane * 16;
    uint4 x[kCopyAhead];
#pragma unroll
    for (int k = 0; k < kCopyAhead; ++k)
      if (k * 512 < left) x[k] = __ldcs(reinterpret_cast<const uint4 *>(src + k * 512));
#pragma unroll
    for (int k = 0; k < kCopyAhead; ++k)
      if (k * 512 < left) __stcs(reinterpret_cast<uint4 *>(dst + k * 512), x[k]);
  }
}

// False where the pieces do not fit 31 bits.
bool lay_out(CopyArgs &a, int n, int rows) {
  const unsigned per_plane = (unsigned)(((long long)rows * a.v.row_bytes + kCopyPiece - 1) / kCopyPiece);
  const unsigned long long per_pair = (unsigned long long)per_plane * a.v.planes, pieces = per_pair * n;
  if (pieces > INT32_MAX) return false;
  a.per_plane = FastDiv(per_plane);
  a.per_pair = FastDiv((unsigned)per_pair);
  a.all_rows = rows;
  a.pieces = (unsigned)pieces;
  return true;
}

unsigned grid_of(const CopyArgs &a) {
  const unsigned need = (a.pieces + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  return need < 148 * 4 ? need : 148 * 4;
}

}  // namespace

cudaError_t copy_blocks(const PoolView &v, const int2 *pairs, int n, int rows, cudaStream_t s) {
  if (rows == 0) return cudaSuccess;
  InlinePairs list;
  for (int at = 0; at < n;) {
    CopyArgs a{};
    a.v = v;
    int m = n - at < kInlinePairs ? n - at : kInlinePairs;
    while (m > 1 && !lay_out(a, m, rows)) m /= 2;
    if (!lay_out(a, m, rows)) return cudaErrorInvalidValue;
    for (int i = 0; i < m; ++i) list.pair[i] = pairs[at + i];
    copy_kernel<<<grid_of(a), kCopyThreads, 0, s>>>(a, list);
    if (const cudaError_t e = cudaGetLastError()) return e;
    at += m;
  }
  return cudaSuccess;
}

}  // namespace kvr

using namespace kvr;

extern "C" kvr_status kvr_cache_copy(const kvr_cache_spec *spec, void *device_pool, const int32_t *pairs, const int32_t *rows, int32_t n_pairs,
                                     int32_t *status, void *stream) {
  CacheView c{};
  if (kvr_status st = layer_view(spec, device_pool, 0, &c)) return st;
  if (n_pairs < 0) return fail_cache(KVR_ERR_INVALID_ARG, "n_pairs < 0");
  if (n_pairs > 0 && !pairs) return fail_cache(KVR_ERR_INVALID_ARG, "pairs is NULL");
  if (((uintptr_t)pairs & 7) || (((uintptr_t)rows | (uintptr_t)status) & 3))
    return fail_cache(KVR_ERR_INVALID_ARG, "pairs must be 8-byte aligned, rows and status 4-byte");
  if (n_pairs == 0) return KVR_OK;
  CopyArgs a{};
  a.v = PoolView{c.base, c.v_offset, c.block_stride, 2 * spec->layers, spec->num_blocks, spec->block_size, c.row_bytes};
  if (2ll * spec->layers > INT32_MAX || !lay_out(a, n_pairs, spec->block_size)) return fail_cache(KVR_ERR_INVALID_ARG, "n_pairs is too large for one call");
  a.pairs = reinterpret_cast<const int2 *>(pairs);
  a.rows = rows;
  a.status = status;
  copy_kernel<<<grid_of(a), kCopyThreads, 0, static_cast<cudaStream_t>(stream)>>>(a, DevicePairs{});
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? KVR_OK : fail_cache(KVR_ERR_CUDA, cudaGetErrorString(e));
}

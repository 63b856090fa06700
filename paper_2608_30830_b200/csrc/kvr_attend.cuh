// Attention over the paged cache: how a call's work is cut up, and what its kernels share.
//
// Work is cut along the keys.  A segment is one request, one group of KV heads and one tile of its query rows (row =
// new token x query heads of one KV head + query head); a unit is `unit_keys` keys of a segment.  Segments follow each
// other request by request, and the units of all of them are dealt out in equal runs, one to each CTA of a grid that
// fills the GPU once: ragged requests keep all SMs busy to the end, and the cut needs nothing from the host but the
// grid's size.  A CTA that holds a whole segment writes its result; the pieces of a cut segment go to the workspace as
// (maximum, sum, accumulator), and the CTA that hands in the last one joins them.  More than 16 pieces are joined by groups of 16
// first, so that one long request is not joined by one CTA.  Pieces are always taken in the order of their keys: results do not
// depend on timing.
#pragma once
#include <cuda.h>

#include "kvr_cache.cuh"

namespace kvr {

struct AttendArgs {
  Batch b;
  CacheView c;
  FastDiv bs, group;         // block size; query heads per KV head
  Rows q, out;
  float *lse;                // or NULL
  const unsigned long long *mask;    // or NULL: causal
  int mask_words;
  float scale_log2;          // scale * log2(e)
  int q_heads;
  int head_groups, group_heads;      // KV heads are taken group_heads at a time
  int row_tile;              // query rows of a segment
  int unit_keys;
  int box_rows;              // tokens of a TMA box (tile kernel): 8 or 16, 0: the block size does not allow one
  int ctas;                  // the grid of the main kernel
  int *handed_in;            // [2][ctas][2]: pieces of a group, groups of a segment; zero between calls
  float *part_o;             // [ctas][2][group_heads][row_tile][head_dim]
  float2 *part_ml;           // [ctas][2][group_heads][row_tile]: maximum (log2), sum
};

// The workspace holds, for every SM, two pieces of this many rows (fp32 accumulators and a pair of statistics each).
constexpr int kPartRows = 256;
constexpr int kMaxSms = 160;
constexpr int kCounterBytes = 4096;
constexpr int kJoinAtOnce = 16;
static_assert(kMaxSms * 4 * 4 <= kCounterBytes, "");

#ifdef __CUDACC__
struct Lengths {
  int first, context, fresh; // of a request: first row, tokens before, new tokens
  int keys;                  // context + fresh
  int units;                 // of one segment
  int segments;
};

__device__ __forceinline__ Lengths attend_lengths(const AttendArgs &a, int r) {
  Lengths l;
  request_lengths(a.b, a.bs.d, r, l.first, l.context, l.fresh);
  l.keys = l.context + l.fresh;
  l.units = (l.keys + a.unit_keys - 1) / a.unit_keys;
  l.segments = l.fresh > 0 ? a.head_groups * (int)(((long long)l.fresh * (int)a.group.d + a.row_tile - 1) / a.row_tile) : 0;
  return l;
}
__device__ __forceinline__ long long units_of(const AttendArgs &a, int r) {
  const Lengths l = attend_lengths(a, r);
  return (long long)l.units * l.segments;
}

// Both for a whole CTA; scratch: 34 words of shared memory.  total_units: of all requests.  find_unit: the request that
// holds a unit (one below the total), and the number of its first unit.
__device__ __forceinline__ long long warp_sum(long long v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ long long total_units(const AttendArgs &a, long long *scratch) {
  long long mine = 0;
  for (int r = threadIdx.x; r < a.b.n_req; r += blockDim.x) {
    int first, context, fresh;
    if (blockIdx.x == 0 && !request_lengths(a.b, a.bs.d, r, first, context, fresh)) report(a.b.status, KVR_DEV_BAD_LENGTH);
    mine += units_of(a, r);
  }
  mine = warp_sum(mine);
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = mine;
  __syncthreads();
  long long total = 0;
  for (int w = 0; w < (int)(blockDim.x + 31) / 32; ++w) total += scratch[w];
  __syncthreads();
  return total;
}
__device__ __forceinline__ void find_unit(const AttendArgs &a, long long unit, long long *scratch, int &r_out, long long &base_out) {
  long long carry = 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (blockDim.x + 31) / 32;
  for (int r0 = 0; r0 < a.b.n_req; r0 += blockDim.x) {
    const int r = r0 + threadIdx.x;
    const long long mine = r < a.b.n_req ? units_of(a, r) : 0;
    long long incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += up;
    }
    if (lane == 31) scratch[warp] = incl;
    __syncthreads();
    long long before = carry, all = carry;
    for (int w = 0; w < warps; ++w) {
      if (w < warp) before += scratch[w];
      all += scratch[w];
    }
    const long long lo = before + incl - mine;
    if (unit >= lo && unit < lo + mine) { scratch[32] = r; scratch[33] = lo; }
    __syncthreads();
    if (unit < all) break;
    carry = all;
  }
  r_out = (int)scratch[32];
  base_out = scratch[33];
  __syncthreads();
}

// units [first_unit(c), first_unit(c + 1)) belong to CTA c
__device__ __forceinline__ long long first_unit(long long total, int ctas, int c) { return total * c / ctas; }
__device__ __forceinline__ int cta_of(long long total, int ctas, long long unit) { return (int)(((unit + 1) * ctas + total - 1) / total) - 1; }

// May row i of a request (of `fresh` new tokens) look at its new token j?
__device__ __forceinline__ bool sees(const AttendArgs &a, int first, int i, int j) {
  if (!a.mask) return j <= i;
  return __ldg(a.mask + (long long)(first + i) * a.mask_words + (j >> 6)) >> (j & 63) & 1;
}
#endif

// warps of a CTA of the row kernel: KV heads of a group x slices of the keys
__host__ __device__ constexpr int rows_warps(int padded_dim) { return padded_dim == 256 ? 4 : 8; }

// By cache format, one translation unit each (kvr_attend_<format>.cu).  tiles: of the row kernel, query rows of a segment / 8,
// 1, 2 or 4 (at most 2 above 128 channels); 0 is the tile kernel (at most 128 channels), for 128 or 256 rows a segment, with its map of
// the layer's K and V planes.
cudaError_t launch_attend_bf16(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s);
cudaError_t launch_attend_f16(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s);
cudaError_t launch_attend_e4m3(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s);
cudaError_t launch_attend_int8(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s);

}  // namespace kvr

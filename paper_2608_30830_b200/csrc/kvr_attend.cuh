// Attention over the paged cache: how a call's work is cut up, and what its kernels share.
//
// Work is cut along the keys.  A segment is one request, one group of KV heads and one tile of its query rows (row =
// new token x query heads of one KV head + query head); a unit is a fixed number of keys of a segment.  Segments follow each
// other request by request, and the units of all of them are dealt out in equal runs (a segment's start may weigh some units of
// its own), one to each CTA of a grid that
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
  FastDiv bs, group, unit;   // block size; query heads per KV head; keys of a unit
  Rows q, out;
  float *lse;                // or NULL
  const unsigned long long *mask;    // or NULL: causal
  int mask_words;
  float scale_log2;          // scale * log2(e)
  int q_heads;
  int head_groups, group_heads;      // KV heads are taken group_heads at a time
  int row_tile, row_shift;   // query rows of a segment, 2^row_shift
  int opening;               // what a segment's start weighs, in units: a CTA that begins one gets fewer keys
  int box_rows;              // tokens of a TMA box (tile kernel): 8 or 16, 0: the block size does not allow one
  int ctas;                  // the grid of the main kernel
  unsigned polls;            // of a barrier, before a wait of the tile kernel gives up; 0: all do at once (tests)
  int *handed_in;            // [2][ctas][2]: pieces of a group, groups of a segment; zero between calls
  float *part_o;             // [ctas][2][group_heads][row_tile][head_dim]; of the tile kernel [ctas][2][head_dim][row_tile]
  float2 *part_ml;           // [ctas][2][group_heads][row_tile]: maximum (log2), sum
};

// The workspace holds, for every SM, two pieces of this many rows (fp32 accumulators and a pair of statistics each).
constexpr int kPartRows = 256;
constexpr int kMaxSms = 160;
constexpr int kCounterBytes = 4096;
constexpr int kJoinAtOnce = 16;
constexpr unsigned kPolls = 1u << 18;
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
  l.units = (int)a.unit.div(l.keys + a.unit.d - 1);
  l.segments = a.head_groups * ((l.fresh * (int)a.group.d + a.row_tile - 1) >> a.row_shift);
  return l;
}

// How the units of a call are dealt out: `ctas` runs, the first `rem` of them one unit longer.  (The host has seen to it that units
// fit 32 bits.)
struct Shares {
  unsigned total, size, rem;
  int ctas;
  __device__ __forceinline__ unsigned first(int c) const { return size * c + min((unsigned)c, rem); }
  __device__ __forceinline__ int cta_of(unsigned unit) const {
    const unsigned longer = rem * (size + 1);
    return (int)(unit < longer ? unit / (size + 1) : rem + (unit - longer) / size);
  }
};

// For a whole CTA: the shares of the call, and the request that this CTA's first unit belongs to with its lengths and the number of
// its own first unit.  False where there is nothing for this CTA.  scratch: 39 words of shared memory.
__device__ __forceinline__ bool find_share(const AttendArgs &a, unsigned *scratch, Shares &sh, int &r_out, unsigned &base_out, Lengths &len_out) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x / 32;
  const bool once = a.b.n_req <= (int)blockDim.x;
  Lengths mine{};
  unsigned units = 0, incl = 0, before = 0;
  // units of request r0 + thread, of all requests up to it within this round (incl) and of the rounds' warps before (before)
  auto scan = [&](int r0) {
    const int r = r0 + threadIdx.x;
    units = 0;
    if (r < a.b.n_req) {
      mine = attend_lengths(a, r);
      units = mine.units ? (unsigned)(mine.units + a.opening) * mine.segments : 0;
      int first, context, fresh;
      if (blockIdx.x == 0 && !request_lengths(a.b, a.bs.d, r, first, context, fresh)) report(a.b.status, KVR_DEV_BAD_LENGTH);
    }
    incl = units;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const unsigned up = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += up;
    }
    if (lane == 31) scratch[warp] = incl;
    __syncthreads();
    unsigned all = 0;
    before = 0;
    for (int w = 0; w < warps; ++w) {
      if (w < warp) before += scratch[w];
      all += scratch[w];
    }
    __syncthreads();
    return all;
  };
  sh.total = 0;
  for (int r0 = 0; r0 < a.b.n_req; r0 += blockDim.x) sh.total += scan(r0);
  sh.ctas = (int)min((unsigned)a.ctas, sh.total);
  if ((int)blockIdx.x >= sh.ctas) return false;
  sh.size = sh.total / sh.ctas;
  sh.rem = sh.total - sh.size * sh.ctas;
  const unsigned unit = sh.first(blockIdx.x);
  unsigned carry = 0;
  for (int r0 = 0; r0 < a.b.n_req; r0 += blockDim.x) {
    const unsigned all = once ? sh.total : scan(r0);
    const unsigned lo = carry + before + incl - units;
    if (unit >= lo && unit - lo < units) {
      scratch[32] = r0 + threadIdx.x; scratch[33] = lo;
      scratch[34] = mine.first; scratch[35] = mine.context; scratch[36] = mine.fresh; scratch[37] = mine.units; scratch[38] = mine.segments;
    }
    carry += all;
    if (unit < carry) break;
    __syncthreads();
  }
  __syncthreads();
  r_out = (int)scratch[32];
  base_out = scratch[33];
  len_out = Lengths{(int)scratch[34], (int)scratch[35], (int)scratch[36], (int)(scratch[35] + scratch[36]), (int)scratch[37], (int)scratch[38]};
  return true;
}

// May row i of a request (of `fresh` new tokens) look at its new token j?
__device__ __forceinline__ bool sees(const AttendArgs &a, int first, int i, int j) {
  if (!a.mask) return j <= i;
  return __ldg(a.mask + (long long)(first + i) * a.mask_words + (j >> 6)) >> (j & 63) & 1;
}
#endif

// chunks of 16 keys that a warp of the row kernel takes at a time (tiles: of 8 rows); a unit holds a multiple of them
__host__ __device__ constexpr int chunks_at_once(int format, int tiles) { return quantised(format) && tiles == 1 ? 2 : 1; }
// warps of a CTA of the row kernel: KV heads of a group x slices of the keys
__host__ __device__ constexpr int rows_warps(int padded_dim) { return padded_dim == 256 ? 4 : 8; }

// By cache format, one translation unit each (kvr_attend_<format>.cu).  tiles: of the row kernel, query rows of a segment / 8,
// 1 or 2; 0 is the tile kernel (at most 128 channels), for 128 or 256 rows a segment, with its map of
// the layer's K and V planes.
cudaError_t launch_attend_bf16(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s);
cudaError_t launch_attend_f16(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s);
cudaError_t launch_attend_e4m3(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s);
cudaError_t launch_attend_int8(const AttendArgs &a, int tiles, int slices, const CUtensorMap &map, cudaStream_t s);

}  // namespace kvr

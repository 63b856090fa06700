// kvr_cache_attend: argument checks and the choice of kernel.
#include "kvr_attend.cuh"

#include <atomic>
#include <cmath>

#include "kvr_once.hpp"

namespace kvr {
namespace {

std::atomic<unsigned> g_polls{kPolls};

int sm_count() {
  static int counts[64];
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if (!counts[dev]) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    counts[dev] = n < kMaxSms ? n : kMaxSms;
  }
  return counts[dev];
}

// The layer's planes as [plane][block][token][head][channel]: boxes are `box_rows` tokens of one head, 128 bytes wide (128-byte
// swizzle, the products' operand layout) or a whole 8-bit head; channels beyond head_dim read as zero.
bool layer_map(const kvr_cache_spec *s, const CacheView &c, int padded, int box_rows, CUtensorMap *map) {
  typedef CUresult (*Encode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                             const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) f = nullptr;
    return reinterpret_cast<Encode>(f);
  }();
  if (!encode) return false;
  const bool quant = quantised(s->format);
  const cuuint64_t element = quant ? 1 : 2;
  const cuuint64_t dims[5] = {(cuuint64_t)s->head_dim, (cuuint64_t)s->kv_heads, (cuuint64_t)s->block_size, (cuuint64_t)s->num_blocks, 2};
  const cuuint64_t strides[4] = {s->head_dim * element, (cuuint64_t)c.row_bytes, (cuuint64_t)c.block_stride, (cuuint64_t)c.v_offset};
  const cuuint32_t box[5] = {(cuuint32_t)(quant ? padded : 64), 1, (cuuint32_t)box_rows, 1, 1}, ones[5] = {1, 1, 1, 1, 1};
  return encode(map, quant ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 5, c.base, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                quant ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace kvr

using namespace kvr;

extern "C" uint64_t kvr_attend_workspace(const kvr_cache_spec *spec) {
  if (check_spec(spec)) return 0;
  return kCounterBytes + (uint64_t)kMaxSms * 2 * kPartRows * (spec->head_dim * 4ull + 8);
}

extern "C" kvr_status kvr_cache_attend(const kvr_cache_spec *spec, const void *device_pool, int32_t layer, const kvr_batch *batch,
                                       const kvr_rows *q, const kvr_rows *out, float *lse, const uint64_t *mask, int32_t mask_words,
                                       float scale, void *workspace, uint64_t workspace_bytes, void *stream) {
  AttendArgs a{};
  if (kvr_status st = layer_view(spec, device_pool, layer, &a.c)) return st;
  if (kvr_status st = check_batch(batch)) return st;
  if (!q || !out) return fail_cache(KVR_ERR_INVALID_ARG, "q and out are needed");
  if (kvr_status st = check_rows(q, "q")) return st;
  if (kvr_status st = check_out(out, "out", spec->head_dim)) return st;
  if (q->type == KVR_F32 || out->type != q->type || out->heads != q->heads)
    return fail_cache(KVR_ERR_INVALID_ARG, "q and out must have one 16-bit type and the same heads");
  if ((spec->format == KVR_CACHE_BF16 && q->type != KVR_BF16) || (spec->format == KVR_CACHE_F16 && q->type != KVR_F16))
    return fail_cache(KVR_ERR_INVALID_ARG, "q must have the type of a 16-bit cache");
  if (q->heads % spec->kv_heads) return fail_cache(KVR_ERR_INVALID_ARG, "q's heads must be a multiple of kv_heads");
  const int group = q->heads / spec->kv_heads;
  if ((int64_t)batch->max_new * group > (1 << 28)) return fail_cache(KVR_ERR_INVALID_ARG, "too many new tokens in one request");
  if (batch->max_tokens > (1 << 30)) return fail_cache(KVR_ERR_INVALID_ARG, "at most 2^30 tokens in one request");
  if (!std::isfinite(scale)) return fail_cache(KVR_ERR_INVALID_ARG, "scale must be finite");
  if (mask && (mask_words < 1 || (int64_t)mask_words * 64 < batch->max_new || ((uintptr_t)mask & 7)))
    return fail_cache(KVR_ERR_INVALID_ARG, "mask must be 8-byte aligned and have a bit for each of max_new tokens");
  if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < kvr_attend_workspace(spec))
    return fail_cache(KVR_ERR_INVALID_ARG, "workspace: kvr_attend_workspace() bytes at a 256-byte boundary are needed");
  if ((uintptr_t)lse & 3) return fail_cache(KVR_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  if (batch->n_tokens == 0) return KVR_OK;
  const int sms = sm_count();
  if (!sms) return fail_cache(KVR_ERR_CUDA, "no current CUDA device");
  a.b = device_batch(batch);
  a.bs = FastDiv(spec->block_size);
  a.group = FastDiv(group);
  a.q = device_rows(q);
  a.out = device_rows(out);
  a.lse = lse;
  a.mask = reinterpret_cast<const unsigned long long *>(mask);
  a.mask_words = mask_words;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.q_heads = q->heads;
  const int padded = spec->head_dim <= 64 ? 64 : spec->head_dim <= 128 ? 128 : 256;
  const int warps = rows_warps(padded);
  const int64_t rows = (int64_t)batch->max_new * group;
  int tiles = 0, slices = 0;
  CUtensorMap map{};
  if (rows > 16 && padded <= 128) {
    // More rows than two tiles of the row kernel.  (us, 8 KV heads of 128, 2 requests of 16k / 32 of 4k.  16 rows: row kernel
    // 44 / 115, tile kernel 54 / 122; int8 44 / 121, 68 / 207.  32 rows, with four tiles of the row kernel, which there was: 198 / 190, tile
    // kernel 57 / 128; int8 228 / 256, 74 / 211.)  Heads of more than 128 channels stay with the row kernel: two jobs' sums and scores
    // would take 768 of tensor memory's 512 columns.  One job of 128 rows would fit (384), but is not built: such rows read the cache once
    // for every 16 of them (8 requests of 4k, 256 channels, trees of 16 tokens 282 us, of 64 1,039, against 42 and 44 for one reading).
    // One kernel for the whole call, by its longest request: a chunk of 512 tokens beside 31 single tokens over 4k each takes 188 us, as two
    // calls 77 + 90 (e4m3 331, 113 + 70).
    a.head_groups = spec->kv_heads;
    a.group_heads = 1;
    a.row_tile = rows <= 128 ? 128 : 256;
    a.unit = FastDiv(128);
    // A segment begun inside a CTA's share costs it a second Q, the wait for the first products and another epilogue: 6 units' worth.
    // (Trees of 64 tokens, 16 requests of 8k, us: 186 without, 179 at 3, 174 at 6, 175 at 9, 180 at 12, 186 at 16; trees of 13
    // over an int8 cache: 134, 130, 126, 127, 131, 135.)  The row kernel's pieces begin while the last one's keys still stream.
    a.opening = 6;
    // (trees of 64 tokens, blocks of 16, us: boxes of 16 tokens 176, of 8 177, copies by the lanes 217; int8, trees of 13: 125, 129, 133)
    a.box_rows = spec->block_size % 16 == 0 ? 16 : spec->block_size % 8 == 0 ? 8 : 0;
    if (a.box_rows && !layer_map(spec, a.c, padded, a.box_rows, &map)) return fail_cache(KVR_ERR_CUDA, "no tensor map could be made of the layer");
  } else {
    tiles = rows <= 8 ? 1 : 2;
    a.row_tile = tiles * 8;
    a.head_groups = (spec->kv_heads + warps - 1) / warps;
    a.group_heads = (spec->kv_heads + a.head_groups - 1) / a.head_groups;
    // Few requests: fewer heads a CTA, its warps then share a head's keys, until no segment is cut into many more than 8 pieces, for
    // a segment's pieces are joined by one CTA.  (us, 8 rows, 16-bit / int8, all heads in a CTA against this: 1 request of 4k 39 / 44,
    // 24 / 20; 2 of 16k 67 / 66, 39 / 33; 8 of 16k 111 / 100, 97 / 85; 4 pieces: 96 / 98, 16 pieces: 95 / 85.)  Not where one tile of
    // rows streams a long 8-bit cache, whose narrow rows and scales are then read in pieces too small: by the caller's bounds, from 512 MB
    // on (int8, 4 rows, 8 requests: of 4k, 67 MB, 49 us whole, 34 split; of 16k 82, 87; of 64k 233, 316).
    const int64_t stream = 2ll * batch->n_req * batch->max_tokens * a.c.row_bytes;
    const bool whole = quantised(spec->format) && tiles == 1 && stream >= 512ll << 20;
    while (!whole && a.group_heads > 1 && (int64_t)batch->n_req * a.head_groups * 8 < sms) {
      a.group_heads = (a.group_heads + 1) / 2;
      a.head_groups = (spec->kv_heads + a.group_heads - 1) / a.group_heads;
    }
    slices = warps / a.group_heads;
    const int turn = 16 * slices * chunks_at_once(spec->format, tiles);      // keys that the warps of a head take at a time
    a.unit = FastDiv((64 + turn - 1) / turn * turn);
    // 64 or more: fewer pieces.  (us, units of 16 / 64 / 128 / 256 / 512 keys, one token, bf16: 32 requests of 333 tokens 21.4 / 18.5 / 18.8 /
    // 25.3 / 23.6, 16 of them 25.9 / 15.6 / 15.7 / 18.6 / 15.8.  Of few requests a turn is 128 keys anyway: one of 333 13.8 / 13.5 /
    // 13.7 / 14.4 / 9.5, of 1,000 15.1 / 15.1 / 15.1 / 15.1 / 16.0.)
  }
  while ((1 << a.row_shift) < a.row_tile) ++a.row_shift;
  // units are numbered in 32 bits; a bound that the lengths on the device keep, whatever they are
  const double most = (double)batch->n_req * (((int64_t)batch->max_new * group + a.row_tile - 1) / a.row_tile) * a.head_groups * (batch->max_tokens / a.unit.d + 1. + a.opening);
  if (most >= INT32_MAX) return fail_cache(KVR_ERR_INVALID_ARG, "n_req, max_new and max_tokens are too large for one call");
  a.ctas = sms;
  a.polls = g_polls.load(std::memory_order_relaxed);
  a.handed_in = static_cast<int *>(workspace);
  a.part_ml = reinterpret_cast<float2 *>(static_cast<char *>(workspace) + kCounterBytes);
  a.part_o = reinterpret_cast<float *>(static_cast<char *>(workspace) + kCounterBytes + (size_t)kMaxSms * 2 * kPartRows * 8);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  switch (spec->format) {
    case KVR_CACHE_BF16: e = launch_attend_bf16(a, tiles, slices, map, s); break;
    case KVR_CACHE_F16: e = launch_attend_f16(a, tiles, slices, map, s); break;
    case KVR_CACHE_E4M3: e = launch_attend_e4m3(a, tiles, slices, map, s); break;
    default: e = launch_attend_int8(a, tiles, slices, map, s);
  }
  return e == cudaSuccess ? KVR_OK : fail_cache(KVR_ERR_CUDA, cudaGetErrorString(e));
}

extern "C" int32_t kvr_test_once(const int32_t *devices, const int32_t *results, int32_t n, int32_t *returned) {
  OncePerDevice once;
  int32_t runs = 0;
  for (int32_t i = 0; i < n; ++i) returned[i] = once(devices[i], [&] { ++runs; return results[i]; });
  return runs;
}

extern "C" uint32_t kvr_test_attend_polls(uint32_t polls) { return g_polls.exchange(polls); }

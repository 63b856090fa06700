// What the operators over the paged cache share: the step's requests and the cache as the kernels see them, checked
// addressing, and conversions.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/kvr.h"

namespace kvr {

// kvr_batch for a kernel
struct Batch {
  const int32_t *token_start, *context, *tables;
  int32_t *status;
  int n_req, n_tokens, max_new, max_tokens, table_stride;
};

// One layer of the cache (or, for keep, all of it).  A plane is K or V of one layer.
struct CacheView {
  char *base;                // K plane of the layer
  long long v_offset;        // from a K plane to its V plane
  long long block_stride;    // from one block to the next within a plane
  int row_bytes, scale_offset;   // of a token's row; the scales lie behind the codes (8-bit: of all heads; 4-bit: of a head)
  int head_bytes;            // from one head's elements to the next's
  int block_size, num_blocks;
  int kv_heads, head_dim;
};

// kvr_rows for a kernel, strides in bytes
struct Rows {
  char *data;
  long long token_stride, head_stride;
  int heads, type;
};

// floor(x / d) for 0 <= x < 2^31 by a multiplication, d > 0 (round-up method: m = ceil(2^(31+s) / d), s = ceil(log2 d);
// the error of m is below 2^s / 2^(31+s), too small to carry any x below 2^31 over a multiple of d)
struct FastDiv {
  unsigned d, m, s;
  FastDiv() = default;
  explicit FastDiv(unsigned div) : d(div), m(0), s(0) {
    while ((1ull << s) < d) ++s;
    const unsigned long long one = 1ull << (31 + s);
    m = (unsigned)((one + d - 1) / d);          // below 2^32, since d > 2^(s-1); d = 1: 2^31
  }
  __device__ __forceinline__ unsigned div(unsigned x) const { return (unsigned)(((unsigned long long)x * m) >> (31 + s)); }
};

#ifdef __CUDACC__
__device__ __forceinline__ void report(int32_t *status, int what) {
  if (status) { *reinterpret_cast<volatile int32_t *>(status) = what; __threadfence_system(); }
}

// last r with token_start[r] <= token
__device__ __forceinline__ int find_request(const Batch &b, int token) {
  int lo = 0, hi = b.n_req - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (__ldg(b.token_start + mid) <= token) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Context and new tokens of request r; false (and both 0) where they do not fit what the host was told.
__device__ __forceinline__ bool request_lengths(const Batch &b, int block_size, int r, int &first, int &context, int &fresh) {
  first = __ldg(b.token_start + r);
  const int end = __ldg(b.token_start + r + 1);
  context = __ldg(b.context + r);
  fresh = end - first;
  const long long total = (long long)context + fresh;
  if (first < 0 || fresh < 0 || end > b.n_tokens || context < 0 || fresh > b.max_new || total > b.max_tokens ||
      total > (long long)b.table_stride * block_size) {
    context = fresh = 0;
    return false;
  }
  return true;
}

// Offset of logical token j of request r inside a plane; -1 where its block id is out of range.
__device__ __forceinline__ long long token_offset(const Batch &b, const CacheView &c, const FastDiv &bs, int r, int j) {
  const unsigned blk = bs.div((unsigned)j);
  if (blk >= (unsigned)b.table_stride) return -1;
  const int id = __ldg(b.tables + (long long)r * b.table_stride + blk);
  if ((unsigned)id >= (unsigned)c.num_blocks) return -1;
  return (long long)id * c.block_stride + (long long)(j - blk * bs.d) * c.row_bytes;
}

// ---- element types: 8 elements of a row as fp32 ------------------------------------

template <int TYPE>
__device__ __forceinline__ void widen8(const uint4 &v, float (&x)[8]) {
  const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (TYPE == KVR_BF16) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
      x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
  }
}
template <int TYPE>
__device__ __forceinline__ void load8(const char *p, float (&x)[8]) {
  if constexpr (TYPE == KVR_F32) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *(reinterpret_cast<const float4 *>(p) + 1);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  } else {
    widen8<TYPE>(*reinterpret_cast<const uint4 *>(p), x);
  }
}

template <int TYPE>
__device__ __forceinline__ float load1(const char *p) {
  if constexpr (TYPE == KVR_F32) return *reinterpret_cast<const float *>(p);
  else if constexpr (TYPE == KVR_BF16) return __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(p));
  else return __half2float(*reinterpret_cast<const __half *>(p));
}

// pairs of fp32 in one 64-bit register
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair(float a, float b) { Pair r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 unpair(Pair v) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v)); return r; }
__device__ __forceinline__ Pair mul2(Pair a, Pair b) { Pair r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Pair add2(Pair a, Pair b) { Pair r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { Pair r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }

__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const unsigned *>(&v);
}
__device__ __forceinline__ unsigned pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const unsigned *>(&v);
}

// Byte BYTE of w, two e2m1 codes, as f16: exact.
template <int BYTE>
__device__ __forceinline__ unsigned widen_e2m1(unsigned w) {
  unsigned r;
  if constexpr (BYTE == 0) asm("{.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;}" : "=r"(r) : "r"(w));
  else if constexpr (BYTE == 1) asm("{.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;}" : "=r"(r) : "r"(w));
  else if constexpr (BYTE == 2) asm("{.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;}" : "=r"(r) : "r"(w));
  else asm("{.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, d;}" : "=r"(r) : "r"(w));
  return r;
}
// 8 numbers as codes: to the nearest, ties to even, at most 6.
__device__ __forceinline__ unsigned narrow_e2m1(const float (&y)[8]) {
  unsigned r;
  asm("{.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};}"
      : "=r"(r) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return r;
}
// The scale of a group of 16 channels by its byte, times 2^-8 (as f16, exact): the fields of an e4m3 number 7 places up lie where f16
// has them.  The sign is not read, and 0x7f is 480: there is no NaN among these.
constexpr float kGroupUnit = 256.f;
__device__ __forceinline__ unsigned group_scale(unsigned byte) { return (byte & 0x7fu) << 7; }

template <int TYPE>
__device__ __forceinline__ void store8(char *p, const float (&x)[8]) {
  if constexpr (TYPE == KVR_F32) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint4 v;
    if constexpr (TYPE == KVR_BF16) v = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    else v = make_uint4(pack_f16(x[0], x[1]), pack_f16(x[2], x[3]), pack_f16(x[4], x[5]), pack_f16(x[6], x[7]));
    *reinterpret_cast<uint4 *>(p) = v;
  }
}
#endif  // __CUDACC__

__host__ __device__ constexpr bool quantised(int format) { return format >= KVR_CACHE_E4M3; }     // codes with scales
__host__ __device__ constexpr bool four_bit(int format) { return format == KVR_CACHE_E2M1; }
// A head's record in a 4-bit row: codes, the head's scale, a scale for each 16 channels, zeros up to a multiple of 16 bytes.
__host__ __device__ constexpr int record_bytes(int head_dim) { return (head_dim / 2 + 4 + head_dim / 16 + 15) / 16 * 16; }

// host side (kvr_cache.cu): argument checks with a message, shared by the entries
kvr_status fail_cache(kvr_status st, const char *msg);
kvr_status check_spec(const kvr_cache_spec *s);
kvr_status check_batch(const kvr_batch *b);
kvr_status check_rows(const kvr_rows *r, const char *what);
kvr_status check_out(const kvr_rows *r, const char *what, int head_dim);   // rows that are written
kvr_status layer_view(const kvr_cache_spec *s, const void *pool, int layer, CacheView *out);
Batch device_batch(const kvr_batch *b);
Rows device_rows(const kvr_rows *r);

}  // namespace kvr

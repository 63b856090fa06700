// Operators that move tokens in and out of the paged cache: append (rotary positions, quantisation, write by block
// table), read (the way back), keep (accepted rows of drafted tokens), and the rotary tables.
//
// A token's rows are read once and written once, with a few operations an element in between: large calls are bound by memory (read,
// keep, append to a 16-bit cache) or, short of it, by what 16 warps an SM can have under way (append to an 8-bit one), small ones by the
// launch and three or four dependent loads.
#include "kvr_cache.cuh"

#include <cmath>
#include <cstdio>

#include "kvr_kernels.cuh"

namespace kvr {

void set_last_error(const char *msg);

namespace {

constexpr int kThreads = 256;
constexpr int kMaxAxes = 4;

struct RopeView {
  const float *table;
  int positions, rot, style;
  float sign;                // of the sine: -1 turns back
  int axes;                  // positions of a token
  uint16_t axis_of[16];      // the axes of pairs 8 i .. 8 i + 7, two bits each
};

struct AppendArgs {
  Batch b;
  CacheView c;
  FastDiv bs;
  Rows q, k, v, q_out;
  RopeView rope;             // table NULL: nothing is turned
  const int32_t *positions;
  int q_heads, k_heads, v_heads;     // 0 where absent
  int per_token;             // groups of lanes that share a token: 1, 2, 4, ...
};

// Where one token of a CTA's lies: filled by one thread per token, read by all.
struct TokenAt {
  long long offset;          // in a plane, -1: not addressable
  int position;              // -1: leave the token out
};

__device__ __forceinline__ TokenAt locate_token(const Batch &b, const CacheView &c, const FastDiv &bs, int token) {
  TokenAt t{-1, -1};
  const int r = find_request(b, token);
  int first, context, fresh;
  if (!request_lengths(b, bs.d, r, first, context, fresh) || token < first || token - first >= fresh) {
    report(b.status, KVR_DEV_BAD_LENGTH);
    return t;
  }
  t.position = context + (token - first);
  t.offset = token_offset(b, c, bs, r, t.position);
  if (t.offset < 0) report(b.status, KVR_DEV_BAD_BLOCK);
  return t;
}

// 8 channels as they lie in memory.
template <int XT>
struct Raw8 {
  static constexpr int kWords = XT == KVR_F32 ? 8 : 4;
  unsigned w[kWords];
  __device__ __forceinline__ void load(const char *p) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
      const uint4 v = *reinterpret_cast<const uint4 *>(p + i * 4);
      w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
  }
  __device__ __forceinline__ void widen(float (&x)[8]) const {
    if constexpr (XT == KVR_F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    } else {
      widen8<XT>(make_uint4(w[0], w[1], w[2], w[3]), x);
    }
  }
};

// The angles of 8 channels d0 .. d0 + 7 at one position (AXES: at the positions of their pairs' axes), and the turn by them.  Products and sums are rounded one by
// one, so the result does not depend on what a compiler contracts.
//   rot % 16 == 0, halves: partners are whole lanes; 8 (cos, sin)
//   rot % 16 == 0, interleaved: partners are the lane's own; 4 (cos, sin)
//   other rot: partners are read again, angles where they are used
template <int XT, bool AXES>
struct Angles {
  const RopeView &rp;
  const float *row;          // (cos, sin) of this position; AXES: of position 0
  const int *where;          // AXES: the token's positions
  Pair c[4], s[4];           // halves: the sine's sign is the channel's side
  __device__ __forceinline__ Angles(const RopeView &rope, const int *position, int d0) : rp(rope), row(nullptr), where(position) {
    if (!rp.table) return;
    row = rp.table + (AXES ? 0ll : (long long)*position * rp.rot);
    const bool low = d0 < (rp.rot >> 1);
    if ((rp.rot & 15) || d0 >= rp.rot) return;
    const bool halves = rp.style == KVR_ROPE_HALF;
    const int pair0 = !halves ? d0 >> 1 : low ? d0 : d0 - (rp.rot >> 1);       // the lane's first pair, a multiple of 4 or 8
    const float sign = halves && low ? -rp.sign : rp.sign;
    const float *from = row + 2 * pair0;
    if constexpr (AXES) {
      const unsigned axes = rp.axis_of[pair0 >> 3] >> (pair0 & 7) * 2 & (halves ? 0xffffu : 0xffu), one = axes & 3;
      if (axes != one * (halves ? 0x5555u : 0x55u)) {        // pair by pair; else the lane's pairs lie side by side
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i >= 2 && !halves) break;
          float2 x[2];
#pragma unroll
          for (int e = 0; e < 2; ++e)
            x[e] = __ldg(reinterpret_cast<const float2 *>(from + (long long)where[axes >> (4 * i + 2 * e) & 3] * rp.rot) + 2 * i + e);
          c[i] = pair(x[0].x, x[1].x);
          s[i] = pair(x[0].y * sign, x[1].y * sign);
        }
        return;
      }
      from += (long long)where[one] * rp.rot;
    }
    const float4 *t = reinterpret_cast<const float4 *>(from);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i >= 2 && !halves) break;
      const float4 x = __ldg(t + i);
      c[i] = pair(x.x, x.z);
      s[i] = pair(x.y * sign, x.w * sign);
    }
  }
  // rot % 16 == 0: N heads at once, turned or (turned: false) only lending their channels to their partners
  template <int LPH, int N>
  __device__ __forceinline__ void turn_lanes(float (&x)[N][8], const Raw8<XT> (&raw)[N], int d0, bool turned) const {
    turned = turned && d0 < rp.rot;
    if (rp.style == KVR_ROPE_HALF) {
      const int half = rp.rot >> 1, partner = (d0 < half ? d0 + half : d0 - half) >> 3;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        Raw8<XT> theirs;               // as they were loaded: half the shuffles for 16-bit types
#pragma unroll
        for (int i = 0; i < Raw8<XT>::kWords; ++i) theirs.w[i] = __shfl_sync(0xffffffffu, raw[k].w[i], partner, LPH);
        if (!turned) continue;
        float y[8];
        theirs.widen(y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // sums one by one: of products by add.f32x2, or by fma.f32x2 with 1, one was not rounded
          const float2 u = unpair(mul2(pair(x[k][2 * i], x[k][2 * i + 1]), c[i])), v = unpair(mul2(pair(y[2 * i], y[2 * i + 1]), s[i]));
          x[k][2 * i] = __fadd_rn(u.x, v.x); x[k][2 * i + 1] = __fadd_rn(u.y, v.y);
        }
      }
    } else if (turned) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float u = x[k][2 * i], v = x[k][2 * i + 1];
          const float2 cs = unpair(c[i >> 1]), sn = unpair(s[i >> 1]);
          const float ci = i & 1 ? cs.y : cs.x, si = i & 1 ? sn.y : sn.x;
          x[k][2 * i] = __fsub_rn(__fmul_rn(u, ci), __fmul_rn(v, si));
          x[k][2 * i + 1] = __fadd_rn(__fmul_rn(u, si), __fmul_rn(v, ci));
        }
      }
    }
  }
  // other rot
  __device__ __forceinline__ void turn(float (&x)[8], const char *src, int d0) const {
    const int half = rp.rot >> 1;
    if (d0 >= rp.rot) return;
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = d0 + i;
      const int partner = rp.style == KVR_ROPE_INTERLEAVED ? (d ^ 1) : d < half ? d + half : d - half;
      y[i] = d < rp.rot ? load1<XT>(src + (long long)partner * (XT == KVR_F32 ? 4 : 2)) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int d = d0 + i;
      if (d >= rp.rot) continue;
      const bool first = rp.style == KVR_ROPE_INTERLEAVED ? (d & 1) == 0 : d < half;
      const int p = rp.style == KVR_ROPE_INTERLEAVED ? d >> 1 : first ? d : d - half;
      const float *from = row;
      if constexpr (AXES) from += (long long)where[rp.axis_of[p >> 3] >> (p & 7) * 2 & 3] * rp.rot;
      const float2 t = __ldg(reinterpret_cast<const float2 *>(from) + p);
      const float sn = t.y * rp.sign;
      x[i] = first ? __fsub_rn(__fmul_rn(x[i], t.x), __fmul_rn(y[i], sn)) : __fadd_rn(__fmul_rn(y[i], sn), __fmul_rn(x[i], t.x));
    }
  }
};

// 8 channels of a head into the cache; LPH lanes hold the head.  A quantised head's largest magnitude is found as an
// integer: for the bits of |x| integer order is numeric order, and infinities and NaN lie above all numbers.
template <int FMT, int LPH>
__device__ __forceinline__ void put8(const float (&x)[8], char *row, int scale_offset, int head, int head_dim, int d0, bool live) {
  if constexpr (!quantised(FMT)) {
    if (live) store8<FMT == KVR_CACHE_BF16 ? KVR_BF16 : KVR_F16>(row + ((long long)head * head_dim + d0) * 2, x);
  } else {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    if (!live) top = 0;
#pragma unroll
    for (int m = LPH / 2; m > 0; m >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, m, LPH));
    const bool finite = top < 0x7f800000u;
    constexpr float kPerLargest = FMT == KVR_CACHE_E4M3 ? 1.f / 448.f : 1.f / 127.f;
    const float scale = finite ? fmaxf(__fmul_rn(__uint_as_float(top), kPerLargest), 1.17549435e-38f) : __uint_as_float(0x7fc00000u);
    if (!live) return;
    unsigned w[2] = {0, 0};
    if (finite) {
      float y[8];
      if (scale > 1e-30f) {
        // x / scale, rounded once: the product with the correctly rounded reciprocal, corrected by its exact remainder (P. Markstein,
        // "Computation of elementary functions on the IBM RISC System/6000", 1990), two numbers to an instruction.  (At
        // scales near 2^-100 the remainder of elements below an eighth of the scale is subnormal: what it loses is 2^-50 in the quotient, whose
        // last bit is 2^-33 where codes are not 0 any more.)  The remainder of -0 is +0, hence the sign.
        const float back = __frcp_rn(scale);
        const Pair r = pair(back, back), minus = pair(-scale, -scale);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const Pair n = pair(x[i], x[i + 1]), q = mul2(n, r);
          const float2 v = unpair(fma2(fma2(q, minus, n), r, q));
          y[i] = copysignf(v.x, x[i]); y[i + 1] = copysignf(v.y, x[i + 1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __fdiv_rn(x[i], scale);
      }
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float a = y[i], b = y[i + 1];
        unsigned pair;
        if constexpr (FMT == KVR_CACHE_E4M3) {
          pair = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
        } else {
          const int ia = min(127, max(-127, __float2int_rn(a))), ib = min(127, max(-127, __float2int_rn(b)));
          pair = (unsigned)(ia & 0xff) | (unsigned)(ib & 0xff) << 8;
        }
        w[i >> 2] |= pair << (8 * (i & 3));
      }
    }
    *reinterpret_cast<uint2 *>(row + (long long)head * head_dim + d0) = make_uint2(w[0], w[1]);
    if (d0 == 0) *reinterpret_cast<float *>(row + scale_offset + 4 * head) = scale;
  }
}

// The largest magnitude of three numbers; NaN if one is.
__device__ __forceinline__ float top3(float a, float b, float c) { float r; asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }

// The same into a 4-bit cache, N heads at once (of the lanes' heads first, first + step, ...): step by step for all of them, for each is a chain of shuffles,
// reciprocals and conversions.  Two lanes hold a group.  Reciprocals and products are rounded one by one, as the header has them.
template <int LPH, int N>
__device__ __forceinline__ void put4(const float (&x)[N][8], char *row, int first, int step, int heads, int head_dim, int d0, bool lane_live) {
  const int lane = d0 >> 3;
  float top[N], most[N], scale[N], back[N];
  unsigned byte[N], codes[N], word[N];
#pragma unroll
  for (int i = 0; i < N; ++i) top[i] = top3(top3(top3(x[i][0], x[i][1], x[i][2]), x[i][3], x[i][4]), top3(x[i][5], x[i][6], x[i][7]), 0.f);
#pragma unroll
  for (int i = 0; i < N; ++i) most[i] = top[i] = top3(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1, LPH), 0.f);
#pragma unroll
  for (int m = 2; m < LPH; m <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) most[i] = top3(most[i], __shfl_xor_sync(0xffffffffu, most[i], m, LPH), 0.f);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    scale[i] = most[i] < INFINITY ? fmaxf(__fmul_rn(most[i], 1.f / 2688.f), 7.8886091e-31f) : __uint_as_float(0x7fc00000u);
    back[i] = __fmul_rn(__frcp_rn(scale[i]), 1.f / 6.f);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) byte[i] = most[i] < INFINITY ? __nv_cvt_float_to_fp8(__fmul_rn(top[i], back[i]), __NV_SATFINITE, __NV_E4M3) : 0u;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float unit = __fmul_rn(__half2float(__ushort_as_half((unsigned short)group_scale(byte[i]))) * kGroupUnit, scale[i]);
    back[i] = byte[i] ? __frcp_rn(unit) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = __fmul_rn(x[i][e], back[i]);
    codes[i] = most[i] < INFINITY ? narrow_e2m1(y) : 0u;
    word[i] = lane & 1 ? 0u : byte[i] << ((lane & 6) * 4);
  }
  // the scales, 8 lanes' (4 groups') to a word, then a word to a lane: the head's scale, the groups', zeros
#pragma unroll
  for (int i = 0; i < N; ++i) word[i] |= __shfl_xor_sync(0xffffffffu, word[i], 2, LPH);
#pragma unroll
  for (int i = 0; i < N; ++i) word[i] |= __shfl_xor_sync(0xffffffffu, word[i], 4, LPH);
#pragma unroll
  for (int i = 0; i < N; ++i) word[i] = __shfl_sync(0xffffffffu, word[i], (lane - 1) * 8, LPH);
  const int bytes = record_bytes(head_dim);
  char *to = row + (long long)first * bytes;
#pragma unroll
  for (int i = 0; i < N; ++i, to += (long long)step * bytes) {
    if (!lane_live || first + i * step >= heads) continue;
    *reinterpret_cast<unsigned *>(to + (d0 >> 1)) = codes[i];
    if (lane * 4 < bytes - head_dim / 2)
      *reinterpret_cast<unsigned *>(to + head_dim / 2 + lane * 4) = lane == 0 ? __float_as_uint(scale[i]) : lane <= LPH / 8 ? word[i] : 0u;
  }
}

// LPH lanes take heads of one token, 8 channels (16 bytes of a 16-bit type) a lane, so a rotation's partner is in a
// neighbouring lane, a scale is a few shuffles, and a lane's angles serve all of its heads.  `per_token` such groups
// share a token's heads; kAhead heads are loaded before the first is worked on.
//
// 32k tokens of 32 query and 8 KV heads of 128 into an e4m3 cache: 734 MB in 156 to 160 us, 4.7 TB/s (int8 165).  Two CTAs an SM (128
// registers) issue in half of the cycles and DRAM is busy for 54 %: neither is full, the warps wait on their loads; bytes alone would
// take 112 us.  Into a bf16 cache 797 MB in 140 us, 5.7 TB/s.  Fewer heads ahead for more CTAs: 170 us (three), 179 us (four).  A step of 32
// tokens takes 5.5 us replayed in a graph (dependent loads: token_start, block table, angles); a call from Python more than that.  Into a 4-bit cache
// 32k tokens take 160 us, 730 MB, 4.6 TB/s: q's half runs at the memory's rate (82 us), k and v wait on the chains of put4 (78 us for 193 MB; one
// head after the other 90).  With positions of three axes 16k tokens take what they take with one (84 us, 4.9 TB/s).
template <int XT, int FMT, int LPH, bool AXES>
__global__ void __launch_bounds__(kThreads, 2) append_kernel(const __grid_constant__ AppendArgs a) {
  constexpr int kGroups = kThreads / LPH, kSize = XT == KVR_F32 ? 4 : 2, kAhead = XT == KVR_F32 ? 2 : 4;
  __shared__ TokenAt at[kGroups];
  __shared__ int places[AXES ? kGroups : 1][kMaxAxes];
  const int per_token = a.per_token, tokens = kGroups / per_token, first = blockIdx.x * tokens;
  const int group = threadIdx.x / LPH, d0 = (threadIdx.x % LPH) * 8;
  const int sub = group % per_token, token = first + group / per_token;
  // The heads of q, then of k, then of v, kAhead at a time; the next are asked for before these are worked on.  The number of
  // turns is the same for all lanes: they shuffle.
  const bool lane_in = token < a.b.n_tokens && d0 < a.c.head_dim;
  auto rows_of = [&](int part) -> const Rows & { return part == 0 ? a.q : part == 1 ? a.k : a.v; };
  auto heads_of = [&](int part) { return part == 0 ? a.q_heads : part == 1 ? a.k_heads : a.v_heads; };
  Raw8<XT> next[kAhead];
  auto ask = [&](int part, int h0) {
    const Rows &src = rows_of(part);
    const int heads = heads_of(part);
    const char *in = src.data + (long long)token * src.token_stride + (long long)(h0 + sub) * src.head_stride + d0 * kSize;
    const long long step = (long long)per_token * src.head_stride;
#pragma unroll
    for (int i = 0; i < kAhead; ++i, in += step) {
      if (lane_in && h0 + i * per_token + sub < heads) next[i].load(in);
      else next[i].clear();
    }
  };
  int part = a.q_heads ? 0 : a.k_heads ? 1 : 2, h0 = 0;
  ask(part, 0);
  if ((int)threadIdx.x < tokens) {
    TokenAt t{-1, -1};
    if (first + (int)threadIdx.x < a.b.n_tokens) {
      t = locate_token(a.b, a.c, a.bs, first + threadIdx.x);
      if (t.position >= 0 && a.rope.table) {
        bool known = true;
        if constexpr (AXES) {
#pragma unroll
          for (int x = 0; x < kMaxAxes; ++x) {
            const int place = x < a.rope.axes ? __ldg(a.positions + (long long)(first + threadIdx.x) * a.rope.axes + x) : 0;
            known = known && (unsigned)place < (unsigned)a.rope.positions;
            places[threadIdx.x][x] = place;
          }
        } else {
          if (a.positions) t.position = __ldg(a.positions + first + threadIdx.x);
          known = (unsigned)t.position < (unsigned)a.rope.positions;
        }
        if (!known) {
          report(a.b.status, KVR_DEV_BAD_POSITION);
          t.position = -1;
        }
      }
    }
    at[threadIdx.x] = t;
  }
  __syncthreads();
  const TokenAt t = at[group / per_token];
  const bool lane_live = t.position >= 0 && d0 < a.c.head_dim;
  const int zero = 0;
  const Angles<XT, AXES> angles(a.rope, AXES ? places[AXES ? group / per_token : 0] : lane_live ? &t.position : &zero, lane_live ? d0 : a.rope.rot);

  while (part < 3) {
    const int now = part, at0 = h0;
    const Rows &src = rows_of(now);
    const int heads = heads_of(now);
    const bool live = lane_live && (now == 0 || t.offset >= 0);
    Raw8<XT> raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) raw[i] = next[i];
    h0 += per_token * kAhead;
    while (part < 3 && h0 >= heads_of(part)) { ++part; h0 = 0; }
    if (part < 3) ask(part, h0);
    float x[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) raw[i].widen(x[i]);
    if (a.rope.table && now < 2) {
      if ((a.rope.rot & 15) == 0) {
        angles.template turn_lanes<LPH, kAhead>(x, raw, d0, lane_live);
      } else {
        const char *in = src.data + (long long)token * src.token_stride;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int head = at0 + i * per_token + sub;
          if (live && head < heads) angles.turn(x[i], in + (long long)head * src.head_stride, d0);
        }
      }
      __syncwarp();                    // q_out may be q: every partner has been read
    }
    if (now == 0) {
      char *to = a.q_out.data + (long long)token * a.q_out.token_stride + (long long)(at0 + sub) * a.q_out.head_stride + d0 * kSize;
      const long long step = (long long)per_token * a.q_out.head_stride;
#pragma unroll
      for (int i = 0; i < kAhead; ++i, to += step)
        if (live && at0 + i * per_token + sub < heads) store8<XT>(to, x[i]);
    } else {
      char *row = a.c.base + (now == 2 ? a.c.v_offset : 0) + t.offset;
      if constexpr (four_bit(FMT)) {
        put4<LPH, kAhead>(x, row, at0 + sub, per_token, heads, a.c.head_dim, d0, live);
      } else {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int head = at0 + i * per_token + sub;
          put8<FMT, LPH>(x[i], row, a.c.scale_offset, head, a.c.head_dim, d0, live && head < heads);
        }
      }
    }
  }
}

struct ReadArgs {
  Batch b;
  CacheView c;
  FastDiv bs;
  Rows k, v;
  int k_heads, v_heads, per_token;
};

// The same division of labour; a lane's 8 channels are 16 bytes of a 16-bit cache, 8 of a quantised one.  32 requests of an int8 cache as
// fp16, 1.93 GB: 306 us, 6.3 TB/s, bound by memory; 8,192 tokens of e4m3, 51 MB, 9 us in a graph.
template <int FMT, int OT, int LPH>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ ReadArgs a) {
  constexpr int kGroups = kThreads / LPH, kAhead = 4;
  __shared__ TokenAt at[kGroups];
  const int per_token = a.per_token, tokens = kGroups / per_token, first = blockIdx.x * tokens;
  if ((int)threadIdx.x < tokens)
    at[threadIdx.x] = first + (int)threadIdx.x < a.b.n_tokens ? locate_token(a.b, a.c, a.bs, first + threadIdx.x) : TokenAt{-1, -1};
  __syncthreads();
  const int group = threadIdx.x / LPH, d0 = (threadIdx.x % LPH) * 8;
  const int sub = group % per_token, token = first + group / per_token;
  const long long offset = at[group / per_token].offset;
  if (d0 >= a.c.head_dim || offset < 0) return;
  const int heads = a.k_heads + a.v_heads;
  for (int h0 = sub; h0 < heads; h0 += per_token * kAhead) {
    uint4 raw[kAhead];
    float scale[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int item = h0 + i * per_token;
      if (item >= heads) break;
      const bool is_v = item >= a.k_heads;
      const int head = is_v ? item - a.k_heads : item;
      const char *row = a.c.base + (is_v ? a.c.v_offset : 0) + offset;
      if constexpr (!quantised(FMT)) {
        raw[i] = *reinterpret_cast<const uint4 *>(row + ((long long)head * a.c.head_dim + d0) * 2);
      } else if constexpr (four_bit(FMT)) {
        const char *record = row + (long long)head * a.c.head_bytes;
        raw[i].x = *reinterpret_cast<const unsigned *>(record + (d0 >> 1));
        raw[i].y = *reinterpret_cast<const unsigned char *>(record + a.c.scale_offset + 4 + (d0 >> 4));
        scale[i] = *reinterpret_cast<const float *>(record + a.c.scale_offset);
      } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(row + (long long)head * a.c.head_dim + d0);
        raw[i].x = w.x; raw[i].y = w.y;
        scale[i] = *reinterpret_cast<const float *>(row + a.c.scale_offset + 4 * head);
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int item = h0 + i * per_token;
      if (item >= heads) break;
      const bool is_v = item >= a.k_heads;
      const int head = is_v ? item - a.k_heads : item;
      float x[8];
      if constexpr (!quantised(FMT)) {
        widen8<FMT == KVR_CACHE_BF16 ? KVR_BF16 : KVR_F16>(raw[i], x);
      } else if constexpr (four_bit(FMT)) {
        const float group = __half2float(__ushort_as_half((unsigned short)group_scale(raw[i].y))) * kGroupUnit;
        const unsigned w[4] = {widen_e2m1<0>(raw[i].x), widen_e2m1<1>(raw[i].x), widen_e2m1<2>(raw[i].x), widen_e2m1<3>(raw[i].x)};
        widen8<KVR_F16>(make_uint4(w[0], w[1], w[2], w[3]), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * group * scale[i];        // code times group is exact
      } else {
        const unsigned u[2] = {raw[i].x, raw[i].y};
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const unsigned pair = u[e >> 2] >> (8 * (e & 3));
          if constexpr (FMT == KVR_CACHE_E4M3) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(pair & 0xffffu), __NV_E4M3);
            const float2 f = __half22float2(__half2(h));
            x[e] = f.x * scale[i];
            x[e + 1] = f.y * scale[i];
          } else {
            x[e] = (float)(signed char)(pair & 0xffu) * scale[i];
            x[e + 1] = (float)(signed char)(pair >> 8 & 0xffu) * scale[i];
          }
        }
      }
      const Rows &dst = is_v ? a.v : a.k;
      store8<OT>(dst.data + (long long)token * dst.token_stride + (long long)head * dst.head_stride + d0 * (OT == KVR_F32 ? 4 : 2), x);
    }
  }
}

struct KeepArgs {
  Batch b;
  CacheView c;               // base: plane 0 of layer 0
  FastDiv bs, per_row;       // per_row: 16-byte columns of a row
  long long plane_stride;
  int columns;               // planes x columns of a row
  const int32_t *index, *count;
  int index_stride;
};

constexpr int kKeepChunk = 64;

// 64 requests, 32 layers of e4m3: 99 MB in 15.5 us, 6.4 TB/s, bound by memory; 32 short lists of one layer 3.9 us, the launch and
// the list.
//
// Requests along y; a thread owns one 16-byte column of one plane and walks the request's list.  Sources ascend and never
// lie before their targets, so target i can only be a source at a place <= i: rows may be read ahead of the writes.
__global__ void __launch_bounds__(kThreads) keep_kernel(const KeepArgs a) {
  __shared__ long long from[kKeepChunk], to[kKeepChunk];
  const int r = blockIdx.y;
  int first, context, fresh;
  if (!request_lengths(a.b, a.bs.d, r, first, context, fresh)) {
    if (threadIdx.x == 0) report(a.b.status, KVR_DEV_BAD_LENGTH);
    return;
  }
  const int n = __ldg(a.count + r);
  const int32_t *list = a.index + (long long)r * a.index_stride;
  // the whole list is checked by every CTA before any of it moves a row
  bool bad = n < 0 || n > a.index_stride || n > fresh, bad_block = false;
  if (!bad) {
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const int s = __ldg(list + i);
      if (s < i || s >= fresh || (i > 0 && s <= __ldg(list + i - 1))) bad = true;
      else if (token_offset(a.b, a.c, a.bs, r, context + s) < 0 || token_offset(a.b, a.c, a.bs, r, context + i) < 0) bad_block = true;
    }
  }
  bad = __syncthreads_or(bad);
  bad_block = __syncthreads_or(bad_block);
  if (bad || bad_block) {
    if (threadIdx.x == 0) report(a.b.status, bad ? KVR_DEV_BAD_INDEX : KVR_DEV_BAD_BLOCK);
    return;
  }
  const int column = blockIdx.x * kThreads + threadIdx.x;
  const bool mine = column < a.columns;
  const unsigned plane = a.per_row.div(mine ? column : 0);
  char *base = a.c.base + plane * a.plane_stride + (long long)((mine ? column : 0) - plane * a.per_row.d) * 16;
  for (int i0 = 0; i0 < n; i0 += kKeepChunk) {
    const int m = min(kKeepChunk, n - i0);
    if ((int)threadIdx.x < m) {
      from[threadIdx.x] = token_offset(a.b, a.c, a.bs, r, context + __ldg(list + i0 + threadIdx.x));
      to[threadIdx.x] = token_offset(a.b, a.c, a.bs, r, context + i0 + threadIdx.x);
    }
    __syncthreads();
    if (mine) {
      for (int i = 0; i < m; i += 4) {
        uint4 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i + k < m && from[i + k] != to[i + k]) x[k] = *reinterpret_cast<const uint4 *>(base + from[i + k]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i + k < m && from[i + k] != to[i + k]) *reinterpret_cast<uint4 *>(base + to[i + k]) = x[k];
      }
    }
    __syncthreads();
  }
}

struct RopeTableArgs {
  float *table;
  double magnitude;
  int first, positions, pairs;
  double freq[128];
};

// cos and sin of position * frequency, reduced and taken in 64 bits (at position 131071 an angle in 32 bits would be off by 2^-8);
// once per model: 131,072 positions of 64 pairs 67 us, bound by the 64-bit operations.
__global__ void __launch_bounds__(kThreads) rope_table_kernel(const __grid_constant__ RopeTableArgs a) {
  const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (i >= (long long)a.positions * a.pairs) return;
  const int pos = (int)(i / a.pairs), pair = (int)(i - (long long)pos * a.pairs);
  double s, c;
  sincos(((double)a.first + pos) * a.freq[pair], &s, &c);
  reinterpret_cast<float2 *>(a.table)[i] = make_float2((float)(c * a.magnitude), (float)(s * a.magnitude));
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// Groups of lanes a token: as few as still fill the GPU four CTAs deep (a lane's angles then serve more heads, and more
// loads of a lane are in flight), as many as there are heads where tokens are few.  (us, one group a token / as many as heads: append of
// 32k tokens 159 / 616, read of 8k tokens 15.6 / 23.4, of 32 x 8k 306 / 782.)
int groups_per_token(int n_tokens, int heads, int groups) {
  int g = 1;
  while (g < groups && g < heads && (long long)n_tokens * g < 148ll * 4 * groups) g *= 2;
  return g;
}

template <int XT, int FMT, bool AXES>
void launch_append(const AppendArgs &a, int lanes, int grid, cudaStream_t s) {
  if (lanes == 8) append_kernel<XT, FMT, 8, AXES><<<grid, kThreads, 0, s>>>(a);
  else if (lanes == 16) append_kernel<XT, FMT, 16, AXES><<<grid, kThreads, 0, s>>>(a);
  else append_kernel<XT, FMT, 32, AXES><<<grid, kThreads, 0, s>>>(a);
}
template <int XT, int FMT>
void launch_append(const AppendArgs &a, int lanes, int grid, cudaStream_t s) {
  if (a.rope.axes > 1) launch_append<XT, FMT, true>(a, lanes, grid, s);
  else launch_append<XT, FMT, false>(a, lanes, grid, s);
}
template <int XT>
void launch_append(const AppendArgs &a, int format, int lanes, int grid, cudaStream_t s) {
  switch (format) {
    case KVR_CACHE_BF16: return launch_append<XT, KVR_CACHE_BF16>(a, lanes, grid, s);
    case KVR_CACHE_F16: return launch_append<XT, KVR_CACHE_F16>(a, lanes, grid, s);
    case KVR_CACHE_E4M3: return launch_append<XT, KVR_CACHE_E4M3>(a, lanes, grid, s);
    case KVR_CACHE_E2M1: return launch_append<XT, KVR_CACHE_E2M1>(a, lanes, grid, s);
    default: return launch_append<XT, KVR_CACHE_INT8>(a, lanes, grid, s);
  }
}

template <int FMT, int OT>
void launch_read(const ReadArgs &a, int lanes, int grid, cudaStream_t s) {
  if (lanes == 8) read_kernel<FMT, OT, 8><<<grid, kThreads, 0, s>>>(a);
  else if (lanes == 16) read_kernel<FMT, OT, 16><<<grid, kThreads, 0, s>>>(a);
  else read_kernel<FMT, OT, 32><<<grid, kThreads, 0, s>>>(a);
}
template <int OT>
void launch_read(const ReadArgs &a, int format, int lanes, int grid, cudaStream_t s) {
  switch (format) {
    case KVR_CACHE_BF16: return launch_read<KVR_CACHE_BF16, OT>(a, lanes, grid, s);
    case KVR_CACHE_F16: return launch_read<KVR_CACHE_F16, OT>(a, lanes, grid, s);
    case KVR_CACHE_E4M3: return launch_read<KVR_CACHE_E4M3, OT>(a, lanes, grid, s);
    case KVR_CACHE_E2M1: return launch_read<KVR_CACHE_E2M1, OT>(a, lanes, grid, s);
    default: return launch_read<KVR_CACHE_INT8, OT>(a, lanes, grid, s);
  }
}

int lanes_of(int head_dim) { return head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32; }

kvr_status launched() {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? KVR_OK : fail_cache(KVR_ERR_CUDA, cudaGetErrorString(e));
}

int64_t row_bytes_of(const kvr_cache_spec *s) {
  if (four_bit(s->format)) return (int64_t)s->kv_heads * record_bytes(s->head_dim);
  const int64_t elements = (int64_t)s->kv_heads * s->head_dim;
  return quantised(s->format) ? elements + (4ll * s->kv_heads + 15) / 16 * 16 : 2 * elements;
}

}  // namespace

kvr_status fail_cache(kvr_status st, const char *msg) { set_last_error(msg); return st; }

kvr_status check_spec(const kvr_cache_spec *s) {
  if (!s) return fail_cache(KVR_ERR_INVALID_ARG, "spec is NULL");
  if (s->layers < 1 || s->kv_heads < 1 || s->block_size < 1 || s->num_blocks < 1)
    return fail_cache(KVR_ERR_GEOMETRY, "layers, kv_heads, block_size and num_blocks must be at least 1");
  if (s->head_dim < 16 || s->head_dim > 256 || s->head_dim % 16) return fail_cache(KVR_ERR_GEOMETRY, "head_dim must be a multiple of 16, at most 256");
  if (s->format < KVR_CACHE_BF16 || s->format > KVR_CACHE_E2M1) return fail_cache(KVR_ERR_INVALID_ARG, "unknown cache format");
  if (four_bit(s->format) && s->head_dim % 32) return fail_cache(KVR_ERR_GEOMETRY, "head_dim of a 4-bit cache must be a multiple of 32");
  if (s->layout != KVR_LAYER_MAJOR && s->layout != KVR_BLOCK_MAJOR) return fail_cache(KVR_ERR_INVALID_ARG, "unknown layout");
  if (row_bytes_of(s) > (1ll << 30) || row_bytes_of(s) * s->block_size > (1ll << 30)) return fail_cache(KVR_ERR_GEOMETRY, "one tile exceeds 1 GiB");
  return KVR_OK;
}

kvr_status check_batch(const kvr_batch *b) {
  if (!b) return fail_cache(KVR_ERR_INVALID_ARG, "batch is NULL");
  if (b->n_req < 0 || b->n_tokens < 0 || b->max_new < 0 || b->max_tokens < 0 || b->table_stride < 0)
    return fail_cache(KVR_ERR_INVALID_ARG, "batch: negative size");
  if (b->n_tokens > 0 && (b->n_req < 1 || !b->token_start || !b->context || !b->tables || b->table_stride < 1))
    return fail_cache(KVR_ERR_INVALID_ARG, "batch: tokens without requests, or a NULL array");
  if (((uintptr_t)b->token_start | (uintptr_t)b->context | (uintptr_t)b->tables | (uintptr_t)b->status) & 3)
    return fail_cache(KVR_ERR_INVALID_ARG, "batch: arrays must be 4-byte aligned");
  return KVR_OK;
}

kvr_status check_rows(const kvr_rows *r, const char *what) {
  char buf[160];
  const char *bad = nullptr;
  if (!r->data) bad = "data is NULL";
  else if (r->type < KVR_BF16 || r->type > KVR_F32) bad = "unknown type";
  else if (r->heads < 1) bad = "heads must be at least 1";
  else {
    const int64_t size = r->type == KVR_F32 ? 4 : 2;
    if (!aligned16(r->data) || r->token_stride * size % 16 || r->head_stride * size % 16) bad = "data and strides must be multiples of 16 bytes";
    else if (r->token_stride < 0 || r->head_stride < 0 || r->token_stride > (1ll << 40) || r->head_stride > (1ll << 40)) bad = "stride out of range";
  }
  if (!bad) return KVR_OK;
  snprintf(buf, sizeof buf, "%s: %s", what, bad);
  return fail_cache(KVR_ERR_INVALID_ARG, buf);
}

kvr_status check_out(const kvr_rows *r, const char *what, int head_dim) {
  if (kvr_status st = check_rows(r, what)) return st;
  char buf[128];
  if (r->token_stride < head_dim || (r->heads > 1 && r->head_stride < head_dim)) {
    snprintf(buf, sizeof buf, "%s: rows that are written must not overlap (stride below head_dim)", what);
    return fail_cache(KVR_ERR_INVALID_ARG, buf);
  }
  return KVR_OK;
}

kvr_status layer_view(const kvr_cache_spec *s, const void *pool, int layer, CacheView *out) {
  if (kvr_status st = check_spec(s)) return st;
  if (!pool || !aligned16(pool)) return fail_cache(KVR_ERR_INVALID_ARG, "device_pool must be a 16-byte aligned pointer");
  if (layer < 0 || layer >= s->layers) return fail_cache(KVR_ERR_INVALID_ARG, "layer out of range");
  const long long row = row_bytes_of(s), tile = row * s->block_size;
  const bool by_layer = s->layout == KVR_LAYER_MAJOR;
  const long long plane = by_layer ? tile * s->num_blocks : tile;
  out->block_stride = by_layer ? tile : tile * 2 * s->layers;
  out->v_offset = plane;
  out->base = static_cast<char *>(const_cast<void *>(pool)) + 2ll * layer * plane;
  out->row_bytes = (int)row;
  out->scale_offset = four_bit(s->format) ? s->head_dim / 2 : s->kv_heads * s->head_dim;
  out->head_bytes = four_bit(s->format) ? record_bytes(s->head_dim) : s->head_dim * (quantised(s->format) ? 1 : 2);
  out->block_size = s->block_size;
  out->num_blocks = s->num_blocks;
  out->kv_heads = s->kv_heads;
  out->head_dim = s->head_dim;
  return KVR_OK;
}

Batch device_batch(const kvr_batch *b) {
  return Batch{b->token_start, b->context, b->tables, b->status, b->n_req, b->n_tokens, b->max_new, b->max_tokens, b->table_stride};
}

Rows device_rows(const kvr_rows *r) {
  const long long size = r->type == KVR_F32 ? 4 : 2;
  return Rows{static_cast<char *>(r->data), r->token_stride * size, r->head_stride * size, r->heads, r->type};
}

}  // namespace kvr

using namespace kvr;

extern "C" kvr_status kvr_cache_geometry(const kvr_cache_spec *spec, kvr_geometry *out) {
  if (!out) return fail_cache(KVR_ERR_INVALID_ARG, "out is NULL");
  if (kvr_status st = check_spec(spec)) return st;
  if (quantised(spec->format)) *out = kvr_geometry{spec->layers, 1, (int32_t)row_bytes_of(spec), 1, spec->block_size};
  else *out = kvr_geometry{spec->layers, spec->kv_heads, spec->head_dim, 2, spec->block_size};
  return KVR_OK;
}

extern "C" kvr_status kvr_rope_frequencies(const kvr_rope_scaling *s, int32_t rot_dim, double *freq, double *magnitude) {
  if (!s || !freq) return fail_cache(KVR_ERR_INVALID_ARG, "scaling or freq is NULL");
  if (rot_dim < 2 || rot_dim > 256 || rot_dim % 2) return fail_cache(KVR_ERR_INVALID_ARG, "rot_dim must be even, in [2, 256]");
  if (!(s->base > 1.0) || !std::isfinite(s->base)) return fail_cache(KVR_ERR_INVALID_ARG, "base must be above 1");
  if (s->kind < KVR_SCALE_NONE || s->kind > KVR_SCALE_RAMP) return fail_cache(KVR_ERR_INVALID_ARG, "unknown scaling");
  if (s->kind != KVR_SCALE_NONE && (!(s->factor >= 1.0) || !std::isfinite(s->factor))) return fail_cache(KVR_ERR_INVALID_ARG, "factor must be at least 1");
  if (s->kind >= KVR_SCALE_BANDS && (!(s->low > 0) || !(s->high > s->low) || !std::isfinite(s->high) || s->original < 1))
    return fail_cache(KVR_ERR_INVALID_ARG, "0 < low < high and a positive original context are needed");
  if (s->kind == KVR_SCALE_BASE && rot_dim < 4) return fail_cache(KVR_ERR_INVALID_ARG, "KVR_SCALE_BASE needs rot_dim >= 4");
  const double two_pi = 6.283185307179586476925, n = rot_dim;
  double base = s->base;
  if (s->kind == KVR_SCALE_BASE) base *= std::pow(s->factor, n / (n - 2));
  auto turns_at = [&](double x) { return n * std::log(s->original / (two_pi * x)) / (2 * std::log(s->base)); };
  double a = 0, b = 0;
  if (s->kind == KVR_SCALE_RAMP) {
    a = std::fmax(std::floor(turns_at(s->high)), 0.0);
    b = std::fmin(std::ceil(turns_at(s->low)), n - 1);
  }
  for (int p = 0; p < rot_dim / 2; ++p) {
    const double theta = std::pow(base, -2.0 * p / n);
    double f = theta;
    if (s->kind == KVR_SCALE_LINEAR) f = theta / s->factor;
    if (s->kind == KVR_SCALE_BANDS) {
      const double turns = s->original * theta / two_pi;
      const double t = std::fmin(std::fmax((turns - s->low) / (s->high - s->low), 0.0), 1.0);
      f = theta * (t + (1 - t) / s->factor);
    }
    if (s->kind == KVR_SCALE_RAMP) {
      const double t = 1 - std::fmin(std::fmax((p - a) / std::fmax(b - a, 0.001), 0.0), 1.0);
      f = theta * (t + (1 - t) / s->factor);
    }
    freq[p] = f;
  }
  if (magnitude) *magnitude = s->kind == KVR_SCALE_RAMP && s->factor > 1 ? 0.1 * std::log(s->factor) + 1 : 1;
  return KVR_OK;
}

extern "C" kvr_status kvr_rope_table(const kvr_rope_scaling *s, int32_t rot_dim, int32_t first, int32_t positions,
                                     float *table_device, void *stream) {
  RopeTableArgs a{};
  if (kvr_status st = kvr_rope_frequencies(s, rot_dim, a.freq, &a.magnitude)) return st;
  if (!table_device || !aligned16(table_device)) return fail_cache(KVR_ERR_INVALID_ARG, "table_device must be a 16-byte aligned pointer");
  if (first < 0 || positions < 0 || (int64_t)first + positions > INT32_MAX) return fail_cache(KVR_ERR_INVALID_ARG, "positions out of range");
  a.table = table_device;
  a.first = first;
  a.positions = positions;
  a.pairs = rot_dim / 2;
  const long long n = (long long)positions * a.pairs;
  if (n == 0) return KVR_OK;
  if ((n + kThreads - 1) / kThreads > INT32_MAX) return fail_cache(KVR_ERR_INVALID_ARG, "table too large for one call");
  rope_table_kernel<<<(unsigned)((n + kThreads - 1) / kThreads), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return launched();
}

static kvr_status append(const kvr_cache_spec *spec, void *device_pool, int32_t layer, const kvr_batch *batch, const kvr_rows *q,
                         const kvr_rows *k, const kvr_rows *v, const kvr_rows *q_out, const kvr_rope *rope, const kvr_rope_axes *axes,
                         const int32_t *positions, void *stream) {
  AppendArgs a{};
  if (kvr_status st = layer_view(spec, device_pool, layer, &a.c)) return st;
  if (kvr_status st = check_batch(batch)) return st;
  if (!q != !q_out) return fail_cache(KVR_ERR_INVALID_ARG, "q and q_out go together");
  int type = -1;
  const kvr_rows *in[3] = {q, k, v};
  const char *names[3] = {"q", "k", "v"};
  for (int i = 0; i < 3; ++i) {
    if (!in[i]) continue;
    if (kvr_status st = check_rows(in[i], names[i])) return st;
    if (i > 0 && in[i]->heads != spec->kv_heads) return fail_cache(KVR_ERR_INVALID_ARG, "k and v must have kv_heads heads");
    if (type >= 0 && in[i]->type != type) return fail_cache(KVR_ERR_INVALID_ARG, "q, k and v must have one type");
    type = in[i]->type;
  }
  if (type < 0) return fail_cache(KVR_ERR_INVALID_ARG, "one of q, k and v is needed");
  if (q) {
    if (kvr_status st = check_out(q_out, "q_out", spec->head_dim)) return st;
    if (q_out->type != q->type || q_out->heads != q->heads) return fail_cache(KVR_ERR_INVALID_ARG, "q_out must have q's type and heads");
    if (q->heads > (1 << 20)) return fail_cache(KVR_ERR_INVALID_ARG, "q: too many heads");
  }
  if (rope) {
    if (!rope->table || !aligned16(rope->table)) return fail_cache(KVR_ERR_INVALID_ARG, "rope: table must be a 16-byte aligned pointer");
    if (rope->rot_dim < 2 || rope->rot_dim % 2 || rope->rot_dim > spec->head_dim) return fail_cache(KVR_ERR_INVALID_ARG, "rope: rot_dim must be even and at most head_dim");
    if (rope->positions < 1) return fail_cache(KVR_ERR_INVALID_ARG, "rope: an empty table");
    if (rope->style != KVR_ROPE_HALF && rope->style != KVR_ROPE_INTERLEAVED) return fail_cache(KVR_ERR_INVALID_ARG, "rope: unknown style");
    a.rope = RopeView{rope->table, rope->positions, rope->rot_dim, rope->style, rope->inverse ? -1.f : 1.f, 1, {}};
  }
  if (axes) {
    if (!rope) return fail_cache(KVR_ERR_INVALID_ARG, "axes without rope");
    if (axes->axes < 1 || axes->axes > kMaxAxes) return fail_cache(KVR_ERR_INVALID_ARG, "axes: 1 to 4 of them");
    if (!positions) return fail_cache(KVR_ERR_INVALID_ARG, "axes: positions are needed");
    a.rope.axes = axes->axes;
    for (int p = 0; p < rope->rot_dim / 2; ++p) {
      if (axes->of_pair[p] >= axes->axes) return fail_cache(KVR_ERR_INVALID_ARG, "axes: a pair's axis is out of range");
      a.rope.axis_of[p >> 3] |= (uint16_t)(axes->of_pair[p] << (p & 7) * 2);
    }
  }
  if (positions && ((uintptr_t)positions & 3)) return fail_cache(KVR_ERR_INVALID_ARG, "positions must be 4-byte aligned");
  if (batch->n_tokens == 0) return KVR_OK;
  a.b = device_batch(batch);
  a.bs = FastDiv(spec->block_size);
  if (q) { a.q = device_rows(q); a.q_out = device_rows(q_out); a.q_heads = q->heads; }
  if (k) { a.k = device_rows(k); a.k_heads = k->heads; }
  if (v) { a.v = device_rows(v); a.v_heads = v->heads; }
  a.positions = positions;
  const int lanes = lanes_of(spec->head_dim), heads = a.q_heads + a.k_heads + a.v_heads;
  const int groups = kThreads / lanes;
  a.per_token = groups_per_token(batch->n_tokens, heads, groups);
  const int tokens = groups / a.per_token, grid = (batch->n_tokens - 1) / tokens + 1;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (type == KVR_BF16) launch_append<KVR_BF16>(a, spec->format, lanes, grid, s);
  else if (type == KVR_F16) launch_append<KVR_F16>(a, spec->format, lanes, grid, s);
  else launch_append<KVR_F32>(a, spec->format, lanes, grid, s);
  return launched();
}

extern "C" kvr_status kvr_cache_append(const kvr_cache_spec *spec, void *device_pool, int32_t layer, const kvr_batch *batch,
                                       const kvr_rows *q, const kvr_rows *k, const kvr_rows *v, const kvr_rows *q_out,
                                       const kvr_rope *rope, const int32_t *positions, void *stream) {
  return append(spec, device_pool, layer, batch, q, k, v, q_out, rope, nullptr, positions, stream);
}

extern "C" kvr_status kvr_cache_append_axes(const kvr_cache_spec *spec, void *device_pool, int32_t layer, const kvr_batch *batch,
                                            const kvr_rows *q, const kvr_rows *k, const kvr_rows *v, const kvr_rows *q_out,
                                            const kvr_rope *rope, const kvr_rope_axes *axes, const int32_t *positions, void *stream) {
  if (!axes) return fail_cache(KVR_ERR_INVALID_ARG, "axes is NULL");
  return append(spec, device_pool, layer, batch, q, k, v, q_out, rope, axes, positions, stream);
}

extern "C" kvr_status kvr_cache_read(const kvr_cache_spec *spec, const void *device_pool, int32_t layer, const kvr_batch *batch,
                                     const kvr_rows *k, const kvr_rows *v, void *stream) {
  ReadArgs a{};
  if (kvr_status st = layer_view(spec, device_pool, layer, &a.c)) return st;
  if (kvr_status st = check_batch(batch)) return st;
  if (!k && !v) return fail_cache(KVR_ERR_INVALID_ARG, "k or v is needed");
  const kvr_rows *out[2] = {k, v};
  for (int i = 0; i < 2; ++i) {
    if (!out[i]) continue;
    if (kvr_status st = check_out(out[i], i ? "v" : "k", spec->head_dim)) return st;
    if (out[i]->heads != spec->kv_heads) return fail_cache(KVR_ERR_INVALID_ARG, "k and v must have kv_heads heads");
  }
  if (k && v && k->type != v->type) return fail_cache(KVR_ERR_INVALID_ARG, "k and v must have one type");
  if (batch->n_tokens == 0) return KVR_OK;
  a.b = device_batch(batch);
  a.bs = FastDiv(spec->block_size);
  if (k) { a.k = device_rows(k); a.k_heads = k->heads; }
  if (v) { a.v = device_rows(v); a.v_heads = v->heads; }
  const int lanes = lanes_of(spec->head_dim), type = k ? k->type : v->type;
  const int groups = kThreads / lanes;
  a.per_token = groups_per_token(batch->n_tokens, a.k_heads + a.v_heads, groups);
  const int tokens = groups / a.per_token, grid = (batch->n_tokens - 1) / tokens + 1;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (type == KVR_BF16) launch_read<KVR_BF16>(a, spec->format, lanes, grid, s);
  else if (type == KVR_F16) launch_read<KVR_F16>(a, spec->format, lanes, grid, s);
  else launch_read<KVR_F32>(a, spec->format, lanes, grid, s);
  return launched();
}

extern "C" kvr_status kvr_cache_keep(const kvr_cache_spec *spec, void *device_pool, const kvr_batch *batch, const int32_t *index,
                                     int32_t index_stride, const int32_t *count, void *stream) {
  KeepArgs a{};
  if (kvr_status st = layer_view(spec, device_pool, 0, &a.c)) return st;
  if (kvr_status st = check_batch(batch)) return st;
  if (index_stride < 0 || (batch->n_tokens > 0 && (!index || !count || index_stride < 1)))
    return fail_cache(KVR_ERR_INVALID_ARG, "index, index_stride and count are needed");
  if (((uintptr_t)index | (uintptr_t)count) & 3) return fail_cache(KVR_ERR_INVALID_ARG, "index and count must be 4-byte aligned");
  if (batch->n_req > 65535) return fail_cache(KVR_ERR_INVALID_ARG, "at most 65535 requests");
  const long long columns = 2ll * spec->layers * (a.c.row_bytes / 16);
  if (columns > INT32_MAX) return fail_cache(KVR_ERR_GEOMETRY, "rows of all layers exceed 32 GiB");
  if (batch->n_tokens == 0) return KVR_OK;
  a.b = device_batch(batch);
  a.bs = FastDiv(spec->block_size);
  a.per_row = FastDiv(a.c.row_bytes / 16);
  a.plane_stride = a.c.v_offset;
  a.columns = (int)columns;
  a.index = index;
  a.count = count;
  a.index_stride = index_stride;
  keep_kernel<<<dim3((unsigned)((columns + kThreads - 1) / kThreads), (unsigned)batch->n_req), kThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return launched();
}

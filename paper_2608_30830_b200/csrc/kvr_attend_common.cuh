// Device helpers of both attention kernels: asynchronous copies, conversions, and the walk over a CTA's pieces.
#pragma once
#include "kvr_attend.cuh"
#include "kvr_once.hpp"

namespace kvr {
namespace {

// Lets `kernel` have `bytes` of dynamic shared memory on the current device.
template <class Kernel>
cudaError_t allow_shared(OncePerDevice &once, Kernel kernel, int bytes) {
  int device = -1;
  if (const cudaError_t e = cudaGetDevice(&device)) return e;
  const cudaError_t e = once(device, [&] { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); });
  if (e != cudaSuccess) cudaGetLastError();      // reported by this call, not by the next one's launch
  return e;
}

__device__ __forceinline__ unsigned shared_at(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(unsigned dst, const void *src, bool valid) {
  const int n = valid ? 16 : 0;
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copy4(unsigned dst, const void *src, bool valid) {
  const int n = valid ? 4 : 0;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---- barriers in shared memory
__device__ __forceinline__ void bar_init(unsigned bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(unsigned bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(unsigned bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(unsigned bar, unsigned parity) {
  unsigned ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// The wait for something that writes shared or tensor memory by itself and was asked for: a CTA must not end with it under way, whatever
// limit its other waits have.  False where kPolls were not enough.
__device__ __forceinline__ bool bar_settle(unsigned bar, unsigned parity) {
  for (unsigned spin = 0; spin < kPolls; ++spin)
    if (bar_try(bar, parity)) return true;
  return false;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The unit of V's scales in a row's sums (8-bit caches): a power of two that scales are multiplied by, between 2^-126 and 2^126.  A
// probability (up to 2^4) times a scale has to fit f16: when a scale that the row sees passes 2^11 units, the unit is set so that
// it lies at 2^7 to 2^8 (2^126 at most, which is where rows begin).  Products stay below 2^15, and what a key adds is rounded to
// 11 bits, or to 2^-32 of the largest scale that the row sees, whichever is more.  Scales that the row does not see have no part in
// it: past the context rows have units of their own.  (One that it sees and that is not finite decides the row's result anyway.)
constexpr float kUnitLimit = 2048.f;
__device__ __forceinline__ float unit_first(bool row) { return __uint_as_float((row ? 253u : 1u) << 23); }   // no row: never passed
__device__ __forceinline__ float unit_of(float scale) { return __uint_as_float(min(253u, 261u - (__float_as_uint(scale) >> 23)) << 23); }   // 2^(7 - e)
__device__ __forceinline__ float unit_back(float unit) { return __uint_as_float((254u << 23) - __float_as_uint(unit)); }       // 1 / unit

// two 8-bit codes (bytes 0 and 1, or 2 and 3, of w) as f16
template <int FMT, bool HIGH>
__device__ __forceinline__ unsigned widen(unsigned w) {
  if constexpr (FMT == KVR_CACHE_E4M3) {
    unsigned r;
    if constexpr (HIGH)
      asm("{.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;}" : "=r"(r) : "r"(w));
    else
      asm("{.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;}" : "=r"(r) : "r"(w));
    return r;
  } else {
    // code + 128 as the low byte of 1024 + (code + 128), minus 1152: exact
    const unsigned u = __byte_perm(w ^ 0x80808080u, 0x64646464u, HIGH ? 0x4342 : 0x4140);
    const __half2 v = __hsub2(*reinterpret_cast<const __half2 *>(&u), __half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480)));
    return *reinterpret_cast<const unsigned *>(&v);
  }
}

// 0x80 in the bytes of w that are NaN as e4m3 (0x7f, 0xff): a sum of 7 bits and one does not carry out of its byte
__device__ __forceinline__ unsigned nan_codes(unsigned w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// A CTA's walk over the pieces of segments in its run of units.
struct Piece {
  unsigned unit, next;       // the CTA's share of the segment, its opening included: units unit .. next - 1
  unsigned base;             // first unit of its request
  int r, head_group, row0;   // request, group of KV heads, first query row
  int begin, end;            // units of the segment
  Lengths len;
};
// The piece that starts at p.unit; false where the share ends within the segment's opening.
__device__ __forceinline__ bool open_piece(const AttendArgs &a, Piece &p, unsigned last) {
  // requests without units are passed over (the bound on r cannot be met while p.unit is below the call's units)
  while (p.len.units == 0 || p.unit - p.base >= (unsigned)(p.len.units + a.opening) * p.len.segments) {
    p.base = p.unit;
    if (++p.r >= a.b.n_req) { p.r = a.b.n_req - 1; return false; }
    p.len = attend_lengths(a, p.r);
  }
  const int span = p.len.units + a.opening, offset = (int)((p.unit - p.base) / span), from = (int)((p.unit - p.base) - offset * span);
  const int to = (int)min((unsigned)span, from + (last - p.unit));
  p.next = p.unit + (to - from);
  p.begin = max(from - a.opening, 0);
  p.end = to - a.opening;
  p.head_group = 0;
  p.row0 = offset << a.row_shift;
  if (a.head_groups > 1) {
    const int tiles = p.len.segments / a.head_groups;
    p.head_group = offset / tiles;
    p.row0 = (offset - p.head_group * tiles) << a.row_shift;
  }
  return p.end > 0;
}
__device__ __forceinline__ bool next_piece(const AttendArgs &a, Piece &p, unsigned last) {
  p.unit = p.next;
  return p.unit < last && open_piece(a, p, last);
}

struct Cut {
  int c0, c1, which0;        // the CTAs of the segment; which of the first one's two pieces it is
  __device__ __forceinline__ int piece(int c) const { return c * 2 + (c == c0 ? which0 : 0); }
};
// The rows of a segment from its pieces of `n` <= 32 CTAs c, c + step, ...: to the output, or (fold) to the first one's place.
// A lane has 4 channels of a 128-channel slab; what costs is latency, so kRows rows and kAhead pieces are read at once.
// Out of line: the kernels' own loops need the registers.
template <int SLABS>
__device__ __noinline__ void join_pieces(const AttendArgs &a, const Piece &p, const Cut &cut, int c, int step, int n, bool fold, int rows, int heads, int warps, int warp, int lane) {
  constexpr int kRows = SLABS > 1 ? 2 : 4, kAhead = 4;
  const int total = rows * heads;
  const long long stride = (long long)step * 2 * a.group_heads * a.row_tile;     // rows from one piece to the next
  // the first CTA of a segment may hold it as its second piece, all others as their first
  auto first_row = [&](int lh, int row) { return ((long long)c * 2 * a.group_heads + lh) * a.row_tile + row; };
  const long long second = c == cut.c0 && cut.which0 ? (long long)a.group_heads * a.row_tile : 0;
#pragma unroll 1
  for (int i0 = warp * kRows; i0 < total; i0 += warps * kRows) {
    float f[kRows], m[kRows], l[kRows], o[kRows][SLABS][4];
    long long at[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int i = min(i0 + u, total - 1), lh = i / rows;
      at[u] = first_row(lh, i - lh * rows);
      float2 ml = make_float2(-INFINITY, 0.f);
      if (lane < n) ml = __ldcg(a.part_ml + at[u] + lane * stride + (lane == 0 ? second : 0));
      f[u] = m[u] = ml.x;
      l[u] = ml.y;
#pragma unroll
      for (int h = 0; h < SLABS; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[u][h][e] = 0.f;
    }
    float4 x[kAhead][kRows][SLABS];
    auto read = [&](int k, float4 (&to)[kRows][SLABS]) {
#pragma unroll
      for (int u = 0; u < kRows; ++u)
#pragma unroll
        for (int h = 0; h < SLABS; ++h) {
          const int d = h * 128 + lane * 4;
          to[u][h] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (k < n && d < a.c.head_dim) to[u][h] = __ldcg(reinterpret_cast<const float4 *>(a.part_o + (at[u] + k * stride + (k == 0 ? second : 0)) * a.c.head_dim + d));
        }
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k) read(k, x[k]);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) m[u] = fmaxf(m[u], __shfl_xor_sync(0xffffffffu, m[u], d));
      f[u] = lane >= n ? 0.f : f[u] == m[u] ? 1.f : exp2_fast(f[u] - m[u]);        // both -infinity: a piece of an empty row
      l[u] *= f[u];
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) l[u] += __shfl_xor_sync(0xffffffffu, l[u], d);
    }
#pragma unroll 1
    for (int k0 = 0; k0 < n; k0 += kAhead) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
          const float w = __shfl_sync(0xffffffffu, f[u], (k0 + k) & 31);           // 0 beyond the last
#pragma unroll
          for (int h = 0; h < SLABS; ++h) {
            if (k0 + k >= n) continue;
            o[u][h][0] += x[k][u][h].x * w; o[u][h][1] += x[k][u][h].y * w; o[u][h][2] += x[k][u][h].z * w; o[u][h][3] += x[k][u][h].w * w;
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) read(k0 + kAhead + k, x[k]);
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      if (i0 + u >= total) break;
      const int lh = (i0 + u) / rows, row = i0 + u - lh * rows;
      if (fold) {
#pragma unroll
        for (int h = 0; h < SLABS; ++h) {
          const int d = h * 128 + lane * 4;
          if (d < a.c.head_dim) *reinterpret_cast<float4 *>(a.part_o + (at[u] + second) * a.c.head_dim + d) = make_float4(o[u][h][0], o[u][h][1], o[u][h][2], o[u][h][3]);
        }
        if (lane == 0) a.part_ml[at[u] + second] = make_float2(m[u], l[u]);
        continue;
      }
      const float inv = l[u] > 0.f ? 1.f / l[u] : l[u] == 0.f ? 0.f : NAN;
      const int t = (int)a.group.div(p.row0 + row), q_head = (p.head_group * a.group_heads + lh) * (int)a.group.d + (p.row0 + row - t * (int)a.group.d);
      char *dst = a.out.data + (long long)(p.len.first + t) * a.out.token_stride + (long long)q_head * a.out.head_stride;
#pragma unroll
      for (int h = 0; h < SLABS; ++h) {
        const int d = h * 128 + lane * 4;
        if (d >= a.c.head_dim) continue;
        uint2 w;
        if (a.out.type == KVR_BF16) w = make_uint2(pack_bf16(o[u][h][0] * inv, o[u][h][1] * inv), pack_bf16(o[u][h][2] * inv, o[u][h][3] * inv));
        else w = make_uint2(pack_f16(o[u][h][0] * inv, o[u][h][1] * inv), pack_f16(o[u][h][2] * inv, o[u][h][3] * inv));
        *reinterpret_cast<uint2 *>(dst + d * 2) = w;
      }
      if (a.lse && lane == 0) a.lse[(long long)(p.len.first + t) * a.q_heads + q_head] = l[u] == 0.f ? -INFINITY : m[u] * 0.69314718f + logf(l[u]);
    }
    __syncwarp();
  }
}

// After this CTA's piece of a cut segment has been stored: joins the segment's pieces if it was the last to come in.  sync() is
// a barrier of the warps that call this (false: given up); `last` is shared memory; join(cut, c, step, n, fold) joins the pieces of
// the n CTAs c, c + step, ...: to the output, or (fold) to the first one's place.
template <class Sync, class Join>
__device__ __forceinline__ bool hand_in(const AttendArgs &a, const Piece &p, const Shares &sh, Sync sync, volatile int *last, int warp, int lane, Join join) {
  const unsigned span = p.len.units + a.opening, begin = p.unit - (p.unit - p.base) % span;
  Cut cut;
  cut.c0 = sh.cta_of(begin + a.opening);       // the first with keys
  cut.c1 = sh.cta_of(begin + span - 1);
  cut.which0 = sh.first(cut.c0) >= begin ? 0 : 1;
  const int all = cut.c1 - cut.c0 + 1, groups = (all + kJoinAtOnce - 1) / kJoinAtOnce;
  const int group = ((int)blockIdx.x - cut.c0) / kJoinAtOnce, leader = cut.c0 + group * kJoinAtOnce, n = min(kJoinAtOnce, cut.c1 - leader + 1);
  auto come_in = [&](int *counter, int of) {
    if (!sync()) return false;
    if (warp == 0 && lane == 0) {
      __threadfence();                   // what the barrier has shown this thread goes before the count
      const bool is_last = atomicAdd(counter, 1) == of - 1;
      if (is_last) atomicExch(counter, 0);
      __threadfence();
      *last = is_last;
    }
    return (bool)sync();
  };
  if (!come_in(a.handed_in + leader * 2 + (leader == cut.c0 ? cut.which0 : 0), n)) return false;
  if (!*last) return true;
  join(cut, leader, 1, n, groups > 1);
  if (groups == 1) return true;
  if (!come_in(a.handed_in + (a.ctas + cut.c0) * 2 + cut.which0, groups)) return false;
  if (!*last) return true;
  join(cut, cut.c0, kJoinAtOnce, groups, false);
  return true;
}

}  // namespace
}  // namespace kvr

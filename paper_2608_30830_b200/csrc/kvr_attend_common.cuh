// Device helpers of both attention kernels: asynchronous copies, conversions, and the walk over a CTA's pieces.
#pragma once
#include "kvr_attend.cuh"

namespace kvr {
namespace {

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

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 2^e exactly; 0 below the normal numbers
__device__ __forceinline__ float power2(int e) { return e < -126 ? 0.f : __uint_as_float((unsigned)(e + 127) << 23); }

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

// A CTA's walk over the pieces of segments in its run of units.
struct Piece {
  long long unit;            // first unit of the piece
  long long base;            // first unit of its request
  int r, head_group, row0;   // request, group of KV heads, first query row
  int begin, end;            // units of the segment
  Lengths len;
};
__device__ __forceinline__ void open_piece(const AttendArgs &a, Piece &p, long long last) {
  // requests without units are passed over (the bound on r cannot be met while p.unit is below the call's units)
  while (p.len.segments == 0 || p.unit - p.base >= (long long)p.len.units * p.len.segments) {
    p.base = p.unit;
    if (++p.r >= a.b.n_req) { p.r = a.b.n_req - 1; p.len = Lengths{0, 0, 0, 0, 1, 1}; break; }
    p.len = attend_lengths(a, p.r);
  }
  const int offset = (int)((p.unit - p.base) / p.len.units);
  p.begin = (int)((p.unit - p.base) - (long long)offset * p.len.units);
  p.end = (int)min((long long)p.len.units, p.begin + (last - p.unit));
  const int tiles = p.len.segments / a.head_groups;
  p.head_group = offset / tiles;
  p.row0 = (offset - p.head_group * tiles) * a.row_tile;
}
__device__ __forceinline__ bool next_piece(const AttendArgs &a, Piece &p, long long last) {
  p.unit += p.end - p.begin;
  if (p.unit >= last) return false;
  open_piece(a, p, last);
  return true;
}

}  // namespace
}  // namespace kvr
